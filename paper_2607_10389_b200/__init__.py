"""B200 data path of an exact-state session mover: per-chunk CRC32C, dirty-chunk diff, lossless
WM1 encode and decode+verify, and the paged 8-bit attention cache of the sessions it moves, as CUDA
kernels behind the C ABI of ``include/wm.h``."""
