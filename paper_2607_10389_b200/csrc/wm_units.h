// How the tiles of an attention call are dealt out to its workers.  Plain C++, for the kernels and for a test on the host.
#pragma once
#include <cstdint>

#ifndef WM_HOST_DEVICE
#ifdef __CUDACC__
#define WM_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define WM_HOST_DEVICE inline
#endif
#endif

namespace wm {

// Worker w's first tile of `total` (the division in 32 bits where they hold it: the long one is a hundred instructions to wait for).
// workers: not above 320; total: below 2^55.
WM_HOST_DEVICE unsigned long long share_of(uint32_t w, unsigned long long total, unsigned long long workers)
{
    if (w >= workers) return total;
    return total < (1u << 23) ? (unsigned long long)(w * (uint32_t)total / (uint32_t)workers) : w * total / workers;
}
// The worker that has a tile.
WM_HOST_DEVICE uint32_t worker_of(unsigned long long tile, unsigned long long total, unsigned long long workers)
{
    return (uint32_t)(((tile + 1) * workers - 1) / total);
}

// Tile `off` of units of nt tiles each, one behind the other.  A request has up to 2^31 units of up to 2^23 tiles: off has 64 bits, and
// is divided in 32 where they hold it, else bit by bit (the long division is a call, whose registers cost the kernels 2 % even where it
// is never made).
struct TileAt {
    uint32_t unit, j;
};
WM_HOST_DEVICE TileAt tile_at(unsigned long long off, uint32_t nt)
{
    TileAt a = {0, 0};
    if (off >> 32 == 0) {
        a.unit = (uint32_t)off / nt;
        a.j = (uint32_t)off - a.unit * nt;
        return a;
    }
#ifdef __CUDACC__
#pragma unroll 1
#endif
    for (int bit = 54; bit >= 0; bit--) {              // (off < 2^55, nt < 2^31)
        a.j = 2u * a.j + (uint32_t)(off >> bit & 1u);
        a.unit = 2u * a.unit + (a.j >= nt ? 1u : 0u);
        if (a.j >= nt) a.j -= nt;
    }
    return a;
}
// Tiles of `units` units.
WM_HOST_DEVICE unsigned long long tiles_of(uint32_t units, uint32_t nt) { return (unsigned long long)units * nt; }

}  // namespace wm
