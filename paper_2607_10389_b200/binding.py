"""Thin Python binding of the C ABI in ``include/wm.h`` (argument marshalling only).

Every step of the path runs in the CUDA library; torch is used for device memory and
streams.  There is no CPU fallback: importing this module without the built library, or
calling it without a CUDA device, raises.
"""
from __future__ import annotations

import ctypes
import os
import struct
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_SO = os.path.join(_HERE, "libwm.so")

STATUS = {
    0: "OK", -1: "ERR_ARG", -2: "ERR_CAPACITY", -3: "ERR_FORMAT", -4: "ERR_META_CRC", -5: "ERR_STRUCT",
    -6: "ERR_DESC", -7: "ERR_CHUNK_CRC", -8: "ERR_STALE", -9: "ERR_CACHE_CRC", -10: "ERR_TIMEOUT",
    -11: "ERR_CUDA",
}
RESULT_BYTES = 40
EXPORTS = ("wm_num_chunks", "wm_num_tiles", "wm_meta_bytes", "wm_wire_bound", "wm_workspace_bytes",
           "wm_checksum", "wm_dirty_diff", "wm_encode", "wm_decode_verify", "wm_last_launch_count",
           "wm_timing_enable", "wm_timing_read_ms", "wm_checksum_noalloc", "wm_encode_leaves",
           "wm_decode_verify_leaves", "wm_zero_tiles_enable", "wm_decode_verify_strict", "wm_checksum_poly", "wm_entropy_enable",
           "wm_encode_opt", "wm_decode_verify_opt", "wm_checksum_xxh64", "wm_wait_budget_ms", "wm_workspace_status",
           "wm_inject_stall", "wm_pages_plan", "wm_pages_append", "wm_pages_workspace_bytes", "wm_pages_attend")


class WmError(RuntimeError):
    pass


def load_library() -> ctypes.CDLL:
    if not os.path.exists(_SO):
        raise WmError(f"{_SO} is missing: build it with `python -m paper_2607_10389_b200.build` "
                      "(there is no CPU fallback)")
    lib = ctypes.CDLL(_SO)
    u64, u32, vp = ctypes.c_uint64, ctypes.c_uint32, ctypes.c_void_p
    lib.wm_num_chunks.restype = u64
    lib.wm_num_chunks.argtypes = [u64, u32]
    lib.wm_num_tiles.restype = u64
    lib.wm_num_tiles.argtypes = [u64]
    for n in ("wm_meta_bytes", "wm_wire_bound", "wm_workspace_bytes"):
        getattr(lib, n).restype = u64
        getattr(lib, n).argtypes = [u64, u32]
    lib.wm_last_launch_count.restype = u32
    lib.wm_last_launch_count.argtypes = []
    lib.wm_timing_enable.restype = None
    lib.wm_timing_enable.argtypes = [ctypes.c_int]
    lib.wm_zero_tiles_enable.restype = None
    lib.wm_zero_tiles_enable.argtypes = [ctypes.c_int]
    lib.wm_entropy_enable.restype = None
    lib.wm_entropy_enable.argtypes = [ctypes.c_int]
    lib.wm_wait_budget_ms.restype = None
    lib.wm_wait_budget_ms.argtypes = [u32]
    lib.wm_inject_stall.restype = None
    lib.wm_inject_stall.argtypes = [ctypes.c_int]
    lib.wm_workspace_status.restype = ctypes.c_int
    lib.wm_workspace_status.argtypes = [vp, vp]
    lib.wm_timing_read_ms.restype = ctypes.c_int
    lib.wm_timing_read_ms.argtypes = [ctypes.c_int, ctypes.POINTER(ctypes.c_float)]
    lib.wm_checksum.restype = ctypes.c_int
    lib.wm_checksum.argtypes = [vp, u64, u32, vp, vp, u64, vp]
    lib.wm_checksum_poly.restype = ctypes.c_int
    lib.wm_checksum_poly.argtypes = [vp, u64, u32, ctypes.c_int, vp, vp, u64, vp]
    lib.wm_checksum_xxh64.restype = ctypes.c_int
    lib.wm_checksum_xxh64.argtypes = [vp, u64, u32, u64, vp, vp]
    lib.wm_checksum_noalloc.restype = ctypes.c_int
    lib.wm_checksum_noalloc.argtypes = [vp, u64, u32, vp, vp]
    lib.wm_dirty_diff.restype = ctypes.c_int
    lib.wm_dirty_diff.argtypes = [vp, vp, u64, u32, vp, vp, vp, vp, u64, vp]
    lib.wm_encode.restype = ctypes.c_int
    lib.wm_encode.argtypes = [vp, u64, u32, vp, vp, vp, u64, vp, u64, vp, vp]
    lib.wm_decode_verify.restype = ctypes.c_int
    lib.wm_decode_verify.argtypes = [vp, u64, vp, u64, u32, vp, vp, u64, vp, vp]
    lib.wm_decode_verify_strict.restype = ctypes.c_int
    lib.wm_decode_verify_strict.argtypes = [vp, u64, vp, u64, u32, vp, vp, u64, vp, vp]
    lib.wm_encode_opt.restype = ctypes.c_int
    lib.wm_encode_opt.argtypes = [vp, vp, u32, u64, u32, vp, vp, vp, u64, vp, u64, u32, vp, vp]
    lib.wm_decode_verify_opt.restype = ctypes.c_int
    lib.wm_decode_verify_opt.argtypes = [vp, u64, vp, vp, u32, u64, u32, vp, vp, u64, u32, vp, vp]
    lib.wm_encode_leaves.restype = ctypes.c_int
    lib.wm_encode_leaves.argtypes = [vp, u32, u64, u32, vp, vp, vp, u64, vp, u64, vp, vp]
    lib.wm_decode_verify_leaves.restype = ctypes.c_int
    lib.wm_decode_verify_leaves.argtypes = [vp, u64, vp, u32, u64, u32, vp, vp, u64, vp, vp]
    lib.wm_pages_workspace_bytes.restype = u64
    lib.wm_pages_workspace_bytes.argtypes = [u32]
    lib.wm_pages_plan.restype = ctypes.c_int
    lib.wm_pages_plan.argtypes = [vp, vp, u32, u32, u32, vp, u32, vp, vp, vp, vp, vp, u32, vp, vp]
    lib.wm_pages_append.restype = ctypes.c_int
    lib.wm_pages_append.argtypes = [vp, vp, vp, ctypes.c_int, vp, u32, vp, vp]
    lib.wm_pages_attend.restype = ctypes.c_int
    lib.wm_pages_attend.argtypes = [vp, vp, u32, vp, vp, u32, vp, vp, ctypes.c_int, vp, u32, u32, u32, ctypes.c_float, u32, u32,
                                    vp, u64, vp, vp]
    return lib


_lib = None


def lib() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        _lib = load_library()
    return _lib


@dataclass
class Result:
    status: int
    first_bad_chunk: int
    n_bad_chunks: int
    n_present: int
    wire_len: int
    payload_bytes: int
    cache_crc: int

    @property
    def status_name(self) -> str:
        return STATUS.get(self.status, str(self.status))

    @property
    def ok(self) -> bool:
        return self.status == 0


def read_result(result_dev: torch.Tensor) -> Result:
    """Copy a 40-byte device result record to the host (synchronises the current stream)."""
    raw = result_dev.cpu().numpy().tobytes()
    st, fb, nb, npres, wl, pb, cc, _ = struct.unpack("<iIIIQQII", raw)
    return Result(st, fb, nb, npres, wl, pb, cc)


def num_chunks(nbytes: int, chunk_bytes: int) -> int:
    return int(lib().wm_num_chunks(nbytes, chunk_bytes))


def num_tiles(nbytes: int) -> int:
    return int(lib().wm_num_tiles(nbytes))


def meta_bytes(nbytes: int, chunk_bytes: int) -> int:
    return int(lib().wm_meta_bytes(nbytes, chunk_bytes))


def wire_bound(nbytes: int, chunk_bytes: int) -> int:
    return int(lib().wm_wire_bound(nbytes, chunk_bytes))


def workspace_bytes(nbytes: int, chunk_bytes: int) -> int:
    return int(lib().wm_workspace_bytes(nbytes, chunk_bytes))


def last_launch_count() -> int:
    return int(lib().wm_last_launch_count())


KIND_CHECKSUM, KIND_DIFF, KIND_ENCODE, KIND_DECODE = 0, 1, 2, 3


def timing_enable(on: bool) -> None:
    lib().wm_timing_enable(1 if on else 0)


def zero_tiles_enable(on: bool) -> None:
    """Encoder option: full tiles of all-zero bytes become table entries without payload."""
    lib().wm_zero_tiles_enable(1 if on else 0)


def entropy_enable(on: bool) -> None:
    """Codec option: entropy-coded exponents (ENT tiles).  Applies to the encode calls (what they
    write) and to the decode calls (what they expect) of this process."""
    lib().wm_entropy_enable(1 if on else 0)


def wait_budget_ms(ms: int) -> None:
    """Upper bound of every device-side wait of the calls issued from now on (default 2000 ms)."""
    lib().wm_wait_budget_ms(int(ms))


def inject_stall(on) -> None:
    """Test hook: calls issued while it is on leave out what their bounded waits wait for, so the
    waits run out after the budget and the calls end in ERR_TIMEOUT.  2: the encode kernel's wait
    for a tile's widths instead of its scanner and the other calls' copies."""
    lib().wm_inject_stall(2 if on == 2 else 1 if on else 0)


def workspace_status(workspace, stream=None) -> int:
    """Device-side outcome (a wm_status) of the last call that used `workspace` on the stream;
    None stands for the built-in scratch of wm_checksum_noalloc.  Synchronises the stream."""
    return int(lib().wm_workspace_status(None if workspace is None else workspace.data_ptr(), _stream(stream)))


def timing_read_ms(kind: int) -> float:
    ms = ctypes.c_float(0.0)
    _check(lib().wm_timing_read_ms(kind, ctypes.byref(ms)), "wm_timing_read_ms")
    return float(ms.value)


def _dev_u8(t: torch.Tensor, what: str) -> torch.Tensor:
    if not t.is_cuda:
        raise WmError(f"{what} must be a CUDA tensor (there is no CPU path)")
    if not t.is_contiguous():
        raise WmError(f"{what} must be contiguous")
    return t


# The current stream's handle without making a Stream object of it: 0.2 us instead of 3.4, where a
# small cache's call is 4 us of host work in all.  The two functions are not public (a PyTorch without
# CUDA has neither); the public way is taken where they are missing.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None or _device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _check(rc: int, what: str) -> None:
    if rc != 0:
        raise WmError(f"{what}: {STATUS.get(rc, rc)}")


def new_workspace(nbytes: int, chunk_bytes: int, device="cuda") -> torch.Tensor:
    n = workspace_bytes(nbytes, chunk_bytes)
    if n == 0:
        raise WmError("bad geometry")
    return torch.empty(n, dtype=torch.uint8, device=device)


def new_result(device="cuda") -> torch.Tensor:
    return torch.zeros(RESULT_BYTES, dtype=torch.uint8, device=device)


def wm_checksum(cache: torch.Tensor, chunk_bytes: int, crc_out: torch.Tensor, workspace: torch.Tensor,
                stream=None) -> None:
    _dev_u8(cache, "cache")
    nbytes = cache.numel() * cache.element_size()
    _check(lib().wm_checksum(cache.data_ptr(), nbytes, chunk_bytes, crc_out.data_ptr(), workspace.data_ptr(),
                             workspace.numel(), _stream(stream)), "wm_checksum")


POLY_CRC32C, POLY_ZLIB = 0, 1


def wm_checksum_poly(cache: torch.Tensor, chunk_bytes: int, polynomial: int, crc_out: torch.Tensor,
                     workspace: torch.Tensor, stream=None) -> None:
    """wm_checksum with the polynomial chosen by the caller (POLY_CRC32C or POLY_ZLIB)."""
    _dev_u8(cache, "cache")
    nbytes = cache.numel() * cache.element_size()
    _check(lib().wm_checksum_poly(cache.data_ptr(), nbytes, chunk_bytes, int(polynomial), crc_out.data_ptr(),
                                  workspace.data_ptr(), workspace.numel(), _stream(stream)), "wm_checksum_poly")


def wm_checksum_xxh64(cache: torch.Tensor, chunk_bytes: int, seed: int, hash_out: torch.Tensor, stream=None) -> None:
    """XXH64 of every chunk into an int64 / uint64 tensor of n_chunks entries."""
    _dev_u8(cache, "cache")
    nbytes = cache.numel() * cache.element_size()
    _check(lib().wm_checksum_xxh64(cache.data_ptr(), nbytes, chunk_bytes, int(seed) & 0xFFFFFFFFFFFFFFFF, hash_out.data_ptr(),
                                   _stream(stream)), "wm_checksum_xxh64")


NOALLOC_MAX_BYTES = 4 << 30


def wm_checksum_noalloc(cache: torch.Tensor, chunk_bytes: int, crc_out: torch.Tensor, stream=None,
                        nbytes: int | None = None) -> None:
    """wm_checksum without a workspace argument: scratch and tables are built into the library,
    for callers that may not allocate device memory.  `nbytes` overrides the tensor's size
    (used to exercise the size limit without allocating a buffer that large)."""
    _dev_u8(cache, "cache")
    n = cache.numel() * cache.element_size() if nbytes is None else int(nbytes)
    _check(lib().wm_checksum_noalloc(cache.data_ptr(), n, chunk_bytes, crc_out.data_ptr(), _stream(stream)),
           "wm_checksum_noalloc")


def wm_dirty_diff(cache: torch.Tensor, prev: torch.Tensor, chunk_bytes: int, dirty_out: torch.Tensor,
                  dirty_idx_out, n_dirty_out: torch.Tensor, workspace: torch.Tensor, stream=None) -> None:
    _dev_u8(cache, "cache")
    _dev_u8(prev, "prev")
    nbytes = cache.numel() * cache.element_size()
    if prev.numel() * prev.element_size() != nbytes:
        raise WmError("snapshots differ in size")
    _check(lib().wm_dirty_diff(cache.data_ptr(), prev.data_ptr(), nbytes, chunk_bytes, dirty_out.data_ptr(),
                               None if dirty_idx_out is None else dirty_idx_out.data_ptr(),
                               n_dirty_out.data_ptr(), workspace.data_ptr(), workspace.numel(),
                               _stream(stream)), "wm_dirty_diff")


def wm_encode(cache: torch.Tensor, chunk_bytes: int, dirty, crc_inout: torch.Tensor, wire: torch.Tensor,
              workspace: torch.Tensor, result: torch.Tensor, stream=None, wire_cap=None) -> None:
    _dev_u8(cache, "cache")
    _dev_u8(wire, "wire")
    nbytes = cache.numel() * cache.element_size()
    cap = wire.numel() if wire_cap is None else int(wire_cap)
    _check(lib().wm_encode(cache.data_ptr(), nbytes, chunk_bytes, None if dirty is None else dirty.data_ptr(),
                           crc_inout.data_ptr(), wire.data_ptr(), cap, workspace.data_ptr(), workspace.numel(),
                           result.data_ptr(), _stream(stream)), "wm_encode")


def wm_decode_verify(wire: torch.Tensor, wire_len: int, dst: torch.Tensor, chunk_bytes: int,
                     dst_crc_inout: torch.Tensor, workspace: torch.Tensor, result: torch.Tensor,
                     stream=None) -> None:
    _dev_u8(wire, "wire")
    _dev_u8(dst, "dst")
    nbytes = dst.numel() * dst.element_size()
    _check(lib().wm_decode_verify(wire.data_ptr(), int(wire_len), dst.data_ptr(), nbytes, chunk_bytes,
                                  dst_crc_inout.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                  result.data_ptr(), _stream(stream)), "wm_decode_verify")


def wm_decode_verify_strict(wire: torch.Tensor, wire_len: int, dst: torch.Tensor, chunk_bytes: int,
                            dst_crc_inout: torch.Tensor, workspace: torch.Tensor, result: torch.Tensor,
                            stream=None) -> None:
    """wm_decode_verify that stores nothing until every check has passed."""
    _dev_u8(wire, "wire")
    _dev_u8(dst, "dst")
    nbytes = dst.numel() * dst.element_size()
    _check(lib().wm_decode_verify_strict(wire.data_ptr(), int(wire_len), dst.data_ptr(), nbytes, chunk_bytes,
                                         dst_crc_inout.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                         result.data_ptr(), _stream(stream)), "wm_decode_verify_strict")


OPT_ZERO_TILES, OPT_ENTROPY, OPT_STRICT = 1, 2, 4


def opt_blocks(n: int) -> int:
    """Option bits that cap the main kernel at n thread blocks (each takes one SM); 0: no cap."""
    return (int(n) & 0xFF) << 8



def wm_encode_opt(cache, chunk_bytes: int, dirty, crc_inout: torch.Tensor, wire: torch.Tensor, workspace: torch.Tensor,
                  result: torch.Tensor, options: int, stream=None, leaf_table=None, nbytes=None) -> None:
    """wm_encode / wm_encode_leaves with the options given per call (OPT_ZERO_TILES, OPT_ENTROPY).
    Flat form: `cache` is a tensor; leaf form: `cache` is None, `leaf_table` and `nbytes` are given."""
    _dev_u8(wire, "wire")
    if leaf_table is None:
        _dev_u8(cache, "cache")
        n, cp, lp, nl = cache.numel() * cache.element_size(), cache.data_ptr(), None, 0
    else:
        n, cp, lp, nl = int(nbytes), None, leaf_table.data_ptr(), leaf_table.shape[0]
    _check(lib().wm_encode_opt(cp, lp, nl, n, chunk_bytes, None if dirty is None else dirty.data_ptr(), crc_inout.data_ptr(),
                               wire.data_ptr(), wire.numel(), workspace.data_ptr(), workspace.numel(), int(options),
                               result.data_ptr(), _stream(stream)), "wm_encode_opt")


def wm_decode_verify_opt(wire: torch.Tensor, wire_len: int, dst, chunk_bytes: int, dst_crc_inout: torch.Tensor,
                         workspace: torch.Tensor, result: torch.Tensor, options: int, stream=None, leaf_table=None,
                         nbytes=None) -> None:
    """The decode calls with the options given per call (OPT_ENTROPY: the image holds ENT tiles;
    OPT_STRICT: nothing is stored before the verdict)."""
    _dev_u8(wire, "wire")
    if leaf_table is None:
        _dev_u8(dst, "dst")
        n, dp, lp, nl = dst.numel() * dst.element_size(), dst.data_ptr(), None, 0
    else:
        n, dp, lp, nl = int(nbytes), None, leaf_table.data_ptr(), leaf_table.shape[0]
    _check(lib().wm_decode_verify_opt(wire.data_ptr(), int(wire_len), dp, lp, nl, n, chunk_bytes, dst_crc_inout.data_ptr(),
                                      workspace.data_ptr(), workspace.numel(), int(options), result.data_ptr(),
                                      _stream(stream)), "wm_decode_verify_opt")


def make_leaf_table(tensors, device="cuda") -> torch.Tensor:
    """Device table of (ptr, nbytes) pairs, one per tensor, in the order given: the `wm_leaf`
    array of the leaf-mode calls.  The tensors must stay alive while the table is in use."""
    rows = []
    for t in tensors:
        if not t.is_cuda or not t.is_contiguous():
            raise WmError("leaves must be contiguous CUDA tensors")
        rows.append((t.data_ptr(), t.numel() * t.element_size()))
    table = torch.tensor(rows, dtype=torch.int64).reshape(-1, 2)
    return table.to(device)


def wm_encode_leaves(leaf_table: torch.Tensor, nbytes: int, chunk_bytes: int, dirty, crc_inout: torch.Tensor,
                     wire: torch.Tensor, workspace: torch.Tensor, result: torch.Tensor, stream=None,
                     wire_cap=None) -> None:
    _dev_u8(wire, "wire")
    cap = wire.numel() if wire_cap is None else int(wire_cap)
    _check(lib().wm_encode_leaves(leaf_table.data_ptr(), leaf_table.shape[0], int(nbytes), chunk_bytes,
                                  None if dirty is None else dirty.data_ptr(), crc_inout.data_ptr(), wire.data_ptr(),
                                  cap, workspace.data_ptr(), workspace.numel(), result.data_ptr(), _stream(stream)),
           "wm_encode_leaves")


def wm_decode_verify_leaves(wire: torch.Tensor, wire_len: int, leaf_table: torch.Tensor, nbytes: int,
                            chunk_bytes: int, dst_crc_inout: torch.Tensor, workspace: torch.Tensor,
                            result: torch.Tensor, stream=None) -> None:
    _dev_u8(wire, "wire")
    _check(lib().wm_decode_verify_leaves(wire.data_ptr(), int(wire_len), leaf_table.data_ptr(), leaf_table.shape[0],
                                         int(nbytes), chunk_bytes, dst_crc_inout.data_ptr(), workspace.data_ptr(),
                                         workspace.numel(), result.data_ptr(), _stream(stream)),
           "wm_decode_verify_leaves")


# ---------------------------------------------------------------- the paged 8-bit cache

class _CPages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("page_stride", ctypes.c_uint64), ("head_stride", ctypes.c_uint64), ("token_stride", ctypes.c_uint64),
                ("n_pages", ctypes.c_uint32), ("page_tokens", ctypes.c_uint32), ("kv_heads", ctypes.c_uint32),
                ("head_dim", ctypes.c_uint32)]


_pack_rows = struct.Struct("=QQQ").pack          # a wm_rows: pointer, strides of rows and heads
TYPE_BF16, TYPE_F16, TYPE_F32 = 0, 1, 2
_TYPES = {torch.bfloat16: TYPE_BF16, torch.float16: TYPE_F16, torch.float32: TYPE_F32}
ATTEND_CAUSAL = 1
PAGES_MAX_REQUESTS = 4000
PAGES_REPORT_BYTES = 16
_WORD = 1 << 32                                  # what ctypes would cut numbers to without a word


class Pages:
    """A pool of 8-bit cache pages: codes of keys and values (n_pages, kv_heads, page_tokens, head_dim) as
    uint8 or float8_e4m3fn tensors (any strides whose last is 1), and their scales (n_pages, kv_heads), float32.
    Holds the tensors; their memory must not be given another use while the pool is in use."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor):
        for t, what in ((k, "k"), (v, "v")):
            if not t.is_cuda:
                raise WmError(f"{what} must be a CUDA tensor (there is no CPU path)")
            if t.dim() != 4 or t.element_size() != 1 or t.stride(3) != 1:
                raise WmError(f"{what} must be 8-bit codes (n_pages, kv_heads, page_tokens, head_dim) whose channels are contiguous")
        if k.shape != v.shape or k.stride() != v.stride() or k.device != v.device:
            raise WmError("keys and values must have the same shape, strides and device")
        for t, what in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t.shape != k.shape[:2] or t.dtype != torch.float32 or t.device != k.device or not t.is_contiguous():
                raise WmError(f"{what} must be a contiguous float32 tensor (n_pages, kv_heads) on the codes' device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.kv_heads, self.page_tokens, self.head_dim = k.shape
        size = self.head_dim                     # (a stride along one page, head or token leads nowhere)
        strides = [s if n > 1 else size for s, n in zip(k.stride(), k.shape)]
        self._c = _CPages(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), strides[0], strides[1], strides[2],
                          self.n_pages, self.page_tokens, self.kv_heads, self.head_dim)
        self._ref, self._device = ctypes.addressof(self._c), k.get_device()

    def handle(self, here: int) -> int:
        """Address of the wm_pages record, for calls on device `here`."""
        if self._device != here:
            _refuse(self.k, "the pool", here)
        return self._ref


def new_pages(n_pages: int, page_tokens: int, kv_heads: int, head_dim: int, device="cuda") -> Pages:
    """A pool with all codes and scales zero."""
    shape = (n_pages, kv_heads, page_tokens, head_dim)
    k, v = (torch.zeros(shape, dtype=torch.uint8, device=device) for _ in range(2))
    return Pages(k, v, *(torch.zeros(shape[:2], dtype=torch.float32, device=device) for _ in range(2)))


def pages_workspace_bytes(head_dim: int) -> int:
    return int(lib().wm_pages_workspace_bytes(head_dim))


def new_pages_workspace(head_dim: int, device="cuda") -> torch.Tensor:
    """Scratch of wm_pages_attend: calls that share it must be ordered."""
    n = pages_workspace_bytes(head_dim)
    if n == 0:
        raise WmError("bad geometry")
    return torch.empty(n, dtype=torch.uint8, device=device)


def new_pages_report(device="cuda") -> torch.Tensor:
    return torch.zeros(PAGES_REPORT_BYTES, dtype=torch.uint8, device=device)


def read_pages_report(report: torch.Tensor):
    """(status name, lowest index concerned or None) of a report; synchronises the current stream."""
    status, first = report[:8].cpu().view(torch.int32).tolist()
    return STATUS.get(status, str(status)), (first & 0xFFFFFFFF) - 1 if first else None


# The arguments' checks.  They are made on every call, so each is one pass of cheap questions; what is wrong is found out
# only when something is.  `here`: the current device, on whose stream the kernels run.
def _here() -> int:
    if _device is None:
        return torch.cuda.current_device()
    try:
        return _device()
    except RuntimeError:                      # (no device at all)
        return -2


def _i32(t: torch.Tensor, n, what: str, here: int) -> int:
    if t.dtype is torch.int32 and t.get_device() == here and t.is_contiguous() and (n is None or t.numel() == n):
        return t.data_ptr()
    _refuse(t, what, here)
    raise WmError(f"{what} must be a contiguous int32 tensor" + (f" of {n} entries" if n is not None else ""))


def _refuse(t: torch.Tensor, what: str, here: int) -> None:
    if not t.is_cuda:
        raise WmError(f"{what} must be a CUDA tensor (there is no CPU path)")
    if t.get_device() != here:
        raise WmError(f"{what} is on device {t.get_device()}, the current device is {here}")


def _table(t: torch.Tensor, n_requests: int, here: int):
    shape = t.shape
    if t.dtype is torch.int32 and t.get_device() == here and len(shape) == 2 and shape[0] == n_requests and t.is_contiguous():
        return t.data_ptr(), shape[1]
    _refuse(t, "the table", here)
    raise WmError(f"the table must be a contiguous int32 tensor of {n_requests} rows")


def _rows(t: torch.Tensor, heads: int, dim: int, what: str, here: int) -> bytes:
    shape, stride = t.shape, t.stride()
    if len(shape) == 3 and shape[1] == heads and shape[2] == dim and stride[2] == 1 and t.dtype in _TYPES and t.get_device() == here:
        return _pack_rows(t.data_ptr(), stride[0] if shape[0] > 1 else 0, stride[1] if heads > 1 else 0)      # (no stride where it leads nowhere)
    _refuse(t, what, here)
    raise WmError(f"{what} must be (rows, {heads}, {dim}) in bfloat16, float16 or float32 with contiguous channels")


def _report(report, here: int):
    if report is None:
        return None
    if report.get_device() == here and report.numel() * report.element_size() >= PAGES_REPORT_BYTES and report.is_contiguous():
        return report.data_ptr()
    _refuse(report, "report", here)
    raise WmError(f"report must be {PAGES_REPORT_BYTES} contiguous bytes")


def wm_pages_plan(old_len: torch.Tensor, new_len: torch.Tensor, page_tokens: int, table: torch.Tensor, free_pages: torch.Tensor,
                  free_count: torch.Tensor, free_count_out: torch.Tensor, start: torch.Tensor, slots: torch.Tensor, report=None,
                  stream=None) -> None:
    """Block tables, free list, row offsets and slot map of a step (see include/wm.h).  All tensors are int32;
    `free_count_out` may be `free_count`."""
    here, n = _here(), old_len.numel()
    if not 0 < page_tokens < _WORD:
        raise WmError("page_tokens must be 16, 32, 64 or 128")
    tab, width = _table(table, n, here)
    n_slots = slots.numel()
    rc = lib().wm_pages_plan(_i32(old_len, None, "old_len", here), _i32(new_len, n, "new_len", here), n, page_tokens, free_pages.numel(),
                             tab, width, _i32(free_pages, None, "free_pages", here), _i32(free_count, 1, "free_count", here),
                             _i32(free_count_out, 1, "free_count_out", here), _i32(start, n + 1, "start", here),
                             _i32(slots, None, "slots", here) if n_slots else None, n_slots, _report(report, here), _stream(stream))
    if rc:
        _check(rc, "wm_pages_plan")


def wm_pages_append(pages: Pages, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, report=None, stream=None) -> None:
    """Rows of keys and values (rows, kv_heads, head_dim) into the slots of the pool (see include/wm.h)."""
    here, n = _here(), k.shape[0]
    if k.dtype is not v.dtype or v.shape[0] != n:
        raise WmError("k and v must have the same type and number of rows")
    rc = lib().wm_pages_append(pages.handle(here), _rows(k, pages.kv_heads, pages.head_dim, "k", here),
                               _rows(v, pages.kv_heads, pages.head_dim, "v", here), _TYPES[k.dtype], _i32(slots, n, "slots", here), n,
                               _report(report, here), _stream(stream))
    if rc:
        _check(rc, "wm_pages_append")


def wm_pages_attend(pages: Pages, table: torch.Tensor, kv_len: torch.Tensor, q_start: torch.Tensor, q: torch.Tensor,
                    out: torch.Tensor, workspace: torch.Tensor, lse=None, scale=None, causal: bool = True, window: int = 0,
                    max_q=None, report=None, stream=None) -> None:
    """Attention of the rows q (rows, q_heads, head_dim) over the pool into `out` (see include/wm.h).  `scale` is
    head_dim ** -0.5 unless given; `max_q` the most rows a request has (all of q's unless given)."""
    here, n, shape, dim = _here(), kv_len.numel(), q.shape, pages.head_dim
    if len(shape) != 3 or out.dtype is not q.dtype or out.shape != shape:
        raise WmError("q must be (rows, heads, channels) and out have its type and shape")
    if window < 0 or (max_q is not None and max_q < 0):
        raise WmError("window and max_q must not be negative")
    window = min(window, _WORD - 1)            # (far beyond every request already)
    rows, heads, _ = shape
    if lse is not None and not (lse.dtype is torch.float32 and lse.get_device() == here and lse.shape == (rows, heads) and lse.is_contiguous()):
        _refuse(lse, "lse", here)
        raise WmError(f"lse must be a contiguous float32 tensor ({rows}, {heads})")
    if workspace.get_device() != here or not workspace.is_contiguous():
        _refuse(workspace, "workspace", here)
        raise WmError("workspace must be contiguous")
    tab, width = _table(table, n, here)
    rc = lib().wm_pages_attend(pages.handle(here), tab, width, _i32(kv_len, None, "kv_len", here), _i32(q_start, n + 1, "q_start", here), n,
                               _rows(q, heads, dim, "q", here), _rows(out, heads, dim, "out", here), _TYPES[q.dtype],
                               None if lse is None else lse.data_ptr(), rows, heads, rows if max_q is None else min(max_q, _WORD - 1),
                               dim ** -0.5 if scale is None else scale, ATTEND_CAUSAL if causal else 0, window, workspace.data_ptr(),
                               workspace.numel() * workspace.element_size(), _report(report, here), _stream(stream))
    if rc:
        _check(rc, "wm_pages_attend")
