"""The paged 8-bit cache at its edges: rows that see nothing of a tile, zeros, extreme scales, long axes, refusals."""
import ctypes
import math

import pytest
import torch

import pages_ref as ref
import pages_ref64 as ref64
import test_pages as tp
from paper_2607_10389_b200 import binding as wm

gpu = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]


def test_the_reference_for_all_rows_at_once_is_the_one_for_a_row():
    g = torch.Generator().manual_seed(30)
    lens, starts, page = [5, 0, 40, 70, 3], [0, 2, 3, 3, 33, 40], 16
    k, v, ks, vs = ref.random_pool(12, 2, page, 64, g, 3)
    table = ref.random_table(lens, page, 5, 12, g)
    q = torch.randn((40, 6, 64), generator=g).double()
    for causal, window in ((True, 0), (True, 7), (False, 0)):
        a = ref.attend(ref.values(k), ref.values(v), ks.double(), vs.double(), table, lens, starts, q, 0.1, causal, window)
        b = ref64.attend(k, v, ks, vs, table, lens, starts, q, 0.1, causal, window)
        for x, y, name in zip(a, b, ("out", "lse", "weight", "reach", "floor", "spread")):
            assert torch.equal(x.isinf(), y.isinf()) and torch.allclose(x.nan_to_num(neginf=0.0), y.nan_to_num(neginf=0.0), rtol=1e-12, atol=1e-13), name


def _alike(arrays, pages, score, dim, g):
    """Keys that all lie one way, so that queries near (1, 1, ..) have scores near `score`."""
    arrays[0].copy_(((score * dim ** -0.5 + 0.3 * torch.randn(arrays[0].shape, generator=g)) * 8.0).to(ref.E4M3).view(torch.uint8))
    arrays[2].fill_(0.125)
    pages.k.copy_(arrays[0]), pages.k_scale.copy_(arrays[2])


@gpu
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("group", [1, 3, 8])
@pytest.mark.parametrize("dim,lens,rows,max_q", [(64, [130], [4], 4), (128, [130, 257, 128], [4, 3, 2], 4), (64, [300, 140], [200, 131], 1)])
@pytest.mark.parametrize("score,zeros", [(-100.0, False), (-20.0, True), (-100.0, True)])
def test_attend_low_scores_where_some_rows_see_nothing_of_a_tile(dtype, group, dim, lens, rows, max_q, score, zeros):
    """Rows on both sides of a tile's border, with scores far below zero or under the smallest value scale."""
    g = torch.Generator().manual_seed(31)
    pages, arrays, table = tp._attend_case(lens, 64, 2, dim, g)
    _alike(arrays, pages, score, dim, g)
    if zeros:
        arrays[1].zero_(), arrays[3].fill_(2.0 ** -126)
        pages.v.copy_(arrays[1]), pages.v_scale.copy_(arrays[3])
    q = 1.0 + 0.25 * torch.randn((sum(rows), 2 * group, dim), generator=g)
    for window in (0, 129):
        tp._attend(pages, arrays, table, lens, rows, 2 * group, dtype, g, max_q=max_q, q=q, window=window)


@gpu
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("group", [1, 3, 8])
@pytest.mark.parametrize("score,zeros", [(-100.0, False), (-20.0, True)])
def test_attend_drafts_across_a_tile_s_border_with_low_scores(dtype, group, score, zeros):
    """Four rows at the end of 130 tokens, in so many requests that a block has both tiles of a unit: the first two rows see nothing
    of the second."""
    g = torch.Generator().manual_seed(39)
    lens, rows = [130] * 200, [4] * 200
    pages, arrays, table = tp._attend_case(lens, 64, 2, 64, g)
    _alike(arrays, pages, score, 64, g)
    if zeros:
        arrays[1].zero_(), arrays[3].fill_(2.0 ** -126)
        pages.v.copy_(arrays[1]), pages.v_scale.copy_(arrays[3])
    q = (1.0 + 0.25 * torch.randn((800, 2 * group, 64), generator=g)).to(dtype).cuda()
    starts = list(range(0, 801, 4))
    out, lse = torch.full_like(q, 7.0), torch.full((800, 2 * group), 7.0, device="cuda")
    wm.wm_pages_attend(pages, tp._dev(table), tp._dev(lens), tp._dev(starts), q, out, wm.new_pages_workspace(64), lse=lse, max_q=4)
    want = ref64.attend(pages.k, pages.v, pages.k_scale, pages.v_scale, table, lens, starts, q, 64 ** -0.5, True, 0)
    far, far_lse = ref.bounds(*want, dtype, 64)
    assert ((out.double() - want[0]).abs() <= far).all() and ((lse.double() - want[1]).abs() <= far_lse).all()


@gpu
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("rows", [[3, 2], [200, 131]])
@pytest.mark.parametrize("dim,page,group", [(64, 16, 1), (128, 64, 4)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 100), (False, 0)])
def test_attend_queries_of_zeros_over_keys_of_zeros(dtype, rows, dim, page, group, causal, window):
    """Factors of scores that are not there any more in 32 bits: zero or tiny queries, keys under the smallest scale
    (as wm_pages_append writes zeros), a tiny softmax scale; ordinary values and zeros."""
    g = torch.Generator().manual_seed(32)
    lens = [300, 131]
    pages, arrays, table = tp._attend_case(lens, page, 2, dim, g)
    q = torch.randn((sum(rows), 2 * group, dim), generator=g)
    q[::3] = 0.0
    q[1::3] *= 2.0 ** -20
    run = lambda **kw: tp._attend(pages, arrays, table, lens, rows, 2 * group, dtype, g, causal, window, q=q, **kw)  # noqa: E731
    run()
    run(scale=2.0 ** -120)
    arrays[2][::2] = 2.0 ** -126                         # codes of any size under it, then zeros everywhere
    pages.k_scale.copy_(arrays[2])
    run()
    arrays[0].zero_(), arrays[2].fill_(2.0 ** -126)
    pages.k.copy_(arrays[0]), pages.k_scale.copy_(arrays[2])
    run()
    arrays[1].zero_(), arrays[3].fill_(2.0 ** -126)
    pages.v.copy_(arrays[1]), pages.v_scale.copy_(arrays[3])
    run()


@gpu
@pytest.mark.parametrize("rows", [5, 150])
def test_a_prompt_of_zeros_through_append_and_attend(rows):
    """What an engine warms up with."""
    pages = wm.new_pages(8, 64, 2, 128)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table, count, start, slots = i32([[-1] * 4]), i32([8]), i32([0, 0]), i32([0] * rows)
    wm.wm_pages_plan(i32([0]), i32([rows]), 64, table, i32(list(range(8))), count, count, start, slots)
    kv = torch.zeros(rows, 2, 128, device="cuda", dtype=torch.bfloat16)
    q = torch.zeros(rows, 8, 128, device="cuda", dtype=torch.bfloat16)
    wm.wm_pages_append(pages, kv, kv + 0.5, slots)
    out, lse = torch.full_like(q, 7.0), torch.full((rows, 8), 7.0, device="cuda")
    wm.wm_pages_attend(pages, table, i32([rows]), start, q, out, wm.new_pages_workspace(128), lse=lse, max_q=rows)
    assert (out == 0.5).all()                            # 0.5 is a code under a power of two, and so is their mean
    want = torch.arange(1, rows + 1, dtype=torch.float64).log()[:, None]
    assert ((lse.cpu().double() - want).abs() <= 2.0 ** -18 + 2.0 ** -22 * want).all()


@gpu
@pytest.mark.parametrize("rows", [12, 150])
def test_attend_rows_that_see_nothing_give_zeros_whatever_their_queries_are(rows):
    g = torch.Generator().manual_seed(33)
    lens = [rows - 5]
    pages, arrays, table = tp._attend_case(lens, 32, 2, 64, g)
    q = torch.randn((rows, 2, 64), generator=g)
    q[0], q[1, 0, 3], q[2, 1, 5], q[3], q[4] = float("nan"), float("inf"), -float("inf"), 0.0, 2.0 ** -24
    for dtype in HALVES:
        out, lse = tp._attend(pages, arrays, table, lens, [rows], 2, dtype, g, q=q)
        assert (out[:5] == 0).all() and (lse[:5] == -float("inf")).all()


def _attend_large(kv_heads, group, dim, page, dtype, lens, rows, causal, window, g, max_q=None, rise=0.0, n_rows_more=3):
    """Against 64 bits on the GPU.  `rise`: how far scores climb from the first token to the last."""
    pages, arrays, table = tp._attend_case(lens, page, kv_heads, dim, g, spread=3)
    heads, n = kv_heads * group, sum(rows)
    q = torch.randn((n + n_rows_more, heads, dim), generator=g)
    if rise:
        q = 1.0 + 0.25 * q
        for i, x in enumerate(lens):
            for j, p in enumerate(table[i][:ref.pages_of(x, page)]):
                t = (j * page + torch.arange(page)) / x
                y = t[None, :, None] * rise * dim ** -0.5 + 0.1 * torch.randn((kv_heads, page, dim), generator=g)
                s = 2.0 ** torch.ceil(torch.log2(y.abs().amax((1, 2)) / 448.0))
                arrays[0][p], arrays[2][p] = (y / s[:, None, None]).to(ref.E4M3).view(torch.uint8), s
        pages.k.copy_(arrays[0]), pages.k_scale.copy_(arrays[2])
    q = q.to(dtype).cuda()
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    out, lse, ws, report = torch.full_like(q, 7.0), torch.full((q.shape[0], heads), 7.0, device="cuda"), wm.new_pages_workspace(dim), wm.new_pages_report()
    ws.fill_(0xFF)
    wm.wm_pages_attend(pages, tp._dev(table), tp._dev(lens), tp._dev(starts), q, out, ws, lse=lse, causal=causal, window=window,
                       max_q=max_q or max(rows), report=report)
    assert wm.read_pages_report(report) == ("OK", None)
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()
    want = ref64.attend(pages.k, pages.v, pages.k_scale, pages.v_scale, table, lens, starts, q[:n], dim ** -0.5, causal, window)
    far, far_lse = ref.bounds(*want, dtype, dim)
    off, off_lse = (out[:n].double() - want[0]).abs(), (lse[:n].double() - want[1]).abs()
    assert (off <= far).all(), (off / far).max()
    fine = ~want[1].isinf()
    assert torch.equal(lse[:n].isinf(), want[1].isinf()) and (off_lse[fine] <= far_lse[fine]).all(), (off_lse / far_lse)[fine].max()


@gpu
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("dim,page", [(64, 64), (128, 16), (128, 128), (64, 32)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 700), (False, 0)])
@pytest.mark.parametrize("rise", [0.0, 60.0])
def test_attend_prompts_of_many_tiles_a_block(dtype, dim, page, causal, window, rise):
    """Some 2000 tiles for the GPU's 148 blocks: units of many tiles, several units a block, parts of many tiles; with scores that
    climb by 60 (86 in powers of two), so that what outputs refer to moves on the way."""
    g = torch.Generator().manual_seed(36)
    _attend_large(8, 4, dim, page, dtype, [2000, 3001, 700, 129], [600, 701, 300, 2], causal, window, g, rise=rise)


@gpu
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("group,rows", [(1, [1, 8, 3, 5]), (4, [1, 4, 3, 2]), (4, [8, 7, 5, 1]), (8, [4, 1, 3, 2]), (32, [1, 1, 1, 1])])
@pytest.mark.parametrize("dim,page", [(64, 32), (128, 64), (128, 16)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1500), (False, 0)])
def test_attend_few_rows_of_many_tiles_a_block(dtype, group, rows, dim, page, causal, window):
    """Some 1300 tiles for the GPU's 296 blocks, with every number of rows that has code of its own."""
    g = torch.Generator().manual_seed(37)
    _attend_large(8, group, dim, page, dtype, [9000, 7003, 300, 4500], rows, causal, window, g, rise=60.0 if page == 64 else 0.0)


@gpu
@pytest.mark.parametrize("max_q", [1, 700])
def test_attend_mixed_batches_of_many_tiles_a_block(max_q):
    g = torch.Generator().manual_seed(38)
    _attend_large(4, 4, 128, 64, torch.bfloat16, [3000, 9000, 1, 4000, 2500, 5000], [700, 1, 1, 5, 300, 1], True, 0, g, max_q=max_q)


def test_attend_of_no_rows_asks_for_no_number_of_rows():
    at, p, r = 1 << 20, tp._c_pages(), tp._c_rows()
    assert wm.lib().wm_pages_attend(ctypes.addressof(p), at, 4, at, at, 1, r, r, 0, None, 0, 8, 0, 1.0, 1, 0, at, 1 << 30, None, None) == 0
    assert wm.last_launch_count() == 0


@gpu
def test_attend_of_no_rows_with_every_number_of_rows_a_caller_may_give():
    pages, none = wm.new_pages(4, 16, 2, 64), torch.zeros(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for kw in ({}, dict(max_q=0), dict(max_q=3)):
        wm.wm_pages_attend(pages, i32([[0, 1]]), i32([3]), i32([0, 0]), none, none.clone(), wm.new_pages_workspace(64), **kw)
    torch.cuda.synchronize()


@gpu
@pytest.mark.parametrize("code,tie", [(9.0, 8.5), (11.0, 9.5), (13.0, 12.5), (15.0, 14.5), (15.0, 7.25), (13.0, 4.5 * 2.0 ** -9)])
def test_append_rounds_kept_codes_once(code, tie):
    """Old scales beside those that would put a code's new value exactly between two codes: the product has more bits than a float,
    and a float of it can lie on the middle where the product does not."""
    page, n, new = 16, 41, 2.0
    near = torch.tensor(tie / code, dtype=torch.float32).view(torch.int32) + torch.arange(n, dtype=torch.int32) - n // 2
    scales = (near.view(torch.float32) * new)[:, None].contiguous()
    k = torch.full((n, 1, page, 64), code).to(ref.E4M3).view(torch.uint8)
    k[:, :, 1::2] = torch.tensor(-code).to(ref.E4M3).view(torch.uint8)
    pages = wm.Pages(k.cuda(), k.cuda(), scales.cuda(), scales.cuda())
    slots = [p * page + 5 for p in range(n)]
    x = torch.full((n, 1, 64), 448.0 * new).cuda()
    want = [ref.values(k), scales.double()]
    ref.append(want[0], want[1], x.cpu(), slots, page)
    assert (want[1] == new).all() and len(want[0][:, 0, 0, 0].unique()) == 2        # the middle is crossed
    wm.wm_pages_append(pages, x, x, torch.tensor(slots, dtype=torch.int32, device="cuda"))
    tp._check_pool(pages, [want[0], want[0], want[1], want[1]])


@gpu
@pytest.mark.parametrize("rows,max_q", [([1, 1], 1), ([3, 8], 8), ([60, 140], 140), ([60, 140], 1)])
@pytest.mark.parametrize("exponent", [119, 110, -120, -126, -130])
def test_attend_values_at_the_ends_of_the_floats(rows, max_q, exponent):
    """Values up to 1.75 * 2^127: their weighted sums leave 32 bits where their means do not."""
    g = torch.Generator().manual_seed(34)
    lens = [300, 5000]
    pages, arrays, table = tp._attend_case(lens, 64, 2, 64, g)
    arrays[1].fill_(0x7E), arrays[3].fill_(2.0 ** exponent)
    pages.v.copy_(arrays[1]), pages.v_scale.copy_(arrays[3])
    q = 0.1 * torch.randn((sum(rows), 2, 64), generator=g)
    tp._attend(pages, arrays, table, lens, rows, 2, torch.bfloat16, g, q=q, max_q=max_q)


@gpu
@pytest.mark.parametrize("exponent", [119, 0, -126])
@pytest.mark.parametrize("requests,rows,heads", [(1, 1, 1), (20, 3, 16), (1, 200, 1), (1, 2560, 16)])
def test_attend_means_of_a_quarter_of_a_million_values_at_the_ends_of_the_floats(exponent, requests, rows, heads):
    """Equal weights and equal values: every sum is a whole number that a float holds, and the mean is the value.  A unit in parts, and
    whole."""
    n, page = 1 << 18, 128
    k, v = torch.zeros((n // page, heads, page, 64), dtype=torch.uint8, device="cuda"), torch.full((n // page, heads, page, 64), 0x7E, dtype=torch.uint8, device="cuda")
    pages = wm.Pages(k, v, torch.ones((n // page, heads), device="cuda"), torch.full((n // page, heads), 2.0 ** exponent, device="cuda"))
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").repeat(requests, 1)
    q = torch.zeros((requests * rows, heads, 64), dtype=torch.bfloat16, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    wm.wm_pages_attend(pages, table, tp._dev([n] * requests), tp._dev([rows * i for i in range(requests + 1)]), q, out, wm.new_pages_workspace(64), lse=lse,
                       causal=False, max_q=rows)
    assert (out.float() == 448.0 * 2.0 ** exponent).all()
    assert (lse.double() - 18 * math.log(2.0)).abs().max() <= 2.0 ** -18 + 2.0 ** -22 * 13


@gpu
@pytest.mark.parametrize("dtype", HALVES)
@pytest.mark.parametrize("rows,heads,dim", [(2560, 16, 64), (64, 1, 128), (8, 16, 64)])
@pytest.mark.parametrize("bits", [20, 27])
def test_attend_one_token_far_above_half_a_million_others(dtype, rows, heads, dim, bits):
    """The first token weighs 2^bits times as much as each of the others, which together still count: 1 / 256 of it where bits is 27.
    In one unit from end to end, and in parts."""
    n, page = 1 << 19, 128
    k = torch.zeros((2, heads, page, dim), dtype=torch.uint8)
    v = torch.full_like(k, 0x38)                         # ones
    k[0, :, 0] = 0x38
    v[0, :, 0, ::2] = 0                                  # half of the channels have nothing of the first token
    ones = torch.ones((2, heads), device="cuda")
    pages = wm.Pages(k.cuda(), v.cuda(), ones, ones.clone())
    table = torch.ones((1, n // page), dtype=torch.int32, device="cuda")
    table[0, 0] = 0
    q = torch.ones((rows, heads, dim), dtype=dtype, device="cuda")
    out, lse = torch.zeros_like(q), torch.zeros((rows, heads), device="cuda")
    score = bits * math.log(2.0)
    wm.wm_pages_attend(pages, table, tp._dev([n]), tp._dev([0, rows]), q, out, wm.new_pages_workspace(dim), lse=lse, scale=score / dim,
                       causal=False, max_q=rows)
    others = (n - 1) * 2.0 ** -bits
    want = torch.ones(dim, dtype=torch.float64, device="cuda")
    want[::2] = others / (1.0 + others)
    # products and sums of ones are exact; the score has a handful of factors, each rounded by 2^-24 of it; weights have 11 bits, and what
    # is below their grid is no more than 2^-12 of the largest in all.  The tensor cores lose what is below 2^-25 of the sum that it
    # is added to: nothing where that holds nothing of the first token
    d = 8 * 2.0 ** -24 * score
    far = want * (2.0 ** -12 + 2 * d + torch.finfo(dtype).eps / 2 + n * 2.0 ** -25) + 2.0 ** -12
    off = (out.double() - want).abs()
    assert (off <= far).all(), (off / far).max()
    assert ((lse.double() - score - math.log1p(others)).abs() <= d + 2.0 ** -18 + 2.0 ** -22 * score).all()


def _plan_args(**change):
    f = {n: 1 << 20 for n in ("old", "new", "table", "free", "count", "count_out", "start", "slots", "report")}
    f.update(change)
    return (f["old"], f["new"], 1, 64, 10, f["table"], 4, f["free"], f["count"], f["count_out"], f["start"], f["slots"], 5, f["report"], None)


# (only what is refused: these addresses are not looked at)
@pytest.mark.parametrize("off", [1, 2, 3])
def test_words_at_odd_addresses_are_refused(off):
    """A slice of a byte tensor can be anywhere; read as words there it would end the context."""
    lib, at, r = wm.lib(), 1 << 20, tp._c_rows()
    for name in ("old", "new", "table", "free", "count", "count_out", "start", "slots", "report"):
        assert lib.wm_pages_plan(*_plan_args(**{name: at + off})) == -1, name
    for change in (dict(k_scale=at + off), dict(v_scale=at + off)):
        p = tp._c_pages(**change)
        assert lib.wm_pages_append(ctypes.addressof(p), r, r, 0, at, 1, None, None) == -1, change
        assert lib.wm_pages_attend(ctypes.addressof(p), at, 4, at, at, 1, r, r, 0, None, 1, 8, 1, 1.0, 1, 0, at, 1 << 30, None, None) == -1, change
    p = tp._c_pages()
    for slots, report in ((at + off, at), (at, at + off)):
        assert lib.wm_pages_append(ctypes.addressof(p), r, r, 0, slots, 1, report, None) == -1
    for i in range(5):
        a = [at + off * (i == j) for j in range(5)]
        assert lib.wm_pages_attend(ctypes.addressof(p), a[0], 4, a[1], a[2], 1, r, r, 0, a[3], 1, 8, 1, 1.0, 1, 0, at, 1 << 30, a[4], None) == -1, i


@gpu
def test_numbers_beyond_32_bits_are_not_cut():
    g = torch.Generator().manual_seed(40)
    lens, rows = [70, 200], [3, 150]
    pages, arrays, table = tp._attend_case(lens, 32, 1, 64, g)
    for window in (2 ** 32, 2 ** 32 + 5, 2 ** 40 + 1):
        for max_q in (2 ** 32, 2 ** 32 + 1):
            tp._attend(pages, arrays, table, lens, rows, 2, torch.bfloat16, g, window=window, max_q=max_q)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    count, start, slots, tab = i32([4]), i32([0, 0]), i32([-9] * 5), i32([[-1, -1]])
    for page in (2 ** 32 + 16, -16, 0):
        with pytest.raises(wm.WmError):
            wm.wm_pages_plan(i32([0]), i32([5]), page, tab, i32([0, 1, 2, 3]), count, count, start, slots)
    assert count.item() == 4 and slots.tolist() == [-9] * 5 and tab.tolist() == [[-1, -1]]


@gpu
@pytest.mark.parametrize("rows", [[1, 1], [4, 2], [200, 131]])
@pytest.mark.parametrize("exponent", [-100, -108, -116, -120, 100, 120])
def test_attend_queries_of_every_size(rows, exponent):
    """Queries at the ends of bf16, over keys at the other end."""
    g = torch.Generator().manual_seed(41)
    lens = [300, 131]
    pages, arrays, table = tp._attend_case(lens, 64, 2, 64, g)
    arrays[2].fill_(2.0 ** (-6 - exponent) if exponent < 0 else 2.0 ** -126)
    pages.k_scale.copy_(arrays[2])
    q = torch.randn((sum(rows), 4, 64), generator=g) * 2.0 ** exponent
    if -113 <= exponent < 0:                             # (rows whose largest element is below 2^-119 are on a coarser grid)
        q[0] *= 2.0 ** -6
    tp._attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g, q=q)


@gpu
@pytest.mark.parametrize("page", [16, 32])
@pytest.mark.parametrize("lens,rows", [([90], [60]), ([90, 220, 35, 350] * 4, [60, 50, 40, 200] * 4)])
def test_attend_gives_the_same_bits_whatever_was_in_shared_memory(page, lens, rows):
    """Rows that fill a tile up see what a call before has left behind the last page: they have no say in how the others are computed."""
    g = torch.Generator().manual_seed(42)
    pages, arrays, table = tp._attend_case(lens, page, 8, 128, g)
    pages.v_scale.fill_(2.0 ** -90)
    before, one = wm.new_pages(1, 128, 16, 128), tp._dev([[0] * 8])
    starts = [0]
    for r in rows:
        starts.append(starts[-1] + r)
    q = torch.randn((starts[-1], 8, 128), generator=g).to(torch.bfloat16).cuda()
    qb, ob, ws = torch.zeros((600, 16, 128), device="cuda", dtype=torch.bfloat16), torch.zeros((600, 16, 128), device="cuda", dtype=torch.bfloat16), wm.new_pages_workspace(128)
    many, at = (tp._dev([1024]), tp._dev([0, 600])), (tp._dev(table), tp._dev(lens), tp._dev(starts))
    got = []
    for code in (0x7F, 0x00, 0x7F, 0x38):
        out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
        before.k.fill_(code), before.v.fill_(code)
        torch.cuda.synchronize()
        wm.wm_pages_attend(before, one, *many, qb, ob, ws, causal=False, max_q=600)
        wm.wm_pages_attend(pages, *at, q, out, ws, lse=lse, causal=False, max_q=max(rows))
        got.append((out.cpu(), lse.cpu()))
    for out, lse in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1])
