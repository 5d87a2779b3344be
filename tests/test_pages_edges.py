"""The paged 8-bit cache at its edges: rows that see nothing of a tile, zeros, extreme scales, long axes, refusals."""
import ctypes

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
