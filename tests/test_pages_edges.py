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
