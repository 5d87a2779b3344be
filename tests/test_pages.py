"""The paged 8-bit cache: block tables from lengths, new tokens in 8 bits, attention over the pool."""
import ctypes
import types
import random

import pytest
import torch

import pages_ref as ref
from paper_2607_10389_b200 import binding as wm

gpu = pytest.mark.gpu


def _dev(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


# ---------------------------------------------------------------- refusals (no device needed: the checks come first)

def _c_pages(**change):
    at = 1 << 20
    f = dict(k=at, v=at, k_scale=at, v_scale=at, page_stride=8 * 64 * 128, head_stride=64 * 128, token_stride=128, n_pages=10,
             page_tokens=64, kv_heads=8, head_dim=128)
    f.update(change)
    return wm._CPages(*[f[n] for n, _ in wm._CPages._fields_])


def _c_rows(**change):
    f = dict(ptr=1 << 20, row_stride=8 * 128, head_stride=128)
    f.update(change)
    return wm._pack_rows(f["ptr"] or 0, f["row_stride"], f["head_stride"])


BAD_PAGES = [dict(k=None), dict(v_scale=None), dict(k=8 + (1 << 20)), dict(page_stride=24), dict(token_stride=64), dict(token_stride=136),
             dict(page_stride=1 << 40), dict(token_stride=1 << 40), dict(page_stride=0), dict(head_stride=64),
             dict(n_pages=0), dict(n_pages=1 << 25), dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=256), dict(kv_heads=0),
             dict(kv_heads=1025), dict(head_dim=96), dict(head_dim=0)]


@pytest.mark.parametrize("change", BAD_PAGES, ids=str)
def test_a_pool_that_breaks_the_rules_is_refused(change):
    lib, at = wm.lib(), 1 << 20
    p, r = _c_pages(**change), _c_rows()
    assert lib.wm_pages_append(ctypes.addressof(p), r, r, 0, at, 1, None, None) == -1
    assert lib.wm_pages_attend(ctypes.addressof(p), at, 4, at, at, 1, r, r, 0, None, 1, 8, 1, 1.0, 1, 0, at,
                               1 << 30, None, None) == -1


@pytest.mark.parametrize("change", [dict(n_rows=1 << 31), dict(type=3), dict(type=-1), dict(slots=None), dict(k=dict(ptr=None)),
                                    dict(v=dict(row_stride=12)), dict(k=dict(head_stride=4)), dict(v=dict(ptr=4 + (1 << 20)))], ids=str)
def test_append_refuses_bad_arguments(change):
    at, p = 1 << 20, _c_pages()
    k, v = _c_rows(**change.get("k", {})), _c_rows(**change.get("v", {}))
    assert wm.lib().wm_pages_append(ctypes.addressof(p), k, v, change.get("type", 0), change.get("slots", at),
                                    change.get("n_rows", 1), None, None) == -1


def test_append_of_no_rows_launches_nothing():
    at, p, r = 1 << 20, _c_pages(), _c_rows()
    assert wm.lib().wm_pages_append(ctypes.addressof(p), r, r, 0, at, 0, None, None) == 0
    assert wm.last_launch_count() == 0


@pytest.mark.parametrize("change", [dict(table=None), dict(stride=0), dict(stride=1 << 26), dict(kv_len=None), dict(q_start=None), dict(n=0), dict(n=4001),
                                    dict(type=2), dict(rows=1 << 24), dict(q_heads=0), dict(q_heads=12), dict(q_heads=8 * 65), dict(max_q=0),
                                    dict(scale=float("nan")), dict(scale=float("inf")), dict(options=2), dict(options=0, window=5),
                                    dict(ws=None), dict(ws=8), dict(ws_bytes=16), dict(q=dict(row_stride=4)), dict(o=dict(ptr=2)),
                                    dict(o=dict(row_stride=0), rows=2), dict(o=dict(head_stride=64)),
                                    dict(q=dict(ptr=None))], ids=str)
def test_attend_refuses_bad_arguments(change):
    at, p = 1 << 20, _c_pages()
    q, o = _c_rows(**change.get("q", {})), _c_rows(**change.get("o", {}))
    g = lambda name, other: change.get(name, other)  # noqa: E731
    assert wm.lib().wm_pages_attend(ctypes.addressof(p), g("table", at), g("stride", 4), g("kv_len", at), g("q_start", at), g("n", 1),
                                    q, o, g("type", 0), None, g("rows", 1), g("q_heads", 8), g("max_q", 1),
                                    g("scale", 1.0), g("options", 1), g("window", 0), g("ws", at), g("ws_bytes", 1 << 30), None, None) == -1


def test_attend_of_no_rows_launches_nothing_and_other_head_sizes_have_no_workspace():
    at, p, r = 1 << 20, _c_pages(), _c_rows()
    assert wm.lib().wm_pages_attend(ctypes.addressof(p), at, 4, at, at, 1, r, r, 0, None, 0, 8, 1, 1.0, 1, 0,
                                    at, 1 << 30, None, None) == 0
    assert wm.last_launch_count() == 0
    assert wm.pages_workspace_bytes(96) == 0 and wm.pages_workspace_bytes(64) > 0
    with pytest.raises(wm.WmError):
        wm.new_pages_workspace(80)


@pytest.mark.parametrize("change", [dict(old=None), dict(free=None), dict(count=None), dict(start=None), dict(slots=None), dict(page=24), dict(n=0),
                                    dict(n=4001), dict(stride=0), dict(stride=1 << 31), dict(n_slots=1 << 31), dict(pool=0), dict(pool=1 << 27)], ids=str)
def test_plan_refuses_bad_arguments(change):
    at = 1 << 20
    g = lambda name, other: change.get(name, other)  # noqa: E731
    assert wm.lib().wm_pages_plan(g("old", at), at, g("n", 1), g("page", 64), g("pool", 10), at, g("stride", 4) & 0xFFFFFFFF, g("free", at),
                                  g("count", at), at, g("start", at), g("slots", at), g("n_slots", 5) & 0xFFFFFFFF, None, None) == -1


def test_the_binding_refuses_negative_windows_and_rows():
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    for what in (dict(window=-1), dict(max_q=-1)):
        with pytest.raises(wm.WmError, match="negative"):
            wm.wm_pages_attend(types.SimpleNamespace(head_dim=64), i[None], i[:1], i, q, torch.empty_like(q), q, **what)


def test_the_binding_refuses_host_tensors():
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(wm.WmError, match="CUDA"):
        wm.wm_pages_plan(i, i, 16, torch.zeros(4, 2, dtype=torch.int32), i, i[:1], i[:1], i, i)
    with pytest.raises(wm.WmError, match="CUDA"):
        wm.Pages(torch.zeros(1, 1, 16, 64, dtype=torch.uint8), torch.zeros(1, 1, 16, 64, dtype=torch.uint8), torch.zeros(1, 1), torch.zeros(1, 1))


# ---------------------------------------------------------------- plan

def _run_plan(old, new, page, table, free, count, n_slots, in_place=False):
    t, f, c = _dev(table), _dev(free), _dev([count])
    c_out = c if in_place else _dev([-7])
    start, slots = _dev([-9] * (len(old) + 1)), _dev([-9] * n_slots)
    report = wm.new_pages_report()
    wm.wm_pages_plan(_dev(old), _dev(new), page, t, f, c, c_out, start, slots, report=report)
    status, first = wm.read_pages_report(report)
    return status, first, t.tolist(), f.tolist(), int(c_out.item()), start.tolist(), slots.tolist()


def _plan_case(r, n, page, most, grow, done, n_free, pad):
    old = [r.randint(0, most) for _ in range(n)]
    new = [0 if r.random() < done else o if r.random() < 0.1 else o + r.randint(1, grow) if r.random() < 0.9 else r.randint(0, o) for o in old]
    width = max(1, max(ref.pages_of(max(o, w), page) for o, w in zip(old, new)) + r.randint(0, 2))
    held = sum(ref.pages_of(o, page) for o in old)
    order = list(range(held + n_free))
    r.shuffle(order)
    table = []
    for o in old:
        h = ref.pages_of(o, page)
        table.append([order.pop() for _ in range(h)] + [-5] * (width - h))
    return old, new, width, table, order + [-3] * held, len(order), sum(max(0, w - o) for o, w in zip(old, new)) + pad


@gpu
@pytest.mark.parametrize("n,page,most,grow,done,pad", [(1, 16, 0, 1, 0, 0), (1, 64, 200, 1, 0, 3), (3, 16, 40, 50, 0.3, 0), (64, 32, 500, 1, 0, 0),
                                                       (257, 64, 300, 40, 0.2, 17), (1024, 16, 60, 3, 0.1, 0), (1025, 128, 700, 1, 0.5, 5),
                                                       (4000, 16, 90, 20, 0.2, 1), (7, 128, 20000, 9000, 0.2, 100), (31, 16, 300, 30, 1.0, 4)])
@pytest.mark.parametrize("in_place", [False, True])
def test_plan(n, page, most, grow, done, pad, in_place):
    r = random.Random(n + page)
    old, new, width, table, free, count, n_slots = _plan_case(r, n, page, most, grow, done, 4 * n + 2 * grow // page * n + 8, pad)
    want = ref.plan(old, new, page, table, free, count, n_slots)
    got = _run_plan(old, new, page, table, free, count, n_slots, in_place)
    assert want[0] == 0 and got[:2] == ("OK", None)
    assert got[2:] == want[1:]


@gpu
@pytest.mark.parametrize("n", [5, 2000])
@pytest.mark.parametrize("spare", [-1, 0, 1])
def test_plan_takes_the_last_page_and_refuses_one_more(n, spare):
    """Pages given back in the call are taken in it, down to the last one."""
    page, r = 16, random.Random(n)
    old = [r.choice([0, 5, 16, 33]) for _ in range(n)]
    new = [0 if i % 3 == 0 else o + r.choice([1, 20, 48]) for i, o in enumerate(old)]
    held, want = [ref.pages_of(o, page) for o in old], [ref.pages_of(x, page) for x in new]
    give, take = sum(max(0, a - b) for a, b in zip(held, want)), sum(max(0, b - a) for a, b in zip(held, want))
    count = max(0, take - give + spare)
    order = list(range(sum(held) + count))
    r.shuffle(order)
    table = [[order.pop() for _ in range(h)] + [-5] * (6 - h) for h in held]
    free = order + [-3] * sum(held)
    n_slots = sum(max(0, b - a) for a, b in zip(old, new))
    expect = ref.plan(old, new, page, table, free, count, n_slots)
    got = _run_plan(old, new, page, table, free, count, n_slots)
    assert got[0] == ("ERR_CAPACITY" if take > count + give else "OK")
    assert got[2:] == expect[1:]


@gpu
@pytest.mark.parametrize("n", [4, 1500])
@pytest.mark.parametrize("what", ["negative", "negative new", "held beyond the row", "want beyond the row", "slots", "count", "double free"])
def test_plan_refuses_on_the_device_and_leaves_everything(n, what):
    r = random.Random(3)
    old, new, width, table, free, count, n_slots = _plan_case(r, n, 16, 60, 10, 0.0, 2 * n, 0)
    at, status = n // 2, -1
    if what == "negative":
        old[at] = -1
    elif what == "negative new":
        new[at] = -2 ** 31
    elif what == "held beyond the row":
        old[at] = width * 16 + 1
    elif what == "want beyond the row":
        new[at], status = 2 ** 31 - 1, -2
    elif what == "slots":
        n_slots, status = n_slots - 1, -2
    elif what == "count":
        count = len(free) + 1
    else:
        new, count = [0] * n, len(free) - 1
    want = ref.plan(old, new, 16, table, free, count, n_slots)
    got = _run_plan(old, new, 16, table, free, count, n_slots)
    assert got[0] == wm.STATUS[status] and want[0] == status
    if "new" in what or "held" in what or "want" in what or what == "negative":
        assert got[1] == at
    assert got[2:] == want[1:]


@gpu
@pytest.mark.parametrize("n", [3, 1200])
def test_plan_leaves_out_the_slots_of_pages_that_are_not_in_the_pool(n):
    old, new = [10] * n, [30] * n
    table = [[2 * i, -5] for i in range(n)]
    free = list(range(1, 2 * n, 2)) + [-3] * n
    table[1][0], free[0] = 2 * n, -1                     # request 1's page so far; the page the last request takes
    got = _run_plan(old, new, 16, table, free, n, 20 * n)
    want = ref.plan(old, new, 16, table, free, n, 20 * n)[5]
    bad = set(range(20, 26)) | set(range(20 * n - 14, 20 * n))
    assert got[0] == "ERR_ARG" and got[1] == 1
    assert got[6] == [-1 if t in bad else s for t, s in enumerate(want)]


# ---------------------------------------------------------------- append

DTYPES = [torch.bfloat16, torch.float16, torch.float32]


def _pool(n, heads, page, dim, g, order="hnd", spread=3):
    """(Pages on the GPU, the four arrays on the CPU): heads before tokens in a page, or tokens before heads, or keys and
    values side by side in one buffer."""
    k, v, ks, vs = ref.random_pool(n, heads, page, dim, g, spread)
    if order == "hnd":
        dk, dv = k.cuda(), v.cuda()
    elif order == "nhd":
        dk, dv = (t.transpose(1, 2).contiguous().cuda().transpose(1, 2) for t in (k, v))
    else:
        both = torch.cat([k, v, torch.full_like(k, 0x7F)[..., :16]], 3).cuda()
        dk, dv = both[..., :dim], both[..., dim:2 * dim]
    return wm.Pages(dk, dv, ks.cuda(), vs.cuda()), (k, v, ks, vs)


def _check_pool(pages, want):
    for got, w, name in ((pages.k, want[0], "k"), (pages.v, want[1], "v")):
        assert torch.equal(ref.values(got).nan_to_num(nan=1e9), w.nan_to_num(nan=1e9)), name
    for got, w, name in ((pages.k_scale, want[2], "k_scale"), (pages.v_scale, want[3], "v_scale")):
        assert torch.equal(got.cpu().double(), w), name


def _append_case(lens_before, lens_after, page, g):
    """Slots of the tokens, the pages in a random order, and the pool's size."""
    n = sum(ref.pages_of(x, page) for x in lens_after) + 2
    table = ref.random_table(lens_after, page, max(1, max(ref.pages_of(x, page) for x in lens_after)), n, g)
    return n, [table[i][p // page] * page + p % page for i, (a, b) in enumerate(zip(lens_before, lens_after)) for p in range(a, b)]


def _run_append(pages, arrays, x, y, slots, page, **kw):
    want = [ref.values(arrays[0]), ref.values(arrays[1]), arrays[2].double(), arrays[3].double()]
    ref.append(want[0], want[2], x.cpu(), slots, page)
    ref.append(want[1], want[3], y.cpu(), slots, page)
    wm.wm_pages_append(pages, x, y, _dev(slots), **kw)
    _check_pool(pages, want)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("heads,dim,page,order", [(8, 128, 64, "hnd"), (1, 64, 16, "nhd"), (3, 64, 32, "both"), (16, 128, 16, "nhd"), (5, 128, 128, "both"),
                                                  (33, 64, 16, "hnd")])
def test_append(dtype, heads, dim, page, order):
    g = torch.Generator().manual_seed(heads + dim)
    before = [0, 1, page - 1, page, page + 1, 3 * page - 2, 7, 0]
    after = [1, 2, page, page + 1, 3 * page + 5, 3 * page, 7, 2 * page]
    n, slots = _append_case(before, after, page, g)
    pages, arrays = _pool(n, heads, page, dim, g, order)
    rows = len(slots) + 3
    x, y = ((torch.randn((rows, heads, dim), generator=g) * 2.0 ** torch.randint(-6, 7, (rows, heads, 1), generator=g)).to(dtype).cuda() for _ in range(2))
    _run_append(pages, arrays, x, y, slots + [-1] * 3, page)


@gpu
def test_append_reads_strided_rows_and_skips_holes():
    g = torch.Generator().manual_seed(5)
    n, slots = _append_case([3, 0, 20], [9, 40, 37], 16, g)
    pages, arrays = _pool(n, 2, 16, 64, g)
    big = torch.randn((len(slots), 7, 64), generator=g).to(torch.bfloat16).cuda()      # queries, keys and values of one product
    keys = torch.randn((2, len(slots), 64), generator=g).to(torch.bfloat16).cuda().transpose(0, 1)
    for at in (0, 5, len(slots) - 1):                    # holes at the ends of runs
        if slots[at] % 16 == 15 or at == len(slots) - 1:
            slots[at] = -1
    _run_append(pages, arrays, keys, big[:, 5:7], slots, 16)


@gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_append_of_extreme_values(dtype):
    """Zeros, the type's largest and smallest values, infinities and NaN; the scale's edge at 448 times a power of two; ties."""
    g = torch.Generator().manual_seed(1)
    info = torch.finfo(dtype)
    rows = [torch.zeros(64), torch.full((64,), info.max), torch.full((64,), info.smallest_normal), torch.full((64,), info.tiny * info.eps),
            torch.tensor([float("inf"), -float("inf"), 3.0, -2.0] * 16), torch.full((64,), float("nan")), torch.tensor([float("nan"), 1.0] * 32),
            torch.full((64,), float("-inf")), torch.tensor([448.0, 1.0] * 32), torch.tensor([450.0, 1.0] * 32), torch.tensor([-7.0, 7.0, 7.03125, 0.0] * 16),
            torch.arange(64) / 64.0 * 17.0, torch.arange(64) * 2.0 ** -9 * 1.5]
    x = torch.stack(rows).to(dtype)[:, None].repeat(1, 2, 1).cuda()
    y = -x.flip(0)
    page = 16
    for before in (0, 3):
        slots = [p * page + before for p in range(len(rows))]
        pages, arrays = _pool(len(rows), 2, page, 64, g)
        arrays[2][3], arrays[2][5] = 0.0, 3.0            # an old scale of zero, and one that is no power of two
        pages.k_scale.copy_(arrays[2])
        _run_append(pages, arrays, x, y, slots, page)


@gpu
def test_append_twice_over_the_same_page_grows_its_scale_once_and_again():
    g = torch.Generator().manual_seed(2)
    pages, arrays = _pool(3, 4, 32, 128, g)
    arrays = list(arrays)
    for step, size in enumerate((0.01, 1.0, 100.0, 0.5)):
        x, y = (torch.randn((2, 4, 128), generator=g).mul(size).to(torch.bfloat16).cuda() for _ in range(2))
        _run_append(pages, arrays, x, y, [32 + 2 * step, 32 + 2 * step + 1], 32)
        arrays = [pages.k.cpu(), pages.v.cpu(), pages.k_scale.cpu(), pages.v_scale.cpu()]


@gpu
def test_append_reports_rows_it_leaves_out():
    g = torch.Generator().manual_seed(3)
    pages, arrays = _pool(4, 2, 16, 64, g)
    x, y = (torch.randn((7, 2, 64), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    report = wm.new_pages_report()
    good = [0, 1, -1, -1, -1, -1, 50]
    want = [ref.values(arrays[0]), ref.values(arrays[1]), arrays[2].double(), arrays[3].double()]
    ref.append(want[0], want[2], x.cpu(), good, 16)
    ref.append(want[1], want[3], y.cpu(), good, 16)
    wm.wm_pages_append(pages, x, y, _dev([0, 1, 5, -2, 64, 2 ** 31 - 1, 50]), report=report)
    assert wm.read_pages_report(report) == ("ERR_ARG", 2)
    _check_pool(pages, want)


# ---------------------------------------------------------------- attend

def _attend(pages, arrays, table, kv_len, rows, heads, dtype, g, causal=True, window=0, scale=None, pad=0, max_q=None, q=None, strided=False,
            check=True, spread_q=False):
    dim = pages.head_dim
    start = [0]
    for r in rows:
        start.append(start[-1] + r)
    n = start[-1] + pad
    if q is None:
        q = torch.randn((n, heads, dim), generator=g)
        if spread_q:
            q = q * 2.0 ** torch.randint(-12, 3, (n, heads, dim), generator=g)
    q = q.to(dtype)
    if strided:
        dq = torch.cat([q, q[:, :1]], 1).cuda()[:, :heads]
        out = torch.full((heads, n, dim), 7.0, dtype=dtype, device="cuda").transpose(0, 1)
    else:
        dq, out = q.cuda(), torch.full((n, heads, dim), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((n, heads), 7.0, device="cuda")
    ws = wm.new_pages_workspace(dim)
    ws.fill_(0xFF)
    report = wm.new_pages_report()
    wm.wm_pages_attend(pages, _dev(table), _dev(kv_len), _dev(start), dq, out, ws, lse=lse, scale=scale, causal=causal, window=window,
                       max_q=max_q if max_q is not None else max(1, max(rows)), report=report)
    torch.cuda.synchronize()
    if not check:
        return out.cpu(), lse.cpu(), wm.read_pages_report(report)
    assert wm.read_pages_report(report) == ("OK", None)
    want = ref.attend(ref.values(arrays[0]), ref.values(arrays[1]), arrays[2].double(), arrays[3].double(), table, kv_len, start,
                      q[:start[-1]].double(), dim ** -0.5 if scale is None else scale, causal, window)
    far, far_lse = ref.bounds(*want, dtype, dim)
    got, got_lse = out.cpu().double(), lse.cpu().double()
    assert (got[start[-1]:] == 7).all() and (got_lse[start[-1]:] == 7).all()
    got, got_lse = got[:start[-1]], got_lse[:start[-1]]
    assert torch.equal(torch.isinf(got_lse), torch.isinf(want[1]))
    bad = ~((got - want[0]).abs() <= far)
    assert not bad.any(), (bad.sum(), bad.nonzero()[:3], ((got - want[0]).abs() / far).max())
    fine = ~torch.isinf(want[1])
    assert ((got_lse - want[1]).abs()[fine] <= far_lse[fine]).all(), ((got_lse - want[1]).abs() / far_lse)[fine].max()
    return out.cpu(), lse.cpu()


def _attend_case(kv_len, page, heads, dim, g, order="hnd", spread=3):
    n = sum(ref.pages_of(x, page) for x in kv_len) + 3
    table = ref.random_table(kv_len, page, max(1, max(ref.pages_of(x, page) for x in kv_len)), n, g)
    return (*_pool(n, heads, page, dim, g, order, spread), table)


LENS = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500]


@gpu
@pytest.mark.parametrize("dtype", DTYPES[:2])
@pytest.mark.parametrize("kv_heads,group,dim,page,order", [(2, 4, 128, 64, "hnd"), (1, 1, 64, 16, "nhd"), (3, 8, 64, 32, "both"), (2, 3, 128, 16, "nhd"),
                                                           (2, 16, 128, 128, "both"), (1, 7, 64, 128, "hnd"), (1, 33, 128, 32, "hnd"), (1, 64, 64, 64, "hnd")])
def test_attend_single_tokens(dtype, kv_heads, group, dim, page, order):
    g = torch.Generator().manual_seed(group + dim)
    pages, arrays, table = _attend_case(LENS, page, kv_heads, dim, g, order)
    _attend(pages, arrays, table, LENS, [1] * len(LENS), kv_heads * group, dtype, g, pad=2)


@gpu
@pytest.mark.parametrize("dtype", DTYPES[:2])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 100), (True, 128), (True, 1000), (False, 0)])
@pytest.mark.parametrize("kv_heads,group,dim,page", [(2, 4, 128, 64), (1, 1, 64, 16), (2, 2, 64, 32), (1, 5, 128, 16)])
def test_attend_drafts(dtype, causal, window, kv_heads, group, dim, page):
    """A few rows a request, among them more rows than tokens (rows that see nothing) and requests without rows or tokens."""
    g = torch.Generator().manual_seed(group + dim + window)
    lens, rows = [5, 0, 0, 3, 128, 129, 130, 300, 131, 64], [2, 0, 3, 7, 8, 1, 5, 6, 4, 3]
    pages, arrays, table = _attend_case(lens, page, kv_heads, dim, g)
    _attend(pages, arrays, table, lens, rows, kv_heads * group, dtype, g, causal, window, pad=1)


@gpu
@pytest.mark.parametrize("dtype", DTYPES[:2])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 37), (True, 200), (False, 0)])
@pytest.mark.parametrize("kv_heads,group,dim,page,order", [(2, 1, 128, 64, "hnd"), (1, 4, 64, 16, "nhd"), (1, 3, 128, 32, "both"), (1, 8, 64, 128, "hnd")])
def test_attend_prompts(dtype, causal, window, kv_heads, group, dim, page, order):
    g = torch.Generator().manual_seed(group + dim + window)
    lens, rows = [300, 129, 128, 511, 40, 260, 1], [300, 100, 128, 77, 60, 129, 1]
    pages, arrays, table = _attend_case(lens, page, kv_heads, dim, g, order)
    _attend(pages, arrays, table, lens, rows, kv_heads * group, dtype, g, causal, window, pad=3)


@gpu
@pytest.mark.parametrize("max_q", [1, 3, 40, 1000])
def test_attend_answers_requests_with_other_numbers_of_rows_than_it_was_told(max_q):
    g = torch.Generator().manual_seed(9)
    lens, rows = [300, 20, 150, 400], [200, 1, 17, 3]
    pages, arrays, table = _attend_case(lens, 32, 2, 128, g)
    _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g, max_q=max_q)


@gpu
@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 1, 2], [150, 130, 260]])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_over_scales_of_very_different_sizes(rows, dim):
    g = torch.Generator().manual_seed(12)
    lens = [300, 131, 260]
    pages, arrays, table = _attend_case(lens, 16, 2, dim, g, spread=0)
    for i in (2, 3):                                     # scales from 2^-40 to 2^3 and zeros (values) in one request
        arrays[i].copy_(2.0 ** torch.randint(-40, 4, arrays[i].shape, generator=g) * (torch.rand(arrays[i].shape, generator=g) + 1.0))
    arrays[3][torch.rand(arrays[3].shape, generator=g) < 0.2] = 0.0
    arrays[2].clamp_(max=0.05)
    pages.k_scale.copy_(arrays[2])
    pages.v_scale.copy_(arrays[3])
    _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g)


@gpu
@pytest.mark.parametrize("rows", [[1, 1], [4, 2], [200, 140]])
@pytest.mark.parametrize("dtype", DTYPES[:2])
def test_attend_with_scores_far_apart_and_queries_of_many_sizes(rows, dtype):
    g = torch.Generator().manual_seed(13)
    lens = [333, 140]
    pages, arrays, table = _attend_case(lens, 64, 2, 128, g, spread=0)
    for scale in (0.0, 1e-6, -0.3, 3.0):
        _attend(pages, arrays, table, lens, rows, 6, dtype, g, scale=scale, spread_q=True)
    _attend(pages, arrays, table, lens, rows, 6, dtype, g, strided=True)


def _poisoned(pages, arrays, table, lens, page):
    """NaN codes behind every request's last token and in all pages that no table names, on both sides."""
    used = set()
    for i, n in enumerate(lens):
        for j, p in enumerate(table[i][:ref.pages_of(n, page)]):
            used.add(p)
            for t in range(page):
                if j * page + t >= n:
                    for k in (arrays[0], arrays[1], pages.k, pages.v):
                        k[p, :, t] = 0x7F
    for p in range(arrays[0].shape[0]):
        if p not in used:
            for k in (arrays[0], arrays[1], pages.k, pages.v):
                k[p] = 0xFF
            pages.k_scale[p] = pages.v_scale[p] = float("nan")


@gpu
@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 1, 2], [150, 130, 260]])
@pytest.mark.parametrize("page,dim", [(16, 128), (64, 64), (128, 128)])
@pytest.mark.parametrize("window", [0, 40])
def test_attend_is_not_touched_by_what_no_row_sees(rows, page, dim, window):
    g = torch.Generator().manual_seed(14)
    lens = [300, 131, 260]
    pages, arrays, table = _attend_case(lens, page, 2, dim, g)
    _poisoned(pages, arrays, table, lens, page)
    _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g, window=window)


@gpu
@pytest.mark.parametrize("rows", [[4, 6], [150, 131]])
@pytest.mark.parametrize("dim,window", [(64, 0), (128, 0), (128, 50)])
def test_attend_rows_are_not_touched_by_codes_that_only_other_rows_see(rows, dim, window):
    """NaN in one value channel and in one key of a token near the end: rows before it are as without it, rows that see it get NaN."""
    g = torch.Generator().manual_seed(15)
    lens = [300, 131]
    pages, arrays, table = _attend_case(lens, 32, 1, dim, g)
    q = torch.randn((sum(rows), 2, dim), generator=g)
    clean, clean_lse = _attend(pages, arrays, table, lens, rows, 2, torch.bfloat16, g, window=window, q=q)
    for i, (n, r) in enumerate(zip(lens, rows)):
        t = n - 2                                        # the last but one token: seen by the last two rows alone
        pages.v[table[i][t // 32], 0, t % 32, 5] = 0x7F
    out, lse, report = _attend(pages, arrays, table, lens, rows, 2, torch.bfloat16, g, window=window, q=q, check=False)
    assert report == ("OK", None)
    start = 0
    for r in rows:
        hit = range(start + r - 2, start + r)
        assert torch.equal(out[start:start + r - 2], clean[start:start + r - 2])
        assert out[list(hit), :, 5].isnan().all()
        rest = [c for c in range(dim) if c != 5]
        assert torch.equal(out[list(hit)][:, :, rest], clean[list(hit)][:, :, rest])
        start += r
    assert torch.equal(lse, clean_lse)
    for i, n in enumerate(lens):
        t = n - 2
        pages.k[table[i][t // 32], 0, t % 32, 9] = 0xFF
    out, lse, _ = _attend(pages, arrays, table, lens, rows, 2, torch.bfloat16, g, window=window, q=q, check=False)
    start = 0
    for r in rows:
        assert torch.equal(out[start:start + r - 2], clean[start:start + r - 2]) and torch.equal(lse[start:start + r - 2], clean_lse[start:start + r - 2])
        assert out[start + r - 2:start + r].isnan().all() and lse[start + r - 2:start + r].isnan().all()
        start += r


@gpu
@pytest.mark.parametrize("rows", [[1, 1, 1], [2, 5, 3], [200, 140, 130]])
def test_attend_gives_nan_in_the_rows_of_a_query_that_is_not_finite_and_in_no_other(rows):
    g = torch.Generator().manual_seed(16)
    lens = [300, 140, 131]
    pages, arrays, table = _attend_case(lens, 64, 2, 128, g)
    q = torch.randn((sum(rows), 4, 128), generator=g)
    clean, clean_lse = _attend(pages, arrays, table, lens, rows, 4, torch.float16, g, q=q)
    r = rows[0]
    q[r, 1, 7], q[r, 3, 100] = float("nan"), float("inf")
    out, lse, _ = _attend(pages, arrays, table, lens, rows, 4, torch.float16, g, q=q, check=False)
    for h in (1, 3):
        assert out[r, h].isnan().all() and not lse[r, h].isfinite()
        out[r, h], lse[r, h] = clean[r, h], clean_lse[r, h]
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)


@gpu
@pytest.mark.parametrize("rows", [[1, 1, 1, 1], [2, 5, 3, 1], [140, 131, 150, 2]])
@pytest.mark.parametrize("what", ["page", "negative page", "length", "long", "start", "rows"])
def test_attend_reports_requests_it_cannot_answer_and_answers_the_others(rows, what):
    g = torch.Generator().manual_seed(17)
    lens = [300, 260, 150, 140]
    pages, arrays, table = _attend_case(lens, 32, 2, 64, g)
    q = torch.randn((sum(rows), 4, 64), generator=g).to(torch.bfloat16).cuda()
    start = [0]
    for r in rows:
        start.append(start[-1] + r)

    def run(table, kv, start, n_rows=None):
        n = q.shape[0] if n_rows is None else n_rows
        out, lse, report = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda"), wm.new_pages_report()
        wm.wm_pages_attend(pages, _dev(table), _dev(kv), _dev(start), q[:n], out[:n], wm.new_pages_workspace(64), lse=lse[:n], max_q=max(rows), report=report)
        return out.cpu(), lse.cpu(), wm.read_pages_report(report)

    clean, clean_lse, report = run(table, lens, start)
    assert report == ("OK", None)
    kv, table, starts = list(lens), [list(r) for r in table], list(start)
    nan = untouched = range(0)
    n_rows, who = None, 1
    if what == "page":
        table[1][1], nan = pages.n_pages, range(start[1], start[2])
    elif what == "negative page":
        table[1][0], nan = -1, range(start[1], start[2])
    elif what == "length":
        kv[1], untouched = -1, range(start[1], start[2])
    elif what == "long":
        kv[1], untouched = 32 * len(table[1]) + 1, range(start[1], start[2])
    elif what == "start":
        starts, kv, table, who = [0, start[2], start[1]] + start[3:], kv, table, 1
        # request 0 now has the rows of 0 and 1, request 1 none (decreasing), request 2 its own from start[1] on: only the last is as before
        out, lse, report = run(table, kv, starts)
        assert report == ("ERR_ARG", 1)
        assert torch.equal(out[start[3]:], clean[start[3]:])
        return
    else:
        n_rows, who, untouched = start[3] - 1, 2, range(start[2], start[4])
        out, lse, report = run(table, kv, starts, n_rows)
        assert report == ("ERR_ARG", 2)
        assert torch.equal(out[:start[2]], clean[:start[2]]) and (out[start[2]:] == 7).all()
        return
    out, lse, report = run(table, kv, starts, n_rows)
    assert report == ("ERR_ARG", who)
    for r in range(q.shape[0]):
        if r in nan:
            assert out[r].isnan().all() and lse[r].isnan().all()
        elif r in untouched:
            assert (out[r] == 7).all() and (lse[r] == 7).all()
        else:
            assert torch.equal(out[r], clean[r]) and torch.equal(lse[r], clean_lse[r])


@gpu
def test_attend_without_lse_and_report_gives_the_same():
    g = torch.Generator().manual_seed(18)
    lens = [70, 300]
    pages, arrays, table = _attend_case(lens, 16, 2, 64, g)
    q = torch.randn((5, 4, 64), generator=g).to(torch.float16)
    want, _ = _attend(pages, arrays, table, lens, [2, 3], 4, torch.float16, g, q=q)
    out = torch.zeros(5, 4, 64, dtype=torch.float16, device="cuda")
    wm.wm_pages_attend(pages, _dev(table), _dev(lens), _dev([0, 2, 5]), q.cuda(), out, wm.new_pages_workspace(64), max_q=3)
    assert torch.equal(out.cpu(), want)


@gpu
@pytest.mark.parametrize("rows", [[1, 1, 1], [2, 5, 3], [200, 140, 130]])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_whose_waits_run_out_reports_it_gives_nan_and_the_next_call_is_right(rows, dim):
    g = torch.Generator().manual_seed(19)
    lens = [300, 140, 131]
    pages, arrays, table = _attend_case(lens, 64, 2, dim, g)
    q = torch.randn((sum(rows), 4, dim), generator=g)
    wm.wait_budget_ms(20)
    wm.inject_stall(1)
    try:
        out, lse, report = _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g, q=q, check=False)
    finally:
        wm.inject_stall(0)
        wm.wait_budget_ms(2000)
    assert report[0] == "ERR_TIMEOUT"
    assert out.isnan().all() and lse.isnan().all()
    _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g, q=q)


@gpu
@pytest.mark.parametrize("rows", [[1, 1, 1], [2, 5, 3], [8, 7, 4], [200, 140, 130]])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_whose_waits_run_out_where_the_tiles_memory_holds_nan_codes(rows, dim):
    """Tiles that never came are looked through for NaN all the same, by threads that are no longer in step: what was in
    their memory before must not send them different ways."""
    g = torch.Generator().manual_seed(20)
    lens = [300, 140, 131]
    pages, arrays, table = _attend_case(lens, 64, 2, dim, g)
    q = torch.randn((sum(rows), 4, dim), generator=g)
    want = _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g, q=q)
    kept = pages.v.clone()
    for _ in range(5):
        pages.v.view(torch.uint8).fill_(0x7F)
        out = _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g, q=q, check=False)[0]
        assert out.isnan().all()
        wm.wait_budget_ms(20)
        wm.inject_stall(1)
        try:
            out, lse, report = _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g, q=q, check=False)
        finally:
            wm.inject_stall(0)
            wm.wait_budget_ms(2000)
        assert report[0] == "ERR_TIMEOUT" and out.isnan().all() and lse.isnan().all()
    pages.v.copy_(kept)
    got = _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g, q=q)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@gpu
@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 1, 2], [150, 130, 260]])
def test_attend_over_keys_whose_scale_is_zero(rows):
    g = torch.Generator().manual_seed(24)
    lens = [300, 131, 260]
    pages, arrays, table = _attend_case(lens, 16, 2, 64, g)
    arrays[2][torch.rand(arrays[2].shape, generator=g) < 0.5] = 0.0
    pages.k_scale.copy_(arrays[2])
    _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g)


@gpu
@pytest.mark.parametrize("rows", [[1, 1, 1], [3, 1, 2], [150, 130, 260]])
def test_attend_over_values_that_are_all_zero(rows):
    """As wm_pages_append stores zeros: codes of zero under the smallest scale, beside pages of ordinary ones."""
    g = torch.Generator().manual_seed(25)
    lens = [300, 131, 260]
    pages, arrays, table = _attend_case(lens, 16, 2, 64, g)
    for i in range(3):
        for p in table[i][:ref.pages_of(lens[i], 16)][::3]:
            arrays[1][p], arrays[3][p] = 0, 2.0 ** -126
    pages.v.copy_(arrays[1]), pages.v_scale.copy_(arrays[3])
    _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g)
    arrays[1].zero_(), arrays[3].fill_(2.0 ** -126)
    pages.v.copy_(arrays[1]), pages.v_scale.copy_(arrays[3])
    _attend(pages, arrays, table, lens, rows, 4, torch.bfloat16, g)


@gpu
@pytest.mark.parametrize("seed", range(24))
def test_attend_of_mixed_batches(seed):
    """Single tokens, drafts and prompts in one batch, any shape; told too few rows, the right number or none."""
    r, g = random.Random(seed), torch.Generator().manual_seed(seed)
    page, dim, kv_heads, group = r.choice([16, 32, 64, 128]), r.choice([64, 128]), r.choice([1, 2, 3]), r.choice([1, 2, 3, 5, 8, 16])
    n = r.randint(1, 9)
    lens = [r.choice([0, 1, 5, r.randint(1, 140), r.randint(100, 700)]) for _ in range(n)]
    rows = [r.choice([0, 1, 1, 3, r.randint(0, 40), r.randint(0, 300)]) for _ in range(n)]
    if not sum(rows):
        rows[0] = 1
    causal = r.random() < 0.7
    window = r.choice([0, 0, 1, 17, 128, 333]) if causal else 0
    pages, arrays, table = _attend_case(lens, page, kv_heads, dim, g, r.choice(["hnd", "nhd", "both"]))
    _attend(pages, arrays, table, lens, rows, kv_heads * group, r.choice(DTYPES[:2]), g, causal, window, pad=r.choice([0, 4]),
            max_q=r.choice([1, max(1, max(rows)), 5000]), strided=r.random() < 0.5)


@gpu
def test_calls_refuse_tensors_of_another_device(monkeypatch):
    pages = wm.new_pages(4, 16, 1, 64)
    i, table, x = _dev([1]), _dev([[0, 1]]), torch.zeros(1, 1, 64, device="cuda", dtype=torch.bfloat16)
    ws = wm.new_pages_workspace(64)
    monkeypatch.setattr(wm, "_device", lambda: 1)
    with pytest.raises(wm.WmError, match="current device is 1"):
        wm.wm_pages_plan(i, i, 16, table, _dev([2, 3]), i, i, _dev([0, 0]), _dev([0]))
    with pytest.raises(wm.WmError, match="current device is 1"):
        wm.wm_pages_append(pages, x, x, i)
    with pytest.raises(wm.WmError, match="current device is 1"):
        wm.wm_pages_attend(pages, table, i, _dev([0, 1]), x, x.clone(), ws)


@gpu
@pytest.mark.parametrize("window", [1, 2 ** 30 - 1, 2 ** 30, 2 ** 31 - 1, 2 ** 32 - 1])
@pytest.mark.parametrize("lens,rows", [([5, 300, 0], [9, 2, 3]), ([100, 300, 0], [200, 150, 40])])
def test_attend_with_windows_of_any_size_and_more_rows_than_tokens(window, lens, rows):
    g = torch.Generator().manual_seed(27)
    pages, arrays, table = _attend_case(lens, 32, 1, 64, g)
    _attend(pages, arrays, table, lens, rows, 2, torch.bfloat16, g, window=window)


@gpu
def test_calls_on_no_rows():
    pages, none = wm.new_pages(4, 16, 2, 64), torch.zeros(0, 2, 64, device="cuda", dtype=torch.bfloat16)
    wm.wm_pages_append(pages, none, none, _dev([]))
    wm.wm_pages_attend(pages, _dev([[0, 1]]), _dev([3]), _dev([0, 0]), none, none.clone(), wm.new_pages_workspace(64), max_q=1)
    count, start = _dev([4]), _dev([9, 9])
    wm.wm_pages_plan(_dev([3]), _dev([3]), 16, _dev([[0, 1]]), _dev([0, 1, 2, 3]), count, count, start, _dev([]))
    torch.cuda.synchronize()
    assert count.item() == 4 and start.tolist() == [0, 0] and not pages.k.any()


@gpu
def test_attention_beside_the_movers_calls_on_another_stream():
    """The encoder takes a whole SM's shared and tensor memory, so blocks of the two take turns; neither waits for the other."""
    g = torch.Generator().manual_seed(28)
    lens = [900, 3000, 1500]
    pages, arrays, table = _attend_case(lens, 64, 4, 128, g)
    tab, kv = _dev(table), _dev(lens)
    n, chunk = 4 << 20, 65536
    cache = torch.randn(n // 2, generator=g).to(torch.bfloat16).cuda()
    mover = [torch.cuda.Stream() for _ in range(2)]
    scratch, res, crc = wm.new_workspace(n, chunk), wm.new_result(), torch.zeros(n // chunk, dtype=torch.int32, device="cuda")
    wires = [torch.zeros(wm.wire_bound(n, chunk), dtype=torch.uint8, device="cuda") for _ in range(2)]
    wm.wm_encode(cache, chunk, None, crc, wires[0], scratch, res)
    length = wm.read_result(res).wire_len
    for rows in ([1, 1, 1], [300, 400, 100]):
        starts = [0, rows[0], rows[0] + rows[1], sum(rows)]
        q = torch.randn((sum(rows), 16, 128), generator=g).to(torch.bfloat16).cuda()
        want, out, ws = torch.zeros_like(q), torch.zeros_like(q), wm.new_pages_workspace(128)
        start = _dev(starts)
        wm.wm_pages_attend(pages, tab, kv, start, q, want, ws, max_q=max(rows))
        torch.cuda.synchronize()
        for _ in range(20):
            wm.wm_pages_attend(pages, tab, kv, start, q, out, ws, max_q=max(rows), stream=mover[0])
            wm.wm_encode(cache, chunk, None, crc, wires[1], scratch, res, stream=mover[1])
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert wm.read_result(res).ok and torch.equal(wires[0][:length], wires[1][:length])


@gpu
def test_many_slots_at_an_address_that_is_not_aligned():
    n, page = 40, 16
    r = random.Random(4)
    old, new, width, table, free, count, n_slots = _plan_case(r, n, page, 300, 400, 0.1, 40 * n, 7)
    assert n_slots > 4096
    want = ref.plan(old, new, page, table, free, count, n_slots)
    t, f, c = _dev(table), _dev(free), _dev([count])
    start, slots = _dev([-9] * (n + 1)), _dev([-9] * (n_slots + 2))
    wm.wm_pages_plan(_dev(old), _dev(new), page, t, f, c, c, start, slots[1:-1])
    assert (t.tolist(), f.tolist(), int(c.item()), start.tolist()) == want[1:5]
    assert slots.tolist() == [-9] + want[5] + [-9]


# ---------------------------------------------------------------- together

class Session:
    """Requests that grow in a pool, and a plain copy of their keys and values."""

    def __init__(self, n, page=16, heads=2, dim=64, pool=200, width=24):
        self.n, self.page, self.heads, self.dim = n, page, heads, dim
        self.pages = wm.new_pages(pool, page, heads, dim)
        self.table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        self.free = torch.arange(pool, dtype=torch.int32, device="cuda")
        self.count = _dev([pool])
        self.lens = _dev([0] * n)
        self.ws, self.report = wm.new_pages_workspace(dim), wm.new_pages_report()

    def step(self, new, k, v, q, start, slots, out, lse=None, max_q=64, stream=None):
        wm.wm_pages_plan(self.lens, new, self.page, self.table, self.free, self.count, self.count, start, slots, report=self.report, stream=stream)
        wm.wm_pages_append(self.pages, k, v, slots, report=self.report, stream=stream)
        wm.wm_pages_attend(self.pages, self.table, new, start, q, out, self.ws, lse=lse, max_q=max_q, report=self.report, stream=stream)


def _check_step(s, lens, start, q, out, lse, dtype):
    want = ref.attend(ref.values(s.pages.k), ref.values(s.pages.v), s.pages.k_scale.cpu().double(), s.pages.v_scale.cpu().double(),
                      s.table.tolist(), lens, start, q[:start[-1]].cpu().double(), s.dim ** -0.5, True, 0)
    far, far_lse = ref.bounds(*want, dtype, s.dim)
    assert ((out[:start[-1]].cpu().double() - want[0]).abs() <= far).all()
    assert ((lse[:start[-1]].cpu().double() - want[1]).abs() <= far_lse).all()


@gpu
def test_requests_arrive_grow_end_and_move():
    """Prompts, tokens, an end, a new request in its place; then one session's pages move as leaves into another pool and go on there."""
    g = torch.Generator().manual_seed(20)
    s = Session(3)
    lens = [0, 0, 0]
    rows = 200
    start, slots = _dev([0] * 4), _dev([0] * rows)
    for new in ([40, 17, 0], [41, 18, 130], [42, 0, 131], [43, 90, 132], [44, 91, 133]):
        q = torch.randn((rows, 6, 64), generator=g).to(torch.bfloat16).cuda()
        k, v = (torch.randn((rows, 2, 64), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
        out, lse = torch.zeros_like(q), torch.zeros((rows, 6), device="cuda")
        s.step(_dev(new), k, v, q, start, slots, out, lse)
        s.lens.copy_(_dev(new))
        more = [max(0, b - a) for a, b in zip(lens, new)]
        lens = new
        assert wm.read_pages_report(s.report) == ("OK", None)
        assert start.tolist() == [0, more[0], more[0] + more[1], sum(more)]
        _check_step(s, lens, start.tolist(), q, out, lse, torch.bfloat16)
    assert int(s.count.item()) == 200 - sum(ref.pages_of(x, 16) for x in lens)
    # request 2 moves: its pages and scales are leaves, the other side has them elsewhere
    ids = s.table[2, :ref.pages_of(lens[2], 16)].long()
    other = Session(3)
    to = torch.randperm(200, generator=g)[:ids.numel()].cuda()
    scales = [s.pages.k_scale[ids], s.pages.v_scale[ids]]
    there = [torch.zeros_like(t) for t in scales]
    leaves = [p[i] for i in ids.tolist() for p in (s.pages.k, s.pages.v)] + scales
    landing = [p[i] for i in to.tolist() for p in (other.pages.k, other.pages.v)] + there
    nbytes = sum(t.numel() * t.element_size() for t in leaves)
    chunk = 16384
    ws, res = wm.new_workspace(nbytes, chunk), wm.new_result()
    crc, crc_there = (torch.zeros(wm.num_chunks(nbytes, chunk), dtype=torch.int32, device="cuda") for _ in range(2))
    wire = torch.zeros(wm.wire_bound(nbytes, chunk), dtype=torch.uint8, device="cuda")
    wm.wm_encode_leaves(wm.make_leaf_table(leaves), nbytes, chunk, None, crc, wire, ws, res)
    r = wm.read_result(res)
    assert r.ok
    wm.wm_decode_verify_leaves(wire, r.wire_len, wm.make_leaf_table(landing), nbytes, chunk, crc_there, ws, res)
    assert wm.read_result(res).ok
    other.pages.k_scale[to], other.pages.v_scale[to] = there
    other.table[0, :to.numel()] = to.to(torch.int32)
    q = torch.randn((1, 6, 64), generator=g).to(torch.bfloat16).cuda()
    outs = []
    for pages, table in ((s.pages, s.table[2:3]), (other.pages, other.table[:1])):
        out, lse = torch.zeros_like(q), torch.zeros((1, 6), device="cuda")
        wm.wm_pages_attend(pages, table.contiguous(), _dev([lens[2]]), _dev([0, 1]), q, out, s.ws, lse=lse, max_q=1)
        outs.append((out, lse))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@gpu
def test_a_step_captured_into_a_graph_and_replayed():
    g = torch.Generator().manual_seed(21)
    n, dim, heads = 5, 128, 2
    a, b = (Session(n, 32, heads, dim) for _ in range(2))
    prompt = [33, 1, 64, 100, 31]
    rows = sum(prompt)
    k, v = (torch.randn((rows, heads, dim), generator=g).to(torch.float16).cuda() for _ in range(2))
    q = torch.randn((rows, 8, dim), generator=g).to(torch.float16).cuda()
    for s in (a, b):
        s.step(_dev(prompt), k, v, q, _dev([0] * (n + 1)), _dev([0] * rows), torch.zeros_like(q))
        s.lens.copy_(_dev(prompt))
    new = _dev(prompt)
    k, v, q = k[:n].clone(), v[:n].clone(), q[:n].clone()
    bufs = {s: (_dev([0] * (n + 1)), _dev([0] * n), torch.zeros_like(q), torch.zeros((n, 8), device="cuda")) for s in (a, b)}

    def step(s):
        start, slots, out, lse = bufs[s]
        s.lens.copy_(new)
        new.add_(1)
        s.step(new, k, v, q, start, slots, out, lse, max_q=1)

    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            step(a)
    torch.cuda.synchronize()
    new.copy_(_dev(prompt))
    steps = [[torch.randn(t.shape, generator=g).to(t.dtype).cuda() for t in (k, v, q)] for _ in range(40)]
    outs = []
    for kk, vv, qq in steps:
        k.copy_(kk), v.copy_(vv), q.copy_(qq)
        graph.replay()
        outs.append((bufs[a][2].clone(), bufs[a][3].clone()))
    new.copy_(_dev(prompt))
    for (kk, vv, qq), (out, lse) in zip(steps, outs):
        k.copy_(kk), v.copy_(vv), q.copy_(qq)
        step(b)
        assert torch.equal(bufs[b][2], out) and torch.equal(bufs[b][3], lse)
    assert wm.read_pages_report(a.report) == ("OK", None) == wm.read_pages_report(b.report)
    assert torch.equal(a.pages.k, b.pages.k) and torch.equal(a.table, b.table) and torch.equal(a.count, b.count)


@gpu
def test_prompts_captured_into_a_graph_and_replayed_with_other_lengths():
    g = torch.Generator().manual_seed(26)
    most, page, dim = [400, 300, 200], 64, 128
    pages, arrays, table = _attend_case(most, page, 2, dim, g)
    tab, kv, start = _dev(table), _dev(most), _dev([0, 0, 0, 0])
    q = torch.randn((500, 8, dim), generator=g).to(torch.bfloat16).cuda()
    out, want, ws = torch.zeros_like(q), torch.zeros_like(q), wm.new_pages_workspace(dim)
    call = lambda o: wm.wm_pages_attend(pages, tab, kv, start, q, o, ws, max_q=300)  # noqa: E731
    call(out)
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            call(out)
    for lens, starts in (([400, 300, 200], [0, 200, 300, 500]), ([400, 1, 128], [0, 300, 301, 301]), ([129, 300, 0], [0, 1, 260, 300]), ([400, 300, 200], [0, 0, 0, 0])):
        kv.copy_(_dev(lens)), start.copy_(_dev(starts))
        out.fill_(3.0), want.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        call(want)
        assert torch.equal(out, want) and (out[starts[-1]:] == 3).all()


_FIRST_IN_A_GRAPH = """
import sys
sys.path.insert(0, {root!r})
import torch
from paper_2607_10389_b200 import binding as wm
p = wm.new_pages(4, 16, 1, 64)
i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
old, new, table, free, count, start, slots = i32([0]), i32([3]), i32([[-1, -1]]), i32([3, 1, 2, 0]), i32([4]), i32([0, 0]), i32([0, 0, 0])
x = torch.ones(3, 1, 64, device="cuda", dtype=torch.bfloat16)
out, ws = torch.zeros_like(x), wm.new_pages_workspace(64)
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    wm.wm_pages_plan(old, new, 16, table, free, count, count, start, slots)
    wm.wm_pages_append(p, x, x, slots)
    wm.wm_pages_attend(p, table, new, start, x, out, ws, max_q=3)
graph.replay()
torch.cuda.synchronize()
assert torch.equal(out, x) and slots.tolist() == [0, 1, 2] and count.item() == 3
print("graph ok")
"""


@gpu
def test_the_first_calls_of_a_process_may_be_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    out = subprocess.run([sys.executable, "-c", _FIRST_IN_A_GRAPH.format(root=root)], capture_output=True, text=True, timeout=600)
    assert out.returncode == 0 and "graph ok" in out.stdout, out.stderr[-2000:]


@gpu
def test_calls_on_two_streams_with_workspaces_of_their_own():
    g = torch.Generator().manual_seed(22)
    lens = [700, 300, 1000, 128]
    pages, arrays, table = _attend_case(lens, 64, 4, 128, g)
    q = torch.randn((4, 16, 128), generator=g).to(torch.bfloat16).cuda()
    tab, kv, start = _dev(table), _dev(lens), _dev([0, 1, 2, 3, 4])
    want = torch.zeros_like(q)
    wm.wm_pages_attend(pages, tab, kv, start, q, want, wm.new_pages_workspace(128), max_q=1)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [[torch.zeros_like(q) for _ in range(30)] for _ in streams]
    ws = [wm.new_pages_workspace(128) for _ in streams]
    torch.cuda.synchronize()
    for j in range(30):
        for s, o, w in zip(streams, outs, ws):
            wm.wm_pages_attend(pages, tab, kv, start, q, o[j], w, max_q=1, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for os in outs for o in os)


@gpu
def test_codes_beyond_four_gigabytes():
    """Pages whose bytes lie more than 2^32 from the pool's first."""
    g = torch.Generator().manual_seed(23)
    page, heads, dim = 128, 8, 128
    n = (5 << 30) // (page * heads * dim)
    k, v = (torch.empty((n, heads, page, dim), dtype=torch.uint8, device="cuda") for _ in range(2))
    pages = wm.Pages(k, v, torch.ones((n, heads), device="cuda"), torch.ones((n, heads), device="cuda"))
    ids = [n - 1, 0, n - 2, n // 2]
    k[ids], v[ids] = 0, 0
    lens = [4 * page - 3]
    x, y = (torch.randn((lens[0], heads, dim), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    wm.wm_pages_append(pages, x, y, _dev([ids[p // page] * page + p % page for p in range(lens[0])]))
    small = [k[ids].cpu(), v[ids].cpu(), pages.k_scale[ids].cpu(), pages.v_scale[ids].cpu()]
    want = [torch.zeros(4, heads, page, dim).double(), torch.ones(4, heads).double()]
    ref.append(want[0], want[1], x.cpu(), list(range(lens[0])), page)
    assert torch.equal(ref.values(small[0]), want[0]) and torch.equal(small[2].double(), want[1])
    for rows in (1, 130):
        q = torch.randn((rows, heads, dim), generator=g).to(torch.bfloat16)
        out = torch.zeros((rows, heads, dim), dtype=torch.bfloat16, device="cuda")
        wm.wm_pages_attend(pages, _dev([ids]), _dev(lens), _dev([0, rows]), q.cuda(), out, wm.new_pages_workspace(dim), max_q=rows)
        w = ref.attend(ref.values(small[0]), ref.values(small[1]), small[2].double(), small[3].double(), [[0, 1, 2, 3]], lens, [0, rows], q.double(),
                       dim ** -0.5, True, 0)
        far, _ = ref.bounds(*w, torch.bfloat16, dim)
        assert ((out.cpu().double() - w[0]).abs() <= far).all()
