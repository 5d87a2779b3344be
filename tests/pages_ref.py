"""Plain 64-bit implementation of the paged 8-bit cache's calls, on the CPU, and makers of their inputs."""
import math

import torch

E4M3 = torch.float8_e4m3fn
SPECIAL = {"nan": 0x7F, "max": 0x7E, "-max": 0xFE}


def pages_of(tokens, page):
    return -(-tokens // page)


def e4m3(x):
    """Doubles to the nearest e4m3 value (ties to even, saturating, NaN stays), as doubles."""
    size = x.abs().clamp(max=448.0)
    step = torch.ldexp(torch.ones_like(size), (torch.frexp(size)[1] - 1).clamp(min=-6) - 3)
    return torch.copysign(torch.round(size / step) * step, x)


def values(codes):
    return codes.view(torch.uint8).cpu().contiguous().view(E4M3).double()


def power_over(x):
    """The smallest power of two that is not below x > 0."""
    m, e = math.frexp(x)
    return math.ldexp(1.0, e - 1 if m == 0.5 else e)


def plan(old, new, page, table, free, count, n_slots):
    """Lists in, lists out: (status, table, free, count, start, slots).  `free`: the whole pool's array."""
    table, free = [list(r) for r in table], list(free)
    start, slots = [0], []
    width, pool = len(table[0]), len(free)
    fail = lambda s: (s, table, free, count, [0] * (len(old) + 1), [-1] * n_slots)  # noqa: E731
    held, want = [pages_of(o, page) for o in old], [pages_of(n, page) for n in new]
    fine = [o >= 0 and n >= 0 and max(h, w) <= width for o, n, h, w in zip(old, new, held, want)]      # the others count for nothing
    give = sum(max(0, h - w) for h, w, f in zip(held, want, fine) if f)
    take = sum(max(0, w - h) for h, w, f in zip(held, want, fine) if f)
    more = sum(max(0, n - o) for o, n, f in zip(old, new, fine) if f)
    status = []
    if min(old) < 0 or min(new) < 0 or max(held) > width or count > pool or count + give - take > pool:
        status.append(-1)
    if max(want) > width or take > count + give or more > n_slots:
        status.append(-2)
    if status:
        return fail(min(status))
    stack = free[:count]
    for i, row in enumerate(table):
        stack += row[want[i]:held[i]]
    for i, row in enumerate(table):
        for j in range(held[i], want[i]):
            row[j] = stack.pop()
        for p in range(old[i], new[i]):
            slots.append(row[p // page] * page + p % page)
        start.append(len(slots))
    kept = min(count, len(stack))
    free[kept:len(stack)] = stack[kept:]
    return 0, table, free, len(stack), start, slots + [-1] * (n_slots - len(slots))


def append(codes, scales, x, slots, page):
    """codes (n, heads, page, dim) as doubles and scales (n, heads) as doubles are updated in place."""
    runs = []
    for r, slot in enumerate(slots):
        if slot < 0:
            continue
        if runs and runs[-1][1] + len(runs[-1][2]) == slot and slot % page:
            runs[-1][2].append(r)
        else:
            runs.append((slot // page, slot, [r]))
    for p, first, rows in runs:
        off = first % page
        for h in range(codes.shape[1]):
            y = x[rows, h].double()
            fine = y[y.isfinite()].abs()
            amax = float(fine.max()) if fine.numel() else 0.0
            scale = max(power_over(amax / 448.0) if amax else 0.0, 2.0 ** -126)
            if off:
                old = float(scales[p, h])
                scale = max(scale, power_over(old) if old else 2.0 ** -126)
                codes[p, h, :off] = e4m3(codes[p, h, :off] * (old / scale))
            scales[p, h] = scale
            codes[p, h, off:off + len(rows)] = e4m3(y / scale)


def attend(k, v, ks, vs, table, kv_len, q_start, q, scale, causal, window):
    """(out, lse, weight, error): doubles.  k, v, ks, vs: values as the codes and scales stand for.  `weight` is sum p |v| of
    each output, `spread` the largest p times sum |v|, `reach` the scores' sum |q||k| scale and qmax sum |k| scale, what the error of a score is counted in."""
    rows, heads, dim = q.shape
    group = heads // k.shape[1]
    page = k.shape[2]
    out = torch.zeros(rows, heads, dim, dtype=torch.float64)
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64)
    weight, reach, floor, spread = torch.zeros_like(out), torch.zeros_like(lse), torch.zeros_like(lse), torch.zeros_like(out)
    for i, n in enumerate(kv_len):
        lo, hi = q_start[i], q_start[i + 1]
        if hi == lo:
            continue
        ids = table[i][:pages_of(n, page)]
        kk = (k[ids] * ks[ids][..., None, None]).transpose(1, 2).reshape(-1, k.shape[1], dim)[:n] if n else torch.zeros(0, k.shape[1], dim).double()
        vv = (v[ids] * vs[ids][..., None, None]).transpose(1, 2).reshape(-1, k.shape[1], dim)[:n] if n else kk
        for j in range(hi - lo):
            p = n - (hi - lo) + j
            a = max(0, p - window + 1) if window else 0
            b = min(n, p + 1) if causal else n
            if b <= a:
                continue
            for h in range(k.shape[1]):
                y = q[lo + j, h * group:(h + 1) * group].double()
                s = y @ kk[a:b, h].T * scale
                w = torch.softmax(s, 1)
                at = (lo + j, slice(h * group, (h + 1) * group))
                out[at] = w @ vv[a:b, h]
                lse[at] = torch.logsumexp(s, 1)
                weight[at] = w @ vv[a:b, h].abs()
                spread[at] = w.amax(1, keepdim=True) * vv[a:b, h].abs().sum(0)
                size = kk[a:b, h].abs()
                reach[at] = (y.abs() @ size.T).amax(1) * abs(scale)
                floor[at] = y.abs().amax(1) * size.sum(1).amax() * abs(scale)
    return out, lse, weight, reach, floor, spread


def bounds(out, lse, weight, reach, floor, spread, dtype, dim):
    """How far a kernel may be off (out, lse).  A score is a sum of dim products in 32 bits, each addition off by less
    than 2^-23 of the sum of the products' sizes, and a handful of factors (scales, the exponential): (dim + 8) 2^-23
    reach.  The queries are held in pieces on a grid of 2^-18 of their row's largest or finer: 2^-18 floor.  An
    error d of the scores moves the softmax's weights by a factor within 1 +- 2 d.  Weights are held in 11 significant
    bits or more (half a step: 2^-12, taken twice for the sum of pieces), sums in 32 bits, and the output is rounded once.
    Small weights lie on a grid: three e4m3 pieces of 2^8 p, each of the remainder times 16, end at steps of
    2^-9 / 16^2 / 2^8 = 2^-25 of the largest weight of the tile, which is not above the row's (twice the true one for errors of
    the scores): half a step, 2^-26, for every value, whatever its weight."""
    d = (dim + 8) * 2.0 ** -23 * reach + 2.0 ** -18 * floor
    rounding = torch.finfo(dtype).eps / 2
    far = 2 * (2 * d[..., None] + 2.0 ** -12) * weight + 2.0 ** -25 * spread
    tiny = torch.finfo(dtype).tiny * torch.finfo(dtype).eps
    return far * (1 + rounding) + rounding * out.abs() + tiny, d + 2.0 ** -18 + 2.0 ** -22 * lse.abs()


def random_pool(n, heads, page, dim, g, spread=0):
    """Codes and power-of-two scales of a pool; `spread`: the scales' exponents lie in -4 .. spread - 4."""
    codes = [(torch.randn((n, heads, page, dim), generator=g) * 60).clamp(-448, 448).to(E4M3).view(torch.uint8) for _ in range(2)]
    scales = [2.0 ** (torch.randint(0, spread + 1, (n, heads), generator=g).float() - 5) for _ in range(2)]
    return codes[0], codes[1], scales[0], scales[1]


def random_table(lens, page, width, n, g):
    order = torch.randperm(n, generator=g).tolist()
    table = []
    for x in lens:
        need = pages_of(x, page)
        table.append([order.pop() for _ in range(need)] + [-1] * (width - need))
    return table
