"""The attention of tests/pages_ref.py, all rows of a request at once: 64 bits, on whatever device its inputs are (the GPU for
cases of millions of pairs)."""
import math

import torch

import pages_ref as ref


def attend(k, v, ks, vs, table, kv_len, q_start, q, scale, causal, window):
    """As pages_ref.attend: (out, lse, weight, reach, floor, spread).  k, v: codes; ks, vs: scales; table: lists."""
    rows, heads, dim = q.shape
    kv_heads, page = k.shape[1], k.shape[2]
    group = heads // kv_heads
    zeros = lambda *s: torch.zeros(s, dtype=torch.float64, device=q.device)  # noqa: E731
    out, weight, spread = zeros(rows, heads, dim), zeros(rows, heads, dim), zeros(rows, heads, dim)
    lse, reach, floor = zeros(rows, heads) - math.inf, zeros(rows, heads), zeros(rows, heads)
    for i, n in enumerate(kv_len):
        lo, hi = q_start[i], q_start[i + 1]
        if hi == lo or n == 0:
            continue
        ids = torch.tensor(table[i][:ref.pages_of(n, page)], device=q.device)
        pos = torch.arange(n - (hi - lo), n, device=q.device).repeat_interleave(group)[:, None]
        col = torch.arange(n, device=q.device)[None]
        seen = (col <= pos) if causal else (col >= 0).expand(pos.shape[0], n)
        if window:
            seen = seen & (col > pos - window)
        some = seen.any(1, keepdim=True)
        for h in range(kv_heads):
            at = (slice(lo, hi), slice(h * group, (h + 1) * group))
            of = lambda c, s: (c[ids, h].view(torch.uint8).view(ref.E4M3).double() * s[ids, h].double()[:, None, None]).reshape(-1, dim)[:n]  # noqa: E731
            kk, vv = of(k, ks), of(v, vs)
            y = q[at].double().reshape(-1, dim)
            s = (y @ kk.T * scale).masked_fill(~seen, -math.inf)
            w = torch.where(some, torch.softmax(s, 1), torch.zeros_like(s))
            back = lambda x: x.reshape(hi - lo, group, *x.shape[1:])  # noqa: E731
            none = lambda x: torch.where(some.squeeze(1) if x.dim() == 1 else some, x, torch.zeros_like(x))  # noqa: E731
            out[at], weight[at] = back(w @ vv), back(w @ vv.abs())
            lse[at] = back(torch.logsumexp(s, 1))
            spread[at] = back(w.amax(1, keepdim=True) * (seen.double() @ vv.abs()))
            reach[at] = back(none((y.abs() @ kk.abs().T).masked_fill(~seen, 0).amax(1) * abs(scale)))
            floor[at] = back(none(y.abs().amax(1) * kk.abs().sum(1)[None].expand_as(seen).masked_fill(~seen, 0).amax(1) * abs(scale)))
    return out, lse, weight, reach, floor, spread
