"""The operators around a block's experts in 64 bits, written from their definitions: the grouped router's choice, the norm, rows in 8 bits, the
4-bit product, and bounds on what fp32 may differ by.  Plain torch on the CPU."""
from __future__ import annotations

import torch

E4M3_MAX = 448.0


def _falling(rows):
    """Indices of a list of (score, ...) tuples in falling order; NaN first, equal ones by rising index."""
    return sorted(range(len(rows)), key=lambda i: tuple((0, 0.0) if v != v else (1, -v) for v in rows[i]) + (i,))


def route_grouped(logits: torch.Tensor, k: int, groups: int, kept: int, top2: bool, bias, sigmoid: bool, renormalize: bool, scale: float):
    """ids [T, k], weights float64 [T, k]; one row after the other."""
    T, E = logits.shape
    each = E // groups
    b = torch.zeros(E, dtype=torch.float64) if bias is None else bias.double()
    ids, weights = torch.zeros(T, k, dtype=torch.int32), torch.zeros(T, k, dtype=torch.float64)
    for t in range(T):
        l = logits[t].double()
        masked = (l == -float("inf")) | (b == -float("inf"))
        if sigmoid:
            p = torch.where(l < -690, 0.0, 1 / (1 + torch.exp(-l)))
        else:
            e = torch.exp(l - l[~masked].max()) if not bool(masked.all()) else torch.zeros(E, dtype=torch.float64)
            e[masked] = 0.0
            p = e / e.sum()
        p = torch.where(masked, 0.0, p)
        s, live, logit = (p + b).tolist(), (~masked).tolist(), l.tolist()
        score = []
        for g in range(groups):
            best = sorted((s[e] for e in range(g * each, (g + 1) * each) if live[e]), key=lambda v: (0, 0.0) if v != v else (1, -v))
            score.append((len(best) > 0, best[0] + (best[1] if top2 and len(best) > 1 else 0.0) if best else 0.0))
        stay = [g for g in _falling(score)][:kept]
        inside = [e for g in sorted(stay) for e in range(g * each, (g + 1) * each)]
        rows = [(True, s[e], logit[e]) if live[e] else (False, 0.0, 0.0) for e in inside]
        order = [inside[i] for i in _falling(rows)][:k]
        w = p[order]
        if renormalize:
            w = torch.zeros_like(w) if float(w.sum()) == 0 else w / w.sum()
        ids[t], weights[t] = torch.tensor(order, dtype=torch.int32), w * scale
    return ids, weights


def add_norm(x, residual, weight, eps: float):
    """(h of the residual's type, y float64)."""
    h = x if residual is None else (x.float() + residual.float()).to(residual.dtype)
    f = h.double()
    mean = f.square().mean(1, keepdim=True) + eps
    y = f / torch.sqrt(mean)
    y = torch.where((f == 0) & (mean == 0), 0.0, y)
    return h, y if weight is None else y * weight.double()


def row_scales(y: torch.Tensor) -> torch.Tensor:
    return (y.abs().amax(1) / E4M3_MAX).clamp(min=2.0 ** -126)


def half_step(v: torch.Tensor) -> torch.Tensor:
    """Half the distance of neighbouring e4m3 values at |v| <= 448 (three bits of mantissa, exponents from -6 on)."""
    e = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    return torch.exp2(e - 4)


def w4_values(q, scales, zeros, group: int) -> torch.Tensor:
    K = q.shape[0]
    z = 8.0 if zeros is None else zeros.double().repeat_interleave(group, dim=0)[:K]
    return (q.double() - z) * scales.double().repeat_interleave(group, dim=0)[:K]


def w4_sum_bound(x, q, scales, zeros, group: int) -> torch.Tensor:
    """Bound on |fp32 sum - exact sum| of x [T, K] times the 4-bit weight.  Within a group the sum starts at -(128 + z) sum x and takes products
    of 128 + q: no partial sum is above 2 * 143 A, A = sum |x|, and there are group additions, those of sum x (each off by 2^-24 A, times 143) and the
    start's rounding: (2 * group + 4) * 2^-24 * 286 A covers them.  The groups' sums, each times its scale (one rounding), are added in any order: as many
    additions and roundings as groups, of partial sums below the sum of |s| (15 A + that error), and 32 more of the wavefronts' sums."""
    K = x.shape[1]
    n = -(-K // group)
    a = torch.zeros(x.shape[0], n * group, dtype=torch.float64)
    a[:, :K] = x.double().abs()
    A = a.reshape(x.shape[0], n, group).sum(2)                       # [T, groups]
    s = scales.double().abs()
    within = (2 * group + 4) * 2.0 ** -24 * 286 * (A @ s)
    return within + (2 * n + 32) * 2.0 ** -24 * (15 * (A @ s) + within)


def silu(g):
    return g / (1 + torch.exp(-g))
