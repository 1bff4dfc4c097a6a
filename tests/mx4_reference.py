"""The 4-bit operators in 64 bits, written from their definitions: block scales, nearest elements, the router's choice, the
products, and bounds on what fp32 sums may differ by.  Plain torch on the CPU."""
from __future__ import annotations

import torch

MAGNITUDES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
BLOCK, ROW_PAD = 32, 128


def quantize(x: torch.Tensor):
    """x [rows, n] -> (codes 0 .. 15 uint8 [rows, Kp], scale bytes uint8 [rows, Kp / 32], values float64 [rows, n]), Kp = n rounded
    up to 128."""
    rows, n = x.shape
    pad = torch.zeros(rows, (n + ROW_PAD - 1) // ROW_PAD * ROW_PAD, dtype=torch.float64)
    pad[:, :n] = x.double()
    b = pad.reshape(rows, -1, BLOCK)
    largest = b.abs().amax(2)
    bad = ~torch.isfinite(b).all(2)
    # floor(log2 a), by counting powers of two (a logarithm may round up to the next integer)
    e = torch.full_like(largest, -1100.0)
    ok = (largest > 0) & ~bad
    guess = torch.floor(torch.log2(largest[ok]))
    guess = torch.where(torch.pow(2.0, guess) > largest[ok], guess - 1, guess)
    guess = torch.where(torch.pow(2.0, guess + 1) <= largest[ok], guess + 1, guess)
    e[ok] = guess
    s = torch.clamp(e - 2, min=-127.0)
    scale = torch.pow(2.0, s)
    a = torch.where(bad[..., None], 0.0, b.abs()) / scale[..., None]
    gap = (a[..., None] - MAGNITUDES).abs()
    # nearest, ties to the even code: an odd code has to be strictly nearer
    order = gap + torch.where(torch.arange(8) % 2 == 1, 1e-12, 0.0)
    code = order.argmin(-1)
    values = torch.copysign(MAGNITUDES[code], torch.where(bad[..., None], 0.0, b)) * scale[..., None]
    code = code + 8 * (torch.signbit(b) & ~bad[..., None])
    values[bad] = float("nan")
    code[bad] = 0
    byte = torch.where(bad, 255.0, s + 127).to(torch.uint8)
    return code.reshape(rows, -1).to(torch.uint8), byte, values.reshape(rows, -1)[:, :n]


def packed_rows(code: torch.Tensor) -> torch.Tensor:
    """Codes [rows, Kp] as bytes [rows, Kp / 2], even elements in the low halves."""
    return code[:, 0::2] | (code[:, 1::2] << 4)


def source_columns(N: int, gated: bool) -> list:
    """Source column of each packed column, padded to 64; -1 is padding."""
    if gated:
        half, cols = N // 2, []
        for u in range((half + 15) // 16):
            idx = range(16 * u, 16 * u + 16)
            cols += [i if i < half else -1 for i in idx] + [half + i if i < half else -1 for i in idx]
    else:
        cols = list(range(N))
    return cols + [-1] * (-len(cols) % 64)


def packed_weights(W: torch.Tensor, gated: bool):
    """W [E, K, N] -> (codes, scales) in the packed layout (flat uint8) and the values [E, K, N] in float64."""
    E, K, N = W.shape
    cols = source_columns(N, gated)
    Kp = (K + ROW_PAD - 1) // ROW_PAD * ROW_PAD
    codes, scales, values = [], [], torch.empty(E, K, N, dtype=torch.float64)
    for e in range(E):
        code, byte, val = quantize(W[e].t())
        values[e] = val.t()
        pc, ps = torch.zeros(len(cols), Kp, dtype=torch.uint8), torch.zeros(len(cols), Kp // BLOCK, dtype=torch.uint8)
        for p, c in enumerate(cols):
            if c >= 0:
                pc[p], ps[p] = code[c], byte[c]
        # [tile n][block j][column c][tile k][g][32] -> [tile n][tile k][j][g][c][32 codes = 16 bytes]
        t = pc.reshape(len(cols) // 64, 4, 16, Kp // 128, 4, 32).permute(0, 3, 1, 4, 2, 5)
        codes.append((t[..., 0::2] | (t[..., 1::2] << 4)).reshape(-1))
        # [tile n][j][c][tile k][g] -> [tile n][tile k][g][c][j]
        scales.append(ps.reshape(len(cols) // 64, 4, 16, Kp // 128, 4).permute(0, 3, 4, 2, 1).reshape(-1))
    return torch.cat(codes), torch.cat(scales), values


def route(logits: torch.Tensor, k: int, sigmoid: bool, renormalize: bool, scale: float):
    """ids [T, k], weights float64 [T, k]; one row after the other."""
    T, E = logits.shape
    ids, weights = torch.zeros(T, k, dtype=torch.int32), torch.zeros(T, k, dtype=torch.float64)
    for t in range(T):
        row = [float(v) for v in logits[t].double()]
        order = sorted(range(E), key=lambda e: (0, 0.0, e) if row[e] != row[e] else (1, -row[e], e))[:k]
        r = torch.tensor(row, dtype=torch.float64)
        if sigmoid:
            p = 1 / (1 + torch.exp(-r))
        elif bool((r == -float("inf")).all()):
            p = torch.zeros(E, dtype=torch.float64)
        else:
            p = torch.exp(r - r.max())
            p = p / p.sum()
        w = p[order]
        if renormalize:
            w = torch.zeros_like(w) if float(w.sum()) == 0 else w / w.sum()
        ids[t], weights[t] = torch.tensor(order, dtype=torch.int32), w * scale
    return ids, weights


def silu(g: torch.Tensor) -> torch.Tensor:
    return g / (1 + torch.exp(-g))


def product_sum_bound(X: torch.Tensor, W: torch.Tensor) -> torch.Tensor:
    """Bound on |fp32 sum - exact sum| of 4-bit products X [T, K] . W [K, N] (float64 values).  How the matrix instructions add
    products of fewer than 16 bits is not documented; the library's tests of 8-bit ones found groups of 8 consecutive k whose products
    keep the bits from 2^(e - 13) up (e: the largest product exponent of the group) and group sums added with 24 bits, and an adder
    for 4-bit products, which are shorter, is assumed to cut off no more: 7 * 2^(e - 13) a group, and 2^-23 of A = sum|x w| twice
    for each group."""
    def exponent(t):
        return torch.where(t == 0, -400.0, torch.floor(torch.log2(t.abs().clamp_min(1e-300))))
    K = X.shape[1]
    bound = (X.abs() @ W.abs()) * (2 * ((K + 7) // 8 + 1) * 2.0 ** -23)
    ex, ew = exponent(X), exponent(W)
    for k in range(0, K, 8):
        e = (ex[:, k: k + 8, None] + ew[None, k: k + 8]).amax(1)
        bound += 7.0 * torch.exp2(e + 1 - 13)      # (a product of two mantissas below 2 may reach the next exponent)
    return bound
