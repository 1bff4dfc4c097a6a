"""The layer for few tokens over 4-bit weights where its matrix instructions add with the fewest bits: channels far above their
neighbours whose products cancel, so that what is left is of the size of what the adder cuts off."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import mx4_reference as ref
from tests.test_gpu_few_tokens import _check, _run, _values

pytestmark = pytest.mark.gpu


def _exponent(v):
    return torch.floor(torch.log2(v.clamp_min(1e-300)))


def _sum_bound(x, err, W):
    """Bound on |sum - exact sum| of a row x [K], whose elements may be off by err and go into the instruction as two e4m3 halves, times
    W [K, N] (values of e2m1 elements with a scale for every 32 k).  Of the 8 products k = 8 i .. 8 i + 7 the instruction keeps the bits
    from 2^(e - 13) up, e the largest sum of two operands' exponents: less than 7 * 2^(e - 13) is lost, and a sixteenth of that in the low halves.
    An operand's exponent: the element's, one more where it rounds up to a power of two, at least that of its type's smallest normal value
    (e4m3: 2^-6 where the block's largest is below 2^8; e2m1: 1).  Sums of groups are added with 24 bits: 2^-23 of A = sum |x w| for a group and for its
    addition, high and low halves (1/16) alike, and so are the wavefronts' sums (16 more)."""
    K = x.shape[0]
    a = torch.nn.functional.pad(x.abs() + err, (0, -K % 32))
    w = torch.nn.functional.pad(W.abs(), (0, 0, 0, -K % 32))
    largest = a.reshape(-1, 32).amax(1).repeat_interleave(32)
    ex = torch.maximum(_exponent(a) + 1, _exponent(largest) + 1 - 13)
    # (the block's scale is not in the values; its largest element is 4 or 6 times it or, where it has nothing else, less)
    top = _exponent(w.reshape(-1, 32, w.shape[1]).amax(1)) - 2
    ew = torch.maximum(_exponent(w), top.repeat_interleave(32, 0))
    e = (ex[:, None] + ew).reshape(-1, 8, w.shape[1]).amax(1)
    return 7.0 * (1 + 1 / 16) * torch.exp2(e - 13).sum(0) + (2 * (2 * (K // 8 + 1)) + 16) * 2.0 ** -23 * 1.1 * (a @ w)


def _expected(X, logits, up, down, k):
    """Output in 64 bits and a bound on what the layer's may differ by."""
    ids, w = ref.route(logits, k, False, True, 1.0)
    U, D, x = _values(up, True), _values(down, True), X.double()
    T, hidden, inter = X.shape[0], X.shape[1], down.shape[1]
    out, tol, mag = (torch.zeros(T, hidden, dtype=torch.float64) for _ in range(3))
    for t in range(T):
        # a token's value: exact, or off by 2^-21 of its block's largest
        largest = torch.nn.functional.pad(x[t].abs(), (0, -hidden % 32)).reshape(-1, 32).amax(1).repeat_interleave(32)[:hidden]
        ex = torch.where(x[t].abs() >= largest * 2.0 ** -13, 0.0, largest * 2.0 ** -21)
        for j in range(k):
            e = int(ids[t, j])
            y, err = x[t] @ U[e], _sum_bound(x[t], ex, U[e]) + ex @ U[e].abs()
            g, u, eg, eu = y[:inter], y[inter:], err[:inter], err[inter:]
            h = ref.silu(g) * u
            eh = 1.1 * eg * (u.abs() + eu) + ref.silu(g).abs() * eu + 32 * 2.0 ** -24 * h.abs()
            top = torch.nn.functional.pad(h.abs() + eh, (0, -inter % 32)).reshape(-1, 32).amax(1).repeat_interleave(32)[:inter]
            eh = eh + torch.maximum(2.0 ** -8 * (h.abs() + eh), 2.0 ** -21 * top)
            z, ez = h @ D[e], eh @ D[e].abs() + _sum_bound(h, eh, D[e])
            p = float(w[t, j])
            out[t] += p * z
            mag[t] += p * (z.abs() + ez)
            tol[t] += p * ez
    tol += mag * (k + 64) * 2.0 ** -24 + 2.0 ** -8 * out.abs() + 2.0 ** -130
    return out, tol, ids, w


def _outliers(X, up, gap, g):
    """Every 32 channels two neighbours are 2^gap above the others in X, and their weights cancel."""
    X, up = X.clone(), up.clone()
    for k in range(3, X.shape[1] - 1, 32):
        X[:, k] = (torch.rand(X.shape[0], generator=g) + 1.0) * 2.0 ** gap
        X[:, k + 1] = X[:, k]
        up[:, k + 1] = -up[:, k]
    return X, up


@pytest.mark.parametrize("gap", [0, 4, 8, 9, 10, 11, 13])
@pytest.mark.parametrize("T,k,E,hidden,inter", [(1, 2, 4, 256, 64), (5, 2, 4, 264, 96), (16, 2, 6, 512, 40), (16, 2, 3, 4712, 40)])
def test_outliers_that_cancel(T, k, E, hidden, inter, gap):
    g = torch.Generator().manual_seed(hidden + gap)
    X = torch.randn(T, hidden, generator=g).to(torch.bfloat16)
    logits = torch.randn(T, E, generator=g)
    up = torch.randn(E, hidden, 2 * inter, generator=g) * hidden ** -0.5
    down = (torch.randn(E, inter, hidden, generator=g) * inter ** -0.5).to(torch.bfloat16)
    X, up = _outliers(X, up, gap, g)
    up = up.to(torch.bfloat16)
    got, want = _run(X, logits, up, down, k, True), _expected(X, logits, up, down, k)
    _check(got, want)
    off = (got[0].double() - want[0]).norm() / want[0].norm()
    print(f"gap 2^{gap}, {T} tokens, {hidden}: off by {float(off):.2e} of the norm, at most {float(((got[0].double() - want[0]).abs() / want[1]).max()):.3f} of the bound")


def test_the_groups_adder():
    """One group of 8: two outliers that cancel and six values at 2^-11 of them, with weights at 1/12 of theirs: 13 bits below the largest product."""
    hidden, inter = 8, 32
    X = torch.tensor([[200.0, 200.0] + 6 * [200.0 * 2.0 ** -11]]).to(torch.bfloat16)
    up = torch.zeros(1, hidden, 2 * inter)
    up[0, 0], up[0, 1], up[0, 2:] = 6.0, -6.0, 0.5
    down = torch.randn(1, inter, hidden, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    logits = torch.zeros(1, 1)
    got, want = _run(X, logits, up.to(torch.bfloat16), down, 1, True), _expected(X, logits, up, down, 1)
    _check(got, want)
