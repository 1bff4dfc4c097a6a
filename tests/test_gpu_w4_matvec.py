"""The product of a few tokens with a dense 4-bit weight, against 64 bits."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import block_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16 = torch.bfloat16, torch.float16


def _weight(K, N, group, seed, zeros=True, dtype=F16):
    g = torch.Generator().manual_seed(seed)
    n = -(-K // group)
    q = torch.randint(0, 16, (K, N), generator=g, dtype=torch.uint8)
    s = ((0.5 + torch.rand(n, N, generator=g)) * K ** -0.5 * torch.where(torch.rand(n, N, generator=g) < 0.1, -1.0, 1.0)).to(dtype)
    z = torch.randint(0, 16, (n, N), generator=g, dtype=torch.uint8) if zeros else None
    return q, s, z


def _tokens(T, K, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, K, generator=g)
    x[:, torch.rand(K, generator=g) < 0.02] *= 16.0
    return x.to(BF16)


def _packed(q, s, z, group, gated):
    K, N = q.shape
    return mb.W4Weights(K, N, group, gated, DEV).pack(q.to(DEV), s.to(DEV), None if z is None else z.to(DEV))


def _expected(x, q, s, z, group, gated, add):
    """(float64 result, bound on the fp32 result's distance before its rounding)"""
    y, bound = x.double() @ ref.w4_values(q, s, z, group), ref.w4_sum_bound(x, q, s, z, group)
    if gated:
        g, u = y.chunk(2, dim=1)
        dg, du = bound.chunk(2, dim=1)
        a = ref.silu(g)
        # |silu'| <= 1.1; exponential, sum, quotient and product: an exponent of up to 88 rounds by 2^-24 of itself, four more roundings
        y, bound = a * u, 1.1 * dg * (u.abs() + du) + a.abs() * du + (a * u).abs() * (88 + 8) * 2.0 ** -24
    if add is not None:
        y, bound = y + add.double(), bound + (y.abs() + add.double().abs()) * 2.0 ** -24
    return y, bound


def _check(x, q, s, z, group, gated=False, add=None, W=None, xg=None):
    T, K, N = x.shape[0], *q.shape
    n = N // 2 if gated else N
    W = W or _packed(q, s, z, group, gated)
    out = torch.full((T + 1, n), 7.0, dtype=BF16, device=DEV)
    mb.moe_w4_matvec(x.to(DEV) if xg is None else xg, W, out, None if add is None else add.to(DEV))
    want, bound = _expected(x, q, s, z, group, gated, add)
    got = out[:T].cpu().double()
    assert bool((out[T] == 7.0).all())
    assert bool(((got - want).abs() <= bound * (1 + 2.0 ** -8) + want.abs() * 2.0 ** -8 + 2.0 ** -133).all())
    # over all outputs the rounding to bf16 is what is left: at most half a step each
    assert float((got - want).norm()) <= 2.0 ** -8 * float(want.norm()) * (1 + 2.0 ** -4)
    return out[:T]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("T,K,N", [(1, 1, 1), (1, 128, 16), (2, 8, 3), (1, 2048, 2816), (3, 33, 17), (16, 256, 48), (5, 1000, 130), (7, 130, 64), (15, 2049, 40), (16, 3584, 160), (4, 4096, 96),
                                   (9, 7168, 34), (1, 14336, 64)])
def test_matvec(T, K, N, group):
    for zeros, dtype in ((True, F16), (False, BF16)):
        q, s, z = _weight(K, N, group, K + N, zeros, dtype)
        x = _tokens(T, K, T)
        _check(x, q, s, z, group)
        _check(x, q, s, z, group, add=_tokens(T, N, 77))


@pytest.mark.parametrize("T,K,N", [(1, 8, 2), (2, 64, 30), (1, 2048, 2816), (16, 512, 66), (5, 777, 320), (3, 4096, 128)])
def test_gated(T, K, N):
    for group in (32, 128):
        q, s, z = _weight(K, N, group, K * N)
        x = _tokens(T, K, T + 1)
        _check(x, q, s, z, group, gated=True)
        _check(x, q, s, z, group, gated=True, add=_tokens(T, N // 2, 78))


@pytest.mark.parametrize("T,K,N,gated", [(1, 300, 4640, False), (7, 129, 4700, False), (16, 256, 5000, False), (8, 257, 12304, False), (16, 300, 12304, False), (9, 128, 12290, True),
                                         (1, 300, 16400, False), (6, 640, 16386, False), (16, 130, 16500, False), (1, 1100, 16420, True), (5, 96, 16402, True), (13, 264, 16400, True)])
def test_many_columns(T, K, N, gated):
    """Workgroups of two and of four tiles of columns, the last of which may not have all of them."""
    for group, zeros in ((32, True), (64, False), (128, True)):
        q, s, z = _weight(K, N, group, K + N, zeros)
        x = _tokens(T, K, T + 2)
        _check(x, q, s, z, group, gated=gated, add=_tokens(T, N // 2 if gated else N, 79) if group == 64 else None)


def test_layouts_give_the_same():
    q, s, z = _weight(520, 70, 64, 3)
    x = _tokens(6, 520, 4)
    a = _check(x, q, s, z, 64)
    W = mb.W4Weights(520, 70, 64, False, DEV)
    W.pack(q.t().contiguous().to(DEV), s.t().contiguous().to(DEV), z.t().contiguous().to(DEV), mb.MOE_W_LAYOUT_NK)
    assert torch.equal(a, _check(x, q, s, z, 64, W=W))


def test_high_bits_of_codes_and_zero_points_are_not_looked_at():
    q, s, z = _weight(256, 32, 32, 5)
    x = _tokens(2, 256, 6)
    _check(x, q, s, z, 32, W=_packed(q | 0x50, s, z | 0xa0, 32, False))


def test_tokens_apart_and_unaligned():
    q, s, z = _weight(640, 48, 128, 7)
    x = _tokens(9, 640, 8)
    same = _check(x, q, s, z, 128)
    for at, pitch in ((3, 700), (8, 704), (0, 641)):
        wide = torch.full((9, pitch), float("nan"), dtype=BF16, device=DEV)
        wide[:, at: at + 640] = x.to(DEV)
        assert torch.equal(same, _check(x, q, s, z, 128, xg=wide[:, at: at + 640]))


def test_added_to_itself():
    q, s, z = _weight(256, 64, 64, 9)
    x, add = _tokens(4, 256, 10), _tokens(4, 64, 11)
    W = _packed(q, s, z, 64, False)
    want = torch.empty(4, 64, dtype=BF16, device=DEV)
    mb.moe_w4_matvec(x.to(DEV), W, want, add.to(DEV))
    out = add.to(DEV)
    mb.moe_w4_matvec(x.to(DEV), W, out, out)
    assert torch.equal(out, want)


def test_a_token_that_is_not_finite_stays_alone():
    q, s, z = _weight(300, 40, 64, 12)
    x = _tokens(16, 300, 13)
    W = _packed(q, s, z, 64, False)
    want = torch.empty(16, 40, dtype=BF16, device=DEV)
    mb.moe_w4_matvec(x.to(DEV), W, want)
    for value in (float("nan"), float("inf")):
        bad = x.clone()
        bad[3, 299] = value
        out = torch.empty(16, 40, dtype=BF16, device=DEV)
        mb.moe_w4_matvec(bad.to(DEV), W, out)
        assert bool(torch.isnan(out[3]).all())
        others = [t for t in range(16) if t != 3]
        assert torch.equal(out[others], want[others])


def test_scales_of_zero_and_of_the_types_ends():
    q, s, z = _weight(256, 32, 64, 14)
    s[0, :8] = 0.0
    s[1, 8:16] = torch.finfo(F16).tiny / 4           # a subnormal
    x = _tokens(3, 256, 15)
    _check(x, q, s, z, 64)


def test_the_same_every_time_and_for_every_number_of_tokens():
    q, s, z = _weight(4096, 256, 128, 16)
    x = _tokens(16, 4096, 17)
    W = _packed(q, s, z, 128, True)
    whole = torch.empty(16, 128, dtype=BF16, device=DEV)
    mb.moe_w4_matvec(x.to(DEV), W, whole)
    for _ in range(3):
        again = torch.empty_like(whole)
        mb.moe_w4_matvec(x.to(DEV), W, again)
        assert torch.equal(whole, again)


@pytest.mark.parametrize("K,N,gated", [(4096, 256, True), (520, 4096, False), (1024, 5632, False), (640, 12304, False), (384, 14336, False), (640, 16400, False), (300, 16420, True)])
def test_a_token_has_the_same_bits_whatever_their_number(K, N, gated):
    """All forms of a token count (up to 4, 8 and 16) and of a workgroup's columns, those that change with the token count among them."""
    q, s, z = _weight(K, N, 64, 21)
    x = _tokens(16, K, 22).to(DEV)
    W = _packed(q, s, z, 64, gated)
    n = N // 2 if gated else N
    whole = torch.empty(16, n, dtype=BF16, device=DEV)
    mb.moe_w4_matvec(x, W, whole)
    for T in (1, 4, 5, 8, 9, 15):
        for first in (0, 16 - T):
            out = torch.empty(T, n, dtype=BF16, device=DEV)
            mb.moe_w4_matvec(x[first: first + T], W, out)
            assert torch.equal(out, whole[first: first + T])


def test_no_tokens():
    q, s, z = _weight(64, 16, 32, 18)
    assert mb.moe_w4_matvec(torch.empty(0, 64, dtype=BF16, device=DEV), _packed(q, s, z, 32, False), torch.empty(0, 16, dtype=BF16, device=DEV)) == mb.MOE_OK


def test_captured_twice_and_on_streams():
    q, s, z = _weight(2048, 512, 128, 19)
    W = _packed(q, s, z, 128, True)
    xs = [_tokens(4, 2048, 20 + i).to(DEV) for i in range(2)]
    outs = [torch.empty(4, 256, dtype=BF16, device=DEV) for _ in range(2)]
    mb.moe_w4_matvec(xs[0], W, outs[0])
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, x, o in zip(graphs, xs, outs):
        with torch.cuda.graph(g):
            mb.moe_w4_matvec(x, W, o)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(3):
        for i, x in enumerate(xs):
            x.copy_(_tokens(4, 2048, 40 + 2 * turn + i))
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):           # (both at once)
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for x, o in zip(xs, outs):
            eager = torch.empty_like(o)
            mb.moe_w4_matvec(x, W, eager)
            assert torch.equal(eager, o)
