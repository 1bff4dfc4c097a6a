"""Residual addition, norm and rows in 8 bits against 64 bits."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import block_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def _rows(T, H, seed, dtype, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, H, generator=g)
    x[:, torch.rand(H, generator=g) < 0.02] *= 16.0
    if kind == "zero rows":
        x[T // 2] = 0.0
        x[0] = 0.0
    elif kind == "tiny":
        x *= 1e-30
    elif kind == "huge":
        x *= 1e36
    return x.to(dtype)


def _relative(H):
    """Of y in fp32: a sum of H squares is at most H / 64 + 16 additions deep where a row is spread over 64 threads at least, and no term is negative;
    its half, and five more roundings of the root, the quotient and the products."""
    return ((H / 64 + 16) / 2 + 5) * 2.0 ** -24


def _check_codes(rows, y, slack):
    """rows against y float64: the scale of the largest, codes nearest to y / scale."""
    T = y.shape[0]
    codes, scales = rows.codes[:T].cpu().view(torch.float8_e4m3fn).double(), rows.scales[:T].cpu().double()
    bad = ~torch.isfinite(y).all(1)
    assert bool(torch.isnan(scales[bad]).all()) and bool(torch.isnan(codes[bad]).all())
    y, codes, scales = y[~bad], codes[~bad], scales[~bad]
    want = ref.row_scales(y)
    assert bool(((scales - want).abs() <= (slack + 2.0 ** -23) * want).all())
    v = y / scales[:, None]
    assert bool(((codes - v).abs() <= ref.half_step(v) * (1 + 2.0 ** -20) + v.abs() * (slack + 2.0 ** -22)).all())


def _check(x, residual, weight, eps=1e-6, want_y=True, want_rows=True, want_sum=True, to=lambda t: t.to(DEV)):
    T, H = x.shape
    xg, rg, wg = (None if t is None else to(t) if t.dim() == 2 else t.to(DEV) for t in (x, residual, weight))
    total = torch.full((T + 1, H), 7.0, dtype=residual.dtype, device=DEV) if residual is not None and want_sum else None
    y = torch.full((T + 1, H), 7.0, dtype=BF16, device=DEV) if want_y else None
    rows = mb.Fp8Rows(T + 1, H, DEV) if want_rows else None
    if rows:
        rows.codes.fill_(9)
        rows.scales.fill_(9.0)
    mb.moe_add_norm(xg, wg, eps, residual=rg, residual_out=total, y=y, rows=rows)
    h, want = ref.add_norm(x, residual, weight, eps)
    slack = _relative(H)
    if total is not None:
        assert torch.allclose(total[:T].cpu(), h, rtol=0, atol=0, equal_nan=True) and bool((total[T] == 7.0).all())
    if want_y:
        got = y[:T].cpu().double()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and bool((y[T] == 7.0).all())
        ok = torch.isfinite(want)
        assert bool(((got - want).abs() <= want.abs() * (2.0 ** -8 + slack) + 2.0 ** -133)[ok].all())
    if rows:
        bad = ~torch.isfinite(want).all(1) | ~torch.isfinite(h.double()).all(1)
        _check_codes(rows, torch.where(bad[:, None], float("nan"), want), slack)
        assert bool((rows.codes[T] == 9).all()) and float(rows.scales[T]) == 9.0


@pytest.mark.parametrize("T,H", [(1, 1), (1, 2048), (3, 7), (5, 64), (2, 65), (33, 520), (7, 1408), (4, 2049), (3, 3583), (2, 7168), (2, 16384), (2, 16385), (1, 20000), (1, 65536),
                                 (9, 9), (17, 4091), (9, 65535)])
@pytest.mark.parametrize("x,residual,weight", [(BF16, BF16, BF16), (BF16, None, BF16), (BF16, F32, F32), (F32, F32, BF16), (F32, BF16, F32), (F32, None, None), (BF16, BF16, None)])
def test_add_norm(T, H, x, residual, weight):
    w = None if weight is None else (1 + 0.2 * torch.randn(H, generator=torch.Generator().manual_seed(H))).to(weight)
    _check(_rows(T, H, 1, x), None if residual is None else _rows(T, H, 2, residual), w)


@pytest.mark.parametrize("outputs", [(True, False, False), (False, True, False), (False, False, True), (True, True, False), (False, True, True)])
def test_outputs_alone(outputs):
    y, rows, total = outputs
    _check(_rows(9, 520, 3, BF16), _rows(9, 520, 4, BF16), _rows(1, 520, 5, F32)[0], want_y=y, want_rows=rows, want_sum=total)


@pytest.mark.parametrize("kind,eps", [("zero rows", 1e-6), ("zero rows", 0.0), ("tiny", 0.0), ("tiny", 1e-6), ("huge", 1e-6)])
@pytest.mark.parametrize("H", [100, 1024])
def test_ranges(kind, eps, H):
    """Rows of zeros; squares that leave fp32 at either end."""
    _check(_rows(5, H, 6, F32, kind), None, _rows(1, H, 7, F32)[0], eps=eps)
    _check(_rows(5, H, 6, BF16, kind), _rows(5, H, 8, BF16, kind), None, eps=eps)


@pytest.mark.parametrize("H", [100, 1024, 7168])
@pytest.mark.parametrize("w_size", [1e-32, 1e-31, 1e-29])
@pytest.mark.parametrize("eps", [0.0, 1e-24])
def test_products_below_fp32(H, w_size, eps):
    """h in range, its products with the weight below fp32's normal numbers (hardly a bit of them left at 1e-32), y in range again.  Scales are above 1e-35, of which a last
    bit of fp32 is 2^-32: the roundings of a small y, of its quotient and of that one's remainder stay below the 2^-30 that the least half step is widened by."""
    w = _rows(1, H, 26, F32)[0] * w_size
    _check(_rows(5, H, 27, F32) * 2e-13, None, w, eps=eps)
    _check((_rows(5, H, 28, BF16).float() * 2e-13).to(BF16), _rows(5, H, 29, F32) * 2e-13, w, eps=eps)


def test_not_finite():
    x, w = _rows(6, 264, 9, BF16), _rows(1, 264, 10, F32)[0]
    x[1, 3], x[2, 263], x[4, 0] = float("nan"), float("inf"), -float("inf")
    _check(x, None, w)
    w[17] = float("inf")                             # every row then
    _check(x, None, w)
    w[17] = float("nan")
    _check(x, _rows(6, 264, 11, F32), w)


def test_rows_apart_and_unaligned():
    def inside(t):
        wide = torch.full((t.shape[0], t.shape[1] + 21), 3.0, dtype=t.dtype, device=DEV)
        wide[:, 5: 5 + t.shape[1]] = t.to(DEV)
        return wide[:, 5: 5 + t.shape[1]]
    _check(_rows(8, 512, 12, BF16), _rows(8, 512, 13, BF16), _rows(1, 512, 14, BF16)[0], to=inside)
    _check(_rows(8, 129, 12, F32), _rows(8, 129, 13, BF16), None, to=inside)

    def in_step(t):                                  # rows that begin as far from 16 bytes as those of the outputs, and do not follow one another
        wide = torch.full((t.shape[0], t.shape[1] + 24), 3.0, dtype=t.dtype, device=DEV)
        wide[:, 8: 8 + t.shape[1]] = t.to(DEV)
        return wide[:, 8: 8 + t.shape[1]]
    for H in (9, 15, 77, 1001, 5143):
        _check(_rows(11, H, 23, BF16), _rows(11, H, 24, F32), _rows(1, H, 25, BF16)[0], to=in_step)
        _check(_rows(11, H, 23, F32), _rows(11, H, 24, BF16), _rows(1, H, 25, F32)[0], to=in_step)

    def every_other(t):
        wide = torch.full((2 * t.shape[0], t.shape[1]), 3.0, dtype=t.dtype, device=DEV)
        wide[::2] = t.to(DEV)
        return wide[::2]
    _check(_rows(8, 512, 15, BF16), _rows(8, 512, 16, F32), None, to=every_other)


def test_in_place():
    """The sum over the residual, and over x."""
    for H in (776, 777, 4099):
        x, r = _rows(11, H, 17, BF16), _rows(11, H, 18, BF16)
        h, want = ref.add_norm(x, r, None, 1e-6)
        for over in (0, 1):
            xg, rg, y = x.to(DEV), r.to(DEV), torch.empty(11, H, dtype=BF16, device=DEV)
            mb.moe_add_norm(xg, None, 1e-6, residual=rg, residual_out=(xg, rg)[over], y=y)
            assert torch.equal((xg, rg)[over].cpu(), h)
            assert bool(((y.cpu().double() - want).abs() <= want.abs() * (2.0 ** -8 + _relative(H))).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,H", [(1, 1), (3, 8), (5, 77), (768, 1408), (9, 3585), (3, 14336), (2, 16392), (1, 40001)])
def test_quantize(T, H, dtype):
    for kind in ("normal", "zero rows", "tiny", "huge"):
        x = _rows(T, H, 19, dtype, kind)
        rows = mb.Fp8Rows(T, H, DEV).quantize(x.to(DEV))
        _check_codes(rows, x.double(), 0.0)
        assert torch.equal(rows.scales.cpu(), (x.float().abs().amax(1) / 448.0).clamp(min=2.0 ** -126))


def test_quantize_not_finite_and_apart():
    x = _rows(7, 400, 20, BF16)
    x[1, 399], x[3, 0], x[5, 7] = float("nan"), float("inf"), -float("inf")
    wide = torch.zeros(7, 433, dtype=BF16, device=DEV)
    wide[:, 3:403] = x.to(DEV)
    rows = mb.Fp8Rows(9, 400, DEV)
    rows.codes.fill_(5)
    rows.quantize(wide[:, 3:403])
    _check_codes(rows, torch.where(torch.isfinite(x.double()).all(1, keepdim=True), x.double(), float("nan")), 0.0)
    assert bool((rows.codes[7:] == 5).all())


def test_no_rows():
    assert mb.moe_add_norm(torch.empty(0, 64, device=DEV), None, 1e-6, y=torch.empty(0, 64, dtype=BF16, device=DEV)) == mb.MOE_OK
    assert mb.moe_fp8_quantize(torch.empty(0, 64, device=DEV), mb.Fp8Rows(0, 64, DEV)) == mb.MOE_OK


def test_captured():
    x, r = _rows(16, 2048, 21, BF16).to(DEV), _rows(16, 2048, 22, BF16).to(DEV)
    y, rows, total = torch.empty(16, 2048, dtype=BF16, device=DEV), mb.Fp8Rows(16, 2048, DEV), torch.empty_like(r)
    mb.moe_add_norm(x, None, 1e-6, residual=r, residual_out=total, y=y, rows=rows)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mb.moe_add_norm(x, None, 1e-6, residual=r, residual_out=total, y=y, rows=rows)
    for turn in range(3):
        x.copy_(_rows(16, 2048, 30 + turn, BF16))
        graph.replay()
        got = [t.clone() for t in (total, y, rows.codes, rows.scales)]
        mb.moe_add_norm(x, None, 1e-6, residual=r, residual_out=total, y=y, rows=rows)
        assert all(torch.equal(a, b) for a, b in zip(got, (total, y, rows.codes, rows.scales)))
