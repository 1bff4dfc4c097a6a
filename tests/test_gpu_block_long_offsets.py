"""Offsets beyond 32 bits in the operators around a block's experts."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import block_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def _memory():
    yield
    torch.cuda.empty_cache()


def test_rows():
    """66000 rows of 65536: the last codes lie beyond 2^32 bytes, the last elements beyond 2^33."""
    T, H = 66000, 65536
    assert T * H > 1 << 32
    x = torch.zeros(T, H, dtype=BF16, device=DEV)
    last = torch.randn(3, H, generator=torch.Generator().manual_seed(1)).to(BF16)
    x[-3:] = last.to(DEV)
    rows = mb.Fp8Rows(T, H, DEV)
    y = torch.empty(T, H, dtype=BF16, device=DEV)
    mb.moe_add_norm(x, None, 1e-6, y=y, rows=rows)
    _, want = ref.add_norm(last, None, None, 1e-6)
    slack = (H / 1024 + 16) * 2.0 ** -24             # as deep as a sum over 1024 threads and its joining, and a few roundings
    assert bool(((y[-3:].cpu().double() - want).abs() <= want.abs() * (2.0 ** -8 + slack)).all())
    v = want / rows.scales[-3:].cpu().double()[:, None]
    codes = rows.codes[-3:].cpu().view(torch.float8_e4m3fn).double()
    assert bool(((codes - v).abs() <= ref.half_step(v) * (1 + 2.0 ** -20) + v.abs() * (slack + 2.0 ** -22)).all())
    assert int(rows.codes[:-3].max()) == 0 and float(y[:-3].abs().max()) == 0.0
    rows.quantize(x)
    assert torch.equal(rows.scales[-3:].cpu(), last.float().abs().amax(1) / 448.0)
    v = last.double() / rows.scales[-3:].cpu().double()[:, None]
    codes = rows.codes[-3:].cpu().view(torch.float8_e4m3fn).double()
    assert bool(((codes - v).abs() <= ref.half_step(v) * (1 + 2.0 ** -20) + v.abs() * 2.0 ** -22).all())


def test_more_rows_than_a_launch():
    T, H = (1 << 22) + 4099, 9
    g = torch.Generator().manual_seed(6)
    x = torch.zeros(T, H, dtype=BF16, device=DEV)
    places = torch.cat([torch.arange(0, 3), torch.arange((1 << 22) - 4, (1 << 22) + 4), torch.arange(T - 3, T)])
    some = torch.randn(len(places), H, generator=g).to(BF16)
    x[places.to(DEV)] = some.to(DEV)
    y, rows = torch.empty(T, H, dtype=BF16, device=DEV), mb.Fp8Rows(T, H, DEV)
    mb.moe_add_norm(x, None, 1e-6, y=y, rows=rows)
    _, want = ref.add_norm(some, None, None, 1e-6)
    at = places.to(DEV)
    assert bool(((y[at].cpu().double() - want).abs() <= want.abs() * (2.0 ** -8 + 32 * 2.0 ** -24)).all())
    assert int((y != 0).any(1).sum()) == len(places) and int((rows.codes != 0).any(1).sum()) == len(places)
    rows.codes.fill_(1)
    rows.quantize(x)
    assert torch.equal(rows.scales[at].cpu(), some.float().abs().amax(1) / 448.0) and int((rows.codes != 0).any(1).sum()) == len(places)


def test_logits_far_apart():
    wide = torch.empty(1100, 1 << 22, dtype=BF16, device=DEV)
    assert wide.numel() > 1 << 32
    x = torch.randn(1100, 64, generator=torch.Generator().manual_seed(2)).to(BF16)
    wide[:, :64] = x.to(DEV)
    ids, w = torch.empty(1100, 6, dtype=torch.int32, device=DEV), torch.empty(1100, 6, device=DEV)
    mb.moe_route_grouped(wide[:, :64], 6, ids, w, 8, 4)
    want, weights = ref.route_grouped(x[-40:], 6, 8, 4, False, None, False, True, 1.0)
    assert torch.equal(ids[-40:].cpu(), want)
    assert bool(((w[-40:].cpu().double() - weights).abs() <= 1.01 * 2.0 ** -24 * weights).all())


def test_weights_of_more_than_four_gibibytes():
    """All codes 0 and all zero points 8, but for the last tile of 16 columns x 128 k, whose codes are 15."""
    K, N = 1 << 16, 1 << 18
    W = mb.W4Weights(K, N, 128, device=DEV)
    assert W.codes.numel() > 1 << 32
    W.codes.zero_()
    scale = 2.0 ** -10
    W.words.view(torch.int32).fill_(int(torch.tensor(scale).view(torch.int32)) | 8)
    W.codes[-1024:] = 0xff
    x = torch.randn(2, K, generator=torch.Generator().manual_seed(3)).to(BF16)
    out = torch.empty(2, N, dtype=BF16, device=DEV)
    mb.moe_w4_matvec(x.to(DEV), W, out)
    total, tail = x.double().sum(1, keepdim=True), x[:, -128:].double().sum(1, keepdim=True)
    want = (-8 * total).expand(2, N).clone()
    want[:, -16:] += 15 * tail
    want *= scale
    bound = (2 * 128 + 4) * 2.0 ** -24 * 286 * scale * x.double().abs().sum(1, keepdim=True) + (2 * K / 128 + 32) * 2.0 ** -24 * 16 * scale * x.double().abs().sum(1, keepdim=True)
    assert bool(((out.cpu().double() - want).abs() <= bound + want.abs() * 2.0 ** -8).all())
    assert bool((out[:, :-16] == out[:, :1]).all()) and not bool((out[:, -16:] == out[:, :1]).any())


def test_tokens_far_apart():
    q = torch.randint(0, 16, (256, 32), generator=torch.Generator().manual_seed(4), dtype=torch.uint8)
    s = torch.full((2, 32), 0.01, dtype=BF16)
    W = mb.W4Weights(256, 32, 128, device=DEV).pack(q.to(DEV), s.to(DEV))
    wide = torch.empty(16, (1 << 28) + 8, dtype=BF16, device=DEV)
    assert wide.numel() > 1 << 32
    x = torch.randn(16, 256, generator=torch.Generator().manual_seed(5)).to(BF16)
    wide[:, :256] = x.to(DEV)
    out, near = torch.empty(16, 32, dtype=BF16, device=DEV), torch.empty(16, 32, dtype=BF16, device=DEV)
    mb.moe_w4_matvec(wide[:, :256], W, out)
    mb.moe_w4_matvec(x.to(DEV), W, near)
    assert torch.equal(out, near)


def test_sizes_beyond_32_bits_are_refused():
    """A row of 2^32 + 64 elements is not one of 64, and 2^32 + 8 rows are not 8."""
    row = torch.empty(1, (1 << 32) + 64, dtype=BF16, device=DEV)
    ids, w = torch.empty(1, 2, dtype=torch.int32, device=DEV), torch.empty(1, 2, device=DEV)
    y = torch.empty(1, 64, dtype=BF16, device=DEV)
    assert mb.moe_route_grouped(row, 2, ids, w, 8, 4, check=False) == mb.MOE_ERR_INVALID_ARG
    assert mb.moe_add_norm(row, None, 1e-6, y=row, check=False) == mb.MOE_ERR_INVALID_ARG
    assert mb.moe_add_norm(row[:, :64], None, 1e-6, y=y, check=False) == mb.MOE_OK
    column = row.reshape(-1, 1)[: (1 << 32) + 8]
    W = mb.W4Weights(1, 1, 32, device=DEV)
    assert mb.moe_w4_matvec(column, W, column, check=False) == mb.MOE_ERR_INVALID_ARG
