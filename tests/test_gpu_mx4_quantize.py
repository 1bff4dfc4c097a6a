"""Quantisation to 4 bits with a scale for every 32: codes, scales and values bit by bit against the definition in 64 bits."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import mx4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _mixed(rows, cols, seed, dtype):
    """Normal values of very different magnitudes from block to block, ties, exact elements, zeros of both signs and whole zero blocks."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g)
    x *= torch.exp2(torch.randint(-40, 40, (rows, (cols + 31) // 32), generator=g).float()).repeat_interleave(32, 1)[:, :cols]
    grid = torch.tensor([0.0, -0.0, 0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0, 7.0, -0.25, -2.5, -5.0, -7.5])
    pick = torch.randint(0, len(grid), (rows, cols), generator=g)
    exact = torch.rand(rows, cols, generator=g) < 0.4
    x = torch.where(exact, grid[pick], x)
    if rows > 2:
        x[rows // 2] = 0.0
        x[rows // 2 + 1, : cols // 2] = -0.0
    return x.to(dtype)


def _check_rows(x_gpu, x_cpu):
    rows, cols = x_cpu.shape
    held = mb.Mx4Rows(rows, cols, DEV)
    held.codes.fill_(0xA5)
    held.scales.fill_(0xA5)
    values = torch.full((rows, cols), 7.0, dtype=torch.bfloat16, device=DEV)
    held.quantize(x_gpu, values=values)
    code, byte, val = ref.quantize(x_cpu)
    assert torch.equal(held.codes.cpu().reshape(rows, -1), ref.packed_rows(code))
    assert torch.equal(held.scales.cpu().reshape(rows, -1), byte)
    got = values.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(val))
    ok = ~torch.isnan(val)
    assert torch.equal(got[ok], val[ok])
    assert torch.equal(torch.signbit(got[ok]), torch.signbit(val[ok]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (3, 33), (7, 127), (2, 128), (5, 129), (130, 264), (64, 2048), (9, 1416), (33, 7168)])
def test_rows(rows, cols, dtype):
    x = _mixed(rows, cols, rows * 10007 + cols, dtype)
    _check_rows(x.to(DEV), x)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_extremes(dtype):
    """Infinities, NaN, the type's largest and smallest values, subnormals: one block each."""
    big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).tiny
    sub = 2.0 ** -133 if dtype == torch.bfloat16 else 2.0 ** -149
    x = torch.zeros(14, 64)
    x[0, 3], x[1, 40], x[2, 0] = float("inf"), float("nan"), -float("inf")
    x[3, :32], x[4, 5], x[5, 7] = big, -big, tiny
    x[6, :4] = torch.tensor([sub, -sub, 3 * sub, tiny / 2])
    x[7, 0], x[7, 1] = big, 1.0
    x[8, 0], x[8, 1], x[8, 2] = 2.0 ** -125, 2.0 ** -127, 2.0 ** -128
    x[9, 0], x[9, 1] = 2.0 ** -124, -(2.0 ** -126)
    x[10, 0] = 1.9921875          # just below 2: exponent 0, and 7.97 / 4 ends at 6
    x[11, 0], x[11, 33] = float("nan"), 5.0
    x[12, 31], x[12, 32] = 6.0, 6.0
    x[13, 0], x[13, 1] = tiny, float("inf")
    x = x.to(dtype)
    _check_rows(x.to(DEV), x)


def test_strided_and_unaligned_rows():
    base = _mixed(20, 900, 5, torch.bfloat16)
    gpu = base.to(DEV)
    for lo, hi in ((0, 256), (8, 264), (1, 257), (3, 500), (16, 900)):
        _check_rows(gpu[:, lo:hi], base[:, lo:hi])
    _check_rows(gpu[::3, 8:136], base[::3, 8:136])
    one = _mixed(6, 161, 8, torch.float32)
    _check_rows(one.to(DEV)[:, 1:], one[:, 1:])
    # values on an odd address
    x = _mixed(4, 256, 9, torch.bfloat16)
    out = torch.empty(4 * 256 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(4, 256)
    mb.Mx4Rows(4, 256, DEV).quantize(x.to(DEV), values=out)
    assert torch.equal(out.cpu().double(), ref.quantize(x)[2])


def test_values_are_a_fixed_point():
    """What the codes stand for is quantised to itself: converting a 4-bit checkpoint through its values loses nothing."""
    x = torch.randn(40, 512, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
    a, b = torch.empty_like(x), torch.empty_like(x)
    mb.Mx4Rows(40, 512, DEV).quantize(x, values=a)
    mb.Mx4Rows(40, 512, DEV).quantize(a, values=b)
    assert torch.equal(a, b)


@pytest.mark.parametrize("layout", [mb.MOE_W_LAYOUT_KN, mb.MOE_W_LAYOUT_NK])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,K,N,gated", [(1, 1, 1, False), (1, 1, 2, True), (2, 32, 64, False), (3, 130, 70, False), (2, 256, 128, True),
                                         (2, 100, 50, True), (1, 264, 98, True), (2, 128, 192, False), (1, 520, 256, True)])
def test_weights(E, K, N, gated, dtype, layout):
    W = _mixed(E * N, K, E * 1000 + K + N, dtype).reshape(E, N, K).transpose(1, 2).contiguous()
    src = W if layout == mb.MOE_W_LAYOUT_KN else W.transpose(1, 2).contiguous()
    codes, scales, val = ref.packed_weights(W, gated)
    held = mb.Mx4Weights(E, K, N, gated, DEV)
    held.codes.fill_(0xA5)
    held.scales.fill_(0xA5)
    values = torch.full(src.shape, 7.0, dtype=torch.bfloat16, device=DEV)
    held.pack(src.to(DEV), layout, values=values)
    assert held.codes.numel() == codes.numel() and held.scales.numel() == scales.numel()
    assert torch.equal(held.codes.cpu(), codes)
    assert torch.equal(held.scales.cpu(), scales)
    got = values.cpu().double() if layout == mb.MOE_W_LAYOUT_KN else values.cpu().double().transpose(1, 2)
    assert torch.equal(got, val)
    # expert by expert: the same bytes
    single = mb.Mx4Weights(E, K, N, gated, DEV)
    for e in range(E):
        single.pack_expert(e, src[e].to(DEV), layout)
    assert torch.equal(single.codes, held.codes) and torch.equal(single.scales, held.scales)


def test_weight_blocks_that_are_not_numbers():
    W = torch.randn(1, 160, 80, generator=torch.Generator().manual_seed(1))
    W[0, 5, 3], W[0, 40, 3], W[0, 159, 79] = float("nan"), float("inf"), -float("inf")
    codes, scales, val = ref.packed_weights(W, False)
    held, values = mb.Mx4Weights(1, 160, 80, False, DEV), torch.empty(1, 160, 80, dtype=torch.bfloat16, device=DEV)
    held.pack(W.to(DEV), values=values)
    assert torch.equal(held.codes.cpu(), codes) and torch.equal(held.scales.cpu(), scales)
    assert torch.equal(torch.isnan(values.cpu()), torch.isnan(val)) and int(torch.isnan(val).sum()) == 32 * 3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,k,E,cols,tile_m", [
    (1, 1, 1, 1, 16), (1, 6, 64, 2048, 16), (7, 3, 5, 130, 32), (128, 6, 64, 264, 16), (500, 2, 8, 136, 128), (1025, 1, 9, 40, 32), (1111, 8, 64, 96, 128),
    (4096, 4, 8, 64, 128), (4097, 4, 256, 33, 128), (16385, 1, 1000, 16, 16)])
def test_map_and_rows_by_one_launch_are_those_of_two(T, k, E, cols, tile_m, dtype):
    g = torch.Generator().manual_seed(T + E)
    ids = torch.rand(T, E, generator=g).topk(k, 1).indices.int().to(DEV)
    if T > 4:
        ids[T // 2] = -1                 # (an id that is no expert: counted as bad by both)
    wide = torch.randn(T, cols + 8, generator=g).to(dtype).to(DEV)
    tiling = mb.Tiling(tile_m, 256)
    for x in (wide[:, :cols], wide[:, :cols].contiguous(), wide[:, 1:cols + 1]):
        got, want = [], []
        for out in (got, want):
            task_map, rows = mb.alloc_task_map(T, k, E, tile_m, 256, 512, DEV), mb.Mx4Rows(T, cols, DEV)
            for t in (task_map, rows.codes, rows.scales):
                t.fill_(77)
            out += [task_map, rows.codes, rows.scales]
        mb.moe_mx4_prepare(ids, T, k, E, 512, tiling, got[0], x, *got[1:])
        mb.moe_build_task_map_ex(ids, T, k, E, 512, tiling, want[0])
        mb.moe_mx4_quantize(x, *want[1:])
        for a, b in zip(got, want):
            assert torch.equal(a, b)
