"""The bindings of the router and of the 4-bit operators refuse buffers that are smaller than what the call would write or read, and
types that it would misread: the C entry points see addresses only.  Nothing is launched."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb

BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
T, K_, E, K, N = 10, 2, 8, 200, 96          # rows of 256 elements in 4 bits: 128 bytes of codes, 8 of scales


def _refused(call, *args, **kw):
    assert call(*args, check=False, **kw) == mb.MOE_ERR_INVALID_ARG
    with pytest.raises(mb.MoeError) as error:
        call(*args, **kw)
    assert error.value.code == mb.MOE_ERR_INVALID_ARG


def _e(*shape, dtype=U8):
    return torch.empty(*shape, dtype=dtype)


@pytest.mark.parametrize("ids,weights", [(_e(T, K_, dtype=torch.int64), _e(T, K_, dtype=F32)), (_e(T, K_, dtype=I32), _e(T, K_, dtype=BF16)),
                                         (_e(T, K_ - 1, dtype=I32), _e(T, K_, dtype=F32)), (_e(T, K_, dtype=I32), _e(T - 1, K_, dtype=F32)),
                                         (_e(K_, T, dtype=I32).t(), _e(T, K_, dtype=F32)), (_e(T, K_, dtype=I32), _e(T, 2 * K_, dtype=F32)[:, :K_])])
def test_route(ids, weights):
    _refused(mb.moe_route, _e(T, E, dtype=F32), K_, ids, weights)


@pytest.mark.parametrize("codes,scales,values", [(_e(T * 128 - 1), _e(T * 8), None), (_e(T * 128), _e(T * 8 - 1), None), (_e(T * 256)[::2], _e(T * 8), None),
                                                 (_e(T * 128), _e(T * 8), _e(T, K - 1, dtype=BF16)), (_e(T * 128), _e(T * 8), _e(T, K, dtype=torch.float16)),
                                                 (_e(T * 128), _e(T * 8), _e(T, K + 8, dtype=BF16)[:, :K])])
def test_quantize(codes, scales, values):
    _refused(mb.moe_mx4_quantize, _e(T, K, dtype=BF16), codes, scales, values)


def _map(rows=T, k=K_):
    return torch.empty(mb.moe_task_map_bytes(rows, k, E, 16, 256, N) // 4, dtype=I32)


@pytest.mark.parametrize("ids,task_map,codes,scales", [(_e(T, K_, dtype=torch.int64), _map(), _e(T * 128), _e(T * 8)), (_e(T - 1, K_, dtype=I32), _map(), _e(T * 128), _e(T * 8)),
                                                       (_e(T, K_, dtype=I32), _map()[:100], _e(T * 128), _e(T * 8)), (_e(T, K_, dtype=I32), _map(), _e(T * 128 - 1), _e(T * 8)),
                                                       (_e(T, K_, dtype=I32), _map(), _e(T * 128), _e(T * 8 - 1)), (_e(K_, T, dtype=I32).t(), _map(), _e(T * 128), _e(T * 8))])
def test_prepare(ids, task_map, codes, scales):
    _refused(mb.moe_mx4_prepare, ids, T, K_, E, N, mb.Tiling(16, 256), task_map, _e(T, K, dtype=BF16), codes, scales)


@pytest.mark.parametrize("W,codes,scales,values", [
    (_e(E, K, N - 1, dtype=BF16), 0, 0, None), (_e(E, N, K, dtype=BF16).transpose(1, 2), 0, 0, None), (_e(E, K, N, dtype=BF16), 1, 0, None),
    (_e(E, K, N, dtype=BF16), 0, 1, None), (_e(E, K, N, dtype=BF16), 0, 0, _e(E, K, N - 1, dtype=BF16)), (_e(E, K, N, dtype=BF16), 0, 0, _e(E, K, N, dtype=F32))])
def test_pack_weights(W, codes, scales, values):
    buffers = _e(mb.moe_mx4_weight_code_bytes(E, K, N) - codes), _e(mb.moe_mx4_weight_scale_bytes(E, K, N) - scales)
    _refused(mb.moe_mx4_pack_weights, W, mb.MOE_W_LAYOUT_KN, E, K, N, False, *buffers, values)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("case", ["rows", "cols", "Y", "Y type", "Y strides", "map", "map type"])
def test_product(case, gated):
    rows = mb.Mx4Rows(T - (case == "rows"), K + 128 * (case == "cols"), device="cpu")
    weights = mb.Mx4Weights(E, K, N, gated, device="cpu")
    out = N // 2 if gated else N
    Y = _e(T, K_, out - (case == "Y"), dtype=F32 if case == "Y type" else BF16)
    if case == "Y strides":
        Y = _e(T, K_, out + 8, dtype=BF16)[:, :, :out]
    task_map = torch.empty(mb.moe_task_map_bytes(T, K_, E, 16, 256, mb.moe_mx4_packed_columns(N, gated)) // 4, dtype=I32)
    if case == "map":
        task_map = task_map[:-64]
    if case == "map type":
        task_map = task_map.view(F32)
    _refused(mb.moe_mx4_grouped_gemm, rows, weights, T, K_, task_map, Y, mb.Tiling(16, 256))
