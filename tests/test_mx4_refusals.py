"""What the 4-bit operators, the router and the layer for few tokens refuse, and what their host-only functions say.  Addresses are
made up: nothing is launched before a check."""
import ctypes

import pytest

from paper_2501_16103_amd import binding as mb

P = 1 << 20          # an aligned address that nobody reads
INVALID, UNSUPPORTED = mb.MOE_ERR_INVALID_ARG, mb.MOE_ERR_UNSUPPORTED


def _route(logits=P, ids=P, weights=P, **kw):
    d = dict(T=4, k=2, E=8, dtype=mb.MOE_DTYPE_FP32, row_stride=8, score=0, renormalize=1, scale=1.0)
    d.update(kw)
    return mb.lib().moe_route(logits, ctypes.byref(mb.moe_route_desc(**d)), ids, weights, None)


@pytest.mark.parametrize("kw,rc", [(dict(T=-1), INVALID), (dict(k=0), INVALID), (dict(k=9), INVALID), (dict(E=0), INVALID), (dict(score=2), INVALID),
                                   (dict(dtype=mb.MOE_DTYPE_FP8_E4M3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(E=1025, row_stride=1025), UNSUPPORTED),
                                   (dict(T=1 << 24), UNSUPPORTED), (dict(row_stride=7), INVALID), (dict(logits=None), INVALID), (dict(ids=None), INVALID),
                                   (dict(weights=None), INVALID), (dict(logits=P + 2), INVALID), (dict(ids=P + 1), INVALID), (dict(weights=P + 2), INVALID),
                                   (dict(dtype=mb.MOE_DTYPE_BF16, logits=P + 1), INVALID), (dict(T=0, logits=None), mb.MOE_OK)])
def test_route(kw, rc):
    assert _route(**kw) == rc


def test_null_descriptions():
    lib = mb.lib()
    assert lib.moe_route(P, None, P, P, None) == INVALID
    assert lib.moe_mx4_grouped_gemm(P, P, P, P, P, P, None, None) == INVALID
    assert lib.moe_layer_few_tokens(P, P, P, P, P, P, None, P, P, P, P, 1 << 30, None) == INVALID
    assert lib.moe_few_tokens_workspace_bytes(None) == 0
    assert lib.moe_mx4_default_tiling(4, 2, 8, 64, 64, 0, None) == INVALID


def _quantize(src=P, dtype=mb.MOE_DTYPE_BF16, rows=4, cols=100, stride=100, codes=P, scales=P, values=None):
    return mb.lib().moe_mx4_quantize(src, dtype, rows, cols, stride, codes, scales, values, None)


@pytest.mark.parametrize("kw,rc", [(dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(stride=99), INVALID), (dict(dtype=mb.MOE_DTYPE_FP8_E4M3), UNSUPPORTED),
                                   (dict(dtype=-1), UNSUPPORTED), (dict(src=None), INVALID), (dict(codes=None), INVALID), (dict(scales=None), INVALID),
                                   (dict(codes=P + 8), INVALID), (dict(scales=P + 2), INVALID), (dict(values=P + 1), INVALID), (dict(src=P + 1), INVALID),
                                   (dict(dtype=mb.MOE_DTYPE_FP32, src=P + 2), INVALID), (dict(rows=1 << 32, cols=8, stride=8), UNSUPPORTED),
                                   (dict(rows=1 << 31, cols=1 << 10, stride=1 << 10), UNSUPPORTED), (dict(rows=0, src=None), mb.MOE_OK)])
def test_quantize(kw, rc):
    assert _quantize(**kw) == rc


def _prepare(ids=P, T=4, k=2, E=8, N=256, tile=(16, 256, 0, 0, 0, 0), task_map=P, X=P, dtype=mb.MOE_DTYPE_BF16, K=100, stride=100, codes=P, scales=P):
    g = ctypes.byref(mb.moe_tiling(*tile)) if tile else None
    return mb.lib().moe_mx4_prepare(ids, T, k, E, N, g, task_map, X, dtype, K, stride, codes, scales, None)


@pytest.mark.parametrize("kw,rc", [(dict(tile=None), INVALID), (dict(T=-1), INVALID), (dict(k=0), INVALID), (dict(k=9), INVALID), (dict(E=0), INVALID), (dict(N=0), INVALID),
                                   (dict(E=1025), UNSUPPORTED), (dict(T=1 << 23, k=8), UNSUPPORTED), (dict(tile=(16, 100, 0, 0, 0, 0)), UNSUPPORTED),
                                   (dict(tile=(16, 256, 5, 0, 0, 0)), INVALID), (dict(tile=(16, 256, 0, 0, 0, 16)), INVALID), (dict(ids=None), INVALID),
                                   (dict(ids=P + 2), INVALID), (dict(task_map=None), INVALID), (dict(task_map=P + 8), INVALID), (dict(X=None), INVALID),
                                   (dict(X=P + 1), INVALID), (dict(dtype=mb.MOE_DTYPE_FP8_E4M3), UNSUPPORTED), (dict(K=0), INVALID), (dict(stride=99), INVALID),
                                   (dict(codes=P + 8), INVALID), (dict(scales=P + 2), INVALID), (dict(codes=None), INVALID), (dict(scales=None), INVALID)])
def test_prepare(kw, rc):
    assert _prepare(**kw) == rc


def _pack(W=P, dtype=mb.MOE_DTYPE_BF16, layout=0, E=2, K=64, N=64, gated=0, codes=P, scales=P, values=None):
    return mb.lib().moe_mx4_pack_weights(W, dtype, layout, E, K, N, gated, codes, scales, values, None)


@pytest.mark.parametrize("kw,rc", [(dict(E=0), INVALID), (dict(K=0), INVALID), (dict(N=0), INVALID), (dict(gated=2), INVALID), (dict(gated=1, N=63), INVALID),
                                   (dict(layout=2), INVALID), (dict(dtype=mb.MOE_DTYPE_FP8_E4M3), UNSUPPORTED), (dict(E=1025), UNSUPPORTED),
                                   (dict(K=(1 << 30) + 1), UNSUPPORTED), (dict(E=1024, K=1 << 15, N=1 << 15), UNSUPPORTED), (dict(W=None), INVALID),
                                   (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(codes=P + 8), INVALID), (dict(scales=P + 4), INVALID),
                                   (dict(values=P + 1), INVALID), (dict(W=P + 1), INVALID), (dict(W=P + 2, dtype=mb.MOE_DTYPE_FP32), INVALID)])
def test_pack(kw, rc):
    assert _pack(**kw) == rc


def _gemm(xc=P, xs=P, wc=P, ws=P, tmap=P, Y=P, **kw):
    d = dict(T=4, k=2, E=8, K=100, N=70, gated=0, tile_m=16, tile_n=256)
    d.update(kw)
    return mb.lib().moe_mx4_grouped_gemm(xc, xs, wc, ws, tmap, Y, ctypes.byref(mb.moe_mx4_gemm_desc(**d)), None)


@pytest.mark.parametrize("kw,rc", [(dict(T=-1), INVALID), (dict(k=0), INVALID), (dict(k=9), INVALID), (dict(E=0, k=1), INVALID), (dict(K=0), INVALID), (dict(N=0), INVALID),
                                   (dict(gated=1, N=71), INVALID), (dict(gated=3), INVALID), (dict(E=1025), UNSUPPORTED), (dict(T=1 << 24), UNSUPPORTED),
                                   (dict(tile_m=48), UNSUPPORTED), (dict(tile_n=512), UNSUPPORTED), (dict(tmap=None), INVALID), (dict(tmap=P + 4), INVALID),
                                   (dict(xc=None), INVALID), (dict(xs=None), INVALID), (dict(wc=None), INVALID), (dict(ws=None), INVALID), (dict(Y=None), INVALID),
                                   (dict(xc=P + 8), INVALID), (dict(xs=P + 2), INVALID), (dict(wc=P + 8), INVALID), (dict(ws=P + 8), INVALID), (dict(Y=P + 2), INVALID),
                                   (dict(T=0, xc=None, Y=None), mb.MOE_OK)])
def test_product(kw, rc):
    assert _gemm(**kw) == rc


def _desc(**kw):
    d = dict(T=4, k=2, E=8, hidden=64, inter=40, w_dtype=mb.MOE_DTYPE_BF16, logits_dtype=mb.MOE_DTYPE_FP32, score=0, renormalize=1, scale=1.0)
    d.update(kw)
    return mb.moe_few_tokens_desc(**d)


def _few(X=P, logits=P, up=P, us=P, down=P, ds=P, ids=P, w=P, out=P, ws=P, nbytes=1 << 40, **kw):
    return mb.lib().moe_layer_few_tokens(X, logits, up, us, down, ds, ctypes.byref(_desc(**kw)), ids, w, out, ws, nbytes, None)


MX4 = dict(w_dtype=mb.MOE_DTYPE_MX4)


@pytest.mark.parametrize("kw,rc", [(dict(T=-1), INVALID), (dict(T=17), UNSUPPORTED), (dict(k=0), INVALID), (dict(k=9), INVALID), (dict(k=17, E=20), UNSUPPORTED),
                                   (dict(E=1025), UNSUPPORTED), (dict(hidden=0), INVALID), (dict(inter=0), INVALID), (dict(hidden=60), UNSUPPORTED),
                                   (dict(inter=44), UNSUPPORTED), (dict(hidden=1 << 21), UNSUPPORTED), (dict(w_dtype=mb.MOE_DTYPE_FP8_E4M3), UNSUPPORTED),
                                   (dict(logits_dtype=mb.MOE_DTYPE_FP8_E4M3), UNSUPPORTED), (dict(logits_dtype=-1), UNSUPPORTED), (dict(score=5), INVALID),
                                   (dict(X=None), INVALID), (dict(logits=None), INVALID), (dict(up=None), INVALID), (dict(down=None), INVALID), (dict(ids=None), INVALID),
                                   (dict(w=None), INVALID), (dict(out=None), INVALID), (dict(ws=None), INVALID), (dict(X=P + 8), INVALID), (dict(up=P + 8), INVALID),
                                   (dict(down=P + 8), INVALID), (dict(out=P + 1), INVALID), (dict(ws=P + 8), INVALID), (dict(ids=P + 2), INVALID), (dict(w=P + 2), INVALID),
                                   (dict(logits=P + 2), INVALID), (dict(us=None, **MX4), INVALID), (dict(ds=None, **MX4), INVALID), (dict(us=P + 8, **MX4), INVALID),
                                   (dict(nbytes=0), INVALID), (dict(T=0, X=None), mb.MOE_OK)])
def test_few_tokens(kw, rc):
    assert _few(**kw) == rc


def test_workspace_is_asked_for():
    for kw in (dict(), MX4):
        need = mb.lib().moe_few_tokens_workspace_bytes(ctypes.byref(_desc(**kw)))
        assert need > 0
        assert _few(nbytes=need - 1, **kw) == INVALID
    assert mb.lib().moe_few_tokens_workspace_bytes(ctypes.byref(_desc(T=17))) == 0
    assert mb.lib().moe_few_tokens_workspace_bytes(ctypes.byref(_desc(T=0))) == 0


def test_sizes():
    assert mb.moe_mx4_row_code_bytes(3, 129) == 3 * 128 and mb.moe_mx4_row_scale_bytes(3, 129) == 3 * 8
    assert mb.moe_mx4_row_code_bytes(0, 64) == 0 and mb.moe_mx4_row_code_bytes(-1, 64) == 0 and mb.moe_mx4_row_code_bytes(4, 0) == 0
    assert mb.moe_mx4_packed_columns(70) == 70 and mb.moe_mx4_packed_columns(70, True) == 96 and mb.moe_mx4_packed_columns(71, True) == 0
    assert mb.moe_mx4_weight_code_bytes(5, 129, 65) == 5 * 2 * 2 * 4096 and mb.moe_mx4_weight_scale_bytes(5, 129, 65) == 5 * 2 * 2 * 256
    assert mb.moe_mx4_weight_code_bytes(1, 128, 66, True) == 2 * 4096          # 33 outputs: three units of gate and up columns
    assert mb.moe_mx4_weight_code_bytes(1, 0, 64) == 0 and mb.moe_mx4_weight_code_bytes(1025, 64, 64) == 0
    assert not mb.moe_mx4_tile_supported(48, 256) and not mb.moe_mx4_tile_supported(16, 512)


def test_default_tiling_is_supported():
    for T in (1, 3, 16, 40, 128, 333, 1000, 4096, 20000):
        for k, E, K, N, gated in ((2, 8, 4096, 28672, True), (6, 64, 2048, 2816, True), (8, 256, 7168, 4096, False), (1, 1, 100, 30, False)):
            g = mb.moe_mx4_default_tiling(T, k, E, K, N, gated)
            assert mb.moe_mx4_tile_supported(g.tile_m, g.tile_n) and g.tile_m_small == 0 and g.tile_m_slack == 0, (T, E, g)
    with pytest.raises(mb.MoeError):
        mb.moe_mx4_default_tiling(4, 9, 8, 64, 64)
