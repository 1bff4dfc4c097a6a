"""What the grouped router, the norm, the row quantiser and the 4-bit product refuse.  Addresses are made up: nothing is launched before a check."""
import ctypes

import pytest
import torch

from paper_2501_16103_amd import binding as mb

P = 1 << 20          # an aligned address that nobody reads
OK, INVALID, UNSUPPORTED = mb.MOE_OK, mb.MOE_ERR_INVALID_ARG, mb.MOE_ERR_UNSUPPORTED
FP32, BF16, FP16, FP8 = mb.MOE_DTYPE_FP32, mb.MOE_DTYPE_BF16, mb.MOE_DTYPE_FP16, mb.MOE_DTYPE_FP8_E4M3


def _route(logits=P, bias=P, groups=4, kept=2, group_score=0, ids=P, weights=P, **kw):
    d = dict(T=4, k=2, E=8, dtype=FP32, row_stride=8, score=0, renormalize=1, scale=1.0)
    d.update(kw)
    return mb.lib().moe_route_grouped(logits, bias, ctypes.byref(mb.moe_route_desc(**d)), groups, kept, group_score, ids, weights, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(T=-1), INVALID), (dict(k=0), INVALID), (dict(k=5), INVALID), (dict(k=9), INVALID), (dict(E=0), INVALID), (dict(score=2), INVALID),
    (dict(groups=0), INVALID), (dict(groups=3), INVALID), (dict(groups=16), INVALID), (dict(kept=0), INVALID), (dict(kept=5), INVALID), (dict(group_score=2), INVALID),
    (dict(group_score=-1), INVALID), (dict(dtype=FP8), UNSUPPORTED), (dict(dtype=FP16), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
    (dict(E=1028, row_stride=1028), UNSUPPORTED), (dict(E=130, groups=65, row_stride=130), UNSUPPORTED), (dict(T=1 << 24), UNSUPPORTED), (dict(row_stride=7), INVALID),
    (dict(logits=None), INVALID), (dict(ids=None), INVALID), (dict(weights=None), INVALID), (dict(logits=P + 2), INVALID), (dict(bias=P + 2), INVALID),
    (dict(ids=P + 1), INVALID), (dict(weights=P + 2), INVALID), (dict(dtype=BF16, logits=P + 1), INVALID), (dict(T=0, logits=None), OK)])
def test_route_grouped(kw, rc):
    assert _route(**kw) == rc


def _norm(x=P, residual=P, weight=P, residual_out=P, y=P, codes=P, scales=P, **kw):
    d = dict(rows=4, x_stride=64, residual_stride=64, cols=64, x_dtype=BF16, residual_dtype=BF16, weight_dtype=BF16, eps=1e-6)
    d.update(kw)
    return mb.lib().moe_add_norm(x, residual, weight, ctypes.byref(mb.moe_norm_desc(**d)), residual_out, y, codes, scales, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(eps=-1e-6), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(x_dtype=FP16), UNSUPPORTED), (dict(residual_dtype=FP8), UNSUPPORTED), (dict(weight_dtype=-1), UNSUPPORTED),
    (dict(cols=65537, x_stride=65537, residual_stride=65537), UNSUPPORTED), (dict(rows=(1 << 24) + 1), UNSUPPORTED), (dict(residual=None), INVALID),
    (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(residual_out=None, y=None, codes=None, scales=None), INVALID), (dict(x=None), INVALID),
    (dict(x_stride=63), INVALID), (dict(residual_stride=63), INVALID), (dict(x=P + 1), INVALID), (dict(residual=P + 1), INVALID), (dict(residual_out=P + 1), INVALID),
    (dict(weight=P + 1), INVALID), (dict(y=P + 1), INVALID), (dict(scales=P + 2), INVALID), (dict(x_dtype=FP32, x=P + 2), INVALID),
    (dict(residual_dtype=FP32, residual=P + 2), INVALID), (dict(weight_dtype=FP32, weight=P + 2), INVALID), (dict(rows=0, x=None), OK)])
def test_add_norm(kw, rc):
    assert _norm(**kw) == rc


def _quantize(src=P, dtype=BF16, rows=4, cols=100, stride=100, codes=P, scales=P):
    return mb.lib().moe_fp8_quantize(src, dtype, rows, cols, stride, codes, scales, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(stride=99), INVALID), (dict(dtype=FP8), UNSUPPORTED), (dict(dtype=FP16), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
    (dict(cols=65537, stride=65537), UNSUPPORTED), (dict(rows=(1 << 24) + 1), UNSUPPORTED), (dict(src=None), INVALID), (dict(codes=None), INVALID),
    (dict(scales=None), INVALID), (dict(scales=P + 2), INVALID), (dict(src=P + 1), INVALID), (dict(dtype=FP32, src=P + 2), INVALID), (dict(rows=0, src=None), OK)])
def test_quantize(kw, rc):
    assert _quantize(**kw) == rc


def _pack(q=P, scales=P, zeros=P, dtype=BF16, layout=0, K=64, N=32, group=32, gated=0, codes=P, words=P):
    return mb.lib().moe_w4_pack_weights(q, scales, zeros, dtype, layout, K, N, group, gated, codes, words, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(K=0), INVALID), (dict(N=0), INVALID), (dict(N=31, gated=1), INVALID), (dict(gated=2), INVALID), (dict(layout=2), INVALID), (dict(group=16), UNSUPPORTED),
    (dict(group=0), UNSUPPORTED), (dict(group=256), UNSUPPORTED), (dict(dtype=FP32), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(K=(1 << 20) + 1), UNSUPPORTED),
    (dict(N=(1 << 20) + 2), UNSUPPORTED), (dict(q=None), INVALID), (dict(scales=None), INVALID), (dict(scales=P + 1), INVALID), (dict(codes=None), INVALID),
    (dict(words=None), INVALID), (dict(codes=P + 8), INVALID), (dict(words=P + 4), INVALID)])
def test_pack(kw, rc):
    assert _pack(**kw) == rc


def _matvec(X=P, stride=64, codes=P, words=P, add=P, out=P, **kw):
    d = dict(T=4, K=64, N=32, group=32, gated=0)
    d.update(kw)
    return mb.lib().moe_w4_matvec(X, stride, codes, words, ctypes.byref(mb.moe_w4_desc(**d)), add, out, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(T=-1), INVALID), (dict(T=17), UNSUPPORTED), (dict(K=0), INVALID), (dict(N=0), INVALID), (dict(N=31, gated=1), INVALID), (dict(gated=-1), INVALID),
    (dict(group=48), UNSUPPORTED), (dict(K=(1 << 20) + 1, stride=1 << 21), UNSUPPORTED), (dict(X=None), INVALID), (dict(codes=None), INVALID), (dict(words=None), INVALID),
    (dict(out=None), INVALID), (dict(stride=63), INVALID), (dict(X=P + 1), INVALID), (dict(codes=P + 8), INVALID), (dict(words=P + 8), INVALID), (dict(add=P + 1), INVALID),
    (dict(out=P + 1), INVALID), (dict(T=0, X=None), OK)])
def test_matvec(kw, rc):
    assert _matvec(**kw) == rc


def test_null_descriptions():
    lib = mb.lib()
    assert lib.moe_route_grouped(P, None, None, 1, 1, 0, P, P, None) == INVALID
    assert lib.moe_add_norm(P, None, None, None, None, P, None, None, None) == INVALID
    assert lib.moe_w4_matvec(P, 64, P, P, None, None, P, None) == INVALID


def test_sizes():
    assert mb.moe_w4_code_bytes(128, 16) == 1024 and mb.moe_w4_code_bytes(129, 17) == 4 * 1024
    assert mb.moe_w4_code_bytes(128, 34, True) == 4 * 1024                      # 17 columns of each half: two tiles each
    assert mb.moe_w4_word_bytes(128, 16, 32) == 4 * 64 and mb.moe_w4_word_bytes(128, 16, 128) == 64
    assert mb.moe_w4_code_bytes(0, 16) == mb.moe_w4_word_bytes(128, 16, 48) == mb.moe_w4_code_bytes(128, 15, True) == 0
    assert mb.moe_w4_code_bytes(1 << 20, 1 << 20) == 1 << 39                    # sizes beyond 32 bits


def test_bindings_refuse_what_does_not_fit():
    """Tensors on the host, of the wrong size, type or layout never reach the library."""
    t = torch.empty
    cpu = dict(check=False)
    ids, w = t(4, 2, dtype=torch.int32), t(4, 2)
    assert mb.moe_route_grouped(t(4, 8), 2, ids, w, 2, 1, **cpu) == INVALID                     # on the host
    assert mb.moe_route_grouped(t(4, 8), 2, t(3, 2, dtype=torch.int32), w, 2, 1, **cpu) == INVALID
    assert mb.moe_route_grouped(t(4, 8), 2, ids, w, 2, 1, bias=t(7), **cpu) == INVALID
    assert mb.moe_route_grouped(t(4, 8), 2, ids, w, 2, 1, bias=t(8, dtype=torch.bfloat16), **cpu) == INVALID
    assert mb.moe_add_norm(t(4, 8), None, 1e-6, y=t(4, 8, dtype=torch.bfloat16), **cpu) == INVALID
    rows = mb.Fp8Rows(4, 8, "cpu")
    assert mb.moe_fp8_quantize(t(4, 8), rows, **cpu) == INVALID
    assert mb.moe_fp8_quantize(t(5, 8), rows, **cpu) == INVALID
    assert mb.moe_fp8_quantize(t(4, 7), rows, **cpu) == INVALID
    W = mb.W4Weights(64, 32, 32, device="cpu")
    q, s = t(64, 32, dtype=torch.uint8), t(2, 32, dtype=torch.float16)
    assert mb.moe_w4_pack_weights(q, s, None, 0, W, **cpu) == INVALID
    assert mb.moe_w4_matvec(t(4, 64, dtype=torch.bfloat16), W, t(4, 32, dtype=torch.bfloat16), **cpu) == INVALID
    for make in (lambda: mb.Fp8Rows(-1, 8, "cpu"), lambda: mb.Fp8Rows(4, 0, "cpu"), lambda: mb.W4Weights(64, 31, 32, True, "cpu"), lambda: mb.W4Weights(64, 32, 48, device="cpu"),
                 lambda: mb.MoeFp8LayerPlan(4, 2, 8, 130, 128, "cpu")):
        with pytest.raises(mb.MoeError):
            make()


class _OnCard(torch.Tensor):
    """A tensor of the host that says it is on the first card, for calls that are looked at before they reach one."""

    def get_device(self):
        return 0


def _card(*shape, dtype=torch.float32):
    return torch.Tensor._make_subclass(_OnCard, torch.empty(*shape, dtype=dtype))


class _Listener:
    """In the library's place: notes the calls that would have launched something, with what their descriptions hold."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        sizes = {"moe_w4_code_bytes", "moe_w4_word_bytes", "moe_strerror"}
        if name in sizes:
            return getattr(self.library, name)

        def call(*args):
            fields = [{n: getattr(a._obj, n) for n, _ in a._obj._fields_} for a in args if hasattr(a, "_obj")]
            self.calls.append((name, args, fields[0] if fields else None))
            return OK
        return call


@pytest.fixture
def listener(monkeypatch):
    there = _Listener()
    there.library = mb.lib()
    monkeypatch.setattr(mb, "_lib", there)
    monkeypatch.setattr(mb, "_current_device", lambda: 0)
    monkeypatch.setattr(mb, "_stream_at", lambda device: 0)
    monkeypatch.setattr(mb, "_stream", lambda: 0)
    return there


MANY = 1 << 32


@pytest.mark.parametrize("K,N,group", [(MANY + 64, 32, 32), (64, MANY + 32, 32), (64, 32, MANY + 32), (MANY + 64, MANY + 32, MANY + 32), (64 - MANY, 32, 32), (64, 32 - MANY, 32)])
def test_weights_of_sizes_beyond_32_bits(K, N, group):
    """Sizes that are others once they are cut off at 32 bits."""
    with pytest.raises(mb.MoeError):
        mb.W4Weights(K, N, group, device="cpu")
    assert mb.moe_w4_word_bytes(K, N, group) == 0
    assert mb.moe_w4_code_bytes(K, N) == (0 if (K, N) != (64, 32) else 2 * 1024)
    with pytest.raises(mb.MoeError):
        mb.W4Weights(64, 32, 32, MANY, "cpu")        # (true, and 0 where it is cut off)


@pytest.mark.parametrize("kw", [dict(groups=MANY + 4), dict(kept=MANY + 2), dict(group_score=MANY), dict(score=MANY + 1), dict(groups=4 - MANY), dict(kept=2 - MANY)])
def test_options_beyond_32_bits(listener, kw):
    good = dict(groups=4, kept=2)
    args = _card(4, 8), 2, _card(4, 2, dtype=torch.int32), _card(4, 2)
    assert mb.moe_route_grouped(*args, **good) == OK and len(listener.calls) == 1
    assert mb.moe_route_grouped(*args, **{**good, **kw}, check=False) == INVALID and len(listener.calls) == 1


def test_choices_beyond_32_bits(listener):
    """No tokens, so that the product of tokens and choices says nothing."""
    args = _card(0, 2), _card(0, 2, dtype=torch.int32), _card(0, 2)
    assert mb.moe_route_grouped(args[0], 2, *args[1:], 1, 1) == OK and len(listener.calls) == 1
    assert mb.moe_route_grouped(args[0], MANY + 2, *args[1:], 1, 1, check=False) == INVALID and len(listener.calls) == 1


def test_layout_beyond_32_bits(listener):
    W = mb.W4Weights(64, 32, 32, device="cpu")
    W.codes, W.words = _card(W.codes.numel(), dtype=torch.uint8), _card(W.words.numel(), dtype=torch.uint8)
    args = _card(64, 32, dtype=torch.uint8), _card(2, 32, dtype=torch.float16), None
    assert mb.moe_w4_pack_weights(*args, mb.MOE_W_LAYOUT_KN, W) == OK and len(listener.calls) == 1
    assert mb.moe_w4_pack_weights(*args, MANY + mb.MOE_W_LAYOUT_NK, W, check=False) == INVALID and len(listener.calls) == 1


def test_what_a_description_holds_is_what_the_call_was_given(listener):
    """Descriptions are kept for each combination of values; a number that a tensor holds may be another one at the next call."""
    scale, renormalize, k, score, eps = torch.tensor(2.5), torch.tensor(True), torch.tensor(2), torch.tensor(0), torch.tensor(0.5)
    for turn in range(2):
        mb.moe_route_grouped(_card(4, 8), k, _card(4, 2, dtype=torch.int32), _card(4, 2), 4, 2, score=score, renormalize=renormalize, scale=scale)
        d = listener.calls[-1][2]
        assert (d["scale"], bool(d["renormalize"]), d["k"], d["score"]) == (scale.item(), renormalize.item(), k.item(), score.item())
        mb.moe_add_norm(_card(4, 8), None, eps, y=_card(4, 8, dtype=torch.bfloat16))
        assert listener.calls[-1][2]["eps"] == eps.item()
        scale.fill_(0.75), renormalize.fill_(False), k.fill_(1), score.fill_(1), eps.fill_(0.25)
    K = torch.tensor(64)
    W = mb.W4Weights(K, torch.tensor(32), torch.tensor(32), device="cpu")
    W.codes, W.words = _card(W.codes.numel(), dtype=torch.uint8), _card(W.words.numel(), dtype=torch.uint8)
    mb.moe_w4_matvec(_card(4, 64, dtype=torch.bfloat16), W, _card(4, 32, dtype=torch.bfloat16))
    K.fill_(96)
    assert W.K == 64
    assert mb.moe_w4_matvec(_card(4, 96, dtype=torch.bfloat16), W, _card(4, 32, dtype=torch.bfloat16), check=False) == INVALID
