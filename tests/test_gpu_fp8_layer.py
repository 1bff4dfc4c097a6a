"""The operators of a block as they are used together: residual addition and norm into 8 bits, the grouped router, an fp8 layer, the shared expert
in 4 bits.  Each step is checked in 64 bits from what the step before it wrote."""
import pytest
import torch

from paper_2501_16103_amd import binding as mb
from tests import block_reference as ref
from tests import helpers as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16 = torch.bfloat16


def _e4m3(w):
    """[E, K, N] -> bytes and a scale for each expert."""
    s = w.abs().amax((1, 2)) / 448.0
    return (w / s[:, None, None]).to(torch.float8_e4m3fn), s


class _Block:
    def __init__(self, T, k, E, hidden, inter, groups, kept, seed):
        g = torch.Generator().manual_seed(seed)
        def normal(*n): return torch.randn(*n, generator=g)
        self.T, self.k, self.E, self.hidden, self.inter, self.groups, self.kept = T, k, E, hidden, inter, groups, kept
        self.norm_weight, self.router, self.bias = 1 + 0.1 * normal(hidden), normal(hidden, E) * hidden ** -0.5, 0.1 * normal(E)
        self.up, self.up_scale = _e4m3(normal(E, hidden, 2 * inter) * hidden ** -0.5)
        self.down, self.down_scale = _e4m3(normal(E, inter, hidden) * inter ** -0.5)
        def shared(K, N):
            return (torch.randint(0, 16, (K, N), generator=g, dtype=torch.uint8), ((0.5 + torch.rand(-(-K // 64), N, generator=g)) * 0.25 * K ** -0.5).half(),
                    torch.randint(6, 10, (-(-K // 64), N), generator=g, dtype=torch.uint8))
        self.shared_up, self.shared_down = shared(hidden, 2 * inter), shared(inter, hidden)
        self.x, self.residual = normal(T, hidden).to(BF16), normal(T, hidden)
        self.plan = mb.MoeFp8LayerPlan(T, k, E, hidden, inter, DEV)
        on = lambda *ts: [t.to(DEV) for t in ts]  # noqa: E731
        self.gpu = on(self.norm_weight, self.router, self.bias, self.up.view(torch.uint8), self.up_scale, self.down.view(torch.uint8), self.down_scale)
        self.W_up = mb.W4Weights(hidden, 2 * inter, 64, True, DEV).pack(*on(*self.shared_up))
        self.W_down = mb.W4Weights(inter, hidden, 64, False, DEV).pack(*on(*self.shared_down))
        self.xg, self.rg = on(self.x, self.residual)
        self.sum, self.y = torch.empty(T, hidden, device=DEV), torch.empty(T, hidden, dtype=BF16, device=DEV)
        self.ids, self.weights = torch.empty(T, k, dtype=torch.int32, device=DEV), torch.empty(T, k, device=DEV)
        self.h, self.out = torch.empty(T, inter, dtype=BF16, device=DEV), torch.empty(T, hidden, dtype=BF16, device=DEV)

    def run(self):
        norm_weight, router, bias, up, up_scale, down, down_scale = self.gpu
        mb.moe_add_norm(self.xg, norm_weight, 1e-6, residual=self.rg, residual_out=self.sum, y=self.y, rows=self.plan.rows)
        self.logits = self.y.float() @ router
        mb.moe_route_grouped(self.logits, self.k, self.ids, self.weights, self.groups, self.kept, mb.MOE_GROUP_TOP2, bias, mb.MOE_SCORE_SIGMOID, scale=2.5)
        routed = self.plan.forward(self.plan.rows, up, up_scale, down, down_scale, self.ids, self.weights)
        if self.T <= 16:
            mb.moe_w4_matvec(self.y, self.W_up, self.h)
            mb.moe_w4_matvec(self.h, self.W_down, self.out, add=routed)
        return self.out if self.T <= 16 else routed


def _near(got, want, bound):
    assert bool(((got.cpu().double() - want).abs() <= bound + want.abs() * 2.0 ** -8 + 2.0 ** -133).all())


@pytest.mark.parametrize("T,k,E,hidden,inter,groups,kept", [(1, 2, 8, 256, 128, 4, 2), (5, 3, 16, 384, 256, 4, 2), (16, 6, 64, 512, 128, 8, 4), (70, 4, 32, 256, 384, 8, 3)])
def test_block(T, k, E, hidden, inter, groups, kept):
    b = _Block(T, k, E, hidden, inter, groups, kept, T)
    b.run()
    plan, R = b.plan, T * k
    h, y = ref.add_norm(b.x, b.residual, b.norm_weight, 1e-6)
    assert torch.equal(b.sum.cpu(), h)
    _near(b.y, y, y.abs() * 32 * 2.0 ** -24)
    ids, weights = ref.route_grouped(b.logits.cpu(), k, groups, kept, True, b.bias, True, True, 2.5)
    assert torch.equal(b.ids.cpu(), ids)
    assert bool(((b.weights.cpu().double() - weights).abs() <= 1.01 * 2.0 ** -24 * weights.abs()).all())
    codes, scales = plan.rows.codes.cpu().view(torch.float8_e4m3fn).double(), plan.rows.scales.cpu().double()
    v = y / scales[:, None]
    assert bool(((codes - v).abs() <= ref.half_step(v) * (1 + 2.0 ** -20) + v.abs() * 64 * 2.0 ** -24).all())
    flat, act = ids.reshape(-1), plan.act.cpu()
    act_codes, act_scales = plan.act_rows.codes.cpu().view(torch.float8_e4m3fn).double(), plan.act_rows.scales.cpu()
    assert torch.equal(act_scales, (act.float().abs().amax(1) / 448.0).clamp(min=2.0 ** -126))
    v = act.double() / act_scales.double()[:, None]
    assert bool(((act_codes - v).abs() <= ref.half_step(v) * (1 + 2.0 ** -20) + v.abs() * 2.0 ** -22).all())
    down = plan.down.cpu()
    for e in torch.unique(flat).tolist():
        rows = torch.nonzero(flat == e).squeeze(1)
        x, w = codes[rows // k], b.up[e].double()
        factor = scales[rows // k, None] * float(b.up_scale[e])
        s, off = x @ w * factor, H.fp8_adder_bound(x.float(), w.float()) * factor
        (g, u), (dg, du) = s.chunk(2, dim=1), off.chunk(2, dim=1)
        a = ref.silu(g)
        # the scales' two products, exponential, sum, quotient and product round by 2^-24 each, an exponent of up to 88 by that of itself
        _near(act[rows], a * u, 1.1 * dg * (u.abs() + du) + a.abs() * du + (a * u).abs() * 100 * 2.0 ** -24)
        x, w = act_codes[rows], b.down[e].double()
        factor = act_scales[rows, None].double() * float(b.down_scale[e])
        _near(down[rows], x @ w * factor, H.fp8_adder_bound(x.float(), w.float()) * factor + (x @ w * factor).abs() * 4 * 2.0 ** -24)
    parts = down.double().reshape(T, k, hidden) * b.weights.cpu().double()[..., None]
    _near(plan.out, parts.sum(1), parts.abs().sum(1) * (k + 1) * 2.0 ** -24)
    if T <= 16:
        yb, hb = b.y.cpu(), b.h.cpu()
        (g, u), (dg, du) = (yb.double() @ ref.w4_values(*b.shared_up, 64)).chunk(2, dim=1), ref.w4_sum_bound(yb, *b.shared_up, 64).chunk(2, dim=1)
        _near(b.h, ref.silu(g) * u, 1.1 * dg * (u.abs() + du) + ref.silu(g).abs() * du + (ref.silu(g) * u).abs() * 100 * 2.0 ** -24)
        want = plan.out.cpu().double() + hb.double() @ ref.w4_values(*b.shared_down, 64)
        _near(b.out, want, ref.w4_sum_bound(hb, *b.shared_down, 64) + (want.abs() + plan.out.cpu().double().abs()) * 2.0 ** -23)


def test_block_captured():
    """A step without the router's library product, captured and replayed over new inputs, with eager work between."""
    b = _Block(4, 2, 8, 256, 128, 4, 2, 40)
    b.run()
    logits = b.logits.clone()
    norm_weight, _, bias, up, up_scale, down, down_scale = b.gpu

    def step():
        mb.moe_add_norm(b.xg, norm_weight, 1e-6, residual=b.rg, residual_out=b.sum, y=b.y, rows=b.plan.rows)
        mb.moe_route_grouped(logits, 2, b.ids, b.weights, 4, 2, mb.MOE_GROUP_TOP2, bias, mb.MOE_SCORE_SIGMOID)
        routed = b.plan.forward(b.plan.rows, up, up_scale, down, down_scale, b.ids, b.weights)
        mb.moe_w4_matvec(b.y, b.W_up, b.h)
        mb.moe_w4_matvec(b.h, b.W_down, b.out, add=routed)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        b.xg.copy_(b.x.roll(turn + 1, 0))
        logits.copy_(logits.roll(1, 1))
        graph.replay()
        torch.cuda.synchronize()
        got = b.out.clone()
        step()
        assert torch.equal(got, b.out)


def test_plan_refuses():
    b = _Block(3, 2, 8, 256, 128, 4, 2, 50)
    _, _, _, up, up_scale, down, down_scale = b.gpu
    ids, w = torch.zeros(3, 2, dtype=torch.int32, device=DEV), torch.ones(3, 2, device=DEV)
    good = dict(X=b.plan.rows, W_gate_up=up, up_scale=up_scale, W_down=down, down_scale=down_scale, topk_ids=ids, topk_weights=w)
    for bad in (dict(X=mb.Fp8Rows(2, 256, DEV)), dict(X=mb.Fp8Rows(3, 128, DEV)), dict(W_gate_up=up[:7]), dict(W_gate_up=up.to(BF16)), dict(W_down=down[:, :, :128]),
                dict(up_scale=up_scale[:7]), dict(down_scale=down_scale.double()), dict(topk_ids=ids.long()), dict(topk_ids=ids[:2]), dict(topk_weights=w.cpu())):
        with pytest.raises(mb.MoeError):
            b.plan.forward(**{**good, **bad})


@pytest.mark.parametrize("other", [torch.float8_e5m2, torch.float8_e4m3fnuz, torch.bool])
def test_plan_refuses_other_types_of_a_byte(other):
    """Weights whose elements are a byte but not e4m3: read as that they would give another product."""
    b = _Block(3, 2, 8, 256, 128, 4, 2, 51)
    _, _, _, up, up_scale, down, down_scale = b.gpu
    ids, w = torch.zeros(3, 2, dtype=torch.int32, device=DEV), torch.ones(3, 2, device=DEV)
    b.plan.rows.quantize(b.xg)
    want = b.plan.forward(b.plan.rows, up, up_scale, down, down_scale, ids, w).clone()
    for same in (torch.float8_e4m3fn, torch.int8):
        assert torch.equal(b.plan.forward(b.plan.rows, up.view(same), up_scale, down.view(same), down_scale, ids, w), want)
    for up_type, down_type in ((other, torch.uint8), (torch.uint8, other)):
        with pytest.raises(mb.MoeError):
            b.plan.forward(b.plan.rows, up.view(up_type), up_scale, down.view(down_type), down_scale, ids, w)


def _bytes(seed, *shape):
    """e4m3 bytes of random numbers, drawn on the GPU, an expert at a time."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    out = torch.empty(shape, dtype=torch.uint8, device=DEV)
    for e in range(shape[0]):
        out[e] = (torch.randn(shape[1:], generator=g, device=DEV) * 100.0).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return out


@pytest.mark.parametrize("T,k,E,hidden,inter", [(1, 6, 64, 2048, 1408), (128, 6, 64, 2048, 1408), (1024, 6, 64, 2048, 1408), (1, 2, 8, 4096, 14336), (128, 2, 8, 4096, 14336)])
def test_layer_at_full_size(T, k, E, hidden, inter):
    """A few rows of three experts and all sums, each step from what the step before it wrote."""
    g = torch.Generator().manual_seed(T + E)
    up, down = _bytes(1, E, hidden, 2 * inter), _bytes(2, E, inter, hidden)
    up_scale, down_scale = ((0.5 + torch.rand(E, generator=g)) * (0.01 * n ** -0.5) for n in (hidden, inter))
    x = torch.randn(T, hidden, generator=g).to(BF16)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)]).to(torch.int32)
    weights = torch.rand(T, k, generator=g)
    plan = mb.MoeFp8LayerPlan(T, k, E, hidden, inter, DEV)
    plan.rows.quantize(x.to(DEV))
    plan.forward(plan.rows, up, up_scale.to(DEV), down, down_scale.to(DEV), ids.to(DEV), weights.to(DEV))
    codes, scales = plan.rows.codes.cpu().view(torch.float8_e4m3fn).double(), plan.rows.scales.cpu().double()
    act_codes, act_scales = plan.act_rows.codes.cpu().view(torch.float8_e4m3fn).double(), plan.act_rows.scales.cpu()
    flat, act, out = ids.reshape(-1).long(), plan.act.cpu(), plan.down.cpu()
    assert torch.equal(act_scales, (act.float().abs().amax(1) / 448.0).clamp(min=2.0 ** -126))
    v = act.double() / act_scales.double()[:, None]
    assert bool(((act_codes - v).abs() <= ref.half_step(v) * (1 + 2.0 ** -20) + v.abs() * 2.0 ** -22).all())
    used = torch.unique(flat)
    for e in used[torch.linspace(0, len(used) - 1, 3).long()].unique().tolist():
        rows = torch.nonzero(flat == e).squeeze(1)
        rows = rows[torch.linspace(0, len(rows) - 1, 3).long().unique()]
        cols = torch.randperm(inter, generator=g)[:200]
        w = up[e].cpu().view(torch.float8_e4m3fn)[:, torch.cat([cols, inter + cols])].double()
        a, factor = codes[rows // k], scales[rows // k, None] * float(up_scale[e])
        s, off = a @ w * factor, H.fp8_adder_bound(a.float(), w.float()) * factor
        (gate, u), (dg, du) = s.chunk(2, dim=1), off.chunk(2, dim=1)
        f = ref.silu(gate)
        _near(act[rows][:, cols], f * u, 1.1 * dg * (u.abs() + du) + f.abs() * du + (f * u).abs() * 100 * 2.0 ** -24)   # (as in test_block)
        cols = torch.randperm(hidden, generator=g)[:200]
        w = down[e].cpu().view(torch.float8_e4m3fn)[:, cols].double()
        a, factor = act_codes[rows], act_scales[rows, None].double() * float(down_scale[e])
        _near(out[rows][:, cols], a @ w * factor, H.fp8_adder_bound(a.float(), w.float()) * factor + (a @ w * factor).abs() * 4 * 2.0 ** -24)
    parts = out.double().reshape(T, k, hidden) * weights.double()[..., None]
    _near(plan.out, parts.sum(1), parts.abs().sum(1) * (k + 1) * 2.0 ** -24)
