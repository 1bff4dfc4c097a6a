"""The operators around a block's experts whose time counts, each in its plain form and as the library's own calls.

  "route"     a router with a balance bias and groups of experts: logits -> each token's k experts and their weights;
  "norm"      the way into a layer: residual addition, root-mean-square norm, and the normed rows in bf16, in e4m3 with a scale
              for each row (what the fp8 product takes), or both;
  "rows"      rows -> e4m3 with a scale for each row: activations on their way into the second fp8 product;
  "matvec"    at most 16 tokens times a dense weight in 4 bits with a scale (and a zero point) for every group of 32, 64 or 128
              along K: the shared expert beside the routed ones, its gated activation and its addition to their sum.

A pass starts from what a serving program has in hand at that point: new tokens, logits or activations, and weights and
buffers that it keeps.  Sizes are those of the repository's own workloads: 64 experts, top-6, 2048 -> 2 x 1408; the
Mixtral-shaped experts (4096 -> 2 x 14336 -> 4096); the evaluation of Sec. 5 of the paper ([3584, 2560]); the fine-grained experts'
hidden size, 7168, and their count, 256, top-8.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda"
EPS = 1e-6
E4M3_MAX = 448.0
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one generated token: a launch's latency
        dict(name="route_T1", op="route", T=1, E=64, k=6, groups=8, kept=4, group_score="max", bias=False, dtype="bf16", score="softmax",
             renormalize=False, scale=1.0, masked=0),
        # a prompt over many experts, sigmoid scores with a bias for balance; every 16th row is padding, all of its experts masked
        dict(name="route_T8192_bias", op="route", T=8192, E=256, k=8, groups=8, kept=4, group_score="top2", bias=True, dtype="fp32",
             score="sigmoid", renormalize=True, scale=2.5, masked=16),
        # a middling prompt, groups of uneven use
        dict(name="route_T700_E160", op="route", T=700, E=160, k=6, groups=8, kept=3, group_score="max", bias=False, dtype="fp32", score="softmax",
             renormalize=False, scale=1.0, masked=0),
        # one generated token on its way into a layer: bf16 for the router's projection, 8 bits for the experts
        dict(name="norm_T1", op="norm", T=1, H=2048, x="bf16", residual="bf16", weight="bf16", outputs="both"),
        # a prompt with a residual stream kept in fp32, an odd width
        dict(name="norm_T777_odd", op="norm", T=777, H=3583, x="bf16", residual="fp32", weight="fp32", outputs="both"),
        # a long prompt
        dict(name="norm_T4096", op="norm", T=4096, H=7168, x="bf16", residual="bf16", weight="bf16", outputs="both"),
        # activated rows of a decoding batch (128 tokens, top-6) on their way into the down product
        dict(name="rows_R768", op="rows", rows=768, cols=1408, dtype="bf16"),
        # those of a long prompt through large experts
        dict(name="rows_R8192", op="rows", rows=8192, cols=14336, dtype="bf16"),
        # generating one sequence: the shared expert's gate and up projections with their activation
        dict(name="matvec_T1", op="matvec", T=1, K=2048, N=2816, group=128, zeros=False, gated=True, add=False, scales="bf16"),
        # the same of a large expert, with zero points
        dict(name="matvec_T1_large", op="matvec", T=1, K=4096, N=28672, group=128, zeros=True, gated=True, add=False, scales="fp16"),
        # a decoding batch, down projection added to the routed experts' sum
        dict(name="matvec_T16_down", op="matvec", T=16, K=14336, N=4096, group=64, zeros=True, gated=False, add=True, scales="fp16"),
        # a few sequences, the finest groups
        dict(name="matvec_T5_g32", op="matvec", T=5, K=3584, N=2560, group=32, zeros=False, gated=False, add=False, scales="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))))), lo), hi)


def _size(rng, lo, hi, step=1):
    return max(_log_int(rng, lo, hi) // step * step, step)


def draw(rng):
    op = rng.choice(["route", "norm", "rows", "matvec", "matvec"])
    if op == "route":
        E, groups = rng.choice([(64, 8), (64, 1), (60, 4), (128, 8), (160, 8), (256, 8), (256, 16), (72, 6), (320, 10), (512, 8)])
        kept = rng.randint(1, groups)
        return dict(op=op, T=_size(rng, 1, 8192 * 256 // max(E, 256)), E=E, k=rng.randint(1, min(8, kept * (E // groups))), groups=groups,
                    kept=kept, group_score=rng.choice(["max", "top2"]), bias=rng.random() < 0.6, dtype=rng.choice(["bf16", "fp32"]),
                    score=rng.choice(["softmax", "sigmoid"]), renormalize=rng.random() < 0.6, scale=rng.choice([1.0, 2.5]),
                    masked=rng.choice([0, 3, 16]))
    if op == "norm":
        x, residual = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("bf16", "fp32"), ("bf16", "none"), ("fp32", "fp32")])
        H = _size(rng, 64, 7168, rng.choice([1, 8, 64]))
        return dict(op=op, T=_size(rng, 1, 4096 if x == "bf16" and residual != "fp32" else 2048), H=H, x=x, residual=residual,
                    weight=rng.choice(["bf16", "fp32"]), outputs=rng.choice(["both", "both", "bf16", "fp8"]))
    if op == "rows":
        cols = _size(rng, 64, 14336, rng.choice([1, 8, 64]))
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        return dict(op=op, rows=_size(rng, 1, 8192 if dtype == "bf16" else 4096), cols=cols, dtype=dtype)
    K = _size(rng, 256, 14336, rng.choice([1, 8, 64, 128]))
    N = _size(rng, 256, min(28672, 4096 * 28672 // K), rng.choice([2, 16, 64]))
    return dict(op=op, T=rng.randint(1, 16), K=K, N=N, group=rng.choice([32, 64, 128, 128]), zeros=rng.random() < 0.5,
                gated=rng.random() < 0.5, add=rng.random() < 0.4, scales=rng.choice(["bf16", "fp16"]))


# ------------------------------------------------------------------------------------------------------------ inputs

def _gen(seed, tag):
    return torch.Generator(device=DEVICE).manual_seed((seed * 1_000_003 + tag) % (1 << 62))


def _normal(seed, tag, *shape):
    return torch.randn(*shape, generator=_gen(seed, tag), device=DEVICE)


def _router(case, seed):
    """Logits as a trained router gives them, some experts favoured; the bias that evens their use out."""
    favour = _normal(seed, 2, case["E"])
    x = (_normal(seed, 1, case["T"], case["E"]) + 0.5 * favour).to(DTYPES[case["dtype"]])
    if case["masked"]:
        x[case["masked"] - 1:: case["masked"]] = float("-inf")            # padding rows
        x[:, case["E"] // 3] = float("-inf")                              # and an expert that is out of service
    return x, -0.1 * favour if case["bias"] else None


def _tokens(seed, tag, T, H, dtype):
    """Rows of a residual stream or of a layer's output: normal, a few channels much larger than the others."""
    x = _normal(seed, tag, T, H)
    big = torch.rand(H, generator=_gen(seed, tag + 1), device=DEVICE) < 0.01
    return torch.where(big, 8.0 * x, x).to(DTYPES[dtype])


def _norm_inputs(case, seed):
    T, H = case["T"], case["H"]
    x = _tokens(seed, 10, T, H, case["x"])
    residual = None if case["residual"] == "none" else _tokens(seed, 12, T, H, case["residual"])
    weight = (1.0 + 0.1 * _normal(seed, 14, H)).to(DTYPES[case["weight"]])
    return x, residual, weight


def _activations(case, seed):
    """What a gated activation leaves: many values near zero, a few large."""
    g, u = _normal(seed, 20, case["rows"], case["cols"]), _normal(seed, 21, case["rows"], case["cols"])
    return (g * torch.sigmoid(g) * u).to(DTYPES[case["dtype"]])


def _matvec_inputs(case, seed):
    """Codes 0 .. 15 [K, N], the scales of their groups, and the zero points (8 where there are none)."""
    T, K, N = case["T"], case["K"], case["N"]
    x = _tokens(seed, 30, T, K, "bf16")
    groups = -(-K // case["group"])
    q = torch.clamp(torch.round(8.0 + 2.6 * _normal(seed, 32, K, N)), 0, 15).to(torch.uint8)
    s = ((0.5 + torch.rand(groups, N, generator=_gen(seed, 33), device=DEVICE)) * (0.4 * K ** -0.5)).to(DTYPES[case["scales"]])
    z = torch.randint(6, 11, (groups, N), generator=_gen(seed, 34), device=DEVICE, dtype=torch.uint8) if case["zeros"] else None
    out = N // 2 if case["gated"] else N
    add = _tokens(seed, 35, T, out, "bf16") if case["add"] else None
    return x, q, s, z, add


# ------------------------------------------------------------------------------------------------------- plain forms

def _plain_route(logits, bias, case):
    x = logits.double()                              # (a score next to another decides which expert is taken)
    T, E = x.shape
    groups, k = case["groups"], case["k"]
    masked = x == -math.inf
    if case["score"] == "softmax":
        top = x.amax(1, keepdim=True)
        p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
        total = p.sum(1, keepdim=True)
        p = torch.where(total > 0, p / total, 0.0)
    else:
        p = 1 / (1 + torch.exp(-x))
    s = p if bias is None else p + bias.double()
    s = torch.where(masked, -math.inf, s)
    g = s.reshape(T, groups, E // groups)
    if case["group_score"] == "top2" and E // groups > 1:
        two = torch.sort(g, dim=2, descending=True).values[..., :2]
        g = two[..., 0] + torch.where(two[..., 1] == -math.inf, 0.0, two[..., 1])
    else:
        g = g.amax(2)
    kept = torch.sort(g, dim=1, descending=True, stable=True).indices[:, : case["kept"]]
    inside = torch.zeros(T, groups, dtype=torch.int32, device=x.device).scatter_(1, kept, 1).repeat_interleave(E // groups, dim=1)
    # falling scores, equal ones by falling logit, equal ones by rising index; the groups that are left out come last
    ids = torch.sort(x, dim=1, descending=True, stable=True).indices
    ids = ids.gather(1, torch.sort(s.gather(1, ids), dim=1, descending=True, stable=True).indices)
    ids = ids.gather(1, torch.sort(inside.gather(1, ids), dim=1, descending=True, stable=True).indices)[:, :k]
    w = torch.where(masked, 0.0, p).gather(1, ids)
    if case["renormalize"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    return ids.to(torch.int32), (w * case["scale"]).float()


def _plain_rows(y):
    """y fp32 -> e4m3 and the scale of each row."""
    scale = (y.abs().amax(1) / E4M3_MAX).clamp(min=2.0 ** -126)
    return (y / scale[:, None]).to(torch.float8_e4m3fn), scale


def _plain_norm(x, residual, weight, outputs):
    h = x if residual is None else (x.float() + residual.float()).to(residual.dtype)
    f = h.float()
    y = f * torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) * weight.float()
    out = {} if residual is None else {"residual": h}
    if outputs != "fp8":
        out["y"] = y.to(torch.bfloat16)
    if outputs != "bf16":
        out["codes"], out["scales"] = _plain_rows(y)
    return out


def _plain_matvec(x, q, s, z, add, group, gated):
    K = q.shape[0]
    zero = 8.0 if z is None else z.float().repeat_interleave(group, dim=0)[:K]
    y = x.float() @ ((q.float() - zero) * s.float().repeat_interleave(group, dim=0)[:K])
    if gated:
        gate, up = y.chunk(2, dim=1)
        y = gate / (1 + torch.exp(-gate)) * up
    return (y if add is None else y + add.float()).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------------- the measured

def prepare(case, seed):
    op, s = case["op"], {"case": case}
    if own:
        from paper_2501_16103_amd import binding as mb
        s["mb"] = mb
    if op == "route":
        s["logits"], s["bias"] = _router(case, seed)
        if own:
            s["ids"] = torch.empty(case["T"], case["k"], dtype=torch.int32, device=DEVICE)
            s["weights"] = torch.empty(case["T"], case["k"], device=DEVICE)
    elif op == "norm":
        s["x"], s["residual"], s["weight"] = _norm_inputs(case, seed)
        if own:
            T, H = case["T"], case["H"]
            s["sum"] = None if s["residual"] is None else torch.empty_like(s["residual"])
            s["y"] = torch.empty(T, H, dtype=torch.bfloat16, device=DEVICE) if case["outputs"] != "fp8" else None
            s["rows"] = mb.Fp8Rows(T, H, DEVICE) if case["outputs"] != "bf16" else None
    elif op == "rows":
        s["x"] = _activations(case, seed)
        if own:
            s["rows"] = mb.Fp8Rows(case["rows"], case["cols"], DEVICE)
    else:
        s["x"], s["q"], s["s"], s["z"], s["add"] = _matvec_inputs(case, seed)
        if own:
            N = case["N"]
            s["W"] = mb.W4Weights(case["K"], N, case["group"], gated=case["gated"], device=DEVICE).pack(s["q"], s["s"], s["z"])
            s["out"] = torch.empty(case["T"], N // 2 if case["gated"] else N, dtype=torch.bfloat16, device=DEVICE)
    return s


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        mb = s["mb"]
        if op == "route":
            mb.moe_route_grouped(s["logits"], case["k"], s["ids"], s["weights"], groups=case["groups"], kept=case["kept"],
                                 group_score=mb.MOE_GROUP_MAX if case["group_score"] == "max" else mb.MOE_GROUP_TOP2, bias=s["bias"],
                                 score=mb.MOE_SCORE_SOFTMAX if case["score"] == "softmax" else mb.MOE_SCORE_SIGMOID,
                                 renormalize=case["renormalize"], scale=case["scale"])
            return s["ids"], s["weights"]
        if op == "norm":
            mb.moe_add_norm(s["x"], s["weight"], EPS, residual=s["residual"], residual_out=s["sum"], y=s["y"], rows=s["rows"])
            out = {} if s["sum"] is None else {"residual": s["sum"]}
            if s["y"] is not None:
                out["y"] = s["y"]
            if s["rows"] is not None:
                out["codes"], out["scales"] = s["rows"].codes.view(torch.float8_e4m3fn), s["rows"].scales
            return out
        if op == "rows":
            s["rows"].quantize(s["x"])
            return {"codes": s["rows"].codes.view(torch.float8_e4m3fn), "scales": s["rows"].scales}
        mb.moe_w4_matvec(s["x"], s["W"], s["out"], add=s["add"])
        return s["out"]
    if op == "route":
        return _plain_route(s["logits"], s["bias"], case)
    if op == "norm":
        return _plain_norm(s["x"], s["residual"], s["weight"], case["outputs"])
    if op == "rows":
        codes, scales = _plain_rows(s["x"].float())
        return {"codes": codes, "scales": scales}
    return _plain_matvec(s["x"], s["q"], s["s"], s["z"], s["add"], case["group"], case["gated"])


def work(case):
    op = case["op"]
    size = {"bf16": 2, "fp16": 2, "fp32": 4, "none": 0}
    if op == "route":
        T, E = case["T"], case["E"]
        return {"bytes": T * (E * size[case["dtype"]] + 8 * case["k"]) + (4 * E if case["bias"] else 0), "flops": 5 * T * E}
    if op == "norm":
        T, H = case["T"], case["H"]
        each = size[case["x"]] + 2 * size[case["residual"]] + {"both": 3, "bf16": 2, "fp8": 1}[case["outputs"]]
        return {"bytes": T * H * each + H * size[case["weight"]] + (4 * T if case["outputs"] != "bf16" else 0), "flops": 6 * T * H}
    if op == "rows":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (size[case["dtype"]] + 1) + 4 * case["rows"], "flops": 2 * n}
    T, K, N = (case[n] for n in ("T", "K", "N"))
    out = N // 2 if case["gated"] else N
    scales = -(-K // case["group"]) * N * (2.5 if case["zeros"] else 2)
    return {"bytes": K * N / 2 + scales + 2 * T * K + (4 if case["add"] else 2) * T * out, "flops": 2 * T * K * N}


# -------------------------------------------------------------------------------------------- the same in 64 bits

def _exact_route(case, seed):
    logits, bias = _router(case, seed)
    l = logits.double().cpu().numpy()
    T, E = l.shape
    off = np.isneginf(l)
    if case["score"] == "softmax":
        e = np.where(off, 0.0, np.exp(l - np.where(off.all(1), 0.0, l.max(1))[:, None]))
        p = e / np.where(off.all(1), 1.0, e.sum(1))[:, None]
    else:
        p = np.where(off, 0.0, 1 / (1 + np.exp(np.where(off, 0.0, -l))))
    s = np.where(off, -np.inf, p + (0.0 if bias is None else bias.double().cpu().numpy()))
    each = E // case["groups"]
    blocks = np.sort(s.reshape(T, case["groups"], each), axis=2)[:, :, ::-1]
    score = blocks[:, :, 0].copy()
    if case["group_score"] == "top2" and each > 1:
        score += np.where(np.isneginf(blocks[:, :, 1]), 0.0, blocks[:, :, 1])
    number = np.broadcast_to(np.arange(case["groups"]), score.shape)
    best = np.lexsort((number, -score), axis=1)[:, : case["kept"]]
    left_out = np.ones((T, E), dtype=bool)
    for j in range(case["kept"]):
        for i in range(each):
            left_out[np.arange(T), best[:, j] * each + i] = False
    ids = np.lexsort((np.broadcast_to(np.arange(E), l.shape), -l, -s, left_out), axis=1)[:, : case["k"]]
    w = np.take_along_axis(p, ids, axis=1)
    if case["renormalize"]:
        total = w.sum(1, keepdims=True)
        w = np.where(total > 0, w / np.where(total > 0, total, 1.0), 0.0)
    return torch.from_numpy(ids.astype(np.int32)), torch.from_numpy(case["scale"] * w)


def _exact_rows(y):
    scale = torch.clamp(y.abs().max(dim=1).values / 448, min=2.0 ** -126)
    return {"codes": torch.div(y, scale.unsqueeze(1)), "scales": scale}


def exact(case, seed):
    op = case["op"]
    if op == "route":
        return _exact_route(case, seed)
    if op == "norm":
        x, residual, weight = _norm_inputs(case, seed)
        out, h = {}, x.double()
        if residual is not None:                     # (the norm is of what the residual's type holds)
            h = (h + residual.double()).to(residual.dtype).double()
            out["residual"] = h
        y = weight.double() * (h / torch.sqrt(h.square().sum(1, keepdim=True) / case["H"] + EPS))
        if case["outputs"] != "fp8":
            out["y"] = y
        return out if case["outputs"] == "bf16" else {**out, **_exact_rows(y)}
    if op == "rows":
        return _exact_rows(_activations(case, seed).double())
    x, q, s, z, add = _matvec_inputs(case, seed)
    x, group = x.double(), case["group"]
    y = torch.zeros(case["T"], case["N"], dtype=torch.float64, device=DEVICE)
    for i, at in enumerate(range(0, case["K"], group)):
        part = x[:, at: at + group]
        y += s[i].double() * (torch.mm(part, q[at: at + group].double()) - part.sum(1, keepdim=True) * (8.0 if z is None else z[i].double()))
    if case["gated"]:
        half = case["N"] // 2
        y = torch.nn.functional.silu(y[:, :half]) * y[:, half:]
    return y if add is None else y + add.double()
