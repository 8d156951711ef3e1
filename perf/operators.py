"""The gated feed-forward block, the norms around it and the clipping of its gradients, as cases to be timed: each operator
as a training step or a serving loop calls it, and the same computed in elementary operations.

With `own` false, `run` computes the plain form in 32 bits, rounded once at the end; with `own` true it calls the library.
Sizes are generic: widths that are multiples of the matrix tiles and widths that are not, from one token to a long batch.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
LOSS_SCALE = 1024.0


def listed():
    return [
        # one new token through a wide block: every weight is read once, for one row
        dict(name="ffn_one_token", kind="ffn", train=False, dtype="f16", act="silu", rows=1, D=4096, F=12288),
        # a batch of requests that each add a token
        dict(name="ffn_requests", kind="ffn", train=False, dtype="bf16", act="gelu_tanh", rows=24, D=2048, F=5632),
        # a long prompt, or many, through a wide block
        dict(name="ffn_prompt", kind="ffn", train=False, dtype="bf16", act="silu", rows=16384, D=4096, F=12288),
        # a training step's pass through one block, forward and backward, with a loss scale
        dict(name="ffn_train", kind="ffn", train=True, dtype="f16", act="silu", rows=8192, D=2048, F=5632),
        # sizes that fill no tile and no 16-byte vector, and an activation with an error function
        dict(name="ffn_ragged", kind="ffn", train=True, dtype="f16", act="gelu", rows=777, D=1000, F=2730),
        # one token through the norms: launches are all there is to it
        dict(name="norm_one_token", kind="norm", train=False, dtype="f16", res="f16", rows=1, C=4096, groups=1, post=True, gate=True),
        # a training step's norms around one block, the residual stream in 32 bits
        dict(name="norm_train", kind="norm", train=True, dtype="f16", res="f32", rows=16384, C=4096, groups=1, post=True, gate=True),
        # gates that belong to each of many short sequences, at an odd width
        dict(name="norm_groups", kind="norm", train=True, dtype="bf16", res="bf16", rows=61 * 67, C=1001, groups=61, post=True, gate=True),
        # the plain layout: a norm in front of every block only
        dict(name="norm_prompt", kind="norm", train=False, dtype="bf16", res="bf16", rows=8192, C=2048, groups=1, post=False, gate=False),
        # gradients of a small network: scales, biases and a few matrices
        dict(name="clip_small", kind="clip", tensors=24, elements=400_000, mix="f16", over=True),
        # the 161 tensors' worth of the headline network's gradients, in FP16 with a loss scale
        dict(name="clip_25m", kind="clip", tensors=161, elements=25_557_032, mix="f16", over=True),
        # a large model's gradients on one card, matrices in BF16 and vectors in 32 bits
        dict(name="clip_600m", kind="clip", tensors=290, elements=600_000_000, mix="bf16+f32", over=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly multiples of 64, often of 8, now and then neither."""
    c, u = _log_int(rng, lo, hi), rng.random()
    if u < 0.15:
        c += c % 2 == 0
        return min(c, hi - 1)
    q = 8 if u < 0.35 else 64
    return max(q, (c + q // 2) // q * q)


def draw(rng):
    kind = rng.choice(["ffn", "ffn", "ffn", "norm", "norm", "clip"])
    if kind == "ffn":
        train = rng.random() < 0.5
        D = _width(rng, 256, 4096)
        F = _width(rng, 2 * D, 4 * D)
        if F == 3072:
            F += 64
        rows = _log_int(rng, 16, 16384) if train or rng.random() < 0.5 else _log_int(rng, 1, 128)
        c = dict(kind=kind, train=train, dtype=rng.choice(["f16", "bf16"]), act=rng.choice(["silu", "silu", "gelu_tanh", "gelu"]),
                 rows=rows, D=D if D != 3072 else 3136, F=F)
        while work(c)["flops"] > 4.9e12:
            c["rows"] = (c["rows"] + 1) // 2
        return c
    if kind == "norm":
        train = rng.random() < 0.5
        dtype = rng.choice(["f16", "f16", "bf16", "bf16", "f32"])
        C = _width(rng, 64, 8192)
        groups = rng.choice([1, 1, 1, 0])
        if groups == 0:
            groups = _log_int(rng, 2, 128)
        per = _log_int(rng, 1, max(1, 16384 // groups))
        post = rng.random() < 0.7
        c = dict(kind=kind, train=train, dtype=dtype, res=rng.choice([dtype, "f32"]), rows=groups * per, C=C if C != 3072 else 3080,
                 groups=groups, post=post, gate=groups > 1 or rng.random() < 0.5)
        return c
    return dict(kind=kind, tensors=_log_int(rng, 1, 400), elements=_log_int(rng, 20_000, 300_000_000), mix=rng.choice(["f16", "f16", "bf16", "f32", "bf16+f32"]),
                over=rng.random() < 0.75)


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _clip_sizes(case):
    """Half of the tensors are short vectors, the rest share the elements unevenly; nothing is aligned on purpose."""
    T, n = case["tensors"], case["elements"]
    short = [64 + 37 * i for i in range(T // 2)]
    while short and sum(short) > n // 2:
        short = [max(1, s // 2) for s in short]
    rest = T - len(short)
    weights = [1 + (7 * i) % 5 for i in range(rest)]
    left, total = n - sum(short), sum(weights)
    big = [left * w // total for w in weights]
    big[0] += left - sum(big)
    sizes = []
    for i in range(T):
        sizes.append(short.pop() if short and i % 2 else big.pop() if big else short.pop())
    return sizes


def _clip_types(case, sizes):
    if case["mix"] != "bf16+f32":
        return [TYPES[case["mix"]]] * len(sizes)
    return [torch.float32 if n < 100_000 else torch.bfloat16 for n in sizes]


def _randn(gen, shape, dtype, std=1.0, mean=0.0):
    """Normal numbers; made in 32 bits slab by slab, kept in the type."""
    t = torch.empty(shape, dtype=dtype, device=DEV)
    flat = t.view(-1)
    for at in range(0, flat.numel(), 1 << 26):
        part = flat[at:at + (1 << 26)]
        part.copy_(torch.randn(part.numel(), generator=gen, device=DEV).mul_(std).add_(mean))
    return t


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case)
    if case["kind"] == "ffn":
        M, D, F, t = case["rows"], case["D"], case["F"], TYPES[case["dtype"]]
        s["x"] = _randn(gen, (M, D), t)
        s["wg"], s["wu"] = _randn(gen, (F, D), t, D ** -0.5), _randn(gen, (F, D), t, D ** -0.5)
        s["wd"] = _randn(gen, (D, F), t, F ** -0.5)
        if case["train"]:
            s["dy"] = _randn(gen, (M, D), t, 0.05)      # the loss scale is in it, backed off until the weight gradients fit FP16
        if own:
            from paper_1807_11205_amd import api
            act = dict(silu=api.JZ_ACT_SILU, gelu=api.JZ_ACT_GELU, gelu_tanh=api.JZ_ACT_GELU_TANH, relu=api.JZ_ACT_RELU)[case["act"]]
            d = s["desc"] = api.ffn_desc(M, D, F, D, act, api.dtype_of(t))
            need = api.jz_ffn_fwd_workspace_bytes(d)
            s["h"], s["y"] = torch.empty((M, F), dtype=t, device=DEV), torch.empty((M, D), dtype=t, device=DEV)
            if case["train"]:
                need = max(need, api.jz_ffn_bwd_workspace_bytes(d))
                s["gate"], s["up"] = torch.empty_like(s["h"]), torch.empty_like(s["h"])
                s["dx"], s["dwg"], s["dwu"], s["dwd"] = (torch.empty_like(s[k]) for k in ("x", "wg", "wu", "wd"))
            s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    elif case["kind"] == "norm":
        M, C, G, t, rt = case["rows"], case["C"], case["groups"], TYPES[case["dtype"]], TYPES[case["res"]]
        s["r"], s["y"] = _randn(gen, (M, C), rt, 2.0), _randn(gen, (M, C), t, 0.7)
        s["w_pre"] = _randn(gen, (C,), torch.float32, 0.1, 1.0)
        s["w_post"] = _randn(gen, (C,), torch.float32, 0.1, 1.0) if case["post"] else None
        s["gate"] = _randn(gen, (G, C), torch.float32, 0.5) if case["gate"] else None
        s["eps"], s["res_scale"], s["branch_scale"] = 1e-5, 1.0, 0.75
        if case["train"]:
            s["dn"], s["dr_out"] = _randn(gen, (M, C), t, 0.05), _randn(gen, (M, C), rt, 0.05)
        if own:
            from paper_1807_11205_amd import api
            d = s["desc"] = api.norm_residual_desc(M, C, M // G, api.dtype_of(t), api.dtype_of(rt), s["eps"], s["res_scale"], s["branch_scale"])
            s["r_out"], s["n"] = torch.empty_like(s["r"]), torch.empty_like(s["y"])
            s["rstd_post"] = torch.empty(M, device=DEV) if case["post"] else None
            s["rstd_pre"] = torch.empty(M, device=DEV)
            if case["train"]:
                s["dr"], s["dy"] = torch.empty_like(s["r"]), torch.empty_like(s["y"])
                s["dw_pre"] = torch.empty(C, dtype=t, device=DEV)
                s["dw_post"] = torch.empty(C, dtype=t, device=DEV) if case["post"] else None
                s["dgate"] = torch.empty((G, C), dtype=t, device=DEV) if case["gate"] else None
                s["ws"] = torch.empty(api.jz_norm_residual_bwd_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    else:
        sizes = _clip_sizes(case)
        types = _clip_types(case, sizes)
        s["scale"] = LOSS_SCALE if case["mix"] == "f16" else 1.0
        # tensors of a network lie orders of magnitude apart
        stds = [1e-4 * 10.0 ** ((5 * i) % 7 / 3.0) for i in range(len(sizes))]
        # fused buffers, one a type, as the optimiser has them: where a tensor starts is as its neighbours' sizes have it
        s["grads"], s["flat"] = [], {}
        for t in dict.fromkeys(types):
            s["flat"][str(t)] = torch.empty(sum(n for n, o in zip(sizes, types) if o is t), dtype=t, device=DEV)
        at = dict.fromkeys(s["flat"], 0)
        for n, t, d in zip(sizes, types, stds):
            k = str(t)
            g = s["flat"][k][at[k]:at[k] + n]
            g.copy_(_randn(gen, (n,), t, d * s["scale"]))
            s["grads"].append(g)
            at[k] += n
        expected = math.sqrt(sum(n * d * d for n, d in zip(sizes, stds)))
        s["max_norm"] = expected * (0.3 if case["over"] else 3.0)
        if own:
            from paper_1807_11205_amd import api
            s["out"] = {k: torch.empty_like(v) for k, v in s["flat"].items()}
            views = [s["out"][str(g.dtype)][g.storage_offset():g.storage_offset() + g.numel()] for g in s["grads"]]
            s["list"] = api.GradList(s["grads"], views)
            s["ws"] = torch.empty(api.jz_grad_clip_workspace_bytes(s["list"]), dtype=torch.uint8, device=DEV)
            api.jz_grad_clip_prepare(s["list"], s["ws"])
            s["norm"] = torch.empty(1, device=DEV)
            s["found_inf"] = torch.empty(1, dtype=torch.int32, device=DEV)
    return s


# ---- the passes ---------------------------------------------------------------------------------------------------------
def run(state):
    if own:
        return dict(ffn=_own_ffn, norm=_own_norm, clip=_own_clip)[state["kind"]](state)
    return dict(ffn=_plain_ffn, norm=_plain_norm, clip=_plain_clip)[state["kind"]](state)


def _given(outputs):
    """Those that the case has."""
    return {k: v for k, v in outputs.items() if v is not None}


def _own_ffn(s):
    from paper_1807_11205_amd import api
    if not s["train"]:
        api.jz_ffn_fwd(s["desc"], s["x"], s["wg"], s["wu"], s["wd"], s["h"], s["y"], ws=s["ws"])
        return dict(y=s["y"])
    api.jz_ffn_fwd(s["desc"], s["x"], s["wg"], s["wu"], s["wd"], s["h"], s["y"], gate=s["gate"], up=s["up"], ws=s["ws"])
    api.jz_ffn_bwd(s["desc"], s["x"], s["wg"], s["wu"], s["wd"], s["gate"], s["up"], s["h"], s["dy"], s["dx"], s["dwg"], s["dwu"], s["dwd"], ws=s["ws"])
    return dict(y=s["y"], dx=s["dx"], dwg=s["dwg"], dwu=s["dwu"], dwd=s["dwd"])


def _own_norm(s):
    from paper_1807_11205_amd import api
    api.jz_norm_residual_fwd(s["desc"], s["r"], s["y"], s["w_post"], s["gate"], s["w_pre"], s["r_out"], s["n"], s["rstd_post"], s["rstd_pre"])
    if not s["train"]:
        return dict(r_out=s["r_out"], n=s["n"])
    api.jz_norm_residual_bwd(s["desc"], s["y"], s["r_out"], s["w_post"], s["gate"], s["w_pre"], s["rstd_post"], s["rstd_pre"], s["dr_out"], s["dn"],
                             s["dr"], s["dy"], s["dw_post"], s["dgate"], s["dw_pre"], s["ws"])
    return _given(dict(r_out=s["r_out"], n=s["n"], dr=s["dr"], dy=s["dy"], dw_post=s["dw_post"], dgate=s["dgate"], dw_pre=s["dw_pre"]))


def _own_clip(s):
    from paper_1807_11205_amd import api
    api.jz_grad_clip(s["list"], s["max_norm"], s["norm"], s["found_inf"], s["ws"], loss_scale=s["scale"])
    return dict(norm=s["norm"], found_inf=s["found_inf"], out=s["out"])


def _act(kind, g):
    """act(g) and its derivative."""
    if kind == "silu":
        a = 1.0 / (1.0 + torch.exp(-g))
        return g * a, a * (1.0 + g * (1.0 - a))
    if kind == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    if kind == "gelu":
        phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    k = math.sqrt(2.0 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * k * (1.0 + 3.0 * 0.044715 * g * g)


def _plain_ffn(s):
    t = s["x"].dtype
    x, wg, wu, wd = (s[k].float() for k in ("x", "wg", "wu", "wd"))
    g, u = x @ wg.t(), x @ wu.t()
    if not s["train"]:
        return dict(y=((_act(s["act"], g)[0] * u) @ wd.t()).to(t))
    a, da = _act(s["act"], g)
    h = a * u
    y = h @ wd.t()
    dy = s["dy"].float()
    dh = dy @ wd
    du, dg = dh * a, dh * u * da
    return dict(y=y.to(t), dx=(dg @ wg + du @ wu).to(t), dwg=(dg.t() @ x).to(t), dwu=(du.t() @ x).to(t), dwd=(dy.t() @ h).to(t))


def _rstd(v, eps):
    return 1.0 / torch.sqrt((v * v).mean(dim=1, keepdim=True) + eps)


def _plain_norm(s):
    t, rt = s["y"].dtype, s["r"].dtype
    M, C = s["y"].shape
    y, r, wq = s["y"].float(), s["r"].float(), s["w_pre"]
    k1 = _rstd(y, s["eps"]) if s["post"] else None
    p = y * k1 * s["w_post"] if s["post"] else y
    gate = s["branch_scale"] * s["gate"].repeat_interleave(M // s["groups"], dim=0) if s["gate"] is not None else s["branch_scale"]
    out = s["res_scale"] * r + gate * p
    k2 = _rstd(out, s["eps"])
    hat = out * k2
    res = dict(r_out=out.to(rt), n=(hat * wq).to(t))
    if not s["train"]:
        return res
    dn = s["dn"].float()
    e = dn * wq
    total = s["dr_out"].float() + k2 * (e - hat * (e * hat).mean(dim=1, keepdim=True))
    dp = gate * total
    res.update(dr=(s["res_scale"] * total).to(rt), dy=None, dw_post=None, dgate=None, dw_pre=(dn * hat).sum(dim=0).to(t))
    if s["gate"] is not None:
        res["dgate"] = (s["branch_scale"] * p * total).view(s["groups"], -1, C).sum(dim=1).to(t)
    if s["post"]:
        yh = y * k1
        e = dp * s["w_post"]
        res["dw_post"] = (dp * yh).sum(dim=0).to(t)
        dp = k1 * (e - yh * (e * yh).mean(dim=1, keepdim=True))
    res["dy"] = dp.to(t)
    return _given(res)


def _plain_clip(s):
    total = torch.zeros((), device=DEV)
    for flat in s["flat"].values():
        f = flat.float() * (1.0 / s["scale"])
        total = total + (f * f).sum()
    norm = torch.sqrt(total)
    bad = torch.logical_not(torch.isfinite(norm))
    c = torch.where(torch.logical_and(norm > s["max_norm"], torch.logical_not(bad)), s["max_norm"] / norm, torch.ones_like(norm))
    return dict(norm=norm.view(1), found_inf=bad.to(torch.int32).view(1), out={k: (v.float() * c).to(v.dtype) for k, v in s["flat"].items()})


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    if case["kind"] == "ffn":
        M, D, F = case["rows"], case["D"], case["F"]
        fwd, weights = 6 * M * D * F, 3 * D * F
        if not case["train"]:
            return dict(bytes=2 * (2 * M * D + weights), flops=fwd)
        return dict(bytes=2 * (4 * M * D + 2 * weights), flops=3 * fwd)     # x, dy in, y, dx out; weights in, their gradients out
    if case["kind"] == "norm":
        n, b, rb = case["rows"] * case["C"], 4 if case["dtype"] == "f32" else 2, 4 if case["res"] == "f32" else 2
        vectors = 4 * case["C"] * (1 + int(case["post"]) + (case["groups"] if case["gate"] else 0))
        moved, flops = n * (2 * rb + 2 * b) + vectors, n * (5 + (5 if case["post"] else 1))
        if case["train"]:
            moved, flops = moved + n * (2 * rb + 2 * b) + vectors * b // 4, flops + n * (11 + (12 if case["post"] else 1))
        return dict(bytes=moved, flops=flops)
    sizes = _clip_sizes(case)
    each = [4 if t is torch.float32 else 2 for t in _clip_types(case, sizes)]
    return dict(bytes=2 * sum(n * b for n, b in zip(sizes, each)), flops=3 * sum(sizes))


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------
def exact(case, seed):
    """What `run` returns, from the formulas in 64 bits."""
    s = prepare(case, seed)
    wide = torch.float64
    if case["kind"] == "ffn":
        x, a, b, c = s["x"].to(wide), s["wg"].to(wide), s["wu"].to(wide), s["wd"].to(wide)
        gate, up = torch.mm(x, a.t()), torch.mm(x, b.t())
        gate.requires_grad_(True)
        act = case["act"]
        if act == "silu":
            f = gate * torch.sigmoid(gate)
        elif act == "relu":
            f = torch.clamp(gate, min=0.0)
        elif act == "gelu":
            f = gate * torch.special.ndtr(gate)
        else:
            f = gate * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (gate + 0.044715 * gate ** 3))
        slope, = torch.autograd.grad(f.sum(), gate) if case["train"] else (None,)
        f = f.detach()
        mid = f * up
        y = torch.mm(mid, c.t())
        if not case["train"]:
            return dict(y=y)
        dy = s["dy"].to(wide)
        dmid = torch.mm(dy, c)
        dgate, dup = dmid * up * slope, dmid * f
        return dict(y=y, dx=torch.mm(dgate, a) + torch.mm(dup, b), dwg=torch.mm(dgate.t(), x), dwu=torch.mm(dup.t(), x), dwd=torch.mm(dy.t(), mid))
    if case["kind"] == "norm":
        leaves = {k: s[k].to(wide).requires_grad_(case["train"]) for k in ("r", "y", "w_pre", "w_post", "gate") if s[k] is not None}

        def rms(v):
            return v / torch.sqrt(v.square().sum(1, keepdim=True) / v.shape[1] + s["eps"])

        p = rms(leaves["y"]) * leaves["w_post"] if case["post"] else leaves["y"]
        if case["gate"]:
            p = (p.view(case["groups"], -1, case["C"]) * leaves["gate"].unsqueeze(1)).view(case["rows"], case["C"])
        out = s["res_scale"] * leaves["r"] + s["branch_scale"] * p
        n = rms(out) * leaves["w_pre"]
        res = dict(r_out=out.detach(), n=n.detach())
        if case["train"]:
            names = list(leaves)
            grads = dict(zip(names, torch.autograd.grad([out, n], [leaves[k] for k in names], [s["dr_out"].to(wide), s["dn"].to(wide)])))
            res.update(dr=grads["r"], dy=grads["y"], dw_post=grads.get("w_post"), dgate=grads.get("gate"), dw_pre=grads["w_pre"])
        return _given(res)
    squares = sum(float(torch.linalg.vector_norm(v, dtype=wide).item()) ** 2 for v in s["flat"].values())
    norm = math.sqrt(squares) / s["scale"]
    c = min(1.0, s["max_norm"] / norm)
    return dict(norm=torch.tensor([norm], dtype=wide, device=DEV), found_inf=torch.zeros(1, dtype=torch.int32, device=DEV),
                out={k: v.to(wide) * c for k, v in s["flat"].items()})
