"""Embedding lookup with its gradient, orthogonalised updates, and products in 8-bit integers, as cases to be timed: each operator as a
training step or a serving loop calls it, and the same computed in elementary operations.

With `own` false, `run` computes the plain form in 32 bits, rounded once at the end; with `own` true it calls the library.
Sizes are generic: widths that are multiples of the matrix tiles and widths that are not, from one token to a long batch.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
COEFS = (3.4445, -4.7750, 2.0315)   # of the fifth-degree polynomial that every step applies to the singular values
EPS = 1e-7
LOSS_SCALE = 1024.0


def listed():
    return [
        # one token's vector into an FP32 residual stream: a launch is all there is to it
        dict(name="embed_one_token", kind="embed", train=False, tokens=1, vocab=50000, D=4096, dtype="f16", out="f32", masked=False),
        # a long prompt, or many
        dict(name="embed_prompt", kind="embed", train=False, tokens=32768, vocab=131072, D=4096, dtype="bf16", out="bf16", masked=False),
        # a training step: lookup into an FP32 stream, and the gradient of the whole table, FP16 with a loss scale, frequent and rare tokens as in a text
        dict(name="embed_train", kind="embed", train=True, tokens=16384, vocab=50001, D=2048, dtype="f16", out="f32", masked=True),
        # short batch, odd sizes: most of the table has no token
        dict(name="embed_train_ragged", kind="embed", train=True, tokens=1777, vocab=32003, D=1001, dtype="bf16", out="bf16", masked=True),
        # a small matrix's update: a chain of short launches
        dict(name="ortho_small", kind="ortho", count=1, rows=128, cols=512, dtype="f16", out="f16"),
        # sizes that fill no tile, more rows than columns, full precision
        dict(name="ortho_ragged", kind="ortho", count=3, rows=1001, cols=333, dtype="f32", out="f32"),
        # the whole update of one kind of weight of a stack of blocks: momentum, orthogonalisation, master weights and their FP16 copy
        dict(name="muon_stack", kind="muon", count=16, rows=2816, cols=1024, dtype="f16"),
        # one matrix of a wide block
        dict(name="ortho_large", kind="ortho", count=1, rows=4096, cols=12288, dtype="bf16", out="bf16"),
        # one new token through a wide layer: every weight is read once, for one row
        dict(name="i8_one_token", kind="i8", rows=1, K=4096, N=12288, dtype="f16"),
        # sizes that fill no tile and no 16-byte vector
        dict(name="i8_ragged", kind="i8", rows=777, K=1001, N=2730, dtype="f16"),
        # a batch of requests that each add a token through a gated block
        dict(name="i8_block_requests", kind="i8ffn", rows=24, D=2048, F=5632, dtype="bf16", act="silu"),
        # a long prompt, or many, through a wide layer
        dict(name="i8_prompt", kind="i8", rows=16384, K=4096, N=12288, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Mostly multiples of 64, often of 8, now and then neither."""
    c, u = _log_int(rng, lo, hi), rng.random()
    if u < 0.2:
        c += c % 2 == 0
        return min(c, hi - 1)
    q = 8 if u < 0.4 else 64
    return min(hi, max(q, (c + q // 2) // q * q))


def draw(rng):
    kind = rng.choice(["embed", "embed", "ortho", "muon", "i8", "i8", "i8ffn"])
    if kind == "embed":
        dtype = rng.choice(["f16", "f16", "bf16", "bf16", "f32"])
        c = dict(kind=kind, train=rng.random() < 0.6, tokens=_log_int(rng, 1, 65536), vocab=_log_int(rng, 500, 200000), D=_width(rng, 64, 8192), dtype=dtype,
                 out=rng.choice([dtype, "f32"]), masked=rng.random() < 0.5)
        while c["vocab"] * c["D"] > 3e8:
            c["vocab"] = c["vocab"] // 2 + 1
        while c["tokens"] * c["D"] > 1.3e8:
            c["tokens"] = c["tokens"] // 2 + 1
        return c
    if kind in ("ortho", "muon"):
        c = dict(kind=kind, count=_log_int(rng, 1, 16), rows=_width(rng, 16, 4096), cols=_width(rng, 16, 4096), dtype=rng.choice(["f16", "bf16"]))
        if kind == "ortho":
            c["dtype"] = rng.choice(["f16", "bf16", "f32"])
            c["out"] = rng.choice([c["dtype"], "f32", "bf16"])
        while work(c)["flops"] > 1.5e12:
            c["count"] = (c["count"] + 1) // 2
        return c
    dtype = rng.choice(["f16", "bf16"])
    rows = _log_int(rng, 1, 128) if rng.random() < 0.5 else _log_int(rng, 64, 8192)
    if kind == "i8":
        return dict(kind=kind, rows=rows, K=_width(rng, 64, 8192), N=_width(rng, 64, 12288), dtype=dtype)
    D = _width(rng, 64, 4096)
    rows = min(rows, 4096)
    return dict(kind=kind, rows=rows, D=D, F=_width(rng, 2 * D, 4 * D), dtype="bf16", act=rng.choice(["silu", "gelu_tanh", "gelu", "relu"]))


# ---- inputs -------------------------------------------------------------------------------------------------------------
def _randn(gen, shape, dtype, std=1.0):
    """Normal numbers; made in 32 bits slab by slab, kept in the type."""
    t = torch.empty(shape, dtype=dtype, device=DEV)
    flat = t.view(-1)
    for at in range(0, flat.numel(), 1 << 26):
        part = flat[at:at + (1 << 26)]
        part.copy_(torch.randn(part.numel(), generator=gen, device=DEV).mul_(std))
    return t


def _token_ids(gen, case):
    """The r-th most frequent token about 1 / r as often as the first, spread over the table; some places masked by -1."""
    n, V = case["tokens"], case["vocab"]
    rank = torch.exp(torch.rand(n, generator=gen, device=DEV, dtype=torch.float64) * math.log(V)).long().clamp_(1, V) - 1
    step = 7919
    while math.gcd(step, V) != 1:
        step += 2
    ids = (rank * step + 13) % V
    if case["masked"]:
        ids[torch.rand(n, generator=gen, device=DEV) < 0.05] = -1
    return ids.to(torch.int32)


def _gradients(gen, case, dtype, scale):
    """[count, rows, cols]: a few strong directions over noise, as gradients and their running means have."""
    B, R, C = case["count"], case["rows"], case["cols"]
    t = torch.empty((B, R, C), dtype=dtype, device=DEV)
    k = max(1, min(12, R // 2, C // 2))
    strength = torch.tensor([0.5 ** i for i in range(k)], device=DEV)
    for b in range(B):
        u = torch.randn((R, k), generator=gen, device=DEV) * strength
        v = torch.randn((k, C), generator=gen, device=DEV)
        noise = torch.randn((R, C), generator=gen, device=DEV)
        t[b].copy_((noise * 0.3 + u @ v) * (1e-3 * scale))
    return t


def _codes(w):
    """int8 codes and FP32 scales of the rows of w, as a model's weights are kept."""
    f = w.float()
    s = f.abs().amax(dim=1) / 127.0
    q = torch.where(s[:, None] > 0, torch.round(f / s[:, None]), torch.zeros_like(f))
    return q.clamp_(-127, 127).to(torch.int8), s


def _weights(gen, rows, cols):
    """Channels of different strength."""
    w = _randn(gen, (rows, cols), torch.float32, cols ** -0.5)
    return _codes(w * (0.5 + torch.rand((rows, 1), generator=gen, device=DEV)))


def _tokens(gen, rows, cols, dtype):
    """Activations: a few channels are ten times as large as the others."""
    x = torch.randn((rows, cols), generator=gen, device=DEV)
    x[:, ::max(1, cols // 6)] *= 10.0
    return x.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = dict(case)
    if own:
        from paper_1807_11205_amd import api
    t = TYPES[case["dtype"]]
    if case["kind"] == "embed":
        n, V, D, o = case["tokens"], case["vocab"], case["D"], TYPES[case["out"]]
        s["ids"] = _token_ids(gen, case)
        s["table"] = _randn(gen, (V, D), t, 0.02)
        s["scale"] = float(D) ** 0.5
        if case["train"]:
            s["dy"] = _randn(gen, (n, D), o, 1e-3)
        if own:
            d = s["desc"] = api.embed_desc(n, V, D, api.dtype_of(t), api.dtype_of(o), s["scale"])
            s["y"] = torch.empty((n, D), dtype=o, device=DEV)
            if case["train"]:
                s["dtable"] = torch.empty_like(s["table"])
                s["ws"] = torch.empty(api.jz_embed_bwd_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    elif case["kind"] == "ortho":
        s["x"] = _gradients(gen, case, t, 1.0)
        if own:
            d = s["desc"] = api.ortho_desc(case["count"], case["rows"], case["cols"], api.dtype_of(t), api.dtype_of(TYPES[case["out"]]), 5, COEFS, EPS)
            s["y"] = torch.empty(s["x"].shape, dtype=TYPES[case["out"]], device=DEV)
            s["ws"] = torch.empty(api.jz_orthogonalize_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    elif case["kind"] == "muon":
        shape = (case["count"], case["rows"], case["cols"])
        s["grad"] = _gradients(gen, case, t, LOSS_SCALE)
        s["momentum"] = _gradients(gen, case, torch.float32, 10.0)
        s["master"] = _randn(gen, shape, torch.float32, case["cols"] ** -0.5)
        s["w16"] = s["master"].to(t)
        s["hp"] = dict(lr=0.02, momentum=0.95, weight_decay=0.01, update_scale=max(1.0, case["rows"] / case["cols"]) ** 0.5, nesterov=True, loss_scale=LOSS_SCALE)
        if own:
            d = s["desc"] = api.ortho_desc(case["count"], case["rows"], case["cols"], api.dtype_of(t), api.dtype_of(t), 5, COEFS, EPS)
            s["own_hp"] = api.muon_hparams(**s["hp"])
            s["found_inf"] = torch.zeros(1, dtype=torch.int32, device=DEV)
            s["ws"] = torch.empty(api.jz_muon_mp_update_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    elif case["kind"] == "i8":
        M, K, N = case["rows"], case["K"], case["N"]
        s["x"] = _tokens(gen, M, K, t)
        s["wq"], s["ws_"] = _weights(gen, N, K)
        if own:
            d = s["desc"] = api.linear_i8_desc(M, K, N, api.dtype_of(t))
            s["wq"] = _own_layout(s["wq"])
            s["y"] = torch.empty((M, N), dtype=t, device=DEV)
            s["ws"] = torch.empty(api.jz_linear_i8_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    else:
        M, D, F = case["rows"], case["D"], case["F"]
        s["x"] = _tokens(gen, M, D, t)
        for k, (a, b) in dict(gate=(F, D), up=(F, D), down=(D, F)).items():
            s["q_" + k], s["s_" + k] = _weights(gen, a, b)
            if own:
                s["q_" + k] = _own_layout(s["q_" + k])
        if own:
            act = dict(silu=api.JZ_ACT_SILU, gelu=api.JZ_ACT_GELU, gelu_tanh=api.JZ_ACT_GELU_TANH, relu=api.JZ_ACT_RELU)[case["act"]]
            d = s["desc"] = api.ffn_desc(M, D, F, D, act, api.dtype_of(t))
            s["y"] = torch.empty((M, D), dtype=t, device=DEV)
            s["ws"] = torch.empty(api.jz_ffn_i8_workspace_bytes(d), dtype=torch.uint8, device=DEV)
    return s


def _own_layout(q):
    """Codes in rows of a multiple of 16 bytes, zeros behind their end: laid out once, with the weights."""
    from paper_1807_11205_amd import api
    to = torch.zeros((q.shape[0], api.i8_pitch(q.shape[1])), dtype=torch.int8, device=DEV)
    to[:, :q.shape[1]] = q
    return to


# ---- the passes ---------------------------------------------------------------------------------------------------------
def run(state):
    if own:
        return dict(embed=_own_embed, ortho=_own_ortho, muon=_own_muon, i8=_own_i8, i8ffn=_own_i8ffn)[state["kind"]](state)
    return dict(embed=_plain_embed, ortho=_plain_ortho, muon=_plain_muon, i8=_plain_i8, i8ffn=_plain_i8ffn)[state["kind"]](state)


def _own_embed(s):
    from paper_1807_11205_amd import api
    api.jz_embed_fwd(s["desc"], s["ids"], s["table"], s["y"])
    if not s["train"]:
        return dict(y=s["y"])
    api.jz_embed_bwd(s["desc"], s["ids"], s["dy"], s["dtable"], s["ws"])
    return dict(y=s["y"], dtable=s["dtable"])


def _own_ortho(s):
    from paper_1807_11205_amd import api
    api.jz_orthogonalize(s["desc"], s["x"], s["y"], s["ws"])
    return dict(y=s["y"])


def _own_muon(s):
    from paper_1807_11205_amd import api
    api.jz_muon_mp_update(s["desc"], s["own_hp"], s["master"], s["momentum"], s["grad"], s["w16"], s["found_inf"], s["ws"])
    return dict(master=s["master"], momentum=s["momentum"], w16=s["w16"], found_inf=s["found_inf"])


def _own_i8(s):
    from paper_1807_11205_amd import api
    api.jz_linear_i8(s["desc"], s["x"], s["wq"], s["ws_"], s["y"], s["ws"])
    return dict(y=s["y"])


def _own_i8ffn(s):
    from paper_1807_11205_amd import api
    api.jz_ffn_i8_fwd(s["desc"], s["x"], s["q_gate"], s["s_gate"], s["q_up"], s["s_up"], s["q_down"], s["s_down"], s["y"], s["ws"])
    return dict(y=s["y"])


def _plain_embed(s):
    ids = s["ids"].long()
    there = (ids >= 0) & (ids < s["vocab"])
    at = torch.where(there, ids, torch.zeros_like(ids))
    y = (s["table"][at].float() * (there.float() * s["scale"])[:, None]).to(TYPES[s["out"]])
    if not s["train"]:
        return dict(y=y)
    total = torch.zeros(s["table"].shape, dtype=torch.float32, device=DEV)
    total.index_add_(0, at, s["dy"].float() * there.float()[:, None])
    return dict(y=y, dtable=(total * s["scale"]).to(s["table"].dtype))


def _polar(x):
    """The polynomial's fifth iterate on the singular values of every matrix of x (32 bits)."""
    a, b, c = COEFS
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2).contiguous()
    x = x / (torch.sqrt((x * x).sum(dim=(1, 2), keepdim=True)) + EPS)
    for _ in range(5):
        g = torch.bmm(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.bmm(b * g + c * torch.bmm(g, g), x)
    return x.transpose(1, 2) if tall else x


def _plain_ortho(s):
    return dict(y=_polar(s["x"].float()).to(TYPES[s["out"]]).contiguous())


def _plain_muon(s):
    hp = s["hp"]
    g = s["grad"].float() * (1.0 / hp["loss_scale"])
    bad = torch.logical_not(torch.isfinite(g).all())
    v = hp["momentum"] * s["momentum"] + g
    o = _polar(g + hp["momentum"] * v)
    w = s["master"] - hp["lr"] * (hp["update_scale"] * o + hp["weight_decay"] * s["master"])
    s["momentum"].copy_(torch.where(bad, s["momentum"], v))
    s["master"].copy_(torch.where(bad, s["master"], w))
    s["w16"].copy_(torch.where(bad, s["w16"], w.to(s["w16"].dtype)))
    return dict(master=s["master"], momentum=s["momentum"], w16=s["w16"], found_inf=bad.to(torch.int32).view(1))


def _plain_product(x, wq, ws):
    """x (32 bits) quantised token by token, times codes: a sum of whole numbers, then both scales."""
    q, s = _codes(x)
    return (q.float() @ wq.float().t()) * s[:, None] * ws


def _plain_i8(s):
    return dict(y=_plain_product(s["x"].float(), s["wq"], s["ws_"]).to(s["x"].dtype))


def _plain_act(kind, g):
    if kind == "silu":
        return g / (1.0 + torch.exp(-g))
    if kind == "relu":
        return g * (g > 0).to(g.dtype)
    if kind == "gelu":
        return g * 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)))


def _plain_i8ffn(s):
    x = s["x"].float()
    g, u = _plain_product(x, s["q_gate"], s["s_gate"]), _plain_product(x, s["q_up"], s["s_up"])
    return dict(y=_plain_product(_plain_act(s["act"], g) * u, s["q_down"], s["s_down"]).to(s["x"].dtype))


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------
def work(case):
    size = {"f16": 2, "bf16": 2, "f32": 4}
    if case["kind"] == "embed":
        n, V, D, b, o = case["tokens"], case["vocab"], case["D"], size[case["dtype"]], size[case["out"]]
        rows = min(n, V)                    # different tokens are fewer still
        moved = 4 * n + rows * D * b + n * D * o
        if case["train"]:
            return dict(bytes=moved + 4 * n + n * D * o + V * D * b, flops=3 * n * D)
        return dict(bytes=moved, flops=n * D)
    if case["kind"] in ("ortho", "muon"):
        B, m, n = case["count"], min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # five steps of three products, two of which are symmetric; or, where one side is much longer, in the space of the shorter one
        each = min(5 * (3 * m * m * n + m ** 3), 6 * m * m * n + 14 * m ** 3)
        elements, b = B * m * n, size[case["dtype"]]
        if case["kind"] == "ortho":
            return dict(bytes=elements * (b + size[case["out"]]), flops=B * each)
        return dict(bytes=elements * (8 + 8 + 2 * b), flops=B * each)   # master and momentum in and out, gradient in, copy out
    if case["kind"] == "i8":
        M, K, N = case["rows"], case["K"], case["N"]
        return dict(bytes=2 * M * K + N * K + 4 * N + 2 * M * N, flops=2 * M * K * N)
    M, D, F = case["rows"], case["D"], case["F"]
    return dict(bytes=4 * M * D + 3 * D * F + 4 * (2 * F + D), flops=6 * M * D * F)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------
def _exact_polar(x):
    """Of one matrix, in the space of its shorter side: with A = X X^T every iterate is P(A) X, so P alone is carried along."""
    a, b, c = COEFS
    tall = x.shape[0] > x.shape[1]
    x = (x.t() if tall else x) / (torch.linalg.vector_norm(x) + EPS)
    A = torch.mm(x, x.t())
    eye = torch.eye(A.shape[0], dtype=A.dtype, device=DEV)
    P = eye
    for _ in range(5):
        G = P @ A @ P
        P = (a * eye + b * G + c * (G @ G)) @ P
    x = P @ x
    return x.t() if tall else x


def _f32(v):
    return v.to(torch.float32).to(torch.float64)


def _exact_product(x, wq, ws):
    """x: 64 bits. A row's scale is its largest magnitude / 127 in FP32, a code the FP32 quotient to the nearest whole number, ties to even."""
    s = _f32(x.abs().max(dim=1).values / 127.0)
    q = torch.clamp(torch.round(_f32(x / s.masked_fill(s == 0, 1.0)[:, None])), -127, 127)
    return torch.mm(q, wq.to(torch.float64).t()) * torch.outer(s, ws.to(torch.float64))


def exact(case, seed):
    """What `run` returns, from the formulas in 64 bits."""
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    wide = torch.float64
    if case["kind"] == "embed":
        ids = s["ids"].long()
        res = dict(y=torch.zeros((case["tokens"], case["D"]), dtype=wide, device=DEV))
        good = torch.nonzero((ids >= 0) & (ids < case["vocab"])).view(-1)
        res["y"][good] = s["table"].index_select(0, ids[good]).to(wide) * s["scale"]
        if case["train"]:
            # tokens in order, running sums, and what they grow by over each token's places
            order = good[torch.argsort(ids[good], stable=True)]
            count = torch.bincount(ids[good], minlength=case["vocab"])
            end = torch.cumsum(count, 0)
            d = torch.zeros(s["table"].shape, dtype=wide, device=DEV)
            for c in range(0, case["D"], 512):
                run_up = torch.cat([torch.zeros((1, min(512, case["D"] - c)), dtype=wide, device=DEV), torch.cumsum(s["dy"][:, c:c + 512].to(wide)[order], 0)])
                d[:, c:c + 512] = (run_up[end] - run_up[end - count]) * s["scale"]
            res["dtable"] = d
        return res
    if case["kind"] == "ortho":
        return dict(y=torch.stack([_exact_polar(x.to(wide)) for x in s["x"]]))
    if case["kind"] == "muon":
        hp = s["hp"]
        g = s["grad"].to(wide) / hp["loss_scale"]
        v = hp["momentum"] * s["momentum"].to(wide) + g
        o = torch.stack([_exact_polar(u) for u in g + hp["momentum"] * v])
        w = (1.0 - hp["lr"] * hp["weight_decay"]) * s["master"].to(wide) - hp["lr"] * hp["update_scale"] * o
        return dict(master=w, momentum=v, w16=w, found_inf=torch.zeros(1, dtype=torch.int32, device=DEV))
    if case["kind"] == "i8":
        return dict(y=_exact_product(s["x"].to(wide), s["wq"], s["ws_"]))
    g, u = (_exact_product(s["x"].to(wide), s["q_" + k], s["s_" + k]) for k in ("gate", "up"))
    act = case["act"]
    if act == "silu":
        h = g * torch.sigmoid(g)
    elif act == "relu":
        h = torch.clamp(g, min=0.0)
    elif act == "gelu":
        h = g * torch.special.ndtr(g)
    else:
        h = g * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3))
    return dict(y=_exact_product(_f32(h * u), s["q_down"], s["s_down"]))
