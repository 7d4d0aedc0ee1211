"""Layers in 8-bit floating point with what surrounds them in a block: activation and residual, the dense MLP, the layer of experts.

Three operators, as a serving program calls them through the package (all with one scale per 128 channels, weights as E4M3 codes):

``linear``   a layer with its epilogue, act(X W + bias) + residual in one call (``Fp8Plan.linear_forward`` and, with ``experts``,
             ``Fp8Plan.grouped_forward`` for rows that lie sorted by expert);
``mlp``      up product, activation (gated: act(gate) * up), quantized again, down product, residual (``mlp_forward``);
``moe``      a whole layer of experts: router product, the k largest logits of every token, the gated MLP of the chosen experts, their
             weighted sum, residual (``moe_forward``), for one token up to a batch of prompts.

The weights are held as codes and scales before the call (in the package's plans, or as they are for the plain form).
"""
from __future__ import annotations

import math
import random

import torch

own = False

BLOCK = 128
E4M3_MAX = 448.0
SMALLEST = 1.75 * 2.0 ** -118  # a block's largest magnitude counts as at least this: its scale is then a normal number


def _case(name=None, **kw):
    c = dict(kw)
    if name is not None:
        c["name"] = name
    return c


def _linear(name=None, **kw):
    return _case(name, **{**dict(op="linear", experts=0, x="bf16", y="bf16", scales="f32", bias=0, act="none", residual=0, pad=0), **kw})


def _mlp(name=None, **kw):
    return _case(name, **{**dict(op="mlp", x="bf16", y="bf16", scales="f32", gated=0, bias=0, act="gelu", residual=1, pad=0), **kw})


def _moe(name=None, **kw):
    return _case(name, **{**dict(op="moe", x="bf16", y="bf16", scales="f32", router="bf16", masked=0.0, act="silu", renormalize=1, residual=1), **kw})


def listed():
    return [
        # one token through the attention's output projection while a model answers, the residual stream added: latency
        _linear("linear_token", rows=1, d_in=4096, d_out=4096, residual=1),
        # a small batch in odd widths, parts of wider buffers, fp32 in and out
        _linear("linear_odd", rows=53, d_in=1001, d_out=2051, x="f32", y="f32", scales="pow2", bias=1, act="gelu", residual=1, pad=7),
        # MLP up-projection of a diffusion transformer, two 64 x 64 token grids
        _linear("linear_image", rows=8192, d_in=1152, d_out=4608, bias=1, act="gelu_tanh"),
        # MLP down-projection over long prompts with the residual stream: the largest layer
        _linear("linear_prompt", rows=16384, d_in=11008, d_out=4096, residual=1),
        # rows sorted by expert through ungated experts' first layer, uneven loads
        _linear("linear_experts", rows=4096, experts=32, d_in=4096, d_out=1536, bias=1, act="relu"),
        # the gated MLP of a language model for one token of an answer
        _mlp("mlp_token", rows=1, d=4096, ff=11008, d_out=4096, gated=1, act="silu"),
        # a small MLP in odd widths, fp32 in and out (a head around the codes)
        _mlp("mlp_odd", rows=100, d=590, ff=1185, d_out=715, x="f32", y="f32", scales="pow2", bias=1, pad=5),
        # the MLP of a diffusion transformer, two 64 x 64 token grids
        _mlp("mlp_image", rows=8192, d=1152, ff=4608, d_out=1152, bias=1, act="gelu_tanh"),
        # the gated MLP of a language model over prompts
        _mlp("mlp_prompt", rows=8192, d=4096, ff=11008, d_out=4096, gated=1, act="silu"),
        # the layer of experts for one token of an answer
        _moe("moe_token", tokens=1, experts=64, top_k=6, d=2048, ff=1408),
        # the same for a batch of answers over many experts
        _moe("moe_batch", tokens=16, experts=256, top_k=8, d=4096, ff=1536),
        # the same over a short prompt, a tenth of the experts masked out
        _moe("moe_prompt", tokens=512, experts=64, top_k=6, d=2048, ff=1408, router="f32", masked=0.1, renormalize=0),
    ]


def draw(rng):
    """One more case: an operator, then its sizes over their range (logarithmic where it is wide)."""
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):  # mostly whole blocks, now and then any number
        n = logint(lo, hi)
        return n if rng.random() < 0.3 else max(BLOCK, (n + 64) // BLOCK * BLOCK)

    op = rng.choice(["linear", "linear", "linear", "mlp", "mlp", "moe", "moe", "moe"])
    kw = dict(scales=rng.choice(["f32", "f32", "pow2"]), x=rng.choice(["bf16", "bf16", "f32"]), y=rng.choice(["bf16", "bf16", "f32"]),
              residual=rng.choice([1, 1, 0]))
    if op == "moe":
        experts = logint(2, 256)
        while True:
            c = _moe(tokens=logint(1, 16) if rng.random() < 0.7 else logint(17, 512), experts=experts, top_k=rng.randint(1, min(8, experts)),
                     d=width(256, 4096), ff=width(256, 2048), router=rng.choice(["bf16", "f32"]), masked=rng.choice([0.0, 0.0, 0.1, 0.6]),
                     act=rng.choice(["silu", "silu", "gelu_tanh"]), renormalize=rng.randrange(2), **kw)
            if experts * c["d"] * c["ff"] <= 2 ** 30 and c["tokens"] * c["top_k"] * c["d"] * c["ff"] <= 2 ** 35:
                return c
    kw["pad"] = rng.choice([0, 0, 8, 5])
    if op == "mlp":
        gated = rng.randrange(2)
        while True:
            d = width(128, 8192)
            c = _mlp(rows=logint(1, 16384), d=d, ff=width(256, 16384), d_out=rng.choice([d, d, width(128, 8192)]), gated=gated,
                     bias=rng.randrange(2), act=rng.choice(["relu", "silu", "gelu", "gelu_tanh"]), **kw)
            if c["rows"] * c["ff"] * ((1 + gated) * d + c["d_out"]) <= 2 ** 39:
                return c
    experts = rng.choice([0, 0, logint(2, 64)])
    while True:
        c = _linear(rows=logint(1, 16384), experts=experts, d_in=width(256, 8192), d_out=width(256, 16384), bias=rng.randrange(2),
                    act=rng.choice(["none", "none", "relu", "silu", "gelu", "gelu_tanh"]), **kw)
        if c["rows"] * c["d_in"] * c["d_out"] <= 2 ** 39 and max(1, experts) * c["d_in"] * c["d_out"] <= 2 ** 30:
            return c


# ---- inputs ----

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(2000003 * (seed + 1))


def _activations(rows, d, dtype, pad, gen):
    """Rows of language-model activations: unit noise, one channel in a hundred 30 times larger, some rows much larger than others."""
    wide = torch.randn((rows, d + pad), device="cuda", generator=gen)
    wide *= torch.where(torch.rand(d + pad, device="cuda", generator=gen) < 0.01, 30.0, 1.0)
    wide *= torch.exp2(torch.randint(-2, 3, (rows, 1), device="cuda", generator=gen).float())
    return wide.to(_DTYPE[dtype])[:, :d]


def _weights(mats, d_out, d_in, pow2, gen):
    """E4M3 codes [mats, d_out, d_in] and the scale of every 128 x 128 block, as a checkpoint holds them; outputs of these activations
    are of the order of one."""
    nr, nc = -(-d_out // BLOCK), -(-d_in // BLOCK)
    codes = torch.empty((mats, d_out, d_in), device="cuda", dtype=torch.float8_e4m3fn)
    scales = torch.empty((mats, nr, nc), device="cuda")
    per = max(1, (1 << 28) // (d_out * d_in))
    for e in range(0, mats, per):
        n = min(per, mats - e)
        w = torch.randn((n, d_out, d_in), device="cuda", generator=gen)
        spread = torch.exp(0.3 * torch.randn((n, nr, nc), device="cuda", generator=gen)) * (0.5 / math.sqrt(d_in))
        s = spread * (4.5 / E4M3_MAX)
        if pow2:
            s = torch.exp2(torch.ceil(torch.log2(s)))
        each = (spread / s).repeat_interleave(BLOCK, 1)[:, :d_out].repeat_interleave(BLOCK, 2)[:, :, :d_in]
        w.mul_(each).clamp_(-E4M3_MAX, E4M3_MAX)
        codes[e:e + n] = w.to(torch.float8_e4m3fn)
        scales[e:e + n] = s
    return codes, scales


def _counts(c):
    """Rows of every expert: falling as the square root of the expert's rank, the last tenth of the experts none."""
    busy = c["experts"] - c["experts"] // 10
    share = [1.0 / math.sqrt(i + 1) for i in range(busy)]
    total, counts, left = sum(share), [], c["rows"]
    for s in share:
        n = min(left, int(c["rows"] * s / total))
        counts.append(n)
        left -= n
    for i in range(left):
        counts[i % busy] += 1
    return counts + [0] * (c["experts"] - busy)


def _made(case, seed):
    """The case's data, the same for either side."""
    c, gen = case, _generator(seed)
    s, pow2 = {"case": c}, c["scales"] == "pow2"

    def residual(rows, d_out):
        wide = torch.randn((rows, d_out + c.get("pad", 0)), device="cuda", generator=gen)
        return wide.to(_DTYPE[c["y"]])[:, :d_out] if c["residual"] else None

    def bias(sets, d_out):
        return 0.5 * torch.randn((sets, d_out), device="cuda", generator=gen) if c["bias"] else None
    if c["op"] == "linear":
        sets = max(1, c["experts"])
        s["x"] = _activations(c["rows"], c["d_in"], c["x"], c["pad"], gen)
        s["w"], s["ws"] = _weights(sets, c["d_out"], c["d_in"], pow2, gen)
        s["bias"], s["residual"] = bias(sets, c["d_out"]), residual(c["rows"], c["d_out"])
        if c["experts"]:
            counts = _counts(c)
            random.Random(seed).shuffle(counts)
            s["counts"] = counts
            s["offsets"] = torch.tensor([sum(counts[:i]) for i in range(sets + 1)], dtype=torch.int32, device="cuda")
    elif c["op"] == "mlp":
        s["x"] = _activations(c["rows"], c["d"], c["x"], c["pad"], gen)
        s["w_up"], s["ws_up"] = _weights(1 + c["gated"], c["ff"], c["d"], pow2, gen)  # gated: gate, up
        s["w_down"], s["ws_down"] = _weights(1, c["d_out"], c["ff"], pow2, gen)
        s["b_up"] = None if c["gated"] else bias(1, c["ff"])
        s["b_down"], s["residual"] = bias(1, c["d_out"]), residual(c["rows"], c["d_out"])
    else:
        E, d, ff = c["experts"], c["d"], c["ff"]
        s["x"] = _activations(c["tokens"], d, c["x"], 0, gen)
        s["router"] = (torch.randn((E, d), device="cuda", generator=gen) / math.sqrt(10.0 * d)).to(_DTYPE[c["router"]])
        s["router_bias"] = None
        if c["masked"]:  # experts that are out of use
            s["router_bias"] = torch.where(torch.rand(E, device="cuda", generator=gen) < c["masked"], -math.inf, 0.0)
        w, ws = _weights(2 * E, ff, d, pow2, gen)
        s["w_up"], s["ws_up"] = w.view(E, 2, ff, d), ws.view(E, 2, *ws.shape[1:])
        s["w_down"], s["ws_down"] = _weights(E, d, ff, pow2, gen)
        s["residual"] = residual(c["tokens"], d)
    return s


def prepare(case, seed):
    s = _made(case, seed)
    if own:
        import paper_2510_26771_amd as st
        c = case
        code = {"f32": st.STAMP_F32, "bf16": st.STAMP_BF16}
        form = {"f32": st.STAMP_SCALE_F32, "pow2": st.STAMP_SCALE_POW2}[c["scales"]]
        x, y = code[c["x"]], code[c["y"]]
        if c["op"] == "linear":
            desc = st.Fp8Desc(d_in=c["d_in"], d_out=c["d_out"], experts=c["experts"], x_dtype=x, y_dtype=y, scale_format=form)
            s["plan"] = st.Fp8Plan(desc, s["w"], s["ws"], s["bias"])
            s["workspace"] = s["plan"].alloc_workspace(c["rows"])
            s["y"] = torch.empty((c["rows"], c["d_out"]), dtype=_DTYPE[c["y"]], device="cuda")
        else:
            moe = c["op"] == "moe"
            E = c["experts"] if moe else c["gated"]  # a gated plan of one expert is a dense gated layer
            up = st.Fp8Desc(d_in=c["d"], d_out=c["ff"], experts=E, gated=int(moe or c["gated"]), x_dtype=x, scale_format=form)
            down = st.Fp8Desc(d_in=c["ff"], d_out=c["d"] if moe else c["d_out"], experts=c["experts"] if moe else 0, y_dtype=y, scale_format=form)
            s["up"] = st.Fp8Plan(up, s["w_up"], s["ws_up"], s.get("b_up"))
            s["down"] = st.Fp8Plan(down, s["w_down"], s["ws_down"], s.get("b_down"))
            rows = c["tokens"] if moe else c["rows"]
            s["y"] = torch.empty((rows, down.d_out), dtype=_DTYPE[c["y"]], device="cuda")
            if moe:
                s["routing"] = st.Routing(rows, E, c["top_k"])
                s["workspace"] = st.moe_workspace(s["up"], s["down"], rows, c["top_k"])
            else:
                s["workspace"] = st.mlp_workspace(s["up"], s["down"], rows)
    return s


# ---- the plain form: elementary torch operations in 32 bits ----

def _blocks(x):
    """[rows, d] -> [rows, blocks, 128], zeros behind the last channel."""
    rows, d = x.shape
    return torch.nn.functional.pad(x, (0, -d % BLOCK)).view(rows, -1, BLOCK)


def _coded(x, pow2):
    """The values that the E4M3 codes and the scales of x's blocks of 128 channels stand for."""
    v = _blocks(x.float())
    a = v.abs().amax(-1, keepdim=True).clamp_min(SMALLEST)
    if pow2:
        m, e = torch.frexp(a)
        e = e - 9 + (m > 0.875).int()
        scale, inv = ((127 + e) << 23).view(torch.float32), ((127 - e) << 23).view(torch.float32)
    else:
        top = torch.full_like(a, E4M3_MAX)
        scale, inv = a / top, top / a
    return ((v * inv).to(torch.float8_e4m3fn).float() * scale).reshape(x.shape[0], -1)[:, :x.shape[1]]


def _values(codes, scales):
    """Weights [d_out, d_in] that codes and block scales stand for."""
    d_out, d_in = codes.shape
    return codes.float() * scales.repeat_interleave(BLOCK, 0)[:d_out].repeat_interleave(BLOCK, 1)[:, :d_in]


def _by_expert(x, counts, w, ws):
    """Rows sorted by expert, each times its expert's weights."""
    return torch.cat([part @ _values(w[e], ws[e]).t() for e, part in enumerate(x.split(counts)) if counts[e]])


def _act(v, name):
    if name == "relu":
        return torch.clamp_min(v, 0.0)
    if name == "silu":
        return v / (1.0 + torch.exp(-v))
    if name == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    return v


def _rounded(y, residual, c):
    return (y if residual is None else y + residual.float()).to(_DTYPE[c["y"]])


def _plain_linear(s):
    c = s["case"]
    x = _coded(s["x"], c["scales"] == "pow2")
    if c["experts"]:
        y = _by_expert(x, s["counts"], s["w"], s["ws"])
        if s["bias"] is not None:
            y += torch.repeat_interleave(s["bias"], s["offsets"].diff().long(), 0, output_size=c["rows"])
    else:
        y = x @ _values(s["w"][0], s["ws"][0]).t()
        y = y if s["bias"] is None else y + s["bias"]
    return _rounded(_act(y, c["act"]), s["residual"], c)


def _plain_mlp(s):
    c, pow2 = s["case"], s["case"]["scales"] == "pow2"
    x = _coded(s["x"], pow2)
    h = x @ _values(s["w_up"][0], s["ws_up"][0]).t()
    if c["gated"]:
        h = _act(h, c["act"]) * (x @ _values(s["w_up"][1], s["ws_up"][1]).t())
    else:
        h = _act(h if s["b_up"] is None else h + s["b_up"], c["act"])
    y = _coded(h, pow2) @ _values(s["w_down"][0], s["ws_down"][0]).t()
    return _rounded(y if s["b_down"] is None else y + s["b_down"], s["residual"], c)


def _plain_moe(s):
    c, pow2, k = s["case"], s["case"]["scales"] == "pow2", s["case"]["top_k"]
    # which of two near logits is larger decides an expert: their sums in 64 bits, rounded once
    l = s["x"].double() @ s["router"].double().t()
    l = (l if s["router_bias"] is None else l + s["router_bias"].double()).float()
    top, ids = torch.sort(l, dim=1, descending=True, stable=True)
    most, top, ids = top[:, :1], top[:, :k], ids[:, :k].int()
    hit = top > -math.inf
    share = torch.where(hit, torch.exp(top - most), 0.0)
    norm = share if c["renormalize"] else torch.where(l > -math.inf, torch.exp(l - most), 0.0)
    weights = torch.where(hit, share / norm.sum(1, keepdim=True), 0.0)
    ids = torch.where(hit, ids, -1)
    flat = torch.where(hit, ids, c["experts"]).reshape(-1).long()
    order = torch.argsort(flat, stable=True)
    counts = torch.bincount(flat, minlength=c["experts"] + 1).tolist()[:-1]
    y = torch.zeros((c["tokens"], c["d"]), device="cuda")
    if sum(counts):
        order = order[:sum(counts)]
        x = _coded(s["x"], pow2)[order // k]
        gate = _by_expert(x, counts, s["w_up"][:, 0], s["ws_up"][:, 0])
        up = _by_expert(x, counts, s["w_up"][:, 1], s["ws_up"][:, 1])
        rows = _by_expert(_coded(_act(gate, c["act"]) * up, pow2), counts, s["w_down"], s["ws_down"])
        slots = torch.zeros((c["tokens"] * k, c["d"]), device="cuda")
        slots[order] = rows * weights.reshape(-1)[order, None]
        y = slots.view(c["tokens"], k, c["d"]).sum(1)
    return {"y": _rounded(y, s["residual"], c), "ids": ids, "weights": weights}


def run(state):
    s, c = state, state["case"]
    if not own:
        return {"linear": _plain_linear, "mlp": _plain_mlp, "moe": _plain_moe}[c["op"]](s)
    import paper_2510_26771_amd as st
    if c["op"] == "linear":
        if c["experts"]:
            s["plan"].grouped_forward(s["x"], s["offsets"], s["y"], s["workspace"], activation=c["act"], residual=s["residual"])
        else:
            s["plan"].linear_forward(s["x"], s["y"], s["workspace"], activation=c["act"], residual=s["residual"])
        return s["y"]
    if c["op"] == "mlp":
        st.mlp_forward(s["up"], s["down"], s["x"], s["y"], s["workspace"], activation=c["act"], residual=s["residual"])
        return s["y"]
    r = s["routing"]
    st.moe_forward(s["router"], s["up"], s["down"], s["x"], r, s["y"], s["workspace"], router_bias=s["router_bias"],
                   renormalize=bool(c["renormalize"]), activation=c["act"], residual=s["residual"])
    return {"y": s["y"], "ids": r.ids, "weights": r.weights}


def work(case):
    c = case
    size = {"f32": 4, "bf16": 2}

    def matrix(d_out, d_in):
        return d_out * d_in + 4 * -(-d_out // BLOCK) * -(-d_in // BLOCK)

    if c["op"] == "linear":
        hit = sum(n > 0 for n in _counts(c)) if c["experts"] else 1
        return {"bytes": hit * (matrix(c["d_out"], c["d_in"]) + 4 * c["d_out"] * c["bias"])
                + c["rows"] * (c["d_in"] * size[c["x"]] + c["d_out"] * size[c["y"]] * (1 + c["residual"])),
                "flops": 2 * c["rows"] * c["d_in"] * c["d_out"]}
    if c["op"] == "mlp":
        n = 1 + c["gated"]
        return {"bytes": n * matrix(c["ff"], c["d"]) + matrix(c["d_out"], c["ff"]) + 4 * c["bias"] * ((1 - c["gated"]) * c["ff"] + c["d_out"])
                + c["rows"] * (c["d"] * size[c["x"]] + c["d_out"] * size[c["y"]] * (1 + c["residual"])),
                "flops": 2 * c["rows"] * c["ff"] * (n * c["d"] + c["d_out"])}
    # rows over experts: as many experts as uniform choices would hit
    used = max(1, round(c["experts"] * (1.0 - c["masked"])))
    k = min(c["top_k"], used)
    slots = c["tokens"] * k
    hit = max(1, round(used * (1.0 - (1.0 - k / used) ** c["tokens"])))
    return {"bytes": hit * (2 * matrix(c["ff"], c["d"]) + matrix(c["d"], c["ff"])) + c["experts"] * c["d"] * size[c["router"]]
            + c["tokens"] * c["d"] * (size[c["x"]] + size[c["y"]] * (1 + c["residual"])) + 8 * c["tokens"] * c["top_k"],
            "flops": 6 * slots * c["d"] * c["ff"] + 2 * c["tokens"] * c["experts"] * c["d"]}


# ---- the definition in 64 bits, written apart from the plain form ----

def _e4m3(v):
    """The nearest E4M3 number: 4 significant bits down to 2^-6, steps of 2^-9 below; halves go to the even one."""
    mag = v.abs().clamp_min(2.0 ** -6)
    step = torch.exp2(torch.floor(torch.log2(mag)) - 3)
    return torch.round(v / step) * step


def _exact_codes(x, pow2):
    """Codes [rows, d] and scales [rows, blocks] in 64 bits.  By definition three values are 32-bit numbers: a scale, what a block is
    multiplied with (448 over its largest magnitude), and that product, of which the code is the nearest E4M3 number."""
    x = x.double()
    codes, scales = torch.empty_like(x), []
    for b in range(0, x.shape[1], BLOCK):
        v = x[:, b:b + BLOCK]
        a = v.abs().max(1).values.clamp(min=SMALLEST)
        if pow2:
            e = torch.floor(torch.log2(a / E4M3_MAX))
            s = torch.exp2(torch.where(torch.exp2(e) * E4M3_MAX >= a, e, e + 1))
            inv = 1.0 / s
        else:
            s, inv = (a / E4M3_MAX).float().double(), (E4M3_MAX / a).float().double()
        codes[:, b:b + BLOCK] = _e4m3((v * inv[:, None]).float().double())
        scales.append(s)
    return codes, torch.stack(scales, 1)


def _exact_product(codes, scales, w, ws):
    """Sum over the blocks of 128 channels of the codes' products times the two scales."""
    d_out = w.shape[0]
    y = torch.zeros((codes.shape[0], d_out), dtype=torch.float64, device=codes.device)
    for b in range(scales.shape[1]):
        part = codes[:, b * BLOCK:(b + 1) * BLOCK] @ w[:, b * BLOCK:(b + 1) * BLOCK].double().t().contiguous()
        part *= scales[:, b, None]
        part *= ws[:, b].double().repeat_interleave(BLOCK)[:d_out]
        y += part
    return y


def _exact_act(v, name):
    if name == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "gelu":
        return 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))
    if name == "gelu_tanh":
        return v * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))
    return v


def _exact_chosen(c, logits):
    """Ids and weights: the largest logit that is left, k times; the lowest expert where several are equal."""
    l = logits.cpu()
    left, column = l.clone(), torch.arange(c["experts"]).expand(l.shape)
    ids, value = torch.full((c["tokens"], c["top_k"]), -1, dtype=torch.int32), torch.full((c["tokens"], c["top_k"]), -math.inf, dtype=torch.float64)
    for j in range(min(c["top_k"], c["experts"])):
        best = left.max(1).values
        first = torch.where(left == best[:, None], column, c["experts"]).min(1).values
        ids[:, j] = torch.where(best > -math.inf, first, -1).int()
        value[:, j] = best
        left.scatter_(1, first[:, None], -math.inf)
    weights = torch.exp(value - torch.logsumexp(value if c["renormalize"] else l, 1, keepdim=True))
    weights[ids < 0] = 0.0
    return ids, weights


def exact(case, seed):
    c, s = case, _made(case, seed)
    pow2 = c["scales"] == "pow2"
    res = 0.0 if s["residual"] is None else s["residual"].double()
    if c["op"] == "linear":
        codes, scales = _exact_codes(s["x"], pow2)
        y = torch.empty((c["rows"], c["d_out"]), dtype=torch.float64, device="cuda")
        end = 0
        for e, n in enumerate(s["counts"] if c["experts"] else [c["rows"]]):
            if n:
                part = _exact_product(codes[end:end + n], scales[end:end + n], s["w"][e], s["ws"][e])
                y[end:end + n] = _exact_act(part if s["bias"] is None else part + s["bias"][e].double(), c["act"])
            end += n
        return y + res
    if c["op"] == "mlp":
        codes, scales = _exact_codes(s["x"], pow2)
        h = _exact_product(codes, scales, s["w_up"][0], s["ws_up"][0])
        if s["b_up"] is not None:
            h += s["b_up"].double()
        h = _exact_act(h, c["act"])
        if c["gated"]:
            h *= _exact_product(codes, scales, s["w_up"][1], s["ws_up"][1])
        y = _exact_product(*_exact_codes(h, pow2), s["w_down"][0], s["ws_down"][0])
        return y + res if s["b_down"] is None else y + s["b_down"].double() + res
    logits = torch.stack([(s["x"].double() * w.double()).sum(1) for w in s["router"]], 1).float().double()  # 32-bit numbers by definition
    if s["router_bias"] is not None:
        logits = logits + s["router_bias"].double()  # 0 or minus infinity
    ids, weights = _exact_chosen(c, logits)
    codes, scales = _exact_codes(s["x"], pow2)
    y = torch.zeros((c["tokens"], c["d"]), dtype=torch.float64, device="cuda")
    for e in range(c["experts"]):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if not t.numel():
            continue
        w = weights[t, j].cuda()
        t = t.cuda()
        gate = _exact_product(codes[t], scales[t], s["w_up"][e, 0], s["ws_up"][e, 0])
        up = _exact_product(codes[t], scales[t], s["w_up"][e, 1], s["ws_up"][e, 1])
        h, hs = _exact_codes(_exact_act(gate, c["act"]) * up, pow2)
        y.index_add_(0, t, w[:, None] * _exact_product(h, hs, s["w_down"][e], s["ws_down"][e]))
    return {"y": y + res, "ids": ids, "weights": weights}
