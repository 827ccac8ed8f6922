"""Expert products in 8-bit integers as cases that can be timed and compared: rows and weights brought into 8 bits, a matrix
product of both with a scale for each token and each channel, the experts' FFNs and a whole MoE layer made of them.

`run` is one pass through an operator: with `own` the calls that a user makes of paper_2201_05596_amd, otherwise the same in
elementary torch operations in 32 bits (64 for what stands next to a border: codes, scales and the choice of an expert).
`exact` is the definition in 64 bits, written apart from both.

  rows     moe_i8_quantize_rows of activations: a scale for each row
  weights  moe_i8_quantize_weights: a scale for each column, codes in the order that the products read
  linear   moe_i8_linear of codes that a program has, with bias and GELU or without
  ffn      moe_i8_expert_ffn on dispatched rows
  layer    moe_i8_layer_forward: gate, experts, combine, with a dense branch or without

A row (or column) whose largest magnitude is m has r = 127 / max(m, 2^-100) rounded to 32 bits, codes round(value r), ties to
even, and the scale max(m, 2^-100) / 127 rounded to 32 bits.  Hidden sizes, experts and tokens are those of the layer's own
configurations, with odd sizes between them.
"""
from __future__ import annotations

import math

import torch

own = False

LEAST = 2.0 ** -100                            # smallest magnitude that a scale is made from


def listed():
    return [
        # a ragged chunk of a prompt in 32 bits, columns of wider rows
        rows_case("rows_chunk_f32", rows=777, cols=1000, wider=512, dtype="f32"),
        # the activations of a prefill of 16384 tokens
        rows_case("rows_prefill", rows=16384, cols=4096),
        # one matrix of a size that fills no block
        weights_case("weights_dense", groups=1, K=1000, N=4000),
        # the first matrices of 64 experts, once per model
        weights_case("weights_experts", groups=64, K=2048, N=8192),
        # a projection of one token: the read of its weights
        linear_case("linear_token", rows=1, K=2048, N=6144, bias=True),
        # a ragged chunk of a prompt with bias and GELU, result in 32 bits
        linear_case("linear_chunk", rows=777, K=1000, N=4000, bias=True, gelu=True, out="f32"),
        # a projection of 8192 tokens: bound by the matrix cores
        linear_case("linear_prefill", rows=8192, K=4096, N=4096),
        # a decode step's rows, none to sixteen for each of 64 experts
        ffn_case("ffn_step", E=64, capacity=16, d=1024, f=4096, bias=True),
        # a prefill's rows, none to 512 for each of 16 experts
        ffn_case("ffn_prefill", E=16, capacity=512, d=2048, f=8192),
        # one token through a dense branch and two of 128 experts: latency is all there is
        layer_case("layer_token", T=1, d=1024, f=4096, E=128, top_k=2, capacity=1, residual=True, bias=True),
        # a decode step of 64 tokens, bound by the read of the experts that they reach
        layer_case("layer_step", T=64, d=2048, f=8192, E=128, top_k=1, capacity=8),
        # a prefill of 8192 tokens beside a dense branch
        layer_case("layer_prefill", T=8192, d=1024, f=4096, E=32, top_k=1, capacity=320, residual=True, bias=True),
    ]


def named(name, c):
    return {"name": name, **c} if name else c


def rows_case(name=None, *, rows, cols, wider=0, dtype="bf16"):
    return named(name, {"op": "rows", "rows": rows, "cols": cols, "wider": wider, "dtype": dtype})


def weights_case(name=None, *, groups, K, N):
    return named(name, {"op": "weights", "groups": groups, "K": K, "N": N})


def linear_case(name=None, *, rows, K, N, bias=False, gelu=False, out="bf16"):
    return named(name, {"op": "linear", "rows": rows, "K": K, "N": N, "bias": bias, "gelu": gelu, "out": out})


def ffn_case(name=None, *, E, capacity, d, f, bias=False):
    return named(name, {"op": "ffn", "E": E, "capacity": capacity, "d": d, "f": f, "bias": bias})


def layer_case(name=None, *, T, d, f, E, top_k, capacity, residual=False, bias=False, skewed=False):
    return named(name, {"op": "layer", "T": T, "d": d, "f": f, "E": E, "top_k": top_k, "capacity": capacity, "residual": residual,
                        "bias": bias, "skewed": skewed})


def draw(rng):
    """One more case: sizes over their logarithm, odd ones among them, no more work than the largest listed cases."""
    spread = lambda lo, hi: max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))  # noqa: E731
    width = lambda hi: rng.choice((8 * spread(1, hi // 8), 128 * spread(1, hi // 128), 1024, 2048))  # noqa: E731
    yes = lambda: rng.random() < 0.5  # noqa: E731
    while True:
        op = rng.choice(("rows", "weights", "linear", "linear", "ffn", "ffn", "layer", "layer", "layer"))
        if op == "rows":
            c = rows_case(rows=spread(1, 16384), cols=width(16384), wider=rng.choice((0, 0, 8 * spread(1, 128))), dtype=rng.choice(("bf16", "bf16", "f32")))
        elif op == "weights":
            c = weights_case(groups=spread(1, 128), K=width(8192), N=width(8192))
        elif op == "linear":
            c = linear_case(rows=spread(1, 8192), K=width(16384), N=width(16384), bias=yes(), gelu=yes(), out=rng.choice(("bf16", "bf16", "f32")))
        elif op == "ffn":
            c = ffn_case(E=spread(1, 128), capacity=spread(1, 512), d=width(4096), f=width(8192), bias=yes())
        else:
            T, E, k = spread(1, 8192), spread(2, 128), rng.choice((1, 1, 2))
            room = min(T, math.ceil(rng.choice((1.0, 1.25, 2.0)) * k * T / E))
            c = layer_case(T=T, d=width(4096), f=width(8192), E=E, top_k=k, capacity=rng.choice((room, room, min(T, max(room, 16)))), residual=yes(),
                           bias=yes(), skewed=rng.random() < 0.3)
        w, held = work(c), 0
        if op in ("ffn", "layer"):             # the plain form multiplies all the room that experts have
            held = c["E"] * (c["d"] * c["f"] + c["capacity"] * (c["d"] + c["f"]))
            w["flops"] = max(w["flops"], 4 * c["E"] * c["capacity"] * c["d"] * c["f"])
        most = {"rows": 2.1e8, "weights": 3.3e9, "linear": 2.8e8, "ffn": 2.2e9, "layer": 4.4e9}[op]
        if w["bytes"] <= most and w["flops"] <= 2.8e11 and held <= 2.2e9:
            return c


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def reached(case):
    """Experts that a layer's tokens reach on average, if they choose evenly."""
    E = case["E"]
    return E * (1 - (1 - 1 / E) ** (case["T"] * case["top_k"]))


def work(case):
    op = case["op"]
    if op == "rows":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (5 if case["dtype"] == "f32" else 3) + 4 * case["rows"], "flops": 2 * n}
    if op == "weights":
        n = case["groups"] * case["K"] * case["N"]
        return {"bytes": 3 * n + 4 * case["groups"] * case["N"], "flops": 2 * n}
    if op == "linear":
        R, K, N = case["rows"], case["K"], case["N"]
        out = 4 if case["out"] == "f32" else 2
        return {"bytes": R * K + 4 * R + N * (K + 4 + 2 * case["bias"]) + R * N * out, "flops": 2 * R * K * N}
    d, f = case["d"], case["f"]
    expert = 2 * d * f + (d + f) * (4 + 2 * case["bias"])
    if op == "ffn":
        rows = case["E"] * case["capacity"] // 2               # on average
        return {"bytes": case["E"] * case["capacity"] // (case["capacity"] + 1) * expert + 4 * rows * d, "flops": 4 * rows * d * f}
    T, k, dense = case["T"], case["top_k"], int(case["residual"])
    kept = min(T * k, case["E"] * case["capacity"])
    return {"bytes": int((reached(case) + dense) * expert) + 4 * T * d + 4 * d * case["E"], "flops": 4 * (kept + T * dense) * d * f + 2 * T * d * case["E"]}


# ---- what a program has in hand before the call ----------------------------------------------------------------

def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def activations(gen, rows, cols):
    """Normal values with a few large channels and rows of different sizes."""
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    x = x * (1 + 7 * (torch.rand((1, cols), generator=gen, device="cuda") > 0.98))
    return x * torch.exp(0.3 * torch.randn((rows, 1), generator=gen, device="cuda"))


def matrix(gen, groups, K, N):
    """bf16 weights [groups, K, N], a few groups at a time."""
    W = torch.empty((groups, K, N), dtype=torch.bfloat16, device="cuda")
    step = max(1, (1 << 28) // (K * N))
    for g in range(0, groups, step):
        W[g:g + step] = torch.randn((min(step, groups - g), K, N), generator=gen, device="cuda") * 0.02
    return W


def scales(m):
    """(127 / m, m / 127) rounded to 32 bits, of largest magnitudes m."""
    m = m.double().clamp(min=LEAST)
    return (127 / m).float(), (m / 127).float()


def quantised(x, dim):
    """(codes, scales) of x along dim; the product of two values of 32 bits is formed whole, so that ties are ties."""
    r, s = scales(x.abs().amax(dim, keepdim=True))
    return torch.round(x.double() * r.double()).to(torch.int8), s.squeeze(dim)


def quantised_matrix(W):
    """The same for weights, a few groups at a time."""
    G, K, N = W.shape
    codes, scale = torch.empty((G, K, N), dtype=torch.int8, device="cuda"), torch.empty((G, N), device="cuda")
    step = max(1, (1 << 28) // (K * N))
    for g in range(0, G, step):
        codes[g:g + step], scale[g:g + step] = quantised(W[g:g + step], 1)
    return codes, scale


def small(gen, groups, n, case):
    """Biases, or None."""
    return (torch.randn((groups, n), generator=gen, device="cuda") * 0.05).to(torch.bfloat16) if case["bias"] else None


def padded(K):
    return (K + 63) // 64 * 64


def tokens(gen, case, Wg, bg):
    """bf16 tokens whose choice of experts does not hang on the last bits of a logit: the others are drawn again."""
    T, k = case["T"], case["top_k"]
    x = activations(gen, T, case["d"]).to(torch.bfloat16)
    if case["E"] > 1:
        for _ in range(8):
            top = torch.topk(x.double() @ Wg.double() + (0 if bg is None else bg.double()), min(k + 1, case["E"]), dim=1).values
            close = ((top[:, :-1] - top[:, 1:]) < 1e-3 * top.abs().amax(1, keepdim=True)).any(1)
            again = activations(gen, T, case["d"]).to(torch.bfloat16)
            x = torch.where(close[:, None], again, x)
    return x


def parts(case, seed):
    """What the seed gives, in the types of a program that has nothing in 8 bits yet."""
    gen, op, s = generator(seed), case["op"], {"case": case}
    if op == "rows":
        x = activations(gen, case["rows"], case["cols"] + case["wider"])
        s["x"] = (x if case["dtype"] == "f32" else x.to(torch.bfloat16))[:, :case["cols"]]
    elif op == "weights":
        s["W"] = matrix(gen, case["groups"], case["K"], case["N"])
    elif op == "linear":
        s["x"] = activations(gen, case["rows"], case["K"]).to(torch.bfloat16)
        s["W"] = matrix(gen, 1, case["K"], case["N"])
        s["b"] = small(gen, 1, case["N"], case)
    else:
        E, d, f = case["E"], case["d"], case["f"]
        s["W1"], s["b1"] = matrix(gen, E, d, f), small(gen, E, f, case)
        s["W2"], s["b2"] = matrix(gen, E, f, d), small(gen, E, d, case)
        if op == "ffn":
            C = case["capacity"]
            s["xe"] = activations(gen, E * C, d).to(torch.bfloat16).view(E, C, d)
            s["rows"] = torch.randint(0, C + 1, (E,), generator=gen, device="cuda", dtype=torch.int32)
        else:
            if case["residual"]:
                s["Wd1"], s["bd1"] = matrix(gen, 1, d, f), small(gen, 1, f, case)
                s["Wd2"], s["bd2"] = matrix(gen, 1, f, d), small(gen, 1, d, case)
            s["Wg"] = torch.randn((d, E), generator=gen, device="cuda") * 0.02
            s["bg"] = 1.5 * torch.log(1 / torch.arange(1, E + 1, device="cuda", dtype=torch.float32)) if case["skewed"] else None
            s["x"] = tokens(gen, case, s["Wg"], s["bg"])
    return s


MATRICES = {"W1": "s1", "W2": "s2", "Wd1": "sd1", "Wd2": "sd2"}


def prepare(case, seed):
    s = parts(case, seed)
    op = case["op"]
    if op == "rows":
        s["codes"] = torch.empty((case["rows"], padded(case["cols"])), dtype=torch.int8, device="cuda")
        s["scale"] = torch.empty(case["rows"], device="cuda")
    elif op == "linear":
        codes, s["s_row"] = quantised(s.pop("x"), 1)
        s["codes"] = torch.zeros((case["rows"], padded(case["K"])), dtype=torch.int8, device="cuda")
        s["codes"][:, :case["K"]] = codes
        s["W"], s["s_col"] = quantised_matrix(s["W"])
        s["out"] = torch.empty((case["rows"], case["N"]), dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16, device="cuda")
    elif op in ("ffn", "layer"):
        for name, scale in MATRICES.items():
            if name in s:
                s[name], s[scale] = quantised_matrix(s[name])
        s["out"] = torch.zeros_like(s["xe"] if op == "ffn" else s["x"])
    if own:
        plan(s)
    return s


def plan(s):
    """What a program keeps between the calls: shapes, weights in the products' order, a workspace."""
    import paper_2201_05596_amd as moe
    c = s["case"]
    s["moe"] = moe
    if c["op"] == "linear":
        s["shape"] = moe.make_i8_linear(c["rows"], c["K"], c["N"], c["out"], c["gelu"])
        s["W"] = moe.moe_i8_pack_weights(s["W"])
    elif c["op"] in ("ffn", "layer"):
        T = c["E"] * c["capacity"] if c["op"] == "ffn" else c["T"]
        s["shape"] = moe.make_shape(T, c["d"], c["f"], c["E"], c.get("top_k", 1), c["capacity"], "bf16", c.get("residual", False))
        for name in MATRICES:
            if name in s:
                s[name] = moe.moe_i8_pack_weights(s[name])
        if c["op"] == "layer" and (gate := moe.moe_pack_gate(s["Wg"])) is not None:
            s["Wg"], s["shape"].flags = gate, moe.MOE_FLAG_PACKED_GATE
        s["weights"] = {n: s.get(n) for m, x in MATRICES.items() for n in (m, x, "b" + m[1:])}
        s["ws"] = torch.empty(moe.moe_i8_workspace_bytes(s["shape"]), dtype=torch.uint8, device="cuda")


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"rows": own_rows, "weights": own_weights, "linear": own_linear, "ffn": own_ffn, "layer": own_layer}[op](s)
    return {"rows": plain_rows, "weights": plain_weights, "linear": plain_linear, "ffn": plain_ffn, "layer": plain_layer}[op](s)


def own_rows(s):
    s["moe"].moe_i8_quantize_rows(s["x"], s["codes"], s["scale"])
    return s["codes"], s["scale"]


def own_weights(s):
    return s["moe"].moe_i8_quantize_weights(s["W"])


def own_linear(s):
    s["moe"].moe_i8_linear(s["shape"], s["codes"], s["s_row"], s["W"], s["s_col"], s["b"], s["out"])
    return s["out"]


def own_ffn(s):
    s["moe"].moe_i8_expert_ffn(s["shape"], s["weights"], s["xe"], s["rows"], s["out"], s["ws"])
    return s["out"]


def own_layer(s):
    s["moe"].moe_i8_layer_forward(s["shape"], s["weights"], s["x"], s["Wg"], s["bg"], s["out"], None, None, None, None, None, None, s["ws"])
    return s["out"]


def plain_rows(s):
    codes, scale = quantised(s["x"], 1)
    return torch.nn.functional.pad(codes, (0, padded(codes.shape[1]) - codes.shape[1])), scale


def plain_weights(s):
    """Codes in the order of moe_i8_pack_weights: blocks of 64 rows and 128 columns, in each 8 x 64 pieces of 16 rows of one column."""
    codes, scale = quantised(s["W"], 1)
    G, K, N = codes.shape
    codes = torch.nn.functional.pad(codes, (0, -N % 128, 0, -K % 64))
    blocks = codes.view(G, codes.shape[1] // 64, 4, 16, codes.shape[2] // 128, 16, 8)
    return blocks.permute(0, 1, 4, 6, 2, 5, 3).reshape(-1), scale


def gelu(v):
    return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))


def product(codes, s_row, W, s_col, b):
    """[G, rows, K] codes times [G, K, N] codes in 32 bits, scaled, with bias."""
    y = torch.matmul(codes.float(), W.float()) * (s_row[..., None] * s_col[:, None, :])
    return y if b is None else y + b.float()[:, None, :]


def plain_linear(s):
    y = product(s["codes"][None, :, :s["case"]["K"]], s["s_row"][None], s["W"], s["s_col"], s["b"])[0]
    return (gelu(y) if s["case"]["gelu"] else y).to(s["out"].dtype)


def plain_experts(codes, s_row, s, one="1", two="2"):
    """The FFNs of all groups in 32 bits; what is between the products is bf16, then 8 bits."""
    h = gelu(product(codes, s_row, s["W" + one], s["s" + one], s["b" + one])).to(torch.bfloat16)
    return product(*quantised(h, 2), s["W" + two], s["s" + two], s["b" + two])


def plain_ffn(s):
    y = plain_experts(*quantised(s["xe"], 2), s)
    there = torch.arange(y.shape[1], device="cuda") < s["rows"][:, None]
    return torch.where(there[..., None], y.to(torch.bfloat16), s["out"])


def plain_layer(s):
    c = s["case"]
    T, E, k, C = c["T"], c["E"], c["top_k"], c["capacity"]
    logits = s["x"].double() @ s["Wg"].double()
    logits = (logits if s["bg"] is None else logits + s["bg"].double()).float()
    gate, expert = torch.topk(torch.softmax(logits, 1), k, dim=1)
    gate = gate / gate.sum(1, keepdim=True) if k == 2 else gate
    claims = expert.T.reshape(-1)                              # every first choice before any second one
    place = torch.nn.functional.one_hot(claims, E).cumsum(0).gather(1, claims[:, None])[:, 0] - 1
    at = torch.where(place < C, claims * C + place, E * C)     # dropped ones behind the last expert's rows
    codes, s_row = quantised(s["x"], 1)
    token = torch.arange(T, device="cuda").repeat(k)
    xe, se = torch.zeros((E * C + 1, c["d"]), dtype=torch.int8, device="cuda"), torch.zeros(E * C + 1, device="cuda")
    xe[at], se[at] = codes[token], s_row[token]
    ye = plain_experts(xe[:E * C].view(E, C, -1), se[:E * C].view(E, C), s).view(E * C, -1)
    kept = (place < C)[:, None]
    part = torch.where(kept, ye[at.clamp(max=E * C - 1)], 0) * gate.T.reshape(-1)[:, None]
    out = part.view(k, T, -1).sum(0)
    if c["residual"]:
        out = out + plain_experts(codes[None], s_row[None], s, "d1", "d2")[0]
    return out.to(torch.bfloat16)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    op, s = case["op"], parts(case, seed)
    if op in ("rows", "weights"):              # codes are what rounding gives; scales have a value in 64 bits
        m = s["x"].double().abs().amax(1) if op == "rows" else s["W"].abs().amax(1).double()
        return None, m.clamp(min=LEAST) / 127
    return {"linear": exact_linear, "ffn": exact_ffn, "layer": exact_layer}[op](s)


def whole(x, dim):
    """(codes, scales) in float64."""
    m = torch.clamp(x.double().abs().max(dim, keepdim=True).values, min=LEAST)
    return (x.double() * (127.0 / m).float().double()).round(), (m / 127.0).float().double()


def exact_product(x, W, b):
    """rows x [R, K] by W [K, N], both brought into codes, plus b."""
    a, s_a = whole(x, 1)
    w, s_w = whole(W, 0)
    y = (a @ w) * s_a * s_w
    return y if b is None else y + b.double()


def exact_gelu(v):
    return v / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))


def exact_linear(s):
    y = exact_product(s["x"], s["W"][0], None if s["b"] is None else s["b"][0])
    return exact_gelu(y) if s["case"]["gelu"] else y


def exact_expert(x, s, g, one="1", two="2"):
    of = lambda n: None if s[n] is None else s[n][g]  # noqa: E731
    h = exact_gelu(exact_product(x, s["W" + one][g], of("b" + one))).to(torch.bfloat16)
    return exact_product(h, s["W" + two][g], of("b" + two))


def exact_ffn(s):
    out = torch.zeros(s["xe"].shape, dtype=torch.float64, device="cuda")
    for e, n in enumerate(s["rows"].tolist()):
        if n:
            out[e, :n] = exact_expert(s["xe"][e, :n], s, e)
    return out


def exact_layer(s):
    c = s["case"]
    T, E, k = c["T"], c["E"], c["top_k"]
    x = s["x"]
    logits = x.double() @ s["Wg"].double()
    if s["bg"] is not None:
        logits = logits + s["bg"].double()
    order = logits.argsort(1, descending=True)[:, :k]
    p = torch.exp(logits - logits.logsumexp(1, keepdim=True)).gather(1, order)
    if k == 2:
        p = p / p.sum(1, keepdim=True)
    out = torch.zeros((T, c["d"]), dtype=torch.float64, device="cuda")
    for e in range(E):
        room = c["capacity"]
        for j in range(k):
            mine = (order[:, j] == e).nonzero()[:, 0][:room]
            room -= len(mine)
            if len(mine):
                out[mine] += p[mine, j, None] * exact_expert(x[mine], s, e)
    if c["residual"]:
        out += exact_expert(x, s, 0, "d1", "d2")
    return out
