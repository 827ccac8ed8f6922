"""Rotary positions, the quantised key/value cache and attention for drafted tokens, as cases that can be timed and compared.

`run` is one pass through an operator: with `own` the calls that a user makes of paper_2201_05596_amd, otherwise the
same in elementary torch operations in 32 bits (64 for the angles of far positions).  `exact` is the definition in 64
bits, written apart from both.

  rope   moe_rope on the query and key heads of a packed projection's rows
  cache  moe_cache_write of new rows' keys and values, then moe_cache_read of the same rows
  read   moe_cache_read of whole prefixes
  tree   moe_tree_attention of the drafted tokens over the cache and over each other

Head counts and sizes are those of the decoder block (hidden sizes 1024, 2048 and 4096, heads of 64 or 128), with and
without shared key/value heads; batches up to 256 sequences and caches up to 131072 positions.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

KINDS = ("bf16", "fp8", "fp4")
TOP = {"fp8": 448.0, "fp4": 6.0}               # largest value of the format
LEAST = -100                                   # smallest exponent of a scale
SCALINGS = ("plain", "linear", "by_parts")
FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # one decode step of a batch of 64: the query and key heads of a hidden size of 2048
        rope_case("rope_step", rows=64, heads=32, values=16, head_dim=128, far=2048),
        # a ragged chunk of a prompt, float32, a quarter of adjacent pairs rotated, positions divided by a factor
        rope_case("rope_chunk_f32", rows=777, heads=24, values=8, head_dim=64, rot=16, layout="interleaved", scaling="linear", dtype="f32", far=32768),
        # a prefill of 16384 tokens of a hidden size of 4096 with shared heads, far beyond the trained length
        rope_case("rope_long", rows=16384, heads=40, values=8, head_dim=128, scaling="by_parts", far=1000000),
        # the rows of one decode step into an 8-bit cache of 64 sequences
        cache_case("cache_step_fp8", n_seq=64, kv_heads=16, head_dim=128, max_len=2048, kind="fp8", chunk=1),
        # a prefill of 8 x 1021 tokens into a 4-bit cache, heads of 64
        cache_case("cache_prefill_fp4", n_seq=8, kv_heads=8, head_dim=64, max_len=2048, kind="fp4", chunk=1021),
        # the prefixes of two long sequences read back from 8 bits
        cache_case("read_prefix_fp8", n_seq=2, kv_heads=8, head_dim=128, max_len=40000, kind="fp8", chunk=32768, op="read"),
        # seven drafted tokens of a single user early in an answer: latency is all there is
        tree_case("tree_single", n_seq=1, draft=7, heads=16, kv_heads=8, head_dim=64, max_len=2048, kind="bf16", lo=37, hi=37),
        # eight drafted tokens of 64 sequences on the decoder block's own cache
        tree_case("tree_block_bf16", n_seq=64, draft=8, heads=16, kv_heads=16, head_dim=128, max_len=2048, kind="bf16", lo=64, hi=2040),
        # plain decoding (one token) of 128 sequences with shared heads on an 8-bit cache
        tree_case("tree_decode_fp8", n_seq=128, draft=1, heads=32, kv_heads=8, head_dim=128, max_len=4096, kind="fp8", lo=1, hi=4095),
        # trees of 32 on long contexts, 8 bits
        tree_case("tree_gqa_fp8", n_seq=16, draft=32, heads=32, kv_heads=8, head_dim=128, max_len=16384, kind="fp8", lo=2000, hi=16001),
        # two documents of 131000 positions in 4 bits, 16 drafted tokens each
        tree_case("tree_long_fp4", n_seq=2, draft=16, heads=32, kv_heads=8, head_dim=128, max_len=131072, kind="fp4", lo=130001, hi=131000),
        # trees of 64 on eight query heads per key/value head: bound by the matrix cores
        tree_case("tree_wide_bf16", n_seq=8, draft=64, heads=32, kv_heads=4, head_dim=128, max_len=8192, kind="bf16", lo=3000, hi=8100),
    ]


def rope_case(name=None, *, rows, heads, values, head_dim, rot=None, layout="half", scaling="plain", dtype="bf16", far):
    c = {"op": "rope", "rows": rows, "heads": heads, "values": values, "head_dim": head_dim, "rot": rot or head_dim, "layout": layout,
         "scaling": scaling, "dtype": dtype, "far": far}
    return {"name": name, **c} if name else c


def cache_case(name=None, *, n_seq, kv_heads, head_dim, max_len, kind, chunk, op="cache"):
    c = {"op": op, "n_seq": n_seq, "kv_heads": kv_heads, "head_dim": head_dim, "max_len": max_len, "kind": kind, "chunk": chunk}
    return {"name": name, **c} if name else c


def tree_case(name=None, *, n_seq, draft, heads, kv_heads, head_dim, max_len, kind, lo, hi):
    c = {"op": "tree", "n_seq": n_seq, "draft": draft, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "max_len": max_len,
         "kind": kind, "lo": lo, "hi": hi}
    return {"name": name, **c} if name else c


def draw(rng):
    """One more case: sizes over their logarithm, odd ones among them, no more work than the largest listed cases."""
    spread = lambda lo, hi: max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))  # noqa: E731
    limit = {"rope": 3.3e8, "cache": 4e8, "read": 4e8, "tree": 5.4e8}
    while True:
        op = rng.choice(("rope", "cache", "read", "tree", "tree", "tree"))
        dh = rng.choice((64, 128))
        if op == "rope":
            heads = spread(1, 40)
            rot = rng.choice((dh, dh, dh // 2, dh // 4, 8 * rng.randint(1, dh // 8)))
            c = rope_case(rows=spread(1, 16384), heads=heads, values=rng.choice((0, 1, 8)), head_dim=dh, rot=rot, layout=rng.choice(("half", "interleaved")),
                          scaling=rng.choice(SCALINGS), dtype=rng.choice(("bf16", "bf16", "f32")), far=spread(16, 1000000))
        elif op == "tree":
            kv = rng.choice((1, 2, 4, 8, 16))
            max_len = spread(16, 131072)
            hi = rng.randint(max_len // 2, max_len)
            c = tree_case(n_seq=spread(1, 256), draft=spread(1, 64), heads=kv * rng.choice((1, 1, 2, 4, 5, 8)), kv_heads=kv, head_dim=dh, max_len=max_len,
                          kind=rng.choice(KINDS), lo=rng.randint(0, hi), hi=hi)
            if c["heads"] > 64 or work(c)["flops"] > 6e10:
                continue
        else:
            max_len = spread(16, 40000)
            c = cache_case(n_seq=spread(1, 256), kv_heads=rng.choice((1, 2, 4, 8, 16)), head_dim=dh, max_len=max_len, kind=rng.choice(KINDS),
                           chunk=spread(1, max_len), op=op)
        if work(c)["bytes"] <= limit[op] and (op == "rope" or c["n_seq"] * c["max_len"] * c["kv_heads"] * dh <= 1 << 29):
            return c


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def row_bytes(kind, head_dim):
    """One position of one head, keys or values: elements and scales."""
    return head_dim * 2 if kind == "bf16" else head_dim // (1 if kind == "fp8" else 2) + head_dim // 32


def written(case):
    """Rows of the chunk that are kept: of every eleven the last is not (a drafted token that was not accepted)."""
    n = case["n_seq"] * case["chunk"]
    return n - n // 11 if case["op"] == "cache" else n


def lengths(case):
    """Cached positions and drafted tokens of the sequences, before they are put in an order by the seed."""
    n, lo, hi, draft = case["n_seq"], case["lo"], case["hi"], case["draft"]
    lens = [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]
    return lens, [max(1, draft - (i % 4) * (draft // 8)) for i in range(n)]


def work(case):
    if case["op"] == "rope":
        n = case["rows"] * case["heads"] * case["head_dim"] * (4 if case["dtype"] == "f32" else 2)
        return {"bytes": 2 * n + 4 * case["rows"] + 4 * case["rot"], "flops": 3 * case["rows"] * case["heads"] * case["rot"]}
    if case["op"] == "tree":
        H, G, dh = case["heads"], case["kv_heads"], case["head_dim"]
        lens, counts = lengths(case)
        rows = sum(counts)
        cached = 2 * G * sum(lens) * row_bytes(case["kind"], dh)
        return {"bytes": cached + rows * (2 * H + 2 * G) * dh * 2 + rows * ((case["draft"] + 31) // 32) * 4,
                "flops": 4 * dh * H * sum(c * (n + (c + 1) // 2) for n, c in zip(lens, counts))}
    rows, G, dh = written(case), case["kv_heads"], case["head_dim"]
    plain, held = 2 * rows * G * dh * 2, 2 * rows * G * row_bytes(case["kind"], dh)
    passes = 2 if case["op"] == "cache" else 1
    return {"bytes": passes * (plain + held + 8 * rows), "flops": passes * 2 * rows * G * dh * 2}


# ---- what a program has in hand before the call ----------------------------------------------------------------

def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def two_to(e):
    """2^e in float32, from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def quantised(x, kind):
    """(codes, scales) of x [..., 32 n] float32: blocks of 32, the smallest power of two with which the block fits the format."""
    blocks = x.unflatten(-1, (-1, 32))
    big = blocks.abs().amax(-1)
    m, e = torch.frexp(big / TOP[kind])        # big / TOP = m 2^e, m in [0.5, 1)
    e = torch.where(m > 0.5, e, e - 1)
    e = torch.where(big > 0, e, torch.full_like(e, LEAST)).clamp(min=LEAST)
    y = blocks * two_to(-e).unsqueeze(-1)
    if kind == "fp8":
        codes = y.to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    else:
        mag = y.abs()
        step = torch.where(mag < 2, 0.5, torch.where(mag < 4, 1.0, 2.0))
        mag = torch.round(mag / step) * step   # halves to even, as the format's codes have it
        code = torch.bucketize(mag, torch.tensor(FP4, device=x.device)).to(torch.uint8) + 8 * (y < 0).to(torch.uint8)
        code = code.flatten(-2)
        codes = code[..., 0::2] | (code[..., 1::2] << 4)
    return codes, (e + 127).to(torch.uint8)


def dequantised(codes, scales, kind):
    """float32 values of a cache's rows."""
    if kind == "bf16":
        return codes.float()
    if kind == "fp8":
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        both = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
        v = torch.tensor(FP4 + tuple(-x for x in FP4), device=codes.device)[both]
    return (v.unflatten(-1, (-1, 32)) * two_to(scales.int() - 127).unsqueeze(-1)).flatten(-2)


def filled_cache(case, gen):
    """Keys and values of every sequence's positions, quantised a sequence at a time; keys have a few large channels."""
    B, G, L, dh, kind = case["n_seq"], case["kv_heads"], case["max_len"], case["head_dim"], case["kind"]
    s = empty_cache(case)
    gain = 1 + 3 * (torch.rand((1, G, 1, dh), generator=gen, device="cuda") > 0.95)
    step = max(1, (1 << 26) // (G * L * dh))
    for b in range(0, B, step):
        n = min(step, B - b)
        for name, g in (("k", gain), ("v", None)):
            x = torch.randn((n, G, L, dh), generator=gen, device="cuda")
            x = x * g * 0.7 if g is not None else x
            if kind == "bf16":
                s[name + "_cache"][b:b + n] = x
            else:
                s[name + "_cache"][b:b + n], s[name + "_scale"][b:b + n] = quantised(x, kind)
    return s


def empty_cache(case):
    B, G, L, dh, kind = case["n_seq"], case["kv_heads"], case["max_len"], case["head_dim"], case["kind"]
    cols = dh // 2 if kind == "fp4" else dh
    s = {n + "_cache": torch.zeros((B, G, L, cols), dtype=torch.bfloat16 if kind == "bf16" else torch.uint8, device="cuda") for n in "kv"}
    s.update({n + "_scale": None if kind == "bf16" else torch.full((B, G, L, dh // 32), 127, dtype=torch.uint8, device="cuda") for n in "kv"})
    return s


def seen(draft, n_seq, rng):
    """[n_seq, draft, words] int32: a drafted token sees itself and its ancestors; its parent is one of the eight before it, or the last cached token."""
    words = (draft + 31) // 32
    bits = np.zeros((n_seq, draft, draft), dtype=bool)
    for i in range(draft):
        parent = i - 1 - rng.integers(0, min(8, i + 1), n_seq)
        at = np.nonzero(parent >= 0)[0]
        bits[at, i] = bits[at, parent[at]]
        bits[:, i, i] = True
    padded = np.zeros((n_seq, draft, words * 32), dtype=np.uint8)
    padded[:, :, :draft] = bits
    packed = np.packbits(padded, axis=-1, bitorder="little").view("<u4").astype(np.uint32)
    return torch.from_numpy(packed.view(np.int32)).cuda()


def prepare(case, seed):
    gen, rng = generator(seed), np.random.default_rng(seed)
    s = {"case": case}
    if case["op"] == "rope":
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        dh, n = case["head_dim"], case["heads"] * case["head_dim"]
        s["rows"] = torch.randn((case["rows"], n + case["values"] * dh), generator=gen, device="cuda").to(dt)
        s["pos"] = torch.randint(0, case["far"], (case["rows"],), generator=gen, device="cuda", dtype=torch.int32)
        s["out"] = torch.empty((case["rows"], n), dtype=dt, device="cuda")
    elif case["op"] == "tree":
        B, N, H, G, dh = case["n_seq"], case["draft"], case["heads"], case["kv_heads"], case["head_dim"]
        s.update(filled_cache(case, gen))
        lens, counts = lengths(case)
        order = rng.permutation(B)
        s["lens"] = torch.tensor(np.array(lens)[order], dtype=torch.int32, device="cuda")
        s["counts"] = torch.tensor(np.array(counts)[order], dtype=torch.int32, device="cuda")
        s["tree"] = seen(N, B, rng)
        s["qkv"] = torch.randn((B * N, (H + 2 * G) * dh), generator=gen, device="cuda").to(torch.bfloat16)
        s["out"] = torch.zeros((B * N, H * dh), dtype=torch.bfloat16, device="cuda")
    else:
        B, G, dh, n = case["n_seq"], case["kv_heads"], case["head_dim"], case["chunk"]
        R = B * n
        first = torch.randint(0, case["max_len"] - n + 1, (B, 1), generator=gen, device="cuda", dtype=torch.int32)
        pos = (first + torch.arange(n, device="cuda", dtype=torch.int32)).reshape(-1)
        s["seq"] = torch.arange(B, device="cuda", dtype=torch.int32).repeat_interleave(n)
        if case["op"] == "cache":
            pos[10::11] = -1                   # not accepted: neither written nor read
            s.update(empty_cache(case))
            x = torch.randn((R, G, 2, dh), generator=gen, device="cuda") * torch.exp(torch.randn((R, G, 2, 1), generator=gen, device="cuda"))
            s["kv"] = x.to(torch.bfloat16).permute(0, 2, 1, 3).reshape(R, 2 * G * dh).contiguous()
        else:
            s.update(filled_cache(case, gen))
        s["pos"] = pos
        s["k_rows"], s["v_rows"] = (torch.zeros((R, G * dh), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    if own:
        plan(s)
    return s


def rope_args(case):
    scaling = {"plain": {}, "linear": {"factor": 8.0}, "by_parts": {"factor": 32.0, "original_len": 8192.0, "low": 1.0, "high": 4.0}}[case["scaling"]]
    return {"base": 10000.0 if case["scaling"] == "plain" else 500000.0, "amplitude": 1.0 if case["scaling"] != "by_parts" else 0.1 * math.log(32.0) + 1.0, **scaling}


def plan(s):
    """What a program keeps between the calls: shapes, the table of frequencies, a workspace."""
    import paper_2201_05596_amd as moe
    case = s["case"]
    s["moe"] = moe
    if case["op"] == "rope":
        s["rope"] = moe.make_rope(case["head_dim"], case["rot"], case["layout"], case["dtype"], scaling=case["scaling"], **rope_args(case))
        s["turns"] = moe.moe_rope_frequencies(s["rope"], "cuda")
    else:
        s["shape"] = moe.make_cache_shape(case["n_seq"], case.get("heads", case["kv_heads"]), case["kv_heads"], case["head_dim"], case["max_len"], case["kind"])
    if case["op"] == "tree":
        s["ws"] = torch.empty(moe.moe_tree_attention_workspace_bytes(s["shape"], case["draft"]), dtype=torch.uint8, device="cuda")


# ---- one pass ---------------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        return {"rope": own_rope, "cache": own_cache, "read": own_read, "tree": own_tree}[op](s)
    return {"rope": plain_rope, "cache": plain_cache, "read": plain_read, "tree": plain_tree}[op](s)


def own_rope(s):
    n = s["out"].shape[1]
    s["moe"].moe_rope(s["rope"], s["rows"][:, :n], s["turns"], s["pos"], s["out"])
    return s["out"]


def own_cache(s):
    n = s["k_rows"].shape[1]
    s["moe"].moe_cache_write(s["shape"], s["kv"][:, :n], s["kv"][:, n:], s["seq"], s["pos"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
    return own_read(s)


def own_read(s):
    s["moe"].moe_cache_read(s["shape"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["seq"], s["pos"], s["k_rows"], s["v_rows"])
    return s["k_rows"], s["v_rows"]


def own_tree(s):
    c = s["case"]
    nq, nk = c["heads"] * c["head_dim"], c["kv_heads"] * c["head_dim"]
    qkv = s["qkv"]
    s["moe"].moe_tree_attention(s["shape"], c["draft"], qkv[:, :nq], qkv[:, nq:nq + nk], qkv[:, nq + nk:], s["k_cache"], s["v_cache"], s["k_scale"],
                                s["v_scale"], s["lens"], s["counts"], s["tree"], s["out"], s["ws"])
    return s["out"]


def plain_rope(s):
    c, a = s["case"], rope_args(s["case"])
    dh, rot = c["head_dim"], c["rot"]
    i = torch.arange(rot // 2, dtype=torch.float64, device="cuda")
    f = a["base"] ** (-2 * i / rot)
    if c["scaling"] == "linear":
        f = f / a["factor"]
    elif c["scaling"] == "by_parts":
        g = ((a["original_len"] * f / (2 * math.pi) - a["low"]) / (a["high"] - a["low"])).clamp(0, 1)
        f = f * (g + (1 - g) / a["factor"])
    angle = (s["pos"].double()[:, None] * f)[:, None, :]
    cos, sin = (angle.cos() * a["amplitude"]).float(), (angle.sin() * a["amplitude"]).float()
    n = s["out"].shape[1]
    x = s["rows"][:, :n].unflatten(1, (-1, dh)).float()
    y = x.clone()
    lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
    y[..., hi] = x[..., hi] * cos + x[..., lo] * sin
    return y.flatten(1).to(s["out"].dtype)


def plain_cache(s):
    c = s["case"]
    n = s["k_rows"].shape[1]
    ok = s["pos"] >= 0
    seq, pos = s["seq"].long(), s["pos"].clamp(min=0).long()
    for name, x in (("k", s["kv"][:, :n]), ("v", s["kv"][:, n:])):
        x = x.unflatten(1, (-1, c["head_dim"]))
        cache, scale = s[name + "_cache"], s[name + "_scale"]
        keep = ok[:, None, None]
        if c["kind"] == "bf16":
            put(cache, seq, pos, x, keep)
        else:
            codes, scales = quantised(x.float(), c["kind"])
            put(cache, seq, pos, codes, keep)
            put(scale, seq, pos, scales, keep)
    return plain_read(s)


def put(cache, seq, pos, x, keep):
    """Rows that are not kept go to a position that no row of the call has: they take what is there."""
    old = cache[seq, :, pos]
    spare = torch.where(keep[:, 0, 0], pos, torch.roll(pos, 1))        # the row before it: written with the same values once more
    x = torch.where(keep, x, torch.where(torch.roll(keep, 1, 0), torch.roll(x, 1, 0), old))
    cache[torch.where(keep[:, 0, 0], seq, torch.roll(seq, 1)), :, spare] = x


def plain_read(s):
    c = s["case"]
    ok = (s["pos"] >= 0)[:, None]
    seq, pos = s["seq"].long(), s["pos"].clamp(min=0).long()
    for name in "kv":
        scale = s[name + "_scale"]
        x = dequantised(s[name + "_cache"][seq, :, pos], None if scale is None else scale[seq, :, pos], c["kind"])
        s[name + "_rows"] = torch.where(ok, x.flatten(1).to(torch.bfloat16), s[name + "_rows"])
    return s["k_rows"], s["v_rows"]


def plain_tree(s):
    c = s["case"]
    B, N, H, G, dh, L = c["n_seq"], c["draft"], c["heads"], c["kv_heads"], c["head_dim"], c["max_len"]
    qkv = s["qkv"].float().view(B, N, H + 2 * G, dh)
    j = torch.arange(N, device="cuda")
    outs = []
    for b in range(B):
        q = qkv[b, :, :H].reshape(N, G, H // G, dh).permute(1, 2, 0, 3).reshape(G, -1, dh)
        scale = lambda n: None if s[n] is None else s[n][b]  # noqa: B023, E731
        k = torch.cat((dequantised(s["k_cache"][b], scale("k_scale"), c["kind"]), qkv[b, :, H:H + G].transpose(0, 1)), 1)
        v = torch.cat((dequantised(s["v_cache"][b], scale("v_scale"), c["kind"]), qkv[b, :, H + G:].transpose(0, 1)), 1)
        sees = ((s["tree"][b][:, j // 32] >> (j % 32)) & 1).bool() & (j < s["counts"][b])
        past = (torch.arange(L, device="cuda") < s["lens"][b]).expand(N, L)
        sees = torch.cat((past, sees), 1).repeat(H // G, 1)
        p = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(dh)
        p = p.masked_fill(~sees, -math.inf)
        p = torch.exp(p - p.amax(-1, keepdim=True).clamp(min=-3e38))
        o = torch.matmul(p, v) / p.sum(-1, keepdim=True).clamp(min=1e-37)
        o = o.view(G, H // G, N, dh).permute(2, 0, 1, 3).reshape(N, H * dh)
        outs.append(torch.where((j < s["counts"][b])[:, None], o.to(torch.bfloat16), s["out"][b * N:(b + 1) * N]))
    return torch.cat(outs)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------

def exact(case, seed):
    return {"rope": exact_rope, "cache": exact_cache, "read": exact_cache, "tree": exact_tree}[case["op"]](prepare(case, seed))


def power(e):
    """2^e in float64."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def held(cache, scale, kind):
    """What stored elements stand for, from their bits."""
    if kind == "bf16":
        return cache.double()
    if kind == "fp8":
        c = cache.to(torch.int64)
        high, part = (c >> 3) & 15, (c & 7).double()
        v = torch.where(high > 0, (8 + part) * power(high - 10), part * 2.0 ** -9)
        v = torch.where(c >= 128, -v, v)
    else:
        c = torch.empty((*cache.shape[:-1], cache.shape[-1] * 2), dtype=torch.int64, device=cache.device)
        c[..., 0::2], c[..., 1::2] = cache.long() % 16, cache.long() // 16
        high, part = (c >> 1) & 3, (c & 1).double()
        v = torch.where(high > 0, (2 + part) * power(high - 2), part * 0.5)
        v = torch.where(c >= 8, -v, v)
    return v * power(scale.long() - 127).repeat_interleave(32, -1)


def exact_rope(s):
    c, a = s["case"], rope_args(s["case"])
    rot, dh = c["rot"], c["head_dim"]
    x = s["rows"][:, :s["out"].shape[1]].double().view(c["rows"], -1, dh)
    out = x.clone()
    for i in range(rot // 2):
        f = a["base"] ** (-2.0 * i / rot)
        if c["scaling"] == "linear":
            f /= a["factor"]
        if c["scaling"] == "by_parts":
            r = a["original_len"] * f / (2 * math.pi)
            g = 0.0 if r < a["low"] else 1.0 if r > a["high"] else (r - a["low"]) / (a["high"] - a["low"])
            f = (1 - g) * f / a["factor"] + g * f
        m, n = (i, i + rot // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
        z = torch.polar(torch.full((c["rows"], 1), a["amplitude"], dtype=torch.float64, device="cuda"), (s["pos"].double() * f)[:, None])
        z = torch.complex(x[..., m], x[..., n]) * z
        out[..., m], out[..., n] = z.real, z.imag
    return out.reshape(c["rows"], -1)


def exact_cache(s):
    c = s["case"]
    G, dh, kind = c["kv_heads"], c["head_dim"], c["kind"]
    outs = []
    for at, name in enumerate("kv"):
        if c["op"] == "read":
            seq, pos = s["seq"].long(), s["pos"].long()
            scale = s[name + "_scale"]
            x = held(s[name + "_cache"][seq, :, pos], None if scale is None else scale[seq, :, pos], kind).reshape(len(pos), -1)
        else:
            x = s["kv"].double()[:, at * G * dh:(at + 1) * G * dh]
            if kind != "bf16":
                values = FP4 if kind == "fp4" else [(8 + c % 8) * 2.0 ** (c // 8 - 10) if c > 7 else c * 2.0 ** -9 for c in range(127)]
                values = torch.tensor(values, dtype=torch.float64, device="cuda")     # rising, in order of their codes
                y = x.reshape(x.shape[0], -1, 32)
                m, e = torch.frexp(y.abs().amax(-1, keepdim=True) / TOP[kind])
                unit = power(torch.where(m == 0.5, e - 1, e).clamp(min=LEAST))
                y = y / unit
                up = torch.searchsorted(values, y.abs().contiguous()).clamp(1, len(values) - 1)
                near, far = y.abs() - values[up - 1], values[up] - y.abs()
                up = torch.where((near < far) | ((near == far) & (up % 2 == 1)), up - 1, up)
                x = (torch.sign(y) * values[up] * unit).reshape(x.shape)
            x = torch.where((s["pos"] >= 0)[:, None], x, torch.zeros((), dtype=torch.float64, device="cuda"))
        outs.append(x)
    return tuple(outs)


def exact_tree(s):
    c = s["case"]
    N, H, G, dh = c["draft"], c["heads"], c["kv_heads"], c["head_dim"]
    out = torch.zeros((c["n_seq"], N, H, dh), dtype=torch.float64, device="cuda")
    qkv = s["qkv"].double().view(c["n_seq"], N, H + 2 * G, dh)
    lens, counts, trees = s["lens"].tolist(), s["counts"].tolist(), s["tree"].cpu().numpy().view(np.uint32)
    for b, (n, m) in enumerate(zip(lens, counts)):
        bits = np.unpackbits(trees[b, :m].copy().view(np.uint8), axis=-1, bitorder="little")[:, :m]
        hidden = torch.from_numpy(bits == 0).cuda()
        for g in range(G):
            ks, vs = (held(s[x + "_cache"][b, g, :n], None if s[x + "_scale"] is None else s[x + "_scale"][b, g, :n], c["kind"]) for x in "kv")
            ks, vs = torch.cat((ks, qkv[b, :m, H + g])), torch.cat((vs, qkv[b, :m, H + G + g]))
            for h in range(g * (H // G), (g + 1) * (H // G)):
                score = qkv[b, :m, h] @ ks.T / dh ** 0.5
                score[:, n:][hidden] = -math.inf
                score -= score.max(1, keepdim=True).values
                score.exp_()
                out[b, :m, h] = score @ vs / score.sum(1, keepdim=True)
    return out.view(c["n_seq"] * N, H * dh)
