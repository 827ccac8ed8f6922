"""moe_draft_block_forward against the oracles, and the operators of a verification step used together.

The block is compared in parts, as moe_decode_block_forward is, because later parts start from numbers that the GPU has rounded:
qkv against the oracle's projection and rotation, x1 against the oracle's attention on the GPU's own qkv, the MoE input against
LayerNorm of the GPU's x1, the output against the MoE oracle on the GPU's MoE input and logits."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as blk
from oracle import draft_oracle as drf
from oracle import moe_oracle as orc
from tests import gpu_util as U
from tests.test_gpu_cache import codes_of
from tests.test_gpu_tree_attention import random_tree, words
from workloads import CONFIGS, make_block_inputs
from workloads.generate import to_f32_numpy

pytestmark = pytest.mark.gpu
DEV = "cuda"
f = to_f32_numpy
ROPE = dict(base=10000.0)


class Model:
    """Weights of one block with G key/value heads, on a cache of `kind`, for B sequences of N tokens."""

    def __init__(self, B, N, H, G, dh, L, kind, layout="half", rot=None, E=4, f_dim=512, residual=False, seed=0, cf=2.0):
        m = U.amd()
        self.m, self.dims, self.kind = m, (B, N, H, G, dh, L), kind
        d = H * dh
        cfg = CONFIGS["c3a" if residual else "c4"].scaled(name="draft", T=B * N, d_model=d, d_ffn=f_dim, E=E, capacity_factor=cf)
        self.bi = bi = make_block_inputs(cfg, H, 8, DEV)
        self.cfg, lay = cfg, bi.layer
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.Wqkv = torch.cat((bi.Wqkv[:, :d], bi.Wqkv[:, d:d + G * dh], bi.Wqkv[:, 2 * d:2 * d + G * dh]), 1).contiguous()
        self.bqkv = torch.cat((bi.bqkv[:d], bi.bqkv[d:d + G * dh], bi.bqkv[2 * d:2 * d + G * dh])).contiguous()
        self.weights = dict(ln1_gamma=bi.ln1_gamma, ln1_beta=bi.ln1_beta, Wqkv=self.Wqkv, bqkv=self.bqkv, Wo=bi.Wo, bo=bi.bo, ln2_gamma=bi.ln2_gamma,
                            ln2_beta=bi.ln2_beta, Wg=lay.Wg, bg=lay.bg, W1=lay.W1, b1=lay.b1, W2=lay.W2, b2=lay.b2, Wd1=lay.Wd1, bd1=lay.bd1,
                            Wd2=lay.Wd2, bd2=lay.bd2)
        self.cache = m.make_cache_shape(B, H, G, dh, L, kind)
        self.caches = m.alloc_cache(self.cache, DEV)
        self.layout, self.rot = layout, rot or dh
        self.rope = None if layout is None else m.make_rope(dh, self.rot, layout, "bf16", **ROPE)
        self.turns = None if layout is None else m.moe_rope_frequencies(self.rope, DEV)
        self.gen = gen

    def step(self, x, N, lens, pos, tree):
        """One call over N tokens per sequence; tree: bits [B, N, N] or None."""
        m = self.m
        B, _, H, G, dh, L = self.dims
        d, T, cfg = H * dh, B * N, self.cfg
        cap = T if cfg.E == 1 else max(1, int(np.ceil(2.0 * T / cfg.E)))
        shape = m.make_shape(T, d, cfg.d_ffn, cfg.E, 1, cap, "bf16", residual=cfg.residual)
        new = lambda *s: torch.full(s, 3.0, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        r = dict(qkv=new(T, (H + 2 * G) * dh), out=new(T, d), x1=new(T, d), moe_in=new(T, d), logits=torch.empty((T, cfg.E), device=DEV), cap=cap)
        ws = torch.full((m.moe_draft_block_workspace_bytes(shape, self.cache, N),), 255, dtype=torch.uint8, device=DEV)
        i32 = lambda v: torch.as_tensor(np.asarray(v, np.int32)).to(DEV)  # noqa: E731
        m.moe_draft_block_forward(shape, self.cache, N, self.rope, self.weights, x, self.turns, None if self.rope is None else i32(pos), *self.caches,
                                  i32(lens), None if tree is None else torch.from_numpy(words(tree)).to(DEV), r["qkv"], r["out"], r["x1"], r["moe_in"],
                                  r["logits"], ws)
        torch.cuda.synchronize()
        return r

    def values(self):
        ks, vs, kx, vx = self.caches
        if self.kind == "bf16":
            return f(ks), f(vs)
        return tuple(drf.dequantise(codes_of(c, self.kind), x.cpu().numpy(), self.kind) for c, x in ((ks, kx), (vs, vx)))

    def check(self, r, x, N, lens, pos, tree):
        B, _, H, G, dh, L = self.dims
        d, T = H * dh, B * N
        w, tol = self.weights, U.TOL["bf16"]
        rows = blk.linear(blk.layer_norm(f(x), f(w["ln1_gamma"]), f(w["ln1_beta"])), f(w["Wqkv"]), f(w["bqkv"])).reshape(T, H + 2 * G, dh)
        if self.rope is not None:
            rows[:, :H + G] = drf.rope(rows[:, :H + G], pos, drf.rope_frequencies(self.rot, **ROPE), self.layout)
        got = f(r["qkv"]).reshape(T, H + 2 * G, dh)
        assert np.max(np.abs(got - rows)) <= tol * np.max(np.abs(rows))
        g = got.astype(np.float64).reshape(B, N, H + 2 * G, dh)
        o, _ = drf.tree_attention(g[:, :, :H], g[:, :, H:H + G], g[:, :, H + G:], *self.values(), lens, None, None if tree is None else words(tree),
                                  np.zeros((B, N, H, dh)))
        x1 = f(x) + blk.linear(o.reshape(T, d), f(w["Wo"]), f(w["bo"]))
        U.assert_close(r["x1"], x1, "bf16", "x1")
        x1g = f(r["x1"])
        U.assert_close(r["moe_in"], blk.layer_norm(x1g, f(w["ln2_gamma"]), f(w["ln2_beta"])), "bf16", "moe input")
        h = U.host(self.bi.layer)
        xin, gl = f(r["moe_in"]), r["logits"].cpu().numpy()
        own = orc.gate_logits(xin, h["Wg"], h.get("bg"))
        assert np.max(np.abs(gl.astype(np.float64) - own)) <= U.LOGIT_RTOL * np.max(np.abs(own))
        ref = blk.moe_half(x1g, None, None, h["Wg"], h.get("bg"), h["W1"], h["b1"], h["W2"], h["b2"], 1, r["cap"], h.get("Wd1"), h.get("bd1"),
                           h.get("Wd2"), h.get("bd2"), moe_input=xin, logits=gl)
        U.assert_close(r["out"], ref["out"], "bf16", "block out")

    def tokens(self, N):
        B, _, H, G, dh, L = self.dims
        return torch.randn((B * N, H * dh), generator=self.gen, device=DEV).to(torch.bfloat16)

    def write(self, r, take, seq, pos):
        """Rows `take` of a step's qkv become positions pos of sequences seq."""
        B, _, H, G, dh, L = self.dims
        seq_all, pos_all = np.full(r["qkv"].shape[0], -1, np.int32), np.full(r["qkv"].shape[0], -1, np.int32)
        seq_all[take], pos_all[take] = seq, pos
        self.m.moe_cache_write(self.cache, r["qkv"][:, H * dh:(H + G) * dh], r["qkv"][:, (H + G) * dh:], torch.from_numpy(seq_all).to(DEV),
                               torch.from_numpy(pos_all).to(DEV), *self.caches)


def fill(model, lens):
    """The caches' first positions from random rows."""
    B, _, H, G, dh, L = model.dims
    n = max(lens)
    if n == 0:
        return
    rows = torch.randn((B * n, 2 * G * dh), generator=model.gen, device=DEV).to(torch.bfloat16)
    seq = np.repeat(np.arange(B, dtype=np.int32), n)
    pos = np.tile(np.arange(n, dtype=np.int32), B)
    pos[pos >= np.repeat(np.asarray(lens), n)] = -1
    model.m.moe_cache_write(model.cache, rows[:, :G * dh], rows[:, G * dh:], torch.from_numpy(seq).to(DEV), torch.from_numpy(pos).to(DEV), *model.caches)


CASES = {
    # B, N, H, G, dh, L, kind, layout, rot, residual, lens
    "one_token": (1, 1, 2, 1, 64, 1, "bf16", "half", 64, False, [0]),
    "few_rows": (3, 5, 4, 2, 64, 40, "fp8", "interleaved", 32, False, [0, 17, 40]),
    "shared": (4, 9, 8, 1, 64, 70, "bf16", "half", 64, False, [70, 1, 33, 64]),
    "no_rope": (2, 20, 2, 2, 128, 100, "fp4", None, None, True, [100, 31]),
    "wide": (2, 64, 4, 1, 128, 150, "fp8", "half", 96, False, [150, 77]),
    "chain": (5, 33, 2, 2, 64, 64, "bf16", "interleaved", 64, True, [64, 0, 5, 31, 32]),
}


@pytest.mark.parametrize("name", sorted(CASES))
def test_draft_block(name):
    B, N, H, G, dh, L, kind, layout, rot, residual, lens = CASES[name]
    print("case draft block", name, flush=True)
    model = Model(B, N, H, G, dh, L, kind, layout, rot, residual=residual)
    fill(model, lens)
    held = [None if t is None else t.clone() for t in model.caches]
    tree = None if name == "chain" else random_tree(B, N, 3)
    depth = np.tile(np.arange(N), (B, 1)) if tree is None else tree.sum(-1) - 1
    pos = (np.asarray(lens)[:, None] + depth).reshape(-1)
    x = model.tokens(N)
    r = model.step(x, N, lens, pos, tree)
    model.check(r, x, N, lens, pos, tree)
    assert all(a is None or torch.equal(a, b) for a, b in zip(held, model.caches)), "the caches were written"


def test_draft_block_one_token_equals_the_decode_block():
    """One token per sequence, bf16, no rotary positions: moe_decode_block_forward's step, whose cache rows moe_cache_write writes."""
    m = U.amd()
    B, H, dh, L = 40, 4, 64, 300
    model = Model(B, 1, H, H, dh, L, "bf16", layout=None)
    bi, lay, d = model.bi, model.bi.layer, H * dh
    model.weights.update(Wqkv=bi.Wqkv, bqkv=bi.bqkv)
    lens = [int(v) for v in np.random.default_rng(2).integers(0, L, B)]
    lens[0], lens[1] = 0, L - 1
    fill(model, lens)
    x = model.tokens(1)
    r = model.step(x, 1, lens, None, None)
    kc, vc = model.caches[0].clone(), model.caches[1].clone()
    shape, block = m.make_shape(B, d, model.cfg.d_ffn, model.cfg.E, 1, r["cap"], "bf16"), m.MoeBlockShape(H, L)
    ws = torch.empty(m.moe_decode_block_workspace_bytes(shape, block), dtype=torch.uint8, device=DEV)
    out, x1 = torch.empty_like(x), torch.empty_like(x)
    m.moe_decode_block_forward(shape, block, model.weights, x, kc, vc, torch.tensor(lens, dtype=torch.int32, device=DEV), out, x1, None, None, ws)
    model.write(r, np.arange(B), np.arange(B), lens)
    torch.cuda.synchronize()
    assert torch.equal(model.caches[0], kc) and torch.equal(model.caches[1], vc)
    # both round sums of the same numbers: probabilities to bf16 here (2^-8 of the attention), both rows to bf16
    assert float((r["x1"].float() - x1.float()).abs().max()) <= 2.0 ** -7 * float(x1.float().abs().max())


@pytest.mark.parametrize("kind", ["bf16", "fp8", "fp4"])
def test_prompt_then_verification_steps(kind):
    """A prompt as a chain of drafted tokens, its rows into the cache, two trees of which a path is accepted, a last token: every step
    against the oracle on what the cache holds by then, and for bf16 the last against full causal attention over the accepted tokens."""
    B, H, G, dh, L, P, N = 2, 4, 2, 64, 60, 21, 12
    print("case verification", kind, flush=True)
    model = Model(B, P, H, G, dh, L, kind, "half", 48)
    x = model.tokens(P)
    pos = np.tile(np.arange(P), B)
    r = model.step(x, P, [0] * B, pos, None)
    model.check(r, x, P, [0] * B, pos, None)
    model.write(r, np.arange(B * P), np.repeat(np.arange(B), P), pos)
    kept = [[f(r["qkv"])[b * P + i] for i in range(P)] for b in range(B)]
    lens = np.full(B, P)
    for s in range(2):
        tree = random_tree(B, N, 20 + s)
        x = model.tokens(N)
        pos = (lens[:, None] + tree.sum(-1) - 1).reshape(-1)
        r = model.step(x, N, lens, pos, tree)
        model.check(r, x, N, lens, pos, tree)
        take, seq, at = [], [], []
        for b in range(B):
            leaf = int(np.argmax(tree[b].sum(-1)))                 # the deepest path, one token fewer for the second sequence
            path = np.flatnonzero(tree[b, leaf])[: None if b == 0 else -1]
            for k, i in enumerate(path):
                take.append(b * N + i), seq.append(b), at.append(lens[b] + k)
                kept[b].append(f(r["qkv"])[b * N + i])
            lens[b] += len(path)
        model.write(r, np.array(take), np.array(seq), np.array(at))
    x = model.tokens(1)
    r = model.step(x, 1, lens, lens, None)
    model.check(r, x, 1, lens, lens, None)
    if kind == "bf16":
        for b in range(B):
            rows = np.array(kept[b] + [f(r["qkv"])[b]]).reshape(-1, H + 2 * G, dh)
            o = np.concatenate([blk.attend(rows[-1, h], rows[:, H + h // (H // G)], rows[:, H + G + h // (H // G)]) for h in range(H)])
            x1 = f(x)[b] + blk.linear(o[None], f(model.weights["Wo"]), f(model.weights["bo"]))[0]
            assert np.max(np.abs(f(r["x1"])[b] - x1)) <= U.TOL["bf16"] * np.max(np.abs(x1))


def test_draft_block_captured():
    """A step recorded into a graph and replayed on other tokens and lengths, against the eager call."""
    m = U.amd()
    B, N, H, G, dh, L = 3, 6, 4, 2, 64, 80
    model = Model(B, N, H, G, dh, L, "fp8")
    fill(model, [80, 80, 80])
    d, T, cfg = H * dh, B * N, model.cfg
    shape = m.make_shape(T, d, cfg.d_ffn, cfg.E, 1, T, "bf16")
    x = model.tokens(N)
    lens = torch.tensor([10, 0, 80], dtype=torch.int32, device=DEV)
    pos = torch.arange(T, dtype=torch.int32, device=DEV)
    tree = torch.from_numpy(words(random_tree(B, N, 1))).to(DEV)
    qkv, out = torch.zeros((T, (H + 2 * G) * dh), dtype=torch.bfloat16, device=DEV), torch.zeros((T, d), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(m.moe_draft_block_workspace_bytes(shape, model.cache, N), dtype=torch.uint8, device=DEV)
    seq = torch.arange(B, dtype=torch.int32, device=DEV).repeat_interleave(N)

    def step():
        m.moe_draft_block_forward(shape, model.cache, N, model.rope, model.weights, x, model.turns, pos, *model.caches, lens, tree, qkv, out, None, None,
                                  None, ws)
        m.moe_cache_write(model.cache, qkv[:, H * dh:(H + G) * dh], qkv[:, (H + G) * dh:], seq, pos, *model.caches)

    start = [t.clone() for t in model.caches]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        x.add_(0.125)
        lens.copy_(torch.tensor([k * 20, 3 * k, 80 - k], dtype=torch.int32))
        for t, s in zip(model.caches, start):
            t.copy_(s)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got, held = out.clone(), [t.clone() for t in model.caches]
        for t, s in zip(model.caches, start):
            t.copy_(s)
        out.zero_()
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, got) and all(torch.equal(a, b) for a, b in zip(held, model.caches))
