"""moe_i8_expert_ffn and moe_i8_layer_forward.

What they are made of is tested by itself (test_gpu_i8_quantize.py, test_gpu_i8_linear.py), so they are held to it here: an FFN
gives the bits of its rows taken one expert at a time through moe_i8_quantize_rows, moe_i8_linear with GELU, moe_i8_quantize_rows and
moe_i8_linear; a layer the sum of these, in 64 bits, with the gate's own tables, up to its roundings to bf16 (2^-8 of a value each) and
its sums in 32 bits.  Against the oracle, whose h may round to its other neighbour now and then, layers are held to the tolerance of
the bf16 layers."""
import numpy as np
import pytest
import torch

from oracle import i8_oracle as o
from oracle import moe_oracle as orc
from tests import gpu_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"
CANARY = 12345.0


def up(n, m):
    return (n + m - 1) // m * m


class Layer:
    def __init__(self, T, d, f, E, k=1, C=4, residual=False, bias=True, seed=0, skew=0.0):
        self.m = m = U.amd()
        g = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
        self.T, self.d, self.f, self.E, self.k, self.C, self.residual = T, d, f, E, k, C, residual
        self.plain = {"W1": r(E, d, f) * d ** -0.5, "W2": r(E, f, d) * f ** -0.5}
        if residual:
            self.plain |= {"Wd1": r(1, d, f) * d ** -0.5, "Wd2": r(1, f, d) * f ** -0.5}
        self.weights = {}
        for n, W in self.plain.items():
            self.plain[n] = W.to(torch.bfloat16)
            self.weights[n], self.weights["s" + n[1:]] = m.moe_i8_quantize_weights(self.plain[n])
            b = (r(W.shape[0], W.shape[2]) * 0.3).to(torch.bfloat16) if bias else None
            self.weights["b" + n[1:]] = b
        self.Wg, self.bg = r(d, E) * 0.5 * d ** -0.5, skew * torch.log(1 / torch.arange(1, E + 1, device=DEV, dtype=torch.float32)) if skew else None
        self.x = r(T, d).to(torch.bfloat16)
        self.shape = m.make_shape(T, d, f, E, k, C, "bf16", residual)
        self.ws = self.workspace()
        self.gen = g

    def workspace(self):
        n = self.m.moe_i8_workspace_bytes(self.shape)
        return torch.full((n,), 0x7f, dtype=torch.uint8, device=DEV)          # scratch memory may hold anything

    def expert(self, rows, e, one="1", two="2", f32=False):
        """FFN of expert e on rows [n, d], from the operators it is made of."""
        m, R = self.m, rows.shape[0]
        part = lambda name, n: None if self.weights[name] is None else self.weights[name].view(-1, n)[e]  # noqa: E731

        def q(x):
            codes, scale = torch.empty((R, up(x.shape[1], 64)), dtype=torch.int8, device=DEV), torch.empty(R, device=DEV)
            m.moe_i8_quantize_rows(x, codes, scale)
            return codes, scale

        def product(x, which, K, N, gelu, dt):
            W = self.weights["W" + which]
            W = W.view(-1, m.moe_i8_weights_bytes(1, K, N))[e]
            out = torch.empty((R, N), dtype=dt, device=DEV)
            m.moe_i8_linear(m.make_i8_linear(R, K, N, dt, gelu), *q(x), W, part("s" + which, N), part("b" + which, N), out)
            return out

        h = product(rows, one, self.d, self.f, True, torch.bfloat16)
        return product(h, two, self.f, self.d, False, torch.float32 if f32 else torch.bfloat16)

    def ffn(self, xe, rows, ye):
        self.m.moe_i8_expert_ffn(self.shape, self.weights, xe, rows, ye, self.ws)

    def forward(self, x=None, out=None, ws=None):
        m, T, E, k, C = self.m, self.T, self.E, self.k, self.C
        x = self.x if x is None else x
        buf = torch.full((T + 8, self.d), CANARY, dtype=torch.bfloat16, device=DEV)
        i32 = dict(dtype=torch.int32, device=DEV)
        r = dict(logits=torch.empty((T, E), device=DEV), expert_idx=torch.empty((T, k), **i32), slot_idx=torch.empty((T, k), **i32),
                 gate_w=torch.empty((T, k), device=DEV), expert_rows=torch.empty(E, **i32), slot_token=torch.empty((E, C), **i32))
        m.moe_i8_layer_forward(self.shape, self.weights, x, self.Wg, self.bg, buf[4:T + 4], *r.values(), self.ws if ws is None else ws)
        torch.cuda.synchronize()
        assert (buf[:4] == CANARY).all() and (buf[T + 4:] == CANARY).all()
        return buf[4:T + 4], r

    def composed(self, r, x=None):
        """(sum in 64 bits, magnitudes of its terms) from the operators and the gate's tables."""
        x = self.x if x is None else x
        out = torch.zeros((self.T, self.d), dtype=torch.float64, device=DEV)
        size = torch.zeros_like(out)
        rows = r["expert_rows"].tolist()
        for e in range(self.E):
            if rows[e] == 0:
                continue
            t = r["slot_token"][e, :rows[e]].long()
            j = (r["expert_idx"][t] == e).int().argmax(1)
            y = r["gate_w"][t, j].double()[:, None] * self.expert(x[t], e, f32=True).double()
            out[t] += y
            size[t] += y.abs()
        if self.residual:
            y = self.expert(x, 0, "d1", "d2", f32=True).double()
            out, size = out + y, size + y.abs()
        return out, size

    def check(self, x=None):
        x = self.x if x is None else x
        got, r = self.forward(x)
        lg = r["logits"].cpu().numpy()
        want = orc.gate(lg, self.k, self.C)
        for n in ("expert_idx", "slot_idx", "expert_rows", "slot_token"):
            assert (r[n].cpu().numpy() == want[n]).all(), n
        ref, size = self.composed(r, x)
        roundings = 1 if self.k == 1 and not self.residual else 2             # of the result, and of the terms
        bound = (2.0 ** -8 * ref.abs() + (roundings - 1) * 2.0 ** -8 * size) * (1 + 2.0 ** -7) + 2.0 ** -20 * size
        assert ((got.double() - ref).abs() <= bound).all(), ((got.double() - ref).abs() - bound).max()
        if self.k == 1 and not self.residual:
            assert (got[r["slot_idx"][:, 0] < 0] == 0).all()
        return got, r, lg

    def check_oracle(self):
        got, r, lg = self.check()
        q = {n: [o.quantise(w, 0) for w in W.float().cpu().numpy()] for n, W in self.plain.items()}
        b = {n: None if self.weights[n] is None else self.weights[n].view(-1, w).float().cpu().numpy()
             for n, w in (("b1", self.f), ("b2", self.d), ("bd1", self.f), ("bd2", self.d)) if n in self.weights}
        one = lambda n: None if b[n] is None else b[n][0]  # noqa: E731
        dense = (q["Wd1"][0], one("bd1"), q["Wd2"][0], one("bd2")) if self.residual else None
        want = o.layer(self.x.float().cpu().numpy(), lg, q["W1"], b["b1"], q["W2"], b["b2"], self.k, self.C, dense)["out"]
        assert np.abs(got.double().cpu().numpy() - want).max() <= U.TOL["bf16"] * np.abs(want).max()


FFNS = [(1, 1, 8, 8), (4, 7, 72, 136), (3, 16, 1000, 264), (5, 17, 136, 1000), (2, 32, 2056, 128), (9, 33, 64, 192), (3, 64, 256, 512), (2, 65, 520, 264),
        (3, 128, 128, 1024), (2, 129, 320, 200), (2, 200, 64, 4104), (1, 300, 1024, 256), (70, 3, 64, 128), (2, 20, 64, 16392)]


@pytest.mark.parametrize("E,C,d,f", FFNS)
@pytest.mark.parametrize("bias", [False, True])
def test_ffn(E, C, d, f, bias):
    """Rows of every kind of number, none among them; other rows stay as they are."""
    L = Layer(E * C, d, f, E, C=C, bias=bias, seed=E + C)
    xe = torch.randn((E, C, d), generator=L.gen, device=DEV).to(torch.bfloat16)
    for counts in ([C] * E, [0] * E, [(7 * e + 1) % (C + 1) for e in range(E)], [C + 5 if e % 2 else -3 for e in range(E)]):
        rows = torch.tensor(counts, dtype=torch.int32, device=DEV)
        ye = torch.full((E * C + 2, d), CANARY, dtype=torch.bfloat16, device=DEV)
        for e, n in enumerate(counts):
            xe[e, max(0, min(n, C)):] = float("nan")                      # what is behind the rows has no part
        L.ffn(xe, rows, ye[1:-1])
        torch.cuda.synchronize()
        want = torch.full_like(ye, CANARY)
        for e, n in enumerate(counts):
            n = max(0, min(n, C))
            if n:
                want[1 + e * C:1 + e * C + n] = L.expert(xe[e, :n].contiguous(), e)
        assert torch.equal(ye, want)
        xe = torch.randn((E, C, d), generator=L.gen, device=DEV).to(torch.bfloat16)


@pytest.mark.parametrize("E,C,d,f", [
    # few rows: 16 to 128 columns of a work-group, K of few blocks and more; 17 rows and more
    (50, 10, 256, 64), (50, 10, 256, 2000), (30, 10, 200, 64), (30, 10, 200, 2000), (5, 10, 200, 64), (5, 10, 200, 2000), (40, 9, 1024, 2048), (37, 9, 1032, 2048),
    (64, 16, 1024, 64), (30, 20, 200, 264), (5, 20, 200, 2000),
    # tiles, with weights in the caches and past them; one row tile and several
    (41, 100, 1024, 64), (41, 100, 1024, 4104), (41, 50, 1024, 4104), (41, 20, 1024, 4104), (41, 20, 1600, 4104),
    # tiles of 256 rows
    (8, 1100, 1024, 64), (8, 1100, 1024, 136), (33, 200, 1024, 4104), (33, 200, 1024, 4224), (17, 300, 1024, 8200), (17, 300, 1024, 8192)])
def test_ffn_on_every_kernel(E, C, d, f):
    L = Layer(E * C, d, f, E, C=C, seed=E + C)
    xe = torch.randn((E, C, d), generator=L.gen, device=DEV).to(torch.bfloat16)
    counts = [C if e == 0 else (37 * e + 5) % (C + 1) for e in range(E)]
    rows = torch.tensor(counts, dtype=torch.int32, device=DEV)
    ye = torch.full((E, C, d), CANARY, dtype=torch.bfloat16, device=DEV)
    L.ffn(xe, rows, ye)
    for e, n in enumerate(counts):
        assert (ye[e, n:] == CANARY).all()
        assert n == 0 or torch.equal(ye[e, :n], L.expert(xe[e, :n].contiguous(), e)), e


def test_ffn_bits_do_not_depend_on_room():
    """The same rows in experts with room for 3, 16, 17, 33, 100, 300: other kernels, the same bits."""
    got = []
    for C in (3, 16, 17, 33, 100, 300):
        L = Layer(64, 264, 520, 4, C=C, seed=3)
        xe = torch.zeros((4, C, 264), dtype=torch.bfloat16, device=DEV)
        xe[:, :3] = torch.randn((4, 3, 264), generator=torch.Generator(device=DEV).manual_seed(8), device=DEV).to(torch.bfloat16)
        ye = torch.zeros((4, C, 264), dtype=torch.bfloat16, device=DEV)
        L.ffn(xe, torch.tensor([3, 2, 0, 3], dtype=torch.int32, device=DEV), ye)
        got.append(ye[:, :3].clone())
    assert all(torch.equal(g, got[0]) for g in got)


@pytest.mark.parametrize("C", [8, 40])
def test_ffn_rows_that_are_not_numbers(C):
    """An infinity in a row, or a hidden value beyond bf16, is NaN in that row alone."""
    L = Layer(2 * C, 64, 128, 2, C=C, seed=1)
    xe = torch.randn((2, C, 64), generator=L.gen, device=DEV).to(torch.bfloat16)
    rows, want, got = torch.full((2,), C, dtype=torch.int32, device=DEV), torch.empty_like(xe), torch.empty_like(xe)
    L.ffn(xe, rows, want)
    xe[0, 1, 5], xe[1, 2, 63], xe[1, 5] = float("inf"), float("nan"), 3e38
    L.ffn(xe, rows, got)
    bad = torch.zeros((2, C), dtype=torch.bool, device=DEV)
    bad[0, 1] = bad[1, 2] = True
    assert got[bad].isnan().all()
    bad[1, 5] = True
    assert torch.equal(got[~bad], want[~bad])
    zero = torch.zeros_like(xe)
    L.ffn(zero, rows, got)
    assert torch.equal(got[0], L.expert(zero[0], 0)) and got.isfinite().all()


LAYERS = {
    # few rows per expert
    "one_token": dict(T=1, d=64, f=128, E=8, C=1), "one_token_top2": dict(T=1, d=1000, f=264, E=4, k=2, C=1), "one_expert": dict(T=5, d=72, f=136, E=1, C=5),
    "one_token_residual": dict(T=1, d=1024, f=512, E=128, k=2, C=1, residual=True), "two_tokens": dict(T=2, d=256, f=1000, E=16, C=2),
    "step": dict(T=64, d=512, f=1024, E=32, C=8), "step_drops": dict(T=64, d=256, f=256, E=4, C=3, skew=1.5), "step_top2": dict(T=33, d=136, f=264, E=8, k=2, C=33),
    "step_residual": dict(T=16, d=512, f=1032, E=8, C=16, residual=True), "step_residual_top2": dict(T=32, d=264, f=520, E=16, k=2, C=32, residual=True, bias=False),
    "many_experts": dict(T=100, d=64, f=72, E=300, C=2), "step_32": dict(T=32, d=256, f=512, E=2, C=32), "odd": dict(T=17, d=8, f=8, E=3, C=17),
    "all_dropped_but_one": dict(T=50, d=64, f=64, E=2, C=1), "step_room": dict(T=4, d=320, f=640, E=8, k=2, C=100),
    # experts of few rows beside a dense branch of more
    "mixed": dict(T=200, d=256, f=512, E=16, C=16, residual=True), "mixed_top2": dict(T=40, d=136, f=264, E=40, k=2, C=8, residual=True),
    # tiles
    "tiles": dict(T=300, d=256, f=512, E=4, C=100), "tiles_drops": dict(T=500, d=136, f=264, E=4, C=60, skew=1.0), "tiles_256": dict(T=900, d=264, f=520, E=3, C=300),
    "tiles_residual": dict(T=400, d=256, f=512, E=4, C=200, residual=True), "tiles_residual_top2": dict(T=300, d=128, f=264, E=8, k=2, C=90, residual=True, skew=0.7),
    "prefill": dict(T=2304, d=256, f=512, E=8, C=360), "prefill_top2": dict(T=2500, d=72, f=200, E=16, k=2, C=400), "f32_gate": dict(T=700, d=1000, f=264, E=5, C=200),
    "prefill_residual": dict(T=2100, d=320, f=384, E=4, C=600, residual=True, bias=False),
}


@pytest.mark.parametrize("name", LAYERS)
def test_layer(name):
    Layer(**LAYERS[name], seed=len(name)).check()


@pytest.mark.parametrize("name", ["one_token_residual", "step", "step_drops", "step_residual_top2", "mixed", "tiles_drops", "tiles_residual_top2", "prefill"])
def test_layer_against_the_oracle(name):
    Layer(**LAYERS[name], seed=5).check_oracle()


@pytest.mark.parametrize("T", [16, 17, 24, 63, 64, 65, 127, 128, 129])
@pytest.mark.parametrize("E,k,C,residual", [(4, 1, 16, False), (4, 1, 16, True), (4, 2, 17, False), (30, 2, 8, False), (24, 1, 16, False), (30, 1, 16, True)])
def test_borders_of_the_few_tokens(T, E, k, C, residual):
    Layer(T, 264, 520, E, k, C, residual, seed=T + E).check()
    Layer(T, 1032, 1024, E, k, C, residual, seed=T + E).check()


@pytest.mark.parametrize("T,E,C,d,f", [(900, 41, 100, 1024, 64), (3000, 41, 100, 1024, 4104), (1500, 41, 50, 1024, 4104), (600, 41, 20, 1024, 4104), (7000, 8, 1100, 1024, 64),
                                       (7000, 8, 1100, 1024, 128), (4000, 33, 200, 1024, 4104), (4000, 33, 200, 1024, 4224), (4000, 17, 300, 1024, 8200),
                                       (4000, 17, 300, 1024, 8192)])
def test_combine_in_every_tile(T, E, C, d, f):
    """Top-1 layers, whose second products' tiles put the tokens back: tiles of 32, 64, 128 and 256 rows, weights in the caches and past them."""
    Layer(T, d, f, E, 1, C, seed=T + f, skew=0.3).check()


@pytest.mark.parametrize("T", list(range(1, 20)) + [31, 32, 33, 63, 64, 65, 255, 256, 257])
def test_every_number_of_tokens(T):
    Layer(T, 64, 136, 4, k=1 + T % 2, C=T, residual=T % 3 == 0, seed=T).check()


@pytest.mark.parametrize("T,k,residual", [(T, k, r) for T in (1, 2, 3, 4, 5) for k in (1, 2) for r in (False, True)])
@pytest.mark.parametrize("d,f,E,C", [(64, 8, 4, 1), (200, 136, 3, 2), (1000, 520, 9, 4), (72, 4104, 2, 4), (136, 5448, 5, 1), (1024, 4096, 128, 4),
                                     (1032, 8200, 3, 2), (64, 16384, 2, 1)])
def test_fewest_tokens(T, k, residual, d, f, E, C):
    """With and without a hand-over between the work-groups; odd numbers of blocks, single columns of a tile, dropped tokens."""
    Layer(T, d, f, E, k, C, residual, seed=T + f).check()


@pytest.mark.parametrize("name", ["step", "step_residual_top2", "tiles_residual"])
def test_layer_twice_is_the_same(name):
    L = Layer(**LAYERS[name], seed=2)
    a = L.forward()[0].clone()
    L.ws.random_(0, 255)
    assert torch.equal(a, L.forward()[0])


def test_a_token_that_is_not_a_number():
    """With room for all, the others' results do not change: not in an FFN, not in the dense branch."""
    for T, C, residual in ((12, 12, False), (12, 12, True), (300, 300, True)):
        L = Layer(T, 64, 136, 4, C=C, residual=residual, seed=T)
        want = L.forward()[0].clone()
        x = L.x.clone()
        x[3, 7] = float("nan")
        got = L.forward(x)[0]
        assert torch.equal(got[:3], want[:3]) and torch.equal(got[4:], want[4:])


def test_packed_gate():
    for name in ("step", "step_residual_top2", "prefill"):
        L = Layer(**LAYERS[name], seed=4)
        want, r = L.forward()
        want = want.clone()
        packed = L.m.moe_pack_gate(L.Wg)
        if packed is None:
            continue
        L.Wg, L.shape.flags = packed, L.m.MOE_FLAG_PACKED_GATE
        got, s = L.forward()
        assert torch.equal(got, want) and all(torch.equal(r[n], s[n]) for n in r)


@pytest.mark.parametrize("name", ["one_token_residual", "step", "step_residual_top2", "mixed", "tiles_residual", "prefill"])
def test_captured_and_replayed(name):
    """Two graphs that share a workspace, replayed in turn with eager calls between."""
    L = Layer(**LAYERS[name], seed=6)
    outs = [torch.empty_like(L.x) for _ in range(2)]
    xs = [L.x.clone(), L.x.clone()]
    call = lambda i: L.m.moe_i8_layer_forward(L.shape, L.weights, xs[i], L.Wg, L.bg, outs[i], *[None] * 6, L.ws)  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(0)
        call(1)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=side):
            call(i)
    for step in range(5):
        for i in range(2):
            xs[i].copy_(torch.randn(L.x.shape, generator=L.gen, device=DEV))
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], L.forward(xs[i])[0]), (step, i)


def test_two_streams():
    """Two layers at once, each with its workspace."""
    for a, b in (("step", "step_residual_top2"), ("one_token_residual", "step"), ("tiles_residual", "mixed")):
        layers = [Layer(**LAYERS[a], seed=1), Layer(**LAYERS[b], seed=2)]
        want = [L.forward()[0].clone() for L in layers]
        streams, outs = [torch.cuda.Stream() for _ in layers], [torch.empty_like(L.x) for L in layers]
        torch.cuda.synchronize()
        for _ in range(20):
            for L, s, out in zip(layers, streams, outs):
                with torch.cuda.stream(s):
                    L.m.moe_i8_layer_forward(L.shape, L.weights, L.x, L.Wg, L.bg, out, *[None] * 6, L.ws)
        torch.cuda.synchronize()
        assert all(torch.equal(out, w) for out, w in zip(outs, want))


@pytest.mark.parametrize("seed", range(12))
def test_random_layers(seed):
    g = np.random.default_rng(seed)
    pick = lambda lo, hi: int(round(np.exp(g.uniform(np.log(lo), np.log(hi)))))  # noqa: E731
    T, E = pick(1, 1500), pick(1, 64)
    k = 1 if E == 1 else int(g.integers(1, 3))
    C = max(1, min(T, round(float(g.choice([0.5, 1.25, 4])) * k * T / E)))
    Layer(T, 8 * pick(1, 100), 8 * pick(1, 200), E, k, C, bool(g.integers(2)), bool(g.integers(2)), seed, float(g.choice([0, 1.5]))).check()


def test_experts_behind_4_gib():
    """Weights and workspace beyond 32 bits: 130 experts of 4096 x 8448."""
    E, C, d, f = 130, 20, 4096, 8448
    L = Layer(E * C, 64, 64, E, C=C)
    m = L.m
    L.d, L.f = d, f
    one = {n: (torch.randn((3, *s), generator=L.gen, device=DEV) * s[0] ** -0.5).to(torch.bfloat16) for n, s in (("1", (d, f)), ("2", (f, d)))}
    for n, W in one.items():
        packed, scale = m.moe_i8_quantize_weights(W)
        at = torch.arange(E, device=DEV) % 3
        L.weights["W" + n] = packed.view(3, -1)[at].view(-1)
        L.weights["s" + n], L.weights["b" + n] = scale[at], None
    L.shape = m.make_shape(E * C, d, f, E, 1, C, "bf16")
    L.ws = L.workspace()
    xe = torch.randn((E, C, d), generator=L.gen, device=DEV).to(torch.bfloat16)
    ye = torch.zeros_like(xe)
    rows = torch.full((E,), C, dtype=torch.int32, device=DEV)
    L.ffn(xe, rows, ye)
    for e in (0, 64, 127, 129):
        assert torch.equal(ye[e], L.expert(xe[e], e)), e


@pytest.mark.parametrize("name", ["one_token_residual", "step", "prefill"])
@pytest.mark.parametrize("pack", [False, True])
def test_layer_object(name, pack):
    """MoELayer(int8=True): the entry point's bits and routing, its weights codes only."""
    L = Layer(**LAYERS[name], seed=2)
    want, r = L.forward()
    plain = {n: W[0] if n[1] == "d" else W for n, W in L.plain.items()}
    bias = {n: L.weights[n] if L.weights[n] is None or n[1] != "d" else L.weights[n][0] for n in L.weights if n[0] == "b"}
    layer = L.m.MoELayer(L.T, L.d, L.f, L.E, L.k, L.C, "bf16", L.Wg, L.bg, **plain, **bias, pack_weights=pack, int8=True)
    for _ in range(2):
        assert torch.equal(layer(L.x), want) and all(torch.equal(layer.routing[n], r[n]) for n in r)
    assert layer.i8["W1"].dtype == torch.int8 and not any(t is W for t in layer.weights for W in plain.values())


def test_binding_refuses():
    L = Layer(**LAYERS["step_residual"], seed=1)
    out = torch.empty_like(L.x)
    args = dict(x=L.x, Wg=L.Wg, bg=None, out=out, logits_out=None, expert_idx_out=None, slot_idx_out=None, gate_w_out=None, expert_rows_out=None, slot_token_out=None, ws=L.ws)
    for name, bad in (("x", L.x.float()), ("Wg", L.Wg[:-1]), ("out", out.cpu()), ("logits_out", out), ("workspace", L.ws[:-1]), ("expert_rows_out", L.x)):
        with pytest.raises(ValueError, match=name):
            L.m.moe_i8_layer_forward(L.shape, L.weights, **{**args, name.replace("workspace", "ws"): bad})
    for name in ("W1", "s1", "b1", "W2", "s2", "b2", "Wd1", "sd1", "bd1", "Wd2", "sd2", "bd2"):
        with pytest.raises(ValueError, match=name):
            L.m.moe_i8_layer_forward(L.shape, {**L.weights, name: L.weights[name].view(-1)[:-1]}, **args)
    with pytest.raises(L.m.MoeError):
        L.m.moe_i8_layer_forward(L.shape, {**L.weights, "Wd1": None}, **args)
