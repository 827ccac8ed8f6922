"""moe_i8_linear against the oracle.

Sums of codes are exact, so without bias and GELU a result in 32 bits is float32(acc) (s_row s_col) in two roundings, to the bit; with bias
the last multiply-add rounds once: a value is off by 2^-24 of |acc s| for the sum's conversion, as much for the scales' product, and 2^-24
of itself.  GELU's slope is below 1.13; its own exponential and reciprocal are good to 2^-22 times the exponent (below 2^5 where the result
is not negligible).  bf16 adds half a step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

from oracle import i8_oracle as o
from oracle import moe_oracle as orc
from tests import gpu_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"


def up(n, m):
    return (n + m - 1) // m * m


class Product:
    def __init__(self, R, K, N, seed=0, bias=False, extremes=False):
        g = np.random.default_rng(seed)
        self.R, self.K, self.N = R, K, N
        self.a = g.integers(-127, 128, (R, K)).astype(np.int8)
        self.w = g.integers(-127, 128, (K, N)).astype(np.int8)
        if extremes:                                                      # sums next to 2^31
            self.a[:], self.w[:] = 127, -128
            self.w[:, ::2] = 127
        self.sr = np.exp(g.standard_normal(R)).astype(np.float32)
        self.sc = (0.01 / K * np.exp(g.standard_normal(N))).astype(np.float32)
        self.b = torch.from_numpy(g.standard_normal(N) * 0.5).to(torch.bfloat16) if bias else None
        self.codes = torch.from_numpy(g.integers(-128, 128, (R, up(K, 64))).astype(np.int8))        # anything behind K
        self.codes[:, :K] = torch.from_numpy(self.a)
        self.codes = self.codes.to(DEV)
        self.W = U.amd().moe_i8_pack_weights(torch.from_numpy(self.w).to(DEV))
        self.row_scale, self.col_scale = torch.from_numpy(self.sr).to(DEV), torch.from_numpy(self.sc).to(DEV)

    def run(self, out="f32", gelu=False, rows=None, out_cols=0):
        m, R, N = U.amd(), self.R if rows is None else rows, self.N
        dt = torch.float32 if out == "f32" else torch.bfloat16
        buf = torch.full((R + 2, N + out_cols), 12345.0, dtype=dt, device=DEV)
        m.moe_i8_linear(m.make_i8_linear(R, self.K, N, out, gelu), self.codes[:R], self.row_scale[:R], self.W, self.col_scale,
                        None if self.b is None else self.b.to(DEV), buf[1:R + 1, :N])
        torch.cuda.synchronize()
        canary = torch.tensor(12345.0).to(dt)
        assert (buf[0].cpu() == canary).all() and (buf[R + 1].cpu() == canary).all() and (buf[:, N:].cpu() == canary).all()
        return buf[1:R + 1, :N]

    def check(self, out="f32", gelu=False, **kw):
        got = self.run(out, gelu, **kw).float().cpu().numpy().astype(np.float64)
        acc = self.a.astype(np.float64) @ self.w.astype(np.float64)
        part = np.abs(acc) * self.sr.astype(np.float64)[:, None] * self.sc.astype(np.float64)
        b = 0.0 if self.b is None else self.b.double().numpy()
        want = o.product(self.a, self.sr, self.w, self.sc) + b
        err = 2.0 ** -23 * part + 2.0 ** -24 * (np.abs(want) + 2.0 ** -23 * part)
        if self.b is None and not gelu and out == "f32":
            exact = acc.astype(np.float32) * (self.sr[:, None] * self.sc)
            assert (got == exact).all()
        if gelu:
            want, err = orc.gelu_tanh(want), 1.13 * err
            err = err + 2.0 ** -17 * np.abs(want) + 1e-9                  # (1e-9: exponents beyond 2^5)
        if out == "bf16":
            err = err + 2.0 ** -8 * (np.abs(want) + err)
        assert (np.abs(got - want) <= err).all(), np.max(np.abs(got - want) - err)


SHAPES = [(1, 8, 8), (1, 64, 128), (3, 72, 136), (16, 1000, 264), (17, 520, 72), (31, 64, 1000), (32, 2056, 128), (33, 128, 256), (63, 200, 264), (64, 1024, 512),
          (65, 136, 520), (127, 64, 264), (128, 256, 256), (129, 1000, 248), (191, 320, 264), (192, 128, 8), (193, 192, 512), (255, 72, 256), (256, 512, 264),
          (257, 640, 264), (300, 1000, 1000), (1025, 264, 520), (1, 8192, 24), (5, 131072, 16), (100, 16384, 40), (2000, 64, 64)]


@pytest.mark.parametrize("R,K,N", SHAPES)
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_linear(R, K, N, out):
    p = Product(R, K, N, seed=R + K + N, bias=N % 16 != 0)
    p.check(out)
    p.check(out, gelu=True, out_cols=8)


@pytest.mark.parametrize("R", [1, 40, 300])
def test_largest_sums(R):
    p = Product(R, 131072, 40, extremes=True)
    p.check("f32")
    got = p.run("f32").cpu().numpy()
    assert (got[0, :2] == (np.array([131072 * 127 * 127, -131072 * 127 * 128], np.int64).astype(np.float32) * (p.sr[0] * p.sc[:2]))).all()


# few rows, by the columns of a work-group and the waves of it; tiles of 256 rows on a K of whole and half chunks
@pytest.mark.parametrize("R,K,N", [(R, K, N) for R in (1, 5, 16, 17, 32) for K in (200, 1160) for N in (520, 5128, 10248)] + [(40, 200, 5000), (64, 2056, 4104)] +
                         [(R, K, N) for R, N in ((2600, 4104), (5000, 2048), (3585, 3080)) for K in (64, 128, 192, 1000)])
def test_many_columns(R, K, N):
    p = Product(R, K, N, seed=R + K + N, bias=N % 16 != 0)
    p.check("bf16")
    p.check("f32", gelu=True, out_cols=8)


@pytest.mark.parametrize("R,K,N", [(200, 4104, 32776), (256, 4224, 32776), (1700, 32776, 4104), (1793, 32768, 4104)])
def test_weights_past_the_caches(R, K, N):
    """128 MB of weights and more, read by one row tile and by several; products of integers in 64 bits are exact."""
    m, g = U.amd(), torch.Generator(device=DEV).manual_seed(R)
    codes = torch.randint(-127, 128, (R, up(K, 64)), generator=g, device=DEV, dtype=torch.int8)
    w = torch.randint(-127, 128, (K, N), generator=g, device=DEV, dtype=torch.int8)
    sr, sc = torch.rand(R, generator=g, device=DEV) + 0.5, (torch.rand(N, generator=g, device=DEV) + 0.5) * (1e-4 * K ** -0.5)
    acc = torch.cat([codes[:, :K].double() @ w[:, n:n + 4096].double() for n in range(0, N, 4096)], 1)
    packed = m.moe_i8_pack_weights(w)
    out = torch.empty((R, N), device=DEV)
    m.moe_i8_linear(m.make_i8_linear(R, K, N, "f32"), codes, sr, packed, sc, None, out)
    assert torch.equal(out, acc.float() * (sr[:, None] * sc))
    exact = out.double()
    m.moe_i8_linear(m.make_i8_linear(R, K, N, "f32", True), codes, sr, packed, sc, None, out)
    want = 0.5 * exact * (1 + torch.tanh(0.7978845608028654 * (exact + 0.044715 * exact ** 3)))
    assert ((out.double() - want).abs() <= 1.13 * 2.0 ** -24 * exact.abs() + 2.0 ** -17 * want.abs() + 1e-9).all()


def test_every_number_of_rows_gives_the_same_bits():
    """Tiles, splits and kernels change with the number of rows; integer sums do not."""
    p = Product(700, 776, 264, bias=True)
    want = {(out, gelu): p.run(out, gelu).clone() for out in ("f32", "bf16") for gelu in (False, True)}
    for R in (1, 2, 15, 16, 17, 31, 32, 33, 47, 48, 63, 64, 65, 90, 96, 127, 128, 129, 160, 192, 200, 255, 256, 257, 384, 511, 513):
        for (out, gelu), w in want.items():
            assert torch.equal(p.run(out, gelu, rows=R), w[:R]), (R, out, gelu)


@pytest.mark.parametrize("R", [5, 40, 300])
def test_a_row_that_is_not_a_number(R):
    p = Product(R, 200, 136)
    want = p.run().clone()
    p.row_scale[3] = float("nan")
    p.col_scale[7] = float("nan")
    got = p.run()
    assert got[3].isnan().all() and got[:, 7].isnan().all()
    keep = torch.ones_like(got, dtype=torch.bool)
    keep[3], keep[:, 7] = False, False
    assert torch.equal(got[keep], want[keep])


def test_codes_of_wider_rows():
    p = Product(40, 200, 136)
    for R in (5, 40):
        want = p.run(rows=R).clone()
        m = U.amd()
        wide = torch.full((R, 512), 99, dtype=torch.int8, device=DEV)
        wide[:, 128:128 + 256] = p.codes[:R]
        out = torch.empty_like(want)
        m.moe_i8_linear(m.make_i8_linear(R, 200, 136, "f32"), wide[:, 128:384], p.row_scale[:R], p.W, p.col_scale, None, out)
        assert torch.equal(out, want)


def test_results_behind_4_gib():
    """2^20 + 5 rows of 2304 results: offsets beyond 32 bits; the same rows repeat."""
    m, n, R, N = U.amd(), 1000, (1 << 20) + 5, 2304
    p = Product(n, 64, N, bias=True)
    want = p.run("bf16", True).clone()
    at = torch.arange(R, device=DEV) % n
    out = torch.empty((R, N), dtype=torch.bfloat16, device=DEV)
    m.moe_i8_linear(m.make_i8_linear(R, 64, N, "bf16", True), p.codes[at], p.row_scale[at], p.W, p.col_scale, p.b.to(DEV), out)
    for r in (0, 65536 * 13, 1 << 19, R - 1000):
        assert torch.equal(out[r:r + 500], want[at[r:r + 500]])


def test_from_values_to_values():
    """Rows and weights into codes, their product: near the product of the values themselves."""
    m = U.amd()
    g = torch.Generator(device=DEV).manual_seed(1)
    for R in (4, 200):
        x, W = torch.randn((R, 1000), generator=g, device=DEV).to(torch.bfloat16), torch.randn((1000, 520), generator=g, device=DEV).to(torch.bfloat16)
        codes, scale = torch.empty((R, 1024), dtype=torch.int8, device=DEV), torch.empty(R, device=DEV)
        m.moe_i8_quantize_rows(x, codes, scale)
        packed, s_col = m.moe_i8_quantize_weights(W)
        out = torch.empty((R, 520), device=DEV)
        m.moe_i8_linear(m.make_i8_linear(R, 1000, 520, "f32"), codes, scale, packed, s_col, None, out)
        xs, ws = x.double(), W.double()
        # a value is off by half a step (and 127 2^-22 of it), so is the other factor
        ds, dw = 0.501 * scale.double()[:, None].expand_as(xs), 0.501 * s_col.double()[None].expand_as(ws)
        bound = ds @ ws.abs() + xs.abs() @ dw + ds @ dw
        assert ((out.double() - xs @ ws).abs() <= bound + 2.0 ** -22 * (xs.abs() @ ws.abs())).all()


def test_captured_and_on_another_stream():
    m = U.amd()
    for R in (7, 300):
        p = Product(R, 328, 264, bias=True)
        b, out, shape = p.b.to(DEV), torch.empty((R, 264), device=DEV), m.make_i8_linear(R, 328, 264, "f32", True)
        call = lambda: m.moe_i8_linear(shape, p.codes, p.row_scale, p.W, p.col_scale, b, out)  # noqa: E731, B023
        call()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        for i in range(4):
            p.codes.copy_(torch.roll(p.codes, i + 1, 0))
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            call()
            torch.cuda.synchronize()
            assert torch.equal(got, out)


def test_binding_refuses():
    m, p = U.amd(), Product(4, 72, 64)
    out = torch.empty((4, 64), device=DEV)
    good = dict(codes=p.codes, row_scale=p.row_scale, W=p.W, col_scale=p.col_scale, bias=None, out=out)
    for name, bad in (("codes", p.codes.cpu()), ("row_scale", p.row_scale[:3]), ("W", p.W[:-16]), ("col_scale", p.col_scale.double()), ("bias", out[0]),
                      ("out", out.to(torch.bfloat16)), ("out", out[:, :32]), ("codes", p.codes[:, :64]), ("codes", p.codes[:3])):
        with pytest.raises(ValueError, match=name):
            m.moe_i8_linear(m.make_i8_linear(4, 72, 64, "f32"), **{**good, name: bad})
