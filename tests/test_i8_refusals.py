"""Refusals of the entry points for 8-bit integers, on the CPU: nothing is launched, so pointers are made up."""
import ctypes

import pytest
import torch

from paper_2201_05596_amd import binding as B

FAKE, ODD, BIG = 0x1000, 0x1008, 1 << 45


def test_weights_bytes():
    for G, K, N, n in ((1, 64, 128, 8192), (3, 8, 8, 3 * 8192), (2, 1000, 4000, 2 * 16 * 32 * 8192), (1, 131072, 8, 2048 * 8192)):
        assert B.moe_i8_weights_bytes(G, K, N) == n
    for bad in ((0, 64, 128), (1, 0, 128), (1, 64, 0), (1, 60, 128), (1, 64, 4), (1, 131080, 8), (1, 8, 131080), (1 << 21, 8, 8), (-1, 64, 128), ((1 << 20) - 3, 8, 8), (1 << 10, 8, 131072)):
        assert B.moe_i8_weights_bytes(*bad) == 0
    assert B.moe_i8_weights_bytes((1 << 20) - 4, 8, 8) == ((1 << 20) - 4) * 8192


@pytest.mark.parametrize("G,K,N,code", [(0, 64, 64, -1), (1, 0, 64, -1), (1, 64, 0, -1), (1, 4, 64, -1), (1, 60, 64, -2), (1, 64, 68, -2), (1, 131080, 64, -2),
                                        (1 << 21, 64, 64, -2)])
def test_weights_sizes(G, K, N, code):
    lib = B.load_library()
    assert lib.moe_i8_quantize_weights(G, K, N, FAKE, FAKE, FAKE, None) == code
    assert lib.moe_i8_pack_weights(G, K, N, FAKE, FAKE, None) == code


def test_weights_pointers():
    lib = B.load_library()
    for p in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None), (ODD, FAKE, FAKE), (FAKE, ODD, FAKE), (FAKE, FAKE, ODD)):
        assert lib.moe_i8_quantize_weights(1, 64, 64, *p, None) == -1
    for p in ((None, FAKE), (FAKE, None), (ODD, FAKE), (FAKE, ODD)):
        assert lib.moe_i8_pack_weights(1, 64, 64, *p, None) == -1


def rows_call(dtype=1, rows=4, cols=1000, x=FAKE, xs=1000, codes=FAKE, cs=1024, scale=FAKE):
    return B.load_library().moe_i8_quantize_rows(dtype, rows, cols, x, xs, codes, cs, scale, None)


def test_rows_arguments():
    for bad in (dict(dtype=2), dict(dtype=-1), dict(rows=0), dict(rows=-1), dict(cols=0), dict(x=None), dict(codes=None), dict(scale=None), dict(x=ODD),
                dict(codes=ODD), dict(scale=ODD), dict(xs=992), dict(xs=1004), dict(dtype=0, xs=1002), dict(xs=(1 << 24) + 8), dict(cs=1008), dict(cs=1032),
                dict(cs=(1 << 24) + 16), dict(xs=-1000)):
        assert rows_call(**bad) == -1, bad
    for bad in (dict(cols=1004), dict(cols=131080, xs=131080, cs=131136), dict(rows=(1 << 24) + 1)):
        assert rows_call(**bad) == -2, bad


def linear_call(patch=None, codes=FAKE, cs=1024, row_scale=FAKE, W=FAKE, col_scale=FAKE, bias=FAKE, out=FAKE, os=4000, null=False):
    p = B.make_i8_linear(4, 1000, 4000, "bf16")
    for k, v in (patch or {}).items():
        setattr(p, k, v)
    return B.load_library().moe_i8_linear(None if null else ctypes.byref(p), codes, cs, row_scale, W, col_scale, bias, out, os, None)


def test_linear_arguments():
    for bad in (dict(n_rows=0), dict(K=0), dict(N=0), dict(out_dtype=2), dict(out_dtype=-1), dict(gelu=2), dict(gelu=-1), dict(n_rows=-5)):
        assert linear_call(bad) == -1, bad
    for bad in (dict(K=1004), dict(N=4004), dict(K=131080), dict(N=131080), dict(n_rows=(1 << 24) + 1), dict(n_rows=1 << 24, N=131072)):
        assert linear_call(bad, cs=1 << 18, os=1 << 18) == -2, bad
    for bad in (dict(null=True), dict(codes=None), dict(row_scale=None), dict(W=None), dict(col_scale=None), dict(out=None), dict(codes=ODD), dict(row_scale=ODD),
                dict(W=ODD), dict(col_scale=ODD), dict(bias=ODD), dict(out=ODD), dict(cs=1008), dict(cs=1032), dict(os=3992), dict(os=4004),
                dict(cs=(1 << 24) + 16), dict(os=(1 << 24) + 8)):
        assert linear_call(**bad) == -1, bad
    assert linear_call(dict(out_dtype=0), os=4002) == -1


BASE = dict(T=64, d_model=1024, d_ffn=4096, E=8, top_k=1, capacity=16, dtype=1, residual=0, flags=0)
BAD_SHAPES = [(dict(T=0), -1), (dict(E=0), -1), (dict(capacity=0), -1), (dict(top_k=0), -1), (dict(top_k=9), -1), (dict(residual=2), -1), (dict(flags=4), -1),
              (dict(flags=1), -1), (dict(dtype=5), -1), (dict(dtype=0), -2), (dict(E=2048), -2), (dict(d_model=1028), -2), (dict(d_ffn=4100), -2),
              (dict(d_model=131080), -2), (dict(d_ffn=131080), -2), (dict(T=(1 << 24) + 1), -2), (dict(capacity=(1 << 21) + 1), -2), (dict(top_k=3, E=8), -2),
              (dict(flags=2, E=200, top_k=1), -2), (dict(capacity=1 << 21, d_ffn=131072), -2)]


def weights(**patch):
    w = {n: FAKE for n in ("W1", "s1", "b1", "W2", "s2", "b2")}
    return B.MoeI8Weights(**{**w, **patch})


def ffn_call(shape, w, xe=FAKE, rows=FAKE, ye=FAKE, ws=FAKE, n=BIG):
    return B.load_library().moe_i8_expert_ffn(shape and ctypes.byref(shape), w and ctypes.byref(w), xe, rows, ye, ws, n, None)


def layer_call(shape, w, x=FAKE, Wg=FAKE, bg=None, out=FAKE, outs=(None,) * 6, ws=FAKE, n=BIG):
    return B.load_library().moe_i8_layer_forward(shape and ctypes.byref(shape), w and ctypes.byref(w), x, Wg, bg, out, *outs, ws, n, None)


@pytest.mark.parametrize("patch,code", BAD_SHAPES)
def test_shapes(patch, code):
    s = B.MoeShape(**{**BASE, **patch})
    assert ffn_call(s, weights()) == code and layer_call(s, weights()) == code
    assert B.moe_i8_workspace_bytes(s) == 0


def test_pointers_and_workspace():
    s = B.MoeShape(**BASE)
    need = B.moe_i8_workspace_bytes(s)
    assert need % 256 == 0 and need >= 8 * 16 * (4096 * 3 + 1024)
    assert ffn_call(None, weights()) == -1 and layer_call(None, weights()) == -1 and ffn_call(s, None) == -1 and layer_call(s, None) == -1
    for n in ("W1", "s1", "W2", "s2"):
        assert ffn_call(s, weights(**{n: None})) == -1 and layer_call(s, weights(**{n: None})) == -1
    for n in ("W1", "s1", "b1", "W2", "s2", "b2"):
        assert ffn_call(s, weights(**{n: ODD})) == -1 and layer_call(s, weights(**{n: ODD})) == -1
    for bad in (dict(xe=None), dict(rows=None), dict(ye=None), dict(xe=ODD), dict(rows=ODD), dict(ye=ODD)):
        assert ffn_call(s, weights(), **bad) == -1, bad
    for bad in (dict(x=None), dict(Wg=None), dict(out=None), dict(x=ODD), dict(Wg=ODD), dict(bg=ODD), dict(out=ODD), *(dict(outs=tuple(ODD if i == j else None for i in range(6))) for j in range(6))):
        assert layer_call(s, weights(), **bad) == -1, bad
    for bad in (dict(ws=None), dict(ws=ODD), dict(n=need - 1)):
        assert ffn_call(s, weights(), **bad) == -3 and layer_call(s, weights(), **bad) == -3, bad
    # the dense branch's weights are there if and only if the layer has one
    dense = dict(Wd1=FAKE, sd1=FAKE, Wd2=FAKE, sd2=FAKE)
    for n in (*dense, "bd1", "bd2"):
        assert layer_call(s, weights(**{n: FAKE})) == -1
    r = B.MoeShape(**{**BASE, "residual": 1})
    for n in dense:
        assert layer_call(r, weights(**{k: v for k, v in dense.items() if k != n})) == -1
    assert B.moe_i8_workspace_bytes(r) > need
    # a missing workspace of a refused shape gives the shape's error
    assert layer_call(B.MoeShape(**{**BASE, "dtype": 0}), weights(), ws=None, n=0) == -2


def test_binding_checks():
    with pytest.raises(ValueError, match="x: expected float32 or bfloat16"):
        B.moe_i8_quantize_rows(torch.zeros(4, 64, dtype=torch.float16), None, None)
    with pytest.raises(ValueError, match="expected \\[K, N\\]"):
        B.moe_i8_pack_weights(torch.zeros(64, dtype=torch.int8))
    with pytest.raises(B.MoeError) as e:
        B.moe_i8_pack_weights(torch.zeros(60, 64, dtype=torch.int8))
    assert e.value.status == -2
    B.moe_i8_quantize_rows(torch.zeros(0, 64), None, None)                # no rows: nothing to do
    B.moe_i8_linear(B.make_i8_linear(0, 64, 64, "bf16"), None, None, None, None, None, None)
