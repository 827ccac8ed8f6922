"""Refusals of moe_rope, moe_cache_write, moe_cache_read and moe_tree_attention, on the CPU: nothing is launched, so pointers are made up."""
import ctypes
import math

import pytest
import torch

from paper_2201_05596_amd import binding as B

FAKE, ODD, BIG = 0x1000, 0x1008, 1 << 40


def rope_call(patch=None, rows=4, heads=2, x=FAKE, xs=256, turns=FAKE, pos=FAKE, out=0x2000, os=256):
    r = B.make_rope(128, 64, "half", "bf16", scaling="by_parts", factor=4.0, original_len=4096.0)
    for k, v in (patch or {}).items():
        setattr(r, k, v)
    return B.load_library().moe_rope(ctypes.byref(r), rows, heads, x, xs, turns, pos, out, os, None)


@pytest.mark.parametrize("patch,code", [
    (dict(layout=2), -1), (dict(dtype=2), -1), (dict(scaling=3), -1), (dict(scaling=-1), -1), (dict(rot_dim=0), -1), (dict(rot_dim=136), -1),
    (dict(head_dim=0), -1), (dict(rot_dim=60), -2), (dict(head_dim=132), -2), (dict(head_dim=520), -2), (dict(base=1.0), -1), (dict(base=math.nan), -1),
    (dict(base=math.inf), -1), (dict(amplitude=math.inf), -1), (dict(amplitude=math.nan), -1), (dict(factor=0.0), -1), (dict(factor=-2.0), -1),
    (dict(factor=math.nan), -1), (dict(original_len=0.0), -1), (dict(low=4.0), -1), (dict(high=math.inf), -1)])
def test_rope_shapes(patch, code):
    assert rope_call(patch) == code
    r = B.make_rope(128, 64, "half", "bf16", scaling="by_parts", factor=4.0, original_len=4096.0)
    for k, v in patch.items():
        setattr(r, k, v)
    assert B.load_library().moe_rope_frequencies(ctypes.byref(r), (ctypes.c_double * 256)()) == code


def test_rope_arguments():
    for bad in (dict(rows=0), dict(heads=0), dict(x=None), dict(turns=None), dict(pos=None), dict(out=None), dict(x=ODD), dict(turns=ODD), dict(pos=ODD),
                dict(out=ODD), dict(xs=248), dict(os=248), dict(xs=260), dict(xs=(1 << 24) + 8), dict(xs=-256), dict(x=0x2000, xs=512)):
        assert rope_call(**bad) == -1, bad
    assert rope_call(rows=(1 << 24) + 1) == -2
    lib, r = B.load_library(), B.make_rope(128, 64, "half", "bf16")
    assert lib.moe_rope(None, 4, 2, FAKE, 256, FAKE, FAKE, FAKE, 256, None) == -1
    assert lib.moe_rope_frequencies(ctypes.byref(r), None) == -1 and lib.moe_rope_frequencies(None, (ctypes.c_double * 64)()) == -1
    # what a scaling does not use is not looked at
    assert lib.moe_rope_frequencies(ctypes.byref(B.make_rope(128, 64, "half", "bf16", factor=0.0, low=5.0)), (ctypes.c_double * 64)()) == 0


BAD_CACHES = [(dict(n_seq=0), -1), (dict(n_heads=0), -1), (dict(n_kv_heads=0), -1), (dict(n_heads=6), -1), (dict(head_dim=0), -1), (dict(max_len=0), -1),
              (dict(kind=3), -1), (dict(kind=-1), -1), (dict(head_dim=96), -2), (dict(head_dim=256), -2), (dict(max_len=(1 << 24) + 1), -2),
              (dict(n_heads=1028), -2), (dict(n_seq=1 << 29), -2)]


def cache_shape(**patch):
    return B.MoeCacheShape(**{**dict(n_seq=2, n_heads=8, n_kv_heads=4, head_dim=64, max_len=100, kind=1), **patch})


def write_call(c, rows=3, k=FAKE, ks=256, v=FAKE, vs=256, seq=FAKE, pos=FAKE, kc=FAKE, vc=FAKE, kx=FAKE, vx=FAKE):
    a = B.load_library().moe_cache_write(c and ctypes.byref(c), rows, k, ks, v, vs, seq, pos, kc, vc, kx, vx, None)
    b = B.load_library().moe_cache_read(c and ctypes.byref(c), rows, kc, vc, kx, vx, seq, pos, k, ks, v, vs, None)
    assert a == b
    return a


def tree_call(c, n=4, q=FAKE, qs=512, k=FAKE, ks=256, v=FAKE, vs=256, kc=FAKE, vc=FAKE, kx=FAKE, vx=FAKE, lens=FAKE, counts=FAKE, tree=FAKE, out=FAKE,
              os=512, ws=FAKE, wsn=BIG):
    return B.load_library().moe_tree_attention(c and ctypes.byref(c), n, q, qs, k, ks, v, vs, kc, vc, kx, vx, lens, counts, tree, out, os, ws, wsn, None)


@pytest.mark.parametrize("patch,code", BAD_CACHES)
def test_cache_shapes(patch, code):
    c = cache_shape(**patch)
    assert write_call(c) == code and tree_call(c) == code
    assert B.moe_cache_bytes(c) == 0 and B.moe_cache_scale_bytes(c) == 0 and B.moe_tree_attention_workspace_bytes(c, 4) == 0


def test_cache_sizes():
    for kind, elements, scales in (("bf16", 128, 0), ("fp8", 64, 2), ("fp4", 32, 2)):
        c = B.make_cache_shape(2, 8, 4, 64, 100, kind)
        assert B.moe_cache_bytes(c) == 800 * elements and B.moe_cache_scale_bytes(c) == 800 * scales
    huge = B.make_cache_shape(1 << 20, 8, 8, 128, 1 << 24, "bf16")
    assert B.moe_cache_bytes(huge) == 1 << (20 + 3 + 24 + 8)


def test_cache_arguments():
    assert write_call(None) == -1 and tree_call(None) == -1
    for kind in range(3):
        c = cache_shape(kind=kind)
        scales = dict(kx=None, vx=None) if kind == 0 else {}
        for bad in (dict(rows=0), dict(rows=-1), dict(k=None), dict(v=None), dict(seq=None), dict(pos=None), dict(kc=None), dict(vc=None), dict(k=ODD),
                    dict(v=ODD), dict(seq=ODD), dict(pos=ODD), dict(kc=ODD), dict(vc=ODD), dict(ks=248), dict(vs=252), dict(vs=260), dict(ks=0)):
            assert write_call(c, **{**scales, **bad}) == -1, bad
        assert write_call(c, **{**scales, "rows": (1 << 24) + 1}) == -2
        wrong = [dict(kx=FAKE, vx=None), dict(kx=None, vx=FAKE), dict(kx=FAKE, vx=FAKE)] if kind == 0 else [dict(kx=None), dict(vx=None), dict(kx=ODD)]
        for bad in wrong:
            assert write_call(c, **bad) == -1 and tree_call(c, **bad) == -1, bad


def test_tree_arguments():
    for kind in range(3):
        c = cache_shape(kind=kind)
        scales = dict(kx=None, vx=None) if kind == 0 else {}
        for bad in (dict(n=0), dict(n=-3), dict(q=None), dict(k=None), dict(v=None), dict(kc=None), dict(vc=None), dict(lens=None), dict(out=None),
                    dict(q=ODD), dict(k=ODD), dict(v=ODD), dict(lens=ODD), dict(counts=ODD), dict(tree=ODD), dict(out=ODD), dict(qs=504), dict(ks=248),
                    dict(vs=0), dict(os=516), dict(os=(1 << 24) + 8)):
            assert tree_call(c, **{**scales, **bad}) == -1, bad
        assert tree_call(c, **{**scales, "n": 257}) == -2
        need = B.moe_tree_attention_workspace_bytes(c, 4)
        assert need > 0
        for bad in (dict(wsn=need - 1), dict(ws=None), dict(ws=ODD)):
            assert tree_call(c, **{**scales, **bad}) == -3, bad
    assert tree_call(cache_shape(n_seq=1 << 22, n_heads=256, n_kv_heads=4), qs=1 << 14) == -2


class FakeDevice:
    """Stands in for a device tensor, so that the binding's checks run without one."""

    def __init__(self, shape, dtype, strides=None, index=0):
        self.shape, self.dtype, self.is_cuda = torch.Size(shape), dtype, True
        self._t = torch.empty(0, dtype=dtype)
        self._s = strides or torch.empty(shape, device="meta").stride()
        self.device = torch.device("cuda", index)

    def stride(self):
        return self._s

    def get_device(self):
        return self.device.index

    def is_contiguous(self):
        return tuple(self._s) == torch.empty(self.shape, device="meta").stride()

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self._t.element_size()

    def data_ptr(self):
        return FAKE


@pytest.fixture
def device0(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)


def test_binding_refuses_what_does_not_fit(device0):
    bf, i32, u8, F = torch.bfloat16, torch.int32, torch.uint8, FakeDevice
    c = cache_shape()
    good = dict(k=F((3, 256), bf), v=F((3, 256), bf), seq=F((3,), i32), pos=F((3,), i32), k_cache=F((2, 4, 100, 64), u8), v_cache=F((2, 4, 100, 64), u8),
                k_scale=F((2, 4, 100, 2), u8), v_scale=F((2, 4, 100, 2), u8))
    for name, bad in (("k", F((3, 128), bf)), ("k", F((3, 256), torch.float32)), ("v", F((4, 256), bf)), ("v", F((3, 256), bf, (512, 2))), ("seq", F((4,), i32)),
                      ("pos", F((3,), torch.int64)), ("k_cache", F((2, 4, 99, 64), u8)), ("v_cache", F((2, 4, 100, 64), bf)), ("k_scale", F((2, 4, 100, 4), u8)),
                      ("v_cache", F((2, 4, 100, 64), u8, (25600, 64, 256, 1)))):
        with pytest.raises(ValueError, match=name):
            B.moe_cache_write(c, **{**good, name: bad})
        with pytest.raises(ValueError, match=name if (name, bad.shape[0]) != ("k", 4) else "seq"):
            B.moe_cache_read(c, **{**good, name: bad})
    with pytest.raises(ValueError, match="cuda:1"):
        B.moe_cache_write(c, **{**good, "pos": F((3,), i32, index=1)})
    tree = dict(q=F((8, 512), bf), k=F((8, 256), bf), v=F((8, 256), bf), lens=F((2,), i32), counts=F((2,), i32), tree=F((2, 4, 1), i32), out=F((8, 512), bf),
                ws=F((BIG,), u8), **{n: good[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale")})
    for name, bad in (("q", F((8, 256), bf)), ("k", F((8, 512), bf)), ("lens", F((3,), i32)), ("counts", F((8,), i32)), ("tree", F((2, 4, 2), i32)),
                      ("out", F((8, 512), torch.float32)), ("workspace", F((16,), u8)), ("v_scale", F((2, 4, 100, 2), torch.int32))):
        with pytest.raises(ValueError, match=name):
            B.moe_tree_attention(c, 4, **{**tree, ("ws" if name == "workspace" else name): bad})
    rope = B.make_rope(64, 64, "half", "bf16")
    ok = dict(x=F((5, 128), bf), turns=F((32,), torch.float64), pos=F((5,), i32), out=F((5, 128), bf))
    for name, bad in (("x", F((5, 100), bf)), ("x", F((5, 128), torch.float32)), ("turns", F((16,), torch.float64)), ("turns", F((32,), torch.float32)),
                      ("pos", F((4,), i32)), ("out", F((5, 64), bf)), ("out", F((5, 128), bf, (1, 5)))):
        with pytest.raises(ValueError, match=name):
            B.moe_rope(rope, **{**ok, name: bad})
    # distances that the library refuses
    with pytest.raises(B.MoeError):
        B.moe_rope(rope, **{**ok, "out": F((5, 128), bf, (132, 1))})
    with pytest.raises(B.MoeError):
        B.moe_cache_write(c, **{**good, "k": F((3, 256), bf, (0, 1))})


def test_names_of_choices():
    assert B.make_rope(64, 64, "interleaved", torch.float32, scaling="linear").layout == B.MOE_ROPE_INTERLEAVED
    with pytest.raises(KeyError):
        B.make_rope(64, 64, "other", "bf16")
    with pytest.raises(KeyError):
        B.make_cache_shape(1, 1, 1, 64, 1, "int8")


def block_call(shape=None, c=None, n=4, rope="own", weights=None, x=FAKE, turns=FAKE, pos=FAKE, kc=FAKE, vc=FAKE, kx=FAKE, vx=FAKE, lens=FAKE, tree=FAKE,
               qkv=FAKE, out=FAKE, x1=None, moe_in=None, logits=None, ws=FAKE, wsn=BIG):
    s = B.MoeShape(**{**dict(T=8, d_model=512, d_ffn=1024, E=4, top_k=1, capacity=8, dtype=1, residual=0, flags=0), **(shape or {})})
    c = cache_shape(**(c or {}))
    r = B.make_rope(64, 64, "half", "bf16") if rope == "own" else rope
    w = {n: FAKE for n in B.BLOCK_WEIGHT_FIELDS if not n.endswith(("d1", "d2"))}
    w.update(weights or {})
    return B.load_library().moe_draft_block_forward(ctypes.byref(s), ctypes.byref(c), n, None if r is None else ctypes.byref(r),
                                                    ctypes.byref(B.MoeBlockWeights(**w)), x, turns, pos, kc, vc, kx, vx, lens, tree, qkv, out, x1, moe_in,
                                                    logits, ws, wsn, None)


def test_draft_block_arguments():
    for patch, code in BAD_CACHES:
        assert block_call(c=patch) == code, patch
    for bad in (dict(shape=dict(T=7)), dict(shape=dict(T=12)), dict(shape=dict(d_model=256)), dict(n=3), dict(n=0), dict(x=None), dict(lens=None),
                dict(qkv=None), dict(out=None), dict(kc=None), dict(vx=None), dict(turns=None), dict(pos=None), dict(x=ODD), dict(qkv=ODD), dict(tree=ODD),
                dict(logits=ODD), dict(x1=ODD), dict(moe_in=ODD), dict(rope=None), dict(rope=None, pos=None), dict(rope=B.make_rope(128, 64, "half", "bf16")),
                dict(rope=B.make_rope(64, 64, "half", "f32")), dict(weights=dict(Wqkv=None)), dict(weights=dict(ln2_beta=None)), dict(weights=dict(W1=ODD)),
                dict(weights=dict(Wd1=FAKE)), dict(shape=dict(residual=1))):
        assert block_call(**bad) == -1, bad
    assert block_call(shape=dict(dtype=0)) == -2
    assert block_call(ws=None) == -3
    s, c = B.make_shape(8, 512, 1024, 4, 1, 8, "bf16"), cache_shape()
    need = B.moe_draft_block_workspace_bytes(s, c, 4)
    assert need > 0 and block_call(wsn=need - 1) == -3
    assert B.moe_draft_block_workspace_bytes(s, c, 3) == 0
    assert B.moe_draft_block_workspace_bytes(B.make_shape(8, 512, 1024, 4, 1, 8, "f32"), c, 4) == 0


def test_binding_without_a_workspace(device0):
    """None is a workspace that is too small, and for a shape that is refused the shape's own error."""
    bf, i32, u8, F = torch.bfloat16, torch.int32, torch.uint8, FakeDevice

    def call(max_len, ws):
        c = B.make_cache_shape(1, 4, 4, 64, max_len, "bf16")
        rows = F((4, 256), bf)
        cache = F((1, 4, max_len, 64), bf)
        B.moe_tree_attention(c, 4, rows, rows, rows, cache, cache, None, None, F((1,), i32), None, None, rows, ws)

    with pytest.raises(ValueError, match="workspace"):
        call(100, None)
    for ws in (None, F((16,), u8)):
        with pytest.raises(B.MoeError, match="unsupported|not supported|shape"):
            call((1 << 24) + 1, ws)
