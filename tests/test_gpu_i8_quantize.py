"""moe_i8_quantize_rows, moe_i8_quantize_weights and moe_i8_pack_weights against the oracle, bit for bit: codes, scales, padding."""
import numpy as np
import pytest
import torch

from oracle import i8_oracle as o
from tests import gpu_util as U

pytestmark = pytest.mark.gpu
DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def up(n, m):
    return (n + m - 1) // m * m


def spread(rows, cols, seed, dtype):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, device=DEV) * torch.exp(4 * torch.randn((rows, 1), generator=g, device=DEV))
    return x.to(DT[dtype])


def check_rows(x, extra=0):
    """x: a view of rows; codes between canaries, `extra` bytes behind the padding."""
    m, (R, N) = U.amd(), x.shape
    pad = up(N, 64)
    buf = torch.full((R + 2, pad + extra), 77, dtype=torch.int8, device=DEV)
    scale = torch.full((R + 8,), 5.0, device=DEV)
    m.moe_i8_quantize_rows(x, buf[1:R + 1], scale[4:R + 4])
    torch.cuda.synchronize()
    want, s = o.quantise(x.float().cpu().numpy(), 1)
    got = buf.cpu().numpy()
    assert (got[0] == 77).all() and (got[R + 1] == 77).all() and (got[:, pad:] == 77).all()
    assert (got[1:R + 1, :N] == want).all() and (got[1:R + 1, N:pad] == 0).all()
    assert np.array_equal(scale[4:R + 4].cpu().numpy(), s, equal_nan=True)
    assert (scale[:4] == 5).all() and (scale[R + 4:] == 5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 8), (1, 64), (3, 72), (5, 520), (2, 2048), (7, 2056), (3, 4096), (4, 4104), (2, 8200), (3, 16384), (2, 16392),
                                       (2, 65536), (1, 65544), (2, 131072), (2048, 8), (2049, 512), (2050, 520), (2048, 1032), (2047, 1024), (2048, 2056),
                                       (2051, 4096), (2048, 4104), (9000, 4096), (5000, 8200)])
def test_rows(dtype, rows, cols):
    check_rows(spread(rows, cols, rows + cols, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 3, 2100])
def test_rows_of_wider_ones(dtype, rows):
    wide = spread(rows, 512, 3, dtype)
    check_rows(wide[:, 8:8 + 200], extra=128)
    check_rows(wide[:, 256:], extra=16)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_and_extremes(dtype):
    """Rows whose r is a power of two, so that halves are ties; rows without numbers, tiny, huge."""
    x = torch.zeros((40, 264))
    half = torch.arange(-127, 127) + 0.5                                  # representable in bf16 up to 128
    for i in range(20):
        x[i, :254] = half * 2.0 ** (6 * i - 60)
        x[i, 254] = 127 * 2.0 ** (6 * i - 60)
    x[21] = 2.0 ** -126
    x[22] = 2.0 ** -133
    x[23, 5], x[23, 6] = 2.0 ** -100, -2.0 ** -108
    x[24, :2] = torch.tensor([3.3e38, -2e36])
    x[25, 7] = float("inf")
    x[26, 9] = -float("inf")
    x[27, 263] = float("nan")
    x[28], x[28, 0] = 1e30, float("inf")
    x[29, 3] = -1.0
    check_rows(x.to(DT[dtype]).to(DEV))
    check_rows(x.to(DT[dtype]).to(DEV).repeat(60, 1))                     # a wave per row


def test_rows_behind_4_gib():
    """Codes and values at offsets beyond 32 bits."""
    x = torch.zeros((300, 1 << 23), dtype=torch.bfloat16, device=DEV)[:, :4096]
    x.copy_(spread(300, 4096, 9, "bf16"))
    m = U.amd()
    codes = torch.empty((300, 1 << 24), dtype=torch.int8, device=DEV)[:, :4096]
    scale = torch.empty(300, device=DEV)
    m.moe_i8_quantize_rows(x, codes, scale)
    want, s = o.quantise(x.float().cpu().numpy(), 1)
    assert (codes.cpu().numpy() == want).all() and (scale.cpu().numpy() == s).all()


@pytest.mark.parametrize("dtype,rows,cols", [("bf16", 70000, 512), ("bf16", 40000, 1000), ("bf16", 17000, 2048), ("bf16", 4100, 8192), ("bf16", 1100, 32768),
                                             ("bf16", 300, 131072), ("f32", 35000, 504), ("f32", 17000, 1024), ("f32", 9000, 2040), ("f32", 5000, 4096),
                                             ("f32", 2500, 8192), ("f32", 1500, 16384), ("f32", 600, 32768), ("f32", 150, 131072)])
def test_large_ones(dtype, rows, cols):
    """Past the caches: 64 MB and more."""
    check_rows(spread(rows, cols, rows, dtype))


def test_more_rows_than_a_launch_has():
    """Launches of 2^21 work-groups, four rows each."""
    n = (1 << 23) + 5
    x = torch.ones((n, 8), device=DEV)
    x[:, 3] = 2 * (torch.arange(n, device=DEV) % 61 + 1)                   # the largest: codes 127 there, 127 / it elsewhere
    codes, scale = torch.full((n + 1, 64), 77, dtype=torch.int8, device=DEV), torch.full((n + 1,), 5.0, device=DEV)
    U.amd().moe_i8_quantize_rows(x, codes[:n], scale[:n])
    want, s = o.quantise(x[:61].cpu().numpy(), 1)
    at = torch.arange(n, device=DEV) % 61
    assert torch.equal(scale[:n], torch.from_numpy(s).to(DEV)[at]) and (codes[n] == 77).all() and scale[n] == 5
    assert torch.equal(codes[:n, :8], torch.from_numpy(want).to(device=DEV, dtype=torch.int8)[at]) and not codes[:n, 8:].any()


WEIGHTS = [(1, 8, 8), (1, 64, 128), (2, 72, 136), (3, 520, 264), (1, 1000, 4000), (2, 1032, 64), (1, 2048, 192), (2, 2056, 72), (1, 8192, 128), (1, 131072, 16),
           (70, 128, 200), (1, 512, 8), (1, 1024, 8), (5, 16, 1000), (1, 4096, 136), (1, 4104, 136),
           # large ones, past the caches
           (9, 1000, 4000), (9, 2048, 2056), (3, 2056, 5448), (1, 16392, 2056), (40, 72, 16384)]


@pytest.mark.parametrize("G,K,N", WEIGHTS)
def test_weights(G, K, N):
    m = U.amd()
    g = torch.Generator(device=DEV).manual_seed(K + N)
    W = (torch.randn((G, K, N), generator=g, device=DEV) * torch.exp(2 * torch.randn((G, 1, N), generator=g, device=DEV))).to(torch.bfloat16)
    W[:, :, N // 2] = 0
    W[-1, K - 1, 0] = float("inf")
    W[0, 0, N - 1] = float("nan")
    packed, scale = m.moe_i8_quantize_weights(W)
    codes, s = o.quantise(W.float().cpu().numpy(), 1)
    assert packed.numel() == m.moe_i8_weights_bytes(G, K, N) and scale.shape == (G, N)
    assert (packed.cpu().numpy() == o.pack(codes)).all()
    assert np.array_equal(scale.cpu().numpy(), s, equal_nan=True)
    again = m.moe_i8_pack_weights(torch.from_numpy(codes).to(DEV))
    assert torch.equal(again, packed)
    if G == 1:
        one, s1 = m.moe_i8_quantize_weights(W[0])
        assert torch.equal(one, packed) and s1.shape == (N,) and torch.equal(m.moe_i8_pack_weights(torch.from_numpy(codes[0]).to(DEV)), packed)


def test_pack_takes_every_code():
    codes = torch.arange(64 * 128, device=DEV).to(torch.int8).view(1, 64, 128)        # -128 among them
    assert (U.amd().moe_i8_pack_weights(codes).cpu().numpy() == o.pack(codes.cpu().numpy())).all()


def test_weights_behind_4_gib():
    m = U.amd()
    W = torch.randn((1, 2048, 512), device=DEV).to(torch.bfloat16).expand(1100, 2048, 512).contiguous()
    W[1099] *= 3
    packed, scale = m.moe_i8_quantize_weights(W)
    n = packed.numel() // 1100
    for g in (0, 511, 1099):
        codes, s = o.quantise(W[g:g + 1].float().cpu().numpy(), 1)
        assert (packed[g * n:(g + 1) * n].cpu().numpy() == o.pack(codes)).all() and (scale[g].cpu().numpy() == s[0]).all()


def test_binding_refuses():
    m = U.amd()
    x, codes, scale = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4)
    for name, args in (("x", (x, codes.to(DEV), scale.to(DEV))), ("codes", (x.to(DEV), codes, scale.to(DEV))), ("scale", (x.to(DEV), codes.to(DEV), scale))):
        with pytest.raises(ValueError, match=f"{name}: device tensor required"):
            m.moe_i8_quantize_rows(*args)
    with pytest.raises(ValueError, match="W: device tensor required"):
        m.moe_i8_quantize_weights(torch.zeros(64, 64, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="codes: contiguous tensor required"):
        m.moe_i8_pack_weights(torch.zeros(64, 128, dtype=torch.int8, device=DEV)[:, ::2])
    with pytest.raises(ValueError, match="scale: expected 4 elements"):
        m.moe_i8_quantize_rows(x.to(DEV), codes.to(DEV), torch.zeros(5, device=DEV))
    with pytest.raises(m.MoeError):
        m.moe_i8_quantize_rows(torch.zeros(4, 68, device=DEV, dtype=torch.bfloat16)[:, :60], codes.to(DEV), scale.to(DEV))
    for bad in (codes.to(DEV)[:, :48], codes.to(DEV)[:3], codes.to(DEV).view(-1), torch.zeros(4, 128, dtype=torch.int8, device=DEV)[:, ::2]):
        with pytest.raises(ValueError, match="codes"):
            m.moe_i8_quantize_rows(x.to(DEV), bad, scale.to(DEV))


def test_captured_and_on_another_stream():
    m = U.amd()
    x, codes, scale = spread(300, 1000, 1, "bf16"), torch.empty((300, 1024), dtype=torch.int8, device=DEV), torch.empty(300, device=DEV)
    m.moe_i8_quantize_rows(x, codes, scale)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        m.moe_i8_quantize_rows(x, codes, scale)
    for seed in range(4):
        x.copy_(spread(300, 1000, seed, "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        want, s = o.quantise(x.float().cpu().numpy(), 1)
        assert (codes.cpu().numpy()[:, :1000] == want).all() and (scale.cpu().numpy() == s).all()
