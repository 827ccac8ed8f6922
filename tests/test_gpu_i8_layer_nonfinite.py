"""A token that is not all numbers, or whose hidden values leave the range of bf16, is NaN in a layer with 8-bit experts, and with room for all no other
token's bits change: on the kernels of the fewest tokens, whose second products find scales of their own, on those of few, and in tiles.  Room for all
is top_k T rows: a token whose logits are all NaN has the last expert as both of its choices, so that expert has more rows than there are tokens."""
import pytest
import torch

from tests.test_gpu_i8_layer import DEV, Layer

pytestmark = pytest.mark.gpu

# experts and tokens: with up to 4 of each the fewest tokens' kernel; a hand-over between work-groups; tiles
SIZES = [(1, 2), (2, 2), (2, 8), (3, 3), (4, 2), (4, 3), (4, 8), (8, 2), (12, 8), (16, 3), (40, 2), (40, 8), (64, 30), (300, 8)]


def check(L, x, bad, want):
    got = L.forward(x)[0]
    rest = torch.ones(L.T, dtype=torch.bool, device=DEV)
    rest[bad] = False
    assert got[bad].isnan().all()
    assert got[rest].isfinite().all() and torch.equal(got[rest], want[rest])


@pytest.mark.parametrize("T,E", SIZES)
@pytest.mark.parametrize("k,residual", [(1, False), (1, True), (2, False), (2, True)])
@pytest.mark.parametrize("more", [0, 3])
def test_tokens(T, E, k, residual, more):
    L = Layer(T, 64, 136, E, k, k * T + more, residual, seed=T + E)
    want = L.forward()[0].clone()
    for bad, at, value in (([0], 63, float("nan")), ([T - 1], 0, float("inf")), ([T // 2], 31, -float("inf")), (list(range(0, T, 2)), 5, float("nan")),
                           (list(range((T + 1) // 2)), 5, float("nan"))):
        x = L.x.clone()
        x[bad, at] = value
        check(L, x, bad, want)


@pytest.mark.parametrize("T,E", SIZES)
@pytest.mark.parametrize("k,residual", [(1, False), (1, True), (2, False), (2, True)])
def test_hidden_values(T, E, k, residual):
    """h[7] is 3e38 x[0] in every expert and in the dense branch: 1.5e38 for a token with x[0] = 0.5, beyond bf16 (and 32 bits) with 2."""
    L = Layer(T, 64, 136, E, k, T, residual, bias=False, seed=T + E)
    for n in ("1", "d1") if residual else ("1",):
        L.plain["W" + n][:, :, 7] = 0
        L.plain["W" + n][:, 0, 7] = 3e38
        L.weights["W" + n], L.weights["s" + n] = L.m.moe_i8_quantize_weights(L.plain["W" + n])
    L.x[:, 0] = 0.5
    want = L.forward()[0].clone()
    for bad in {0, T // 2, T - 1}:
        x = L.x.clone()
        x[bad, 0] = 2
        check(L, x, [bad], want)


@pytest.mark.parametrize("T", [3, 12, 300])
@pytest.mark.parametrize("residual", [False, True])
def test_all_tokens(T, residual):
    """Nothing but tokens that are not numbers: 2 T rows of the last expert."""
    L = Layer(T, 64, 136, 4, 2, 2 * T, residual, seed=T)
    got, r = L.forward(torch.full_like(L.x, float("nan")))
    assert got.isnan().all() and (r["expert_idx"] == 3).all() and r["expert_rows"].tolist() == [0, 0, 0, 2 * T]
