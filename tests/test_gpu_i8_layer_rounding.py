"""A layer with 8-bit experts rounds once, whatever the number of its tokens.

From the experts' (and the dense branch's) results in 32 bits, as moe_i8_linear gives them, and the gate's own tables, a token's result is a chain of
multiply-adds in 32 bits that begins with the dense branch's value, and one rounding to bf16.  Each multiply-add is formed here in 64 bits, where the
product of two values of 32 bits is exact, and rounded to 32: the layer's bits, on every kernel."""
import pytest
import torch

from tests.test_gpu_i8_layer import DEV, Layer

pytestmark = pytest.mark.gpu


def chain(L, r):
    terms = torch.zeros((L.k, L.T, L.d), device=DEV)
    for e, n in enumerate(r["expert_rows"].tolist()):
        if n:
            t = r["slot_token"][e, :n].long()
            terms[(r["expert_idx"][t] == e).int().argmax(1), t] = L.expert(L.x[t], e, f32=True)
    v = L.expert(L.x, 0, "d1", "d2", f32=True) if L.residual else torch.zeros_like(terms[0])
    for j in range(L.k):
        kept = (r["slot_idx"][:, j] >= 0)[:, None]
        v = torch.where(kept, (r["gate_w"][:, j, None].double() * terms[j].double() + v.double()).float(), v)
    return v.to(torch.bfloat16)


@pytest.mark.parametrize("T,d,f,E,k,C,residual", [
    # the kernels of few tokens, with a hand-over between work-groups and without
    (2, 256, 512, 8, 2, 2, True), (16, 512, 1032, 8, 1, 16, True), (12, 264, 520, 16, 2, 12, True), (60, 136, 264, 16, 2, 16, False),
    # tiles of 32, 64, 128 and 256 rows; experts and dense branch in one launch, with dropped tokens
    (24, 264, 520, 8, 1, 8, True), (40, 136, 264, 40, 2, 8, True), (200, 256, 512, 16, 1, 12, True), (300, 256, 512, 4, 2, 100, False), (300, 128, 264, 8, 2, 90, True),
    (1000, 1024, 512, 16, 2, 150, False), (2100, 320, 384, 4, 1, 600, True), (3000, 1024, 256, 8, 2, 700, True), (3000, 2048, 256, 8, 2, 900, False),
    (700, 1000, 264, 5, 1, 200, True)])
def test_one_rounding(T, d, f, E, k, C, residual):
    L = Layer(T, d, f, E, k, C, residual, seed=T + E)
    got, r = L.forward()
    assert torch.equal(got, chain(L, r))
