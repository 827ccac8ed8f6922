"""moe_draft_block_forward on many rows, and on steps where some sequences have fewer tokens than others."""
import numpy as np
import pytest
import torch

from tests import gpu_util as U
from tests.test_gpu_draft_block import DEV, Model, fill
from tests.test_gpu_tree_attention import random_tree, words

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,N,kind,residual", [(40, 256, "fp8", False), (64, 8, "bf16", True)])
def test_draft_block_many_rows(B, N, kind, residual):
    """A chunk of a prompt, and a batch of short chains: rows enough for many tiles of the projections."""
    H, G, dh, L = 2, 1, 64, 60
    print("case draft block rows", B, N, kind, flush=True)
    model = Model(B, N, H, G, dh, L, kind, "half", 64, residual=residual)
    lens = [int(v) for v in np.random.default_rng(1).integers(0, L + 1, B)]
    fill(model, lens)
    pos = (np.asarray(lens)[:, None] + np.arange(N)).reshape(-1)
    x = model.tokens(N)
    model.check(model.step(x, N, lens, pos, None), x, N, lens, pos, None)


@pytest.mark.parametrize("chain", [True, False])
@pytest.mark.parametrize("residual", [False, True])
def test_draft_block_rows_behind_a_sequence(chain, residual):
    """With a capacity that drops nothing, what the rows behind a sequence's tokens hold changes no token: not a bit up to the MoE layer,
    whose sums in 32 bits may have other parts (a step of bf16 at most)."""
    m = U.amd()
    B, N, H, G, dh, L = 4, 20, 4, 2, 64, 70
    model = Model(B, N, H, G, dh, L, "fp8", residual=residual)
    lens, counts = [70, 0, 33, 64], [20, 7, 1, 13]
    fill(model, lens)
    d, T, cfg = H * dh, B * N, model.cfg
    real = torch.tensor([i < counts[b] for b in range(B) for i in range(N)], device=DEV)
    bits = random_tree(B, N, 2)                        # a token sees itself and tokens before it: never those behind the count
    tree = None if chain else torch.from_numpy(words(bits)).to(DEV)
    pos = torch.from_numpy((np.asarray(lens)[:, None] + np.arange(N)).reshape(-1).astype(np.int32)).to(DEV)
    shape = m.make_shape(T, d, cfg.d_ffn, cfg.E, 1, T, "bf16", residual=residual)
    ws = torch.empty(m.moe_draft_block_workspace_bytes(shape, model.cache, N), dtype=torch.uint8, device=DEV)
    x, found = model.tokens(N), []
    print("case draft block behind", chain, residual, flush=True)
    for other in (None, 0.0, 1000.0, -1.0):
        y = x if other is None else torch.where(real[:, None], x, torch.full_like(x, other) * torch.arange(d, device=DEV).remainder(7).to(x.dtype))
        new = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)  # noqa: E731
        qkv, out, x1, moe_in, logits = new(T, d + 2 * G * dh), new(T, d), new(T, d), new(T, d), torch.zeros((T, cfg.E), device=DEV)
        m.moe_draft_block_forward(shape, model.cache, N, model.rope, model.weights, y, model.turns, pos, *model.caches,
                                  torch.tensor(lens, dtype=torch.int32, device=DEV), tree, qkv, out, x1, moe_in, logits, ws)
        torch.cuda.synchronize()
        found.append((out[real].float(), [t[real].clone() for t in (qkv, x1, moe_in, logits)]))
    out, exact = found[0]
    for o, e in found[1:]:
        assert all(torch.equal(a, b) for a, b in zip(e, exact))
        assert bool(((o - out).abs() <= 2.0 ** -7 * torch.maximum(o.abs(), out.abs()) + 2.0 ** -20 * out.abs().max()).all())
