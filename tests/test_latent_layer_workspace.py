"""CPU check of the latent-attention layer example: every attention call gets a workspace of the size that the library
asks for that call's tokens and sequences. The library is a stand-in that asks for more the more tokens there are."""
import os
import sys

import pytest
import torch

import paper_2607_12875_gb300 as gb

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from latent_layer import LatentLayer  # noqa: E402


@pytest.fixture
def calls(monkeypatch):
    seen = []

    def size(cfg, T, B):
        return 256 * T * B

    def prompt(cfg, q, k, k_rope, v, cu_q, cu_k, out, ws, **kw):
        seen.append(("prompt", q.shape[0], ws.numel(), size(cfg, q.shape[0], cu_q.numel() - 1)))
        out.zero_()

    def cached(cfg, batch, q, cache, out, ws, **kw):
        seen.append(("cached", q.shape[0], ws.numel(), size(cfg, q.shape[0], batch.B)))
        out.zero_()

    def norm(cfg, x, residual, gamma, eps, total, y, **kw):
        total.copy_(x + residual)
        y.copy_(total)
    for name, stand_in in {"latent_workspace_size": size, "latent_prompt": prompt, "latent_cached": cached, "moe_rmsnorm_add": norm,
                           "workspace_size": lambda cfg: 1, "latent_append": lambda *a, **kw: None,
                           "moe_forward": lambda cfg, x, w, lb, sb, e, s, out, ws: out.zero_(),
                           "attn_rope_table": lambda P, *a, **kw: torch.zeros(P // 2, dtype=torch.int64)}.items():
        monkeypatch.setattr(gb, name, stand_in)
    return seen


def test_workspace_is_large_enough_for_every_call(calls):
    """Prompts that fill the context, then single and draft tokens."""
    def rows(n):
        return torch.zeros((n, 256), dtype=torch.bfloat16)

    def offsets(*n):
        return torch.tensor([0, *torch.tensor(n).cumsum(0).tolist()], dtype=torch.int32)
    layer = LatentLayer(3, 20, hidden=256, heads=2, latent=64, rope=16, nope=16, value=16, experts=2, top_k=1, intermediate=128, page=16,
                        device="cpu")
    layer.forward(rows(45), rows(45), offsets(20, 15, 10))
    layer.forward(rows(3), rows(3), offsets(1, 1, 1))
    layer.forward(rows(6), rows(6), offsets(2, 2, 2))
    assert [c[:2] for c in calls] == [("prompt", 45), ("cached", 3), ("cached", 6)]
    assert all(given >= asked for _, _, given, asked in calls), calls
