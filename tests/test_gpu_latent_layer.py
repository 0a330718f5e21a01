"""The latent-attention layer example: both forms, the norm with the residual and the MoE together, prompts then
single tokens."""
import os
import sys

import pytest
import torch

import paper_2607_12875_gb300 as gb

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from latent_layer import LatentLayer  # noqa: E402

pytestmark = pytest.mark.gpu


def offsets(n):
    return torch.tensor([0, *torch.tensor(n).cumsum(0).tolist()], dtype=torch.int32, device="cuda")


def test_tokens_one_at_a_time_give_what_the_whole_prompt_gives():
    """Three sequences as whole prompts (expanded form), and the same sequences with their last 5 tokens one by one
    (absorbed form over the cache). The same attention but for bf16's rounding of the expanded keys and values there, of
    the absorbed queries and sums here, and of both forms' weights; routing may move a token's near-ties to another
    expert, so the median token is held to the bound and every token to a looser one."""
    lens, tail, bound = [130, 9, 64], 5, 0.02
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x, res = (torch.empty((sum(lens), 1024), device="cuda").normal_(generator=g).to(torch.bfloat16) for _ in range(2))
    y, total = LatentLayer(3, 140).forward(x, res, offsets(lens))
    whole = (y.float() + total.float()).split(lens)
    layer = LatentLayer(3, 140)
    head = [n - tail for n in lens]
    layer.forward(*(torch.cat([p[:n] for p, n in zip(t.split(lens), head)]) for t in (x, res)), offsets(head))
    errs = []
    for i in range(tail):
        y, total = layer.forward(*(torch.stack([p[n + i] for p, n in zip(t.split(lens), head)]) for t in (x, res)), offsets([1, 1, 1]))
        want = torch.stack([w[n + i] for w, n in zip(whole, head)])
        errs.append((y.float() + total.float() - want).norm(dim=1) / want.norm(dim=1))
    errs = torch.cat(errs)
    assert gb.moe_device_status(layer.ws) == gb.OK
    assert float(errs.median()) <= bound and float(errs.max()) <= 6 * bound, errs
