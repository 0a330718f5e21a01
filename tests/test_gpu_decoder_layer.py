"""The decoder-layer example: attention and MoE together, prompts then single tokens."""
import os
import sys

import pytest
import torch

import paper_2607_12875_gb300 as gb

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

from decoder_layer import DecoderLayer  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache,bound", [("act", 0.02), ("e4m3", 0.06)])
def test_tokens_one_at_a_time_give_what_the_whole_prompt_gives(cache, bound):
    """Three sequences as whole prompts, and the same sequences with their last 5 tokens decoded one by one. The
    attention sees the same keys (bf16 cache: the same values, rounded weights apart; e4m3: 3 bits of mantissa, an
    error of at most 2^-4 of a value and on average far less), and routing may move a token's near-ties to another
    expert, so the median token is held to the bound and every token to a looser one."""
    lens, tail = [130, 9, 64], 5
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.empty((sum(lens), 1024), device="cuda").normal_(generator=g).to(torch.bfloat16)

    def offsets(n):
        return torch.tensor([0, *torch.tensor(n).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    whole = DecoderLayer(3, 140, cache=cache).forward(x, offsets(lens))
    layer = DecoderLayer(3, 140, cache=cache)
    parts = torch.split(x, lens)
    head = [n - tail for n in lens]
    layer.forward(torch.cat([p[:n] for p, n in zip(parts, head)]), offsets(head))
    errs = []
    for i in range(tail):
        y = layer.forward(torch.stack([p[n + i] for p, n in zip(parts, head)]), offsets([1, 1, 1]))
        want = torch.stack([w[n + i] for w, n in zip(torch.split(whole, lens), head)]).float()
        errs.append((y.float() - want).norm(dim=1) / want.norm(dim=1))
    errs = torch.cat(errs)
    assert gb.moe_device_status(layer.ws) == gb.OK
    assert float(errs.median()) <= bound and float(errs.max()) <= 6 * bound, errs
