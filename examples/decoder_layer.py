"""One decoder layer of an MoE model, served: packed prompts, then a token of each
sequence at a time. Random weights; run it on the GPU:

    python examples/decoder_layer.py [--cache e4m3|act] [--steps N]

    x -> moe_rmsnorm -> q, k, v projections -> attn_append (rotation, paged cache)
      -> attn_prompt (prompts) or attn_cached (one token) -> output projection, + x
      -> moe_rmsnorm -> moe_forward, + x

The projections are plain library products; everything else is this framework.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_12875_gb300 as gb  # noqa: E402


class DecoderLayer:
    """Weights of one layer, its paged cache for up to `batch` sequences of up to `context` tokens, and the
    handles that the calls take."""

    def __init__(self, batch, context, *, hidden=1024, heads=16, kv_heads=4, head_dim=64, experts=16, top_k=4,
                 intermediate=768, cache="e4m3", page=64, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(*shape, sigma):
            return torch.empty(shape, device=device).normal_(0.0, sigma, generator=g).to(torch.bfloat16)
        self.device, self.hidden, self.heads, self.kv_heads, self.head_dim = device, hidden, heads, kv_heads, head_dim
        self.w_qkv = weight(hidden, (heads + 2 * kv_heads) * head_dim, sigma=hidden ** -0.5)
        self.w_out = weight(heads * head_dim, hidden, sigma=(heads * head_dim) ** -0.5)
        self.gamma = [torch.ones(hidden, dtype=torch.bfloat16, device=device) for _ in range(2)]
        self.w_router = weight(experts, hidden, sigma=0.02)
        self.ffn = [weight(experts, intermediate, hidden, sigma=0.02), weight(experts, intermediate, hidden, sigma=0.02),
                    weight(experts, hidden, intermediate, sigma=0.02)]
        self.experts = gb.weights(*self.ffn)
        self.moe = dict(H=hidden, I=intermediate, E=experts, top_k=top_k)
        # attention: config, rotation table, a pool of pages and the table that deals them out
        self.attn = gb.attn_config(heads, kv_heads, head_dim, rotary_dim=head_dim, cache=cache, page=page)
        self.rope = gb.attn_rope_table(head_dim, 10000.0, device=device)
        per = -(-context // page)
        shape = (batch * per, kv_heads, page, head_dim)
        dt = torch.uint8 if cache == "e4m3" else torch.bfloat16
        self.k_pool, self.v_pool = (torch.zeros(shape, dtype=dt, device=device) for _ in range(2))
        self.scales = [torch.zeros(shape[:2], dtype=torch.uint8, device=device) for _ in range(2)] if cache == "e4m3" else [None] * 2
        self.cache = gb.attn_cache(self.k_pool, self.v_pool, *self.scales)
        order = torch.randperm(batch * per, generator=g, device=device).to(torch.int32)
        self.pages = order.view(batch, per)  # (an engine would hand pages out as sequences grow)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=device)
        self.ws, self.moe_ws = None, {}

    def _norm(self, x, which):
        y = torch.empty_like(x)
        gb.moe_rmsnorm(gb.make_config(x.shape[0], **self.moe), x, self.gamma[which], 1e-6, y)
        return y

    def _moe(self, x):
        cfg = gb.make_config(x.shape[0], **self.moe)
        ws = self.moe_ws.get(x.shape[0])
        if ws is None:
            ws = self.moe_ws[x.shape[0]] = torch.empty(gb.workspace_size(cfg), dtype=torch.uint8, device=self.device)
        out = torch.empty_like(x)
        gb.moe_forward(cfg, x, self.w_router, None, None, self.experts, None, out, ws)
        return out

    def forward(self, x, cu):
        """x [T, hidden]: new tokens of every sequence, packed (cu [batch + 1] int32 offsets on the device)."""
        T, batch = x.shape[0], self.lens.numel()
        prompts = bool((self.lens == 0).all())  # (an engine knows; this example asks the device)
        if self.ws is None:
            self.ws = torch.zeros(gb.attn_workspace_size(self.attn, T, batch), dtype=torch.uint8, device=self.device)
        qkv = (self._norm(x, 0) @ self.w_qkv).view(T, -1, self.head_dim)
        q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)  # slices of one projection's rows
        self.lens += cu[1:] - cu[:-1]
        new = gb.attn_batch(cu, self.lens, self.pages)
        out = torch.empty((T, self.heads, self.head_dim), dtype=x.dtype, device=x.device)
        if prompts:
            # rotated in place: the prompt attends to its own rows, the cache serves the tokens to come
            gb.attn_append(self.attn, new, k, v, self.rope, self.cache, q=q, q_out=q, k_out=k)
            gb.attn_prompt(self.attn, q, k, v, cu, cu, out, self.ws)
        else:
            gb.attn_append(self.attn, new, k, v, self.rope, self.cache, q=q, q_out=q)
            gb.attn_cached(self.attn, new, q, self.cache, out, self.ws)
        x = x + out.view(T, -1) @ self.w_out
        return x + self._moe(self._norm(x, 1))


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--cache", choices=("e4m3", "act"), default="e4m3")
    ap.add_argument("--steps", type=int, default=32)
    a = ap.parse_args()
    lens = [300, 17, 1024, 128]
    layer = DecoderLayer(len(lens), max(lens) + a.steps, cache=a.cache)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.empty((sum(lens), layer.hidden), device="cuda").normal_(generator=g).to(torch.bfloat16)
    cu = torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    one = torch.arange(len(lens) + 1, dtype=torch.int32, device="cuda")
    y = layer.forward(x, cu)
    y = y[cu[1:].long() - 1]  # each sequence's last token (a model would sample from the logits of the last layer)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(a.steps):
        y = layer.forward(y, one)
    end.record()
    torch.cuda.synchronize()
    if gb.moe_device_status(layer.ws) != gb.OK:
        raise SystemExit("a device-side wait gave up")
    print(f"{sum(lens)} prompt tokens, then {a.steps} steps of {len(lens)} sequences: "
          f"{start.elapsed_time(end) / a.steps * 1e3:.0f} us a step, |y| {float(y.float().abs().mean()):.3f}")


if __name__ == "__main__":
    main()
