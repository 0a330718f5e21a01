"""One decoder layer of an MoE model with latent attention, served: packed prompts in
the expanded form, then a token of each sequence at a time in the absorbed form over
the cached latents. Random weights; run it on the GPU:

    python examples/latent_layer.py [--steps N]

    x, residual -> moe_rmsnorm_add -> queries; latent and rotary key
      -> latent_append (norm, rotation, paged cache)
      -> latent_prompt (prompts) or latent_cached (one token) -> output projection
      -> moe_rmsnorm_add -> moe_forward

The projections are plain library products; everything else is this framework.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_12875_gb300 as gb  # noqa: E402


class LatentLayer:
    """Weights of one layer, its paged cache for up to `batch` sequences of up to `context` tokens, and the
    handles that the calls take."""

    def __init__(self, batch, context, *, hidden=1024, heads=20, latent=256, rope=32, nope=64, value=64, experts=16, top_k=4,
                 intermediate=768, page=64, seed=0, device="cuda"):
        g = torch.Generator(device=device)
        g.manual_seed(seed)

        def weight(*shape, sigma):
            return torch.empty(shape, device=device).normal_(0.0, sigma, generator=g).to(torch.bfloat16)
        self.device, self.hidden, self.heads = device, hidden, heads
        self.latent, self.rope, self.nope, self.value = latent, rope, nope, value
        self.w_q = weight(hidden, heads * (nope + rope), sigma=hidden ** -0.5)
        self.w_kv = weight(hidden, latent + rope, sigma=hidden ** -0.5)
        self.w_key = weight(heads, latent, nope, sigma=latent ** -0.5)      # latent -> a head's keys
        self.w_value = weight(heads, latent, value, sigma=latent ** -0.5)   # latent -> a head's values
        self.w_out = weight(heads * value, hidden, sigma=(heads * value) ** -0.5)
        self.gamma = [torch.ones(n, dtype=torch.bfloat16, device=device) for n in (hidden, hidden, latent)]
        self.w_router = weight(experts, hidden, sigma=0.02)
        self.ffn = [weight(experts, intermediate, hidden, sigma=0.02), weight(experts, intermediate, hidden, sigma=0.02),
                    weight(experts, hidden, intermediate, sigma=0.02)]
        self.experts = gb.weights(*self.ffn)
        self.moe = dict(H=hidden, I=intermediate, E=experts, top_k=top_k)
        self.attn = gb.latent_config(heads, latent_dim=latent, rope_dim=rope, nope_dim=nope, value_dim=value, page=page)
        self.table = gb.attn_rope_table(rope, 10000.0, device=device)
        per = -(-context // page)
        self.pool = torch.zeros((batch * per, page, latent + rope), dtype=torch.bfloat16, device=device)
        self.cache = gb.latent_cache(self.pool)
        order = torch.randperm(batch * per, generator=g, device=device).to(torch.int32)
        self.pages = order.view(batch, per)  # (an engine would hand pages out as sequences grow)
        self.lens = torch.zeros(batch, dtype=torch.int32, device=device)
        # (no call has more query tokens than whole prompts of all sequences)
        self.ws = torch.zeros(gb.latent_workspace_size(self.attn, batch * context, batch), dtype=torch.uint8, device=device)
        self.moe_ws = {}

    def _norm(self, x, residual, which):
        total, y = torch.empty_like(x), torch.empty_like(x)
        gb.moe_rmsnorm_add(gb.make_config(x.shape[0], **self.moe), x, residual, self.gamma[which], 1e-6, total, y)
        return total, y

    def _moe(self, x):
        cfg = gb.make_config(x.shape[0], **self.moe)
        ws = self.moe_ws.get(x.shape[0])
        if ws is None:
            ws = self.moe_ws[x.shape[0]] = torch.empty(gb.workspace_size(cfg), dtype=torch.uint8, device=self.device)
        out = torch.empty_like(x)
        gb.moe_forward(cfg, x, self.w_router, None, None, self.experts, None, out, ws)
        return out

    def forward(self, x, residual, cu):
        """x [T, hidden]: what the layer before adds to the residual, for the new tokens of every sequence, packed (cu
        [batch + 1] int32 offsets on the device); returns this layer's addition and the residual so far."""
        T, R, N = x.shape[0], self.latent, self.nope
        prompts = bool((self.lens == 0).all())  # (an engine knows; this example asks the device)
        residual, y = self._norm(x, residual, 0)
        q = (y @ self.w_q).view(T, self.heads, -1)
        kv = y @ self.w_kv
        self.lens += cu[1:] - cu[:-1]
        new = gb.attn_batch(cu, self.lens, self.pages)
        if prompts:
            # normed and rotated in place: the prompt attends to keys and values expanded from its own rows
            gb.latent_append(self.attn, new, kv, self.gamma[2], self.table, self.cache, q=q[..., N:], q_out=q[..., N:], kv_out=kv)
            k, v = (torch.einsum("tr,hrn->thn", kv[:, :R], w) for w in (self.w_key, self.w_value))
            out = torch.empty((T, self.heads, self.value), dtype=x.dtype, device=x.device)
            gb.latent_prompt(self.attn, q, k, kv[:, R:], v, cu, cu, out, self.ws)
        else:
            # the key's weights go into the query, the value's behind the sum: the cached rows serve all heads
            absorbed = torch.empty((T, self.heads, R + self.rope), dtype=x.dtype, device=x.device)
            absorbed[..., :R] = torch.einsum("thn,hrn->thr", q[..., :N], self.w_key)
            gb.latent_append(self.attn, new, kv, self.gamma[2], self.table, self.cache, q=q[..., N:], q_out=absorbed[..., R:])
            sums = torch.empty((T, self.heads, R), dtype=x.dtype, device=x.device)
            gb.latent_cached(self.attn, new, absorbed, self.cache, sums, self.ws)
            out = torch.einsum("thr,hrv->thv", sums, self.w_value)
        residual, y = self._norm(out.reshape(T, -1) @ self.w_out, residual, 1)
        return self._moe(y), residual


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=32)
    a = ap.parse_args()
    lens = [300, 17, 1024, 128]
    layer = LatentLayer(len(lens), max(lens) + a.steps)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.empty((sum(lens), layer.hidden), device="cuda").normal_(generator=g).to(torch.bfloat16)
    cu = torch.tensor([0, *torch.tensor(lens).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    one = torch.arange(len(lens) + 1, dtype=torch.int32, device="cuda")
    y, residual = layer.forward(x, torch.zeros_like(x), cu)
    last = cu[1:].long() - 1  # each sequence's last token (a model would sample from the logits of the last layer)
    y, residual = y[last], residual[last]
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(a.steps):
        y, residual = layer.forward(y, residual, one)
    end.record()
    torch.cuda.synchronize()
    if gb.moe_device_status(layer.ws) != gb.OK:
        raise SystemExit("a device-side wait gave up")
    print(f"{sum(lens)} prompt tokens, then {a.steps} steps of {len(lens)} sequences: "
          f"{start.elapsed_time(end) / a.steps * 1e3:.0f} us a step, |y| {float(y.float().abs().mean()):.3f}")


if __name__ == "__main__":
    main()
