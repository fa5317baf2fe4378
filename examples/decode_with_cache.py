"""A small decoder whose layers run on the library from end to end: prompt, then one token at a time.

    python examples/decode_with_cache.py [--prompt 600] [--steps 32] [--budget 256] [--layers 4] [--bits 16]

Per layer and prompt: the projections' output is the key/value cache of the prefill (no copy: the cache is described by
strides), si_attn_prefill attends to it, si_attn_weights ranks its entries by the attention the prompt's last queries gave
them, si_kv_evict keeps `budget` of them in the decode cache, and si_prefill_forward runs the FFN over the loaded neurons and
picks the ones that decoding will compute.  Per layer and token: si_attn_decode (which stores the new entry and adds up the
weights), si_kv_evict in place, si_ffn_forward over the chosen neurons.  With --bits 4 the decode caches are held in 4 bits: what
the eviction keeps of a prompt is quantised by si_kv4_store, and si_kv4_attn_decode and si_kv4_evict take the place of the two.  The model is random (there are no checkpoints here);
projections and norms are plain torch.  One decode step is captured in a CUDA graph and replayed.
"""
import argparse
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2607_18081_b200 import api  # noqa: E402


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-5)).to(x.dtype)


class Decoder:
    def __init__(self, layers=4, d_model=1024, n_q_heads=8, n_kv_heads=2, head_dim=128, d_ff=2816, loaded=1971, budget=256, n_sink=4,
                 n_recent=32, window=0, observe=32, dtype=torch.bfloat16, seed=0, bits=16):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g, device="cuda") * s[-1] ** -0.5).to(dtype)  # noqa: E731
        self.layers, self.d, self.hq, self.hkv, self.hd = layers, d_model, n_q_heads, n_kv_heads, head_dim
        self.budget, self.n_sink, self.n_recent, self.window, self.observe, self.dtype = budget, n_sink, n_recent, window, observe, dtype
        self.scale = 1.0 / math.sqrt(head_dim)
        self.w_qkv = [w((n_q_heads + 2 * n_kv_heads) * head_dim, d_model) for _ in range(layers)]
        self.w_out = [w(d_model, n_q_heads * head_dim) for _ in range(layers)]
        # the FFN: the first `loaded` neurons of a ranking are kept in the store, the first 30 % of d_ff are always computed
        self.n_loaded, self.n_static = loaded, min(loaded, 3 * d_ff // 10)
        self.active = min(loaded, 4 * d_ff // 10)
        self.store = api.NeuronStore(layers, d_model, d_ff, [loaded] * layers, dtype)
        for l in range(layers):
            ids = torch.randperm(d_ff, generator=g, device="cuda")[:loaded].cpu().numpy()
            self.store.load(l, w(d_ff, d_model), w(d_ff, d_model), w(d_model, d_ff), ids, self.n_static)
        self.lists = [torch.zeros(self.active, dtype=torch.int32, device="cuda") for _ in range(layers)]
        # decode caches: room for the budget and the entry of the step
        i32 = dict(dtype=torch.int32, device="cuda")
        self.bits = bits
        shape = (1, n_kv_heads, budget + 8 if bits == 16 else (budget + 32) // 32 * 32)
        self.length, self.position = torch.zeros(1, **i32), torch.zeros(1, **i32)      # shared by all layers
        self.wide = lambda length: api.KVCache(*(torch.zeros(*shape, head_dim, dtype=dtype, device="cuda") for _ in range(2)), length,  # noqa: E731
                                               torch.zeros(shape, **i32), torch.zeros(shape, device="cuda"))
        if bits == 16:
            self.caches = [self.wide(self.length) for _ in range(layers)]
            self.ws = self.caches[0].workspace(n_q_heads, 1)
        else:
            self.caches = [api.KV4Cache.empty(*shape, head_dim, 32, dtype, self.length, torch.zeros(shape, **i32), torch.zeros(shape, device="cuda"))
                           for _ in range(layers)]
            self.ws = self.caches[0].workspace(n_q_heads)
        self.status = torch.zeros(1, **i32)
        self.ffn_ws = self.store.workspace(1, self.active, 1)

    def split(self, qkv):
        """q [.., n_q_heads, head_dim] and k, v [.., n_kv_heads, head_dim] as views of a fused projection."""
        parts = qkv.view(*qkv.shape[:-1], self.hq + 2 * self.hkv, self.hd)
        return parts.split([self.hq, self.hkv, self.hkv], dim=-2)

    def prompt(self, x):
        """x: [T, d_model] of the prompt's tokens; fills the decode caches and the neuron lists; returns the last row."""
        T = x.shape[0]
        length = torch.full((1,), T, dtype=torch.int32, device="cuda")
        lse = torch.empty(1, T, self.hq, dtype=torch.float32, device="cuda")
        out = torch.empty(1, T, self.hq, self.hd, dtype=self.dtype, device="cuda")
        n_out = torch.zeros(1, dtype=torch.int32, device="cuda")
        ffn_ws = self.store.workspace(max(T, 2), self.n_loaded, 1)
        alpha, beta = self.active, self.n_loaded
        vote_ws = torch.zeros(api.si_prefill_vote_workspace_bytes(T, self.n_loaded, alpha) + 256, dtype=torch.uint8, device="cuda")
        vote_ws = vote_ws[(-vote_ws.data_ptr()) % 256:]
        kept_len = torch.full((1,), min(T, self.budget), dtype=torch.int32, device="cuda")
        kept = None if self.bits == 16 else self.wide(kept_len)          # what is kept of a layer, on its way into 4 bits
        self.length.copy_(kept_len if self.bits == 16 else torch.zeros_like(kept_len))
        self.position.fill_(T)
        for l in range(self.layers):
            q, k, v = self.split(torch.matmul(norm(x), self.w_qkv[l].T)[None])
            weight = torch.zeros(1, self.hkv, T, device="cuda")
            scratch = api.KVCache(k.transpose(1, 2), v.transpose(1, 2), length, None, weight)
            ws = scratch.workspace(self.hq, T)
            api.si_attn_prefill(scratch, q, self.window, self.n_sink, self.scale, out, lse, ws, self.status)
            last = min(T, self.observe)
            api.si_attn_weights(scratch, q[:, T - last:], self.window, self.n_sink, self.scale, lse[:, T - last:].contiguous(), ws, self.status)
            api.si_kv_evict(scratch, self.caches[l] if kept is None else kept, None, 0, self.budget, self.n_sink, self.n_recent, None, None, ws, self.status)
            if kept is not None:
                api.si_kv4_store(kept, self.caches[l], None, self.status)
            x = x + torch.matmul(out.view(T, -1), self.w_out[l].T)
            y = torch.empty_like(x)
            api.si_prefill_forward(self.store.handle, l, norm(x), T, y, alpha, beta, self.n_static, self.active, api.SI_FLAG_SCORE_ABS,
                                   self.lists[l], n_out, None, ffn_ws, vote_ws, self.status)
            x = x + y
        self.length.copy_(kept_len)
        return x[-1:]

    def attend(self, l, x):
        """The attention of layer l for the token in x [1, d_model]: new entry stored, weights added, one entry evicted."""
        q, k, v = self.split(torch.matmul(norm(x), self.w_qkv[l].T))
        out = torch.empty(1, self.hq, self.hd, dtype=self.dtype, device="cuda")
        decode, evict = (api.si_attn_decode, api.si_kv_evict) if self.bits == 16 else (api.si_kv4_attn_decode, api.si_kv4_evict)
        decode(self.caches[l], q, self.position, k, v, self.window, self.n_sink, self.scale, out, None, api.SI_FLAG_ACC_WEIGHT,
               self.ws, self.status)
        evict(self.caches[l], self.caches[l], self.position, 1, self.budget, self.n_sink, self.n_recent, None, None, self.ws, self.status)
        return out

    def step(self, x):
        """One token, x [1, d_model], through all layers; the caches stay at their budget."""
        for l in range(self.layers):
            x = x + torch.matmul(self.attend(l, x).view(1, -1), self.w_out[l].T)
            y = torch.empty_like(x)
            api.si_ffn_forward(self.store.handle, l, norm(x), 1, self.lists[l], None, self.active, y, 0, self.ffn_ws, self.status)
            x = x + y
        self.length.add_(1).clamp_(max=self.budget)
        self.position.add_(1)
        return x


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("prompt", 600), ("steps", 32), ("budget", 256), ("layers", 4)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--bits", type=int, default=16, choices=(4, 16))
    a = ap.parse_args()
    model = Decoder(layers=a.layers, budget=a.budget, bits=a.bits)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = model.prompt(torch.randn(a.prompt, model.d, generator=g, device="cuda").to(model.dtype))
    x = model.step(x)                                  # first use of every kernel, outside the capture
    torch.cuda.synchronize()
    buf = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        buf.copy_(norm(model.step(buf)))               # a random model has no vocabulary: the hidden state is the next input
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(a.steps):
        graph.replay()
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    assert model.status.item() == 0, api.strerror(model.status.item())
    entries = int(model.length.item())
    print(f"{a.layers} layers, prompt {a.prompt}, cache {entries} of {int(model.position.item())} positions per head, "
          f"{model.active} of {model.n_loaded} loaded neurons: {a.steps / took:.0f} tokens/s, |x| {buf.float().norm().item():.1f}")


if __name__ == "__main__":
    main()
