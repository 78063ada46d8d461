"""Decoding with draft trees, end to end: a small transformer with random weights, its paged cache and the STAND step.

    python examples/tree_decode.py [--batch 4] [--steps 64] [--dtype bf16]

The model is a stand-in; everything around it is what a server runs per step, all of it on the GPU and on one stream:

    serving.TreeAttention     attention of the tree's nodes over the cache, per layer
    serving.LogitsProcessor   penalties and a grammar mask on the nodes' logits
    binding.Stand.step        verification, table update, next tree
    serving.PageMap           pages and slots for the accepted nodes
    serving.KvCommit          their keys and values, all layers
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

from paper_2506_04708_b200 import binding, inputs, serving


class Model:
    """Pre-norm transformer with grouped heads and rotary positions; weights from a seed."""

    def __init__(self, V=2000, layers=2, heads_q=8, heads_kv=2, dim=64, dtype=torch.bfloat16, device="cuda:0", seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.V, self.layers, self.hq, self.hkv, self.dim, self.dtype, self.dev = V, layers, heads_q, heads_kv, dim, dtype, device
        width = heads_q * dim
        w = lambda *s: (torch.randn(s, generator=g, device=device) / s[0] ** 0.5).to(dtype)  # noqa: E731
        self.embed = (torch.randn((V, width), generator=g, device=device)).to(dtype)
        self.blocks = [dict(qkv=w(width, (heads_q + 2 * heads_kv) * dim), out=w(width, width), up=w(width, 2 * width), down=w(2 * width, width))
                       for _ in range(layers)]
        self.head = (w(width, V).float() * 4).to(dtype)  # peaked enough for drafts to be accepted now and then
        self.freq = 10000.0 ** (-torch.arange(0, dim, 2, device=device, dtype=torch.float32) / dim)

    def rotate(self, x, pos):
        a = pos.float()[..., None, None] * self.freq
        x0, x1 = x.float().unflatten(-1, (-1, 2)).unbind(-1)
        return torch.stack([x0 * a.cos() - x1 * a.sin(), x0 * a.sin() + x1 * a.cos()], -1).flatten(-2).to(x.dtype)

    @staticmethod
    def norm(x):
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def forward(self, tokens, pos, attend):
        """tokens, pos [B, N]; attend(layer, q, k, v) -> [B, N, heads_q, dim].  Returns logits, keys and values of all
        layers [layers, B, N, heads_kv, dim]."""
        x = self.embed[tokens.clamp(min=0).long()]  # a node that was not drafted gets some token: nobody looks at it
        ks, vs = [], []
        for i, w in enumerate(self.blocks):
            qkv = (self.norm(x) @ w["qkv"]).unflatten(-1, (-1, self.dim))
            q, k, v = qkv.split([self.hq, self.hkv, self.hkv], 2)
            q, k = self.rotate(q, pos), self.rotate(k, pos)
            ks.append(k)
            vs.append(v)
            x = x + attend(i, q, k, v).flatten(2) @ w["out"]
            h = self.norm(x) @ w["up"]
            x = x + torch.nn.functional.silu(h) @ w["down"]
        return self.norm(x) @ self.head, torch.stack(ks), torch.stack(vs)


class Decoder:
    """A batch of sequences, decoded with draft trees of one static shape."""

    def __init__(self, model, prompts, N=16, depth=5, kids=3, page=16, most=512, temperature=0.7, seed=1, mask=None):
        m, dev, B = model, model.dev, len(prompts)
        self.m, self.B, self.N, self.page = m, B, N, page
        self.parent = inputs.topology(N, depth, kids)
        self.depth = torch.from_numpy(inputs.node_depths(self.parent)).to(dev)
        cols = -(-most // page)
        pool = B * cols
        self.cache_k = torch.zeros((m.layers, pool, m.hkv, page, m.dim), dtype=m.dtype, device=dev)
        self.cache_v = torch.zeros_like(self.cache_k)
        self.table = torch.full((B, cols), -1, dtype=torch.int32, device=dev)
        self.free = torch.arange(pool, dtype=torch.int32, device=dev)
        self.n_free = torch.tensor([pool], dtype=torch.int32, device=dev)
        self.len = torch.zeros(B, dtype=torch.int64, device=dev)  # tokens in the cache: the text without its last one
        self.text = torch.zeros((B, most), dtype=torch.int32, device=dev)
        self.n_text = torch.tensor([len(p) for p in prompts], dtype=torch.int64, device=dev)
        self.n_prompt = self.n_text.clone()
        for b, p in enumerate(prompts):
            self.text[b, : len(p)] = torch.as_tensor(p, dtype=torch.int32)
        order = 3
        logits_dtype = binding.DTYPE_F32 if m.dtype == torch.float32 else binding.DTYPE_BF16
        self.stand = binding.Stand(B, N, m.V, 8, order, logits_dtype, temperature, seed, 1 << 16, self.parent, device=dev)
        width = self.stand.D + 1
        self.attention = serving.TreeAttention(B, N, m.hq, m.hkv, m.dim, m.dtype, page, pool, cols, parent=self.parent, device=dev)
        self.map = serving.PageMap(B, width, page, cols, pool, device=dev)
        self.commit = serving.KvCommit(m.layers, B, N, m.hkv, m.dim, m.dtype, page, pool, width, device=dev)
        self.processor = serving.LogitsProcessor(B, N, m.V, torch.float32 if m.dtype == torch.float32 else torch.bfloat16,
                                                 parent=self.parent, device=dev)
        self.presence = torch.full((B,), 0.2, device=dev)
        self.mask = mask
        self.mask_row = None if mask is None else torch.zeros((B, N), dtype=torch.int32, device=dev)
        self.path = torch.full((B, width), -1, dtype=torch.int32, device=dev)
        self.short = torch.zeros(B, dtype=torch.bool, device=dev)  # sequences that outgrew their pages: their text is no longer to be trusted
        self.prefill(max(len(p) for p in prompts) - 1)
        tail = np.full((B, order), -1, np.int32)
        for b, p in enumerate(prompts):
            tail[b, max(0, order - len(p)):] = p[-order:]
        self.stand.reset_sequences(torch.from_numpy(tail), self.n_text)
        self.tree = torch.full((B, N), -1, dtype=torch.int32, device=dev)
        self.tree[:, 0] = self.text.gather(1, self.n_text[:, None] - 1)[:, 0]

    def attend(self, attention):
        def f(layer, q, k, v):
            return attention(q, k, v, self.cache_k[layer], self.cache_v[layer], self.table, self.len, tree_tokens=self.seen)[0]
        return f

    def prefill(self, n):
        """All prompts in one pass (a chain of n nodes per sequence, shorter prompts padded)."""
        m, dev = self.m, self.m.dev
        if n == 0:
            return
        new = (self.n_text - 1).to(torch.int32)
        chain = serving.TreeAttention(self.B, n, m.hq, m.hkv, m.dim, m.dtype, self.page, self.cache_k.shape[1], self.table.shape[1], device=dev)
        slots_of = serving.PageMap(self.B, n, self.page, self.table.shape[1], self.free.numel(), device=dev)
        store = serving.KvCommit(m.layers, self.B, n, m.hkv, m.dim, m.dtype, self.page, self.cache_k.shape[1], n, device=dev)
        pos = torch.arange(n, device=dev)[None].expand(self.B, n)
        self.seen = torch.where(pos < new[:, None], self.text[:, :n], -1).contiguous()
        _, k, v = m.forward(self.text[:, :n], pos, self.attend(chain))
        slots, granted, length, self.n_free = slots_of(self.len, new, self.table, self.free, self.n_free)
        self.short |= granted < 0
        store(k, v, slots, self.cache_k, self.cache_v)
        self.len = length.clone()

    def step(self):
        """One step; returns the nodes' logits before processing (for checks), emitted tokens and their number."""
        self.seen = self.tree
        pos = self.len[:, None] + self.depth[None]
        raw, k, v = self.m.forward(self.tree, pos, self.attend(self.attention))
        logits = self.processor(raw, self.text, self.n_text, n_prompt=self.n_prompt, tree_tokens=self.tree, presence=self.presence,
                                mask=self.mask, mask_row=self.mask_row)
        emitted, n, tree = self.stand.step(logits)
        self.stand.path_device(self.path)
        slots, granted, self.len, self.n_free = self.map(self.len, n, self.table, self.free, self.n_free)
        self.short |= granted < 0  # looked at when the host has a reason to wait anyway
        self.commit(k, v, slots, self.cache_k, self.cache_v, path=self.path)
        j = torch.arange(emitted.shape[1], device=self.text.device)[None]
        at = (self.n_text[:, None] + j).clamp(max=self.text.shape[1] - 1)
        keep = self.text.gather(1, at)
        self.text.scatter_(1, at, torch.where(j < n[:, None], emitted, keep))
        self.n_text = self.n_text + n
        self.tree = tree
        return raw, emitted, n


def prompts_for(batch, V, seed=0):
    rng = np.random.default_rng(seed)
    return [rng.integers(0, V, rng.integers(5, 40)).astype(np.int32) for _ in range(batch)]


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    a = ap.parse_args()
    model = Model(dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    most = 40 + a.steps * 6 + 16
    dec = Decoder(model, prompts_for(a.batch, model.V), most=most)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    dec.step()
    start.record()
    for _ in range(a.steps):
        dec.step()
    end.record()
    torch.cuda.synchronize()
    if dec.short.any():
        raise SystemExit("a sequence outgrew its pages")
    made = int((dec.n_text - dec.n_prompt).sum())
    print(f"{a.batch} sequences, {a.steps + 1} steps: {made} tokens ({made / (a.steps + 1) / a.batch:.2f} per step and sequence), "
          f"{start.elapsed_time(end) / a.steps:.3f} ms per step")


if __name__ == "__main__":
    main()
