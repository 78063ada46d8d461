"""Decoding with draft trees, end to end: a small transformer with random weights, its paged cache and the STAND step.

    python examples/tree_decode.py [--batch 4] [--steps 64] [--dtype bf16] [--cache 16]

The model is a stand-in; everything around it is what a server runs per step, all of it on the GPU and on one stream:

    serving.HeadRotation      norms of queries and keys per head and their rotation, per layer
    serving.TreeAttention     attention of the tree's nodes over the cache, per layer
    serving.LogitsProcessor   penalties and a grammar mask on the nodes' logits
    binding.Stand.step        verification, table update, next tree
    serving.PageMap           pages and slots for the accepted nodes
    serving.KvCommit          their keys and values, all layers

With --cache 4 the cache is held in 4 bits: serving.PackedTreeAttention reads it, and serving.KvAppend takes the accepted nodes' keys as the
projections left them, and normalises, turns and quantises them on the way (no other rotated keys are kept).
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

    def __init__(self, V=2000, layers=2, heads_q=8, heads_kv=2, dim=64, dtype=torch.bfloat16, device="cuda:0", seed=0, head_norm=False):
        g = torch.Generator(device=device).manual_seed(seed)
        self.V, self.layers, self.hq, self.hkv, self.dim, self.dtype, self.dev = V, layers, heads_q, heads_kv, dim, dtype, device
        width = heads_q * dim
        w = lambda *s: (torch.randn(s, generator=g, device=device) / s[0] ** 0.5).to(dtype)  # noqa: E731
        self.embed = (torch.randn((V, width), generator=g, device=device)).to(dtype)
        self.blocks = [dict(qkv=w(width, (heads_q + 2 * heads_kv) * dim), out=w(width, width), up=w(width, 2 * width), down=w(2 * width, width))
                       for _ in range(layers)]
        self.head = (w(width, V).float() * 4).to(dtype)  # peaked enough for drafts to be accepted now and then
        self.freq = 10000.0 ** (-torch.arange(0, dim, 2, device=device, dtype=torch.float32) / dim)
        self.head_norm = head_norm
        one = lambda: (1 + 0.2 * torch.randn((layers, dim), generator=g, device=device)).to(dtype)  # noqa: E731
        self.weight_q, self.weight_k = (one(), one()) if head_norm else (None, None)
        self.turns = {}  # by shape: the nodes' positions, and the layers' rotations by them

    def turn(self, pos):
        """The layers' rotations for tokens at pos [B, N]."""
        B, N = pos.shape
        if (B, N) not in self.turns:
            at = torch.zeros((B, N), dtype=torch.int32, device=self.dev)
            row = lambda w, i: None if w is None else w[i]  # noqa: E731
            self.turns[B, N] = at, [serving.HeadRotation(B, N, self.hq, self.hkv, self.dim, self.dtype, freq=self.freq, offset=at, interleaved=True,
                                                         norm=self.head_norm, weight_q=row(self.weight_q, i), weight_k=row(self.weight_k, i),
                                                         device=self.dev) for i in range(self.layers)]
        at, turns = self.turns[B, N]
        at.copy_(pos)
        return turns

    @staticmethod
    def norm(x):
        f = x.float()
        return (f * torch.rsqrt(f.square().mean(-1, keepdim=True) + 1e-6)).to(x.dtype)

    def forward(self, tokens, pos, attend, raw_keys=False):
        """tokens, pos [B, N]; attend(layer, q, k, v) -> [B, N, heads_q, dim].  Returns logits, keys (raw_keys: before norm and
        rotation) and values of all layers [layers, B, N, heads_kv, dim]."""
        turns = self.turn(pos)
        x = self.embed[tokens.clamp(min=0).long()]  # a node that was not drafted gets some token: nobody looks at it
        ks, vs = [], []
        for i, w in enumerate(self.blocks):
            qkv = (self.norm(x) @ w["qkv"]).unflatten(-1, (-1, self.dim))
            q, k, v = qkv.split([self.hq, self.hkv, self.hkv], 2)
            raw = k
            q, k = turns[i](q, k)
            ks.append(raw if raw_keys else k)
            vs.append(v)
            x = x + attend(i, q, k, v).flatten(2) @ w["out"]
            h = self.norm(x) @ w["up"]
            x = x + torch.nn.functional.silu(h) @ w["down"]
        return self.norm(x) @ self.head, torch.stack(ks), torch.stack(vs)


class Decoder:
    """A batch of sequences, decoded with draft trees of one static shape."""

    def __init__(self, model, prompts, N=16, depth=5, kids=3, page=16, most=512, temperature=0.7, seed=1, mask=None, packed=False):
        m, dev, B = model, model.dev, len(prompts)
        self.m, self.B, self.N, self.page = m, B, N, page
        self.parent = inputs.topology(N, depth, kids)
        self.depth = torch.from_numpy(inputs.node_depths(self.parent)).to(dev)
        cols = -(-most // page)
        pool = B * cols
        self.packed = packed
        if packed:
            self.cache_k = torch.zeros((m.layers, pool, m.hkv, serving.packed_block_bytes(page, m.dim)), dtype=torch.uint8, device=dev)
        else:
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
        self.attention = self.attention_of(N, parent=self.parent)
        self.map = serving.PageMap(B, width, page, cols, pool, device=dev)
        self.commit = self.commit_of(N, width, self.depth.to(torch.int32))
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

    def attention_of(self, N, parent=None):
        m, kind = self.m, serving.PackedTreeAttention if self.packed else serving.TreeAttention
        return kind(self.B, N, m.hq, m.hkv, m.dim, m.dtype, self.page, self.cache_k.shape[1], self.table.shape[1], parent=parent, device=m.dev)

    def commit_of(self, N, width, offset=None):
        """commit(k, v, slots, length, path): rows of N nodes, at positions length + offset (None: their number), into the cache."""
        m, shape = self.m, (self.m.layers, self.B, N, self.m.hkv, self.m.dim, self.m.dtype, self.page, self.cache_k.shape[1], width)
        if not self.packed:
            store = serving.KvCommit(*shape, device=m.dev)
            return lambda k, v, slots, length, path=None: store(k, v, slots, self.cache_k, self.cache_v, path=path)
        store = serving.KvAppend(*shape, packed=True, freq=m.freq, offset=offset, interleaved=True, norm=m.head_norm, weight_k=m.weight_k, device=m.dev)
        return lambda k, v, slots, length, path=None: store(k, v, slots, self.cache_k, self.cache_v, base=length, path=path)

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
        chain = self.attention_of(n)
        slots_of = serving.PageMap(self.B, n, self.page, self.table.shape[1], self.free.numel(), device=dev)
        store = self.commit_of(n, n)
        pos = torch.arange(n, device=dev)[None].expand(self.B, n)
        self.seen = torch.where(pos < new[:, None], self.text[:, :n], -1).contiguous()
        _, k, v = m.forward(self.text[:, :n], pos, self.attend(chain), raw_keys=self.packed)
        slots, granted, length, self.n_free = slots_of(self.len, new, self.table, self.free, self.n_free)
        self.short |= granted < 0
        store(k, v, slots, self.len)
        self.len = length.clone()

    def step(self):
        """One step; returns the nodes' logits before processing (for checks), emitted tokens and their number."""
        self.seen = self.tree
        pos = self.len[:, None] + self.depth[None]
        raw, k, v = self.m.forward(self.tree, pos, self.attend(self.attention), raw_keys=self.packed)
        logits = self.processor(raw, self.text, self.n_text, n_prompt=self.n_prompt, tree_tokens=self.tree, presence=self.presence,
                                mask=self.mask, mask_row=self.mask_row)
        emitted, n, tree = self.stand.step(logits)
        self.stand.path_device(self.path)
        before = self.len
        slots, granted, self.len, self.n_free = self.map(self.len, n, self.table, self.free, self.n_free)
        self.short |= granted < 0  # looked at when the host has a reason to wait anyway
        self.commit(k, v, slots, before, self.path)
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
    ap.add_argument("--cache", choices=("16", "4"), default="16", help="4: keys and values are held in 4 bits")
    a = ap.parse_args()
    model = Model(dtype=torch.bfloat16 if a.dtype == "bf16" else torch.float32)
    most = 40 + a.steps * 6 + 16
    dec = Decoder(model, prompts_for(a.batch, model.V), most=most, packed=a.cache == "4")
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
