"""Serving a decoder with the library: prompts in chunks, forks, decoding in a graph.

A stack of decoder layers with random weights (head norms and rotation, attention over a
paged cache, the routed sparse MLP), driven as a serving program drives one:

    extend the sequences' pages -> per layer: project, append (norm, rotation, cache),
    attend, project, sparse MLP -> logits -> sample

    python examples/serve.py [--layers 4] [--prompts 4] [--prompt 512] [--samples 2] [--tokens 64]
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_08991_amd as sats  # noqa: E402


class Decoder:
    """Weights of a small decoder, and the cache of its sequences."""

    def __init__(self, layers=4, heads=8, kv_heads=2, dim=64, d_ff=1024, vocab=4096, max_seqs=16, max_len=2048,
                 page=16, pages=None, dtype=torch.bfloat16, threshold=0.05, theta=10000.0, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        d = heads * dim

        def w(*shape, std):
            return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)

        self.layers, self.heads, self.kv_heads, self.dim, self.d, self.d_ff = layers, heads, kv_heads, dim, d, d_ff
        self.vocab, self.dtype, self.max_len, self.page = vocab, dtype, max_len, page
        self.embed = w(vocab, d, std=1.0)
        self.unembed = w(vocab, d, std=d ** -0.5)
        self.qkv = w(layers, (heads + 2 * kv_heads) * dim, d, std=d ** -0.5)
        self.q_norm, self.k_norm = (1 + w(layers, dim, std=0.1) for _ in range(2))
        self.o = w(layers, d, d, std=d ** -0.5)
        self.gate, self.up, self.down = (w(layers, d_ff, d, std=1.28 * d ** -0.5) for _ in range(3))
        self.thresholds = torch.full((layers,), threshold, device="cuda")
        self.lut = (torch.rand(vocab, generator=g, device="cuda") < 0.25).to(torch.uint8)  # 1: the dense path
        angle = torch.arange(max_len, device="cuda", dtype=torch.float64)[:, None] * theta ** (
            -torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim)
        self.rope = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        pages = pages or max_seqs * max_len // page
        shape = (layers, pages, kv_heads, page, dim)
        self.cache = sats.KVCache(torch.zeros(shape, device="cuda", dtype=dtype),
                                  torch.zeros(shape, device="cuda", dtype=dtype))
        self.pages = sats.KVPages(torch.full((max_seqs, max_len // page), -1, device="cuda", dtype=torch.int32),
                                  torch.zeros(max_seqs, device="cuda", dtype=torch.int32),
                                  torch.zeros(pages, device="cuda", dtype=torch.int32))
        self.status = torch.zeros(2, device="cuda", dtype=torch.int32)

    def forward(self, ids, batch, last):
        """Logits of rows `last` for the new tokens `ids`, whose pages are there already."""
        n = ids.numel()
        x = self.embed[ids.long()].float()
        q = torch.empty((n, self.heads, self.dim), device="cuda", dtype=self.dtype)
        att, mlp = torch.empty_like(q), torch.empty((n, self.d), device="cuda", dtype=self.dtype)
        for i in range(self.layers):
            h = rms(x).to(self.dtype)
            qkv = (h @ self.qkv[i].T).view(n, -1, self.dim)
            a, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), 1)
            sats.sats_qkv_append(a, k, v, self.rope, q, self.cache, i, batch, q_norm=self.q_norm[i],
                                 k_norm=self.k_norm[i])
            sats.sats_paged_attention(q, self.cache, i, batch, att, self.dim ** -0.5)
            x = x + (att.view(n, -1) @ self.o[i].T).float()
            h = rms(x).to(self.dtype)
            sats.sats_mlp_forward(h, ids, self.gate[i], self.up[i], self.down[i], self.thresholds[i:i + 1], self.lut,
                                  mlp, n, self.d, self.d_ff, 1)
            x = x + mlp.float()
        return (rms(x[last]).to(self.dtype) @ self.unembed.T).float()

    def prefill(self, seqs, prompts):
        """Runs the prompts (lists of ids) of the sequences `seqs`; logits of each one's last token."""
        lens = [len(p) for p in prompts]
        start = [0]
        for m in lens:
            start.append(start[-1] + m)
        seq, add = ints(seqs), ints(lens)
        sats.sats_cache_extend(self.cache, self.pages, seq, add, self.status)
        batch = sats.KVBatch(self.pages.table[seq.long()], ints(start), self.pages.len[seq.long()], start[-1],
                             max(lens), self.max_len)
        ids = ints([t for p in prompts for t in p])
        return self.forward(ids, batch, ints(start[1:]).long() - 1)

    def missing(self):
        """Pages that the last extension or fork lacked, and items it left out."""
        return tuple(self.status.tolist())


class DecodeLoop:
    """One token a step for the sequences 0 .. n - 1, the whole step in one graph."""

    def __init__(self, model, n, temperature=0.8, top_k=50, top_p=0.95, min_p=0.0):
        self.model, self.n = model, n
        f = lambda v: torch.full((n,), float(v), device="cuda")  # noqa: E731
        self.rules = dict(temperature=f(temperature), top_k=ints([top_k] * n), top_p=f(top_p), min_p=f(min_p))
        self.ids, self.u, self.one = ints([0] * n), f(0), ints([1] * n)
        self.start, self.rows = ints(list(range(n + 1))), torch.arange(n, device="cuda")
        self.batch = sats.KVBatch(model.pages.table[:n], self.start, model.pages.len[:n], n, 1, model.max_len)
        self.graph = None

    def _step(self):
        m = self.model
        sats.sats_cache_extend(m.cache, m.pages, None, self.one, m.status)
        logits = m.forward(self.ids, self.batch, self.rows)
        sats.sats_sample(logits, self.u, self.ids, **self.rules)

    def capture(self):
        m = self.model
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            sats.sats_reserve(self.n, m.d, m.d_ff, 1, m.embed.element_size(), stream=s)
            sats.sats_reserve_serving(self.n, m.pages.n_pages, self.n, m.vocab, m.dim, stream=s)
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph, stream=s):
                self._step()
        torch.cuda.current_stream().wait_stream(s)

    def step(self, u):
        """Decodes `ids` (in place): the next ids for the random numbers u [n]."""
        self.u.copy_(u)
        if self.graph is not None:
            self.graph.replay()
        else:
            self._step()
        return self.ids


def rms(x):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6)


def ints(v):
    return torch.tensor(v, device="cuda", dtype=torch.int32)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("prompts", 4), ("prompt", 512), ("samples", 2), ("tokens", 64)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    n = a.prompts * a.samples
    model = Decoder(layers=a.layers, max_seqs=n, max_len=-(-(a.prompt + a.tokens + 1) // 16) * 16)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    first = list(range(0, n, a.samples))
    prompts = torch.randint(0, model.vocab, (a.prompts, a.prompt), generator=g, device="cuda").tolist()
    model.prefill(first, prompts)  # (first calls)
    sats.sats_cache_free(model.cache, model.pages, ints(first))
    torch.cuda.synchronize()
    t = time.perf_counter()
    logits = model.prefill(first, prompts)
    torch.cuda.synchronize()
    print(f"prompts: {a.prompts} x {a.prompt} tokens in {1e3 * (time.perf_counter() - t):.2f} ms")
    # further samples share the prompts' full pages
    src = [s for s in first for _ in range(a.samples - 1)]
    dst = [s + i for s in first for i in range(1, a.samples)]
    if src:
        sats.sats_cache_fork(model.cache, model.pages, ints(src), ints(dst), model.status)
    shared = int((model.pages.refs > 1).sum())
    print(f"forked to {n} sequences: {int((model.pages.refs > 0).sum())} pages in use, {shared} shared")
    loop = DecodeLoop(model, n)
    sats.sats_sample(logits.repeat_interleave(a.samples, 0), torch.rand(n, generator=g, device="cuda"), loop.ids,
                     **loop.rules)
    loop.capture()
    out = [loop.ids.tolist()]
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(a.tokens):
        out.append(loop.step(torch.rand(n, generator=g, device="cuda")).clone())
    torch.cuda.synchronize()
    dt = time.perf_counter() - t
    print(f"decoded: {a.tokens} steps of {n} sequences, {1e3 * dt / a.tokens:.3f} ms a step, {n * a.tokens / dt:.0f} tok/s")
    assert model.missing() == (0, 0)
    print("first ids of sequence 0:", [int(o[0]) for o in out[:8]])


if __name__ == "__main__":
    main()
