"""A small serving loop: decoder layers of W4A4 linears over a paged key-value cache.

Prompts of several lengths are taken in (append with rotary positions, then attention
of the packed tokens), tokens are decoded one a sequence (the step captured into a HIP
graph and replayed), a sequence forks into two that go on by themselves, one ends, and
the cache is compacted.  The output head is a linear in 8 bits, and the next tokens are
sampled from its logits (temperature 0: the largest).  Weights are random: it shows how
the calls go together, and times them.

    python examples/serve_layers.py [--layers 4] [--batch 8] [--prompt 500] [--steps 32]
                                    [--cache fp16|int4] [--window 0] [--sinks 0]
                                    [--temperature 0] [--top-k 0] [--top-p 1] [--min-p 0]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2606_08761_amd as apex4  # noqa: E402


def norm(x):
    return (x.float() * torch.rsqrt(x.float().pow(2).mean(dim=-1, keepdim=True) + 1e-6)).to(torch.float16)


class Layer:
    """qkv and output projections around the attention, gate + up and down ones
    around the activation."""

    def __init__(self, hidden, heads, kv_heads, head_dim, inner, generator):
        def linear(n, k):
            w = torch.empty((n, k), dtype=torch.float16, device="cuda").normal_(0.0, k ** -0.5, generator=generator)
            return apex4.W4A4Linear(w, G=128)
        self.heads, self.kv_heads, self.head_dim, self.inner = heads, kv_heads, head_dim, inner
        self.qkv = linear((heads + 2 * kv_heads) * head_dim, hidden)
        self.out = linear(hidden, heads * head_dim)
        self.gate_up, self.down = linear(2 * inner, hidden), linear(hidden, inner)

    def split(self, x):
        """q, k and v as views of the fused projection's rows."""
        qkv = self.qkv(norm(x)).view(x.shape[0], -1, self.head_dim)
        return torch.split(qkv, [self.heads, self.kv_heads, self.kv_heads], dim=1)

    def finish(self, x, attention):
        x = x + self.out(attention.view(x.shape[0], -1))
        gate, up = self.gate_up(norm(x)).split(self.inner, dim=1)
        return x + self.down((torch.nn.functional.silu(gate.float()) * up.float()).to(torch.float16))


class Model:
    def __init__(self, layers=4, hidden=1024, heads=8, kv_heads=2, head_dim=128, inner=2816, vocab=4096, slots=16,
                 pages=1024, page=16, max_len=2048, cache="fp16", window=0, sinks=0, seed=0, temperature=0.0, top_k=0, top_p=1.0,
                 min_p=0.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.layers = [Layer(hidden, heads, kv_heads, head_dim, inner, g) for _ in range(layers)]
        self.embed = torch.empty((vocab, hidden), dtype=torch.float16, device="cuda").normal_(0.0, 1.0, generator=g)
        self.cache = apex4.PagedKVCache(layers, pages, slots, kv_heads, head_dim, page, max_len, cache)
        self.mask = {"window": window, "sinks": sinks}
        self.freq, _ = apex4.apex4_rope_freq(head_dim)
        self.lm_head = apex4.W8A8Linear(torch.empty((vocab, hidden), dtype=torch.float16, device="cuda").normal_(0.0, hidden ** -0.5, generator=g))
        self.settings = {"temperature": temperature, "top_k": top_k, "top_p": top_p, "min_p": min_p}
        self.generator = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.u = torch.zeros(slots, device="cuda")  # a random number for each sequence of a step

    def draw(self):
        self.u.uniform_(generator=self.generator)

    def head(self, x):
        tokens, _ = apex4.apex4_sample(self.lm_head(norm(x)), self.u[:x.shape[0]], **self.settings)
        return tokens.long()

    def take_in(self, prompts, seqs):
        """Prompts (lists of token numbers) into the empty slots seqs; the next tokens."""
        n = [len(p) for p in prompts]
        if not self.cache.reserved(self.cache.reserve(seqs, n)):
            raise RuntimeError("no pages left for the prompts")
        start = torch.tensor([0, *n], device="cuda").cumsum(0).to(torch.int32)
        batch = self.cache.batch(seqs)
        x = self.embed[torch.tensor([t for p in prompts for t in p], device="cuda")]
        for i, layer in enumerate(self.layers):
            q, k, v = layer.split(x)
            q = self.cache.append_rope(i, q, k, v, batch, self.freq, start)
            x = layer.finish(x, self.cache.prefill(i, q, batch, start, max(n), **self.mask))
        self.draw()
        return self.head(x[start[1:].long() - 1])

    def step(self, tokens, batch):
        """One token a sequence, whose places are reserved and counted in batch."""
        x = self.embed[tokens]
        for i, layer in enumerate(self.layers):
            q, k, v = layer.split(x)
            q = self.cache.append_rope(i, q, k, v, batch, self.freq)
            x = layer.finish(x, self.cache.decode(i, q, batch, **self.mask))
        return self.head(x)

    def decode(self, tokens, seqs, lens, steps):
        """steps tokens for each of the slots seqs, lens tokens long so far, from one
        captured step; all tokens, [steps, sequences]."""
        if not self.cache.reserved(self.cache.reserve(seqs, [n + steps for n in lens])):
            raise RuntimeError("no pages left for the steps")
        table, _ = self.cache.batch(seqs)
        kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda") + 1
        out = torch.empty((steps, len(seqs)), dtype=torch.int64, device="cuda")
        # steps outside the capture: the kernels are loaded, the linears' buffers made
        # (on the sequences' own next places, which the captured steps write again)
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        current = tokens.clone()
        with torch.cuda.stream(stream):
            self.step(current, (table, kv_len))
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            following = self.step(current, (table, kv_len))
        for i in range(steps):
            self.draw()
            graph.replay()
            out[i] = following
            current.copy_(following)
            kv_len += 1
        return out


def serve(layers=4, batch=8, prompt=500, steps=32, cache="fp16", window=0, sinks=0, say=print, **sizes):
    """Returns the tokens of every part, for the tests."""
    model = Model(layers=layers, cache=cache, window=window, sinks=sinks, slots=batch + 1,
                  max_len=prompt + 2 * steps + 16, pages=(batch + 1) * (-(-(prompt + 2 * steps + 16) // 16)), **sizes)
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, model.embed.shape[0], (max(1, prompt - 37 * i),), generator=g).tolist() for i in range(batch)]
    seqs, lens = list(range(batch)), [len(p) for p in prompts]

    model.take_in([[0] * 20], [batch])  # the kernels are loaded
    model.cache.free([batch])
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    first = model.take_in(prompts, seqs)
    torch.cuda.synchronize()
    t1 = time.perf_counter()
    tokens = model.decode(first, seqs, lens, steps)
    torch.cuda.synchronize()
    t2 = time.perf_counter()
    lens = [n + steps for n in lens]
    say(f"{sum(len(p) for p in prompts)} prompt tokens in {1e3 * (t1 - t0):.1f} ms, {steps} steps of {batch} in {1e3 * (t2 - t1):.1f} ms")

    # slot 0 goes on in the spare slot too; the last sequence ends; what is left moves together
    spare = batch
    if not model.cache.reserved(model.cache.fork([0], [spare])):
        raise RuntimeError("no page left for the fork")
    if batch > 1:
        model.cache.free([batch - 1])
        seqs, lens = seqs[:-1], lens[:-1]
    live = int(model.cache.compact().item())
    say(f"{live} pages in use")
    more = model.decode(torch.cat((tokens[-1][:len(seqs)], tokens[-1][:1])), [*seqs, spare], [*lens, lens[0]], steps)
    if not model.settings["temperature"] > 0:
        assert torch.equal(more[:, 0], more[:, -1]), "a fork without a change goes on as its parent"
    return first, tokens, more


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("layers", 4), ("batch", 8), ("prompt", 500), ("steps", 32), ("window", 0), ("sinks", 0), ("top-k", 0)):
        ap.add_argument(f"--{name}", type=int, default=value)
    for name, value in (("temperature", 0.0), ("top-p", 1.0), ("min-p", 0.0)):
        ap.add_argument(f"--{name}", type=float, default=value)
    ap.add_argument("--cache", choices=sorted(apex4.KV_CACHES), default="fp16")
    serve(**vars(ap.parse_args()))


if __name__ == "__main__":
    main()
