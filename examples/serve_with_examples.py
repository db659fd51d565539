"""Retrieval and serving together: the cached example that is most similar to a request goes in front of it, and its keys and
values are not computed again but shared.

    python examples/serve_with_examples.py

The "model" is a stand-in (random projections per layer, no weights are to be had offline): what is shown is the order of the
calls around it.  An example is run through the model once, into a sequence of the paged cache that stays; a request finds its
example with ICCache, forks from that sequence (full pages shared, the tail copied), appends and attends its own tokens (a second
example would be among them: its keys and values depend on what stands before it), and
then decodes, here with a few samples per request that fork from the request in turn."""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2501_12689_b200 import ICCache, ICPagedKV  # noqa: E402


class Model:
    """Stand-in layers: queries, keys and values of a token are projections of its hidden state."""

    def __init__(self, layers=2, heads=8, kv_heads=2, dim=64, device="cuda:0", dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.layers, self.heads, self.kv_heads, self.dim, self.hidden = layers, heads, kv_heads, dim, heads * dim
        wide = (heads + 2 * kv_heads) * dim
        self.proj = [(torch.randn(self.hidden, wide, device=device, generator=g) / self.hidden ** 0.5).to(dtype) for _ in range(layers)]

    def run(self, x, kv: ICPagedKV, seqs, starts=None, trace=None):
        """x [tokens, hidden]: the newest tokens of `seqs`, already reserved.  One extend (or, without starts, decode) per layer."""
        for layer, w in enumerate(self.proj):
            qkv = (x @ w).view(-1, self.heads + 2 * self.kv_heads, self.dim)
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)      # strided views: taken as they are
            kv.write(layer, k, v, seqs, starts)
            o = kv.decode(layer, q, seqs) if starts is None else kv.extend(layer, q, seqs, starts)
            if trace is not None:
                trace.append((layer, q, o))
            x = torch.nn.functional.normalize(x.float() + o.reshape(x.shape).float(), dim=-1).mul(self.hidden ** 0.5).to(x.dtype)
        return x


def serve(n_examples=40, n_requests=6, samples=2, steps=4, seed=0, check=None):
    """Returns (kv, example of each request, hidden state of each sample after the last step).  check(kv, layer, q, out, seqs, counts)
    is called after every attention."""
    dev = "cuda:0"
    g = torch.Generator(device=dev).manual_seed(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    model = Model(device=dev)
    dtype = torch.bfloat16

    def look(trace, seqs, counts):
        if check is not None:
            for layer, q, o in trace:
                check(kv, layer, q, o, seqs, counts)

    # the store: an embedding per example for retrieval, a sequence per example for its keys and values
    emb = torch.nn.functional.normalize(torch.randn(n_examples, 64, device=dev, generator=g), dim=-1).to(dtype)
    store = ICCache(64, n_examples)
    store.insert(emb, torch.arange(n_examples, device=dev))
    rows = n_examples + n_requests * (1 + samples)            # examples first, then requests, then samples
    kv = ICPagedKV(n_pages=1024, n_layers=model.layers, n_kv_heads=model.kv_heads, page_size=16, head_dim=model.dim, max_seqs=rows,
                   max_pages=32)
    lengths = torch.randint(20, 200, (n_examples,), generator=torch.Generator().manual_seed(seed)).tolist()
    which = list(range(n_examples))
    starts = ints([0] + torch.tensor(lengths).cumsum(0).tolist())
    kv.reserve(ints(which), ints(lengths))
    trace = []
    model.run(torch.randn(sum(lengths), model.hidden, device=dev, generator=g).to(dtype), kv, ints(which), starts, trace)
    look(trace, which, lengths)

    # requests: similar to some example each
    near = torch.randint(0, n_examples, (n_requests,), device=dev, generator=g)
    asked = torch.nn.functional.normalize(emb[near].float() + 0.05 * torch.randn(n_requests, 64, device=dev, generator=g), dim=-1).to(dtype)
    found, _ = store.query(asked, 1)                          # ids are the examples' sequence numbers, and stay on the device
    requests = [n_examples + i for i in range(n_requests)]
    kv.fork(found[:, 0].to(torch.int32), ints(requests))
    fresh = [5 + 7 * i for i in range(n_requests)]
    kv.reserve(ints(requests), ints(fresh))
    trace = []
    x = model.run(torch.randn(sum(fresh), model.hidden, device=dev, generator=g).to(dtype), kv, ints(requests),
                  ints([0] + torch.tensor(fresh).cumsum(0).tolist()), trace)
    look(trace, requests, fresh)

    # samples: each request's are forks of it; the last token's state is where they begin
    drawn = [n_examples + n_requests + i for i in range(n_requests * samples)]
    kv.fork(ints([r for r in requests for _ in range(samples)]), ints(drawn))
    last = torch.tensor(fresh, device=dev).cumsum(0) - 1
    x = x[last].repeat_interleave(samples, 0)
    for _ in range(steps):
        x = (x.float() + 0.5 * torch.randn(x.shape, device=dev, generator=g)).to(dtype)      # the next token, sampled
        kv.reserve(ints(drawn), ints([1] * len(drawn)))
        trace = []
        x = model.run(x, kv, ints(drawn), None, trace)
        look(trace, drawn, [1] * len(drawn))
    kv.sync()
    store.sync()
    assert torch.equal(found[:, 0], near)
    return kv, found[:, 0], x, requests + drawn


def main():
    kv, found, x, used = serve()
    free = int((kv.refs == 0).sum())
    shared = int((kv.refs > 1).sum())
    print(f"requests were answered behind examples {found.tolist()}; {shared} pages are shared, {free} of {kv.n_pages} free")
    kv.free(torch.tensor(used, dtype=torch.int32, device=kv.device))
    kv.compact()
    kv.sync()
    print(f"after the requests: {int((kv.refs == 0).sum())} pages free, the examples in pages 0 .. {int((kv.refs > 0).sum()) - 1}")


if __name__ == "__main__":
    main()
