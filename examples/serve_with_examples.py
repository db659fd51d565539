"""Retrieval and serving together: the cached example that is most similar to a request goes in front of it, and its keys and
values are not computed again but shared.

    python examples/serve_with_examples.py

The "model" is a stand-in (random projections per layer, no weights are to be had offline): what is shown is the order of the
calls around it.  It has attention layers with rotary positions, whose keys and values are in the paged cache, and between them recurrent ones, whose
states are in the state cache.  An example is run through the model once, into a sequence of both caches that stays; a request finds its
example with ICCache, forks from that sequence (full pages shared, the tail and the states copied), appends and attends its own tokens (a second
example would be among them: its keys and values depend on what stands before it), and
then decodes, here with a few samples per request that fork from the request in turn.  What the model thought of the answers, from the scores of
their tokens, is added to the utility of the examples that stood in front of them."""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2501_12689_b200 import ICCache, ICPagedKV, ICStates, ICTokenScores  # noqa: E402


class Model:
    """Stand-in layers: queries, keys and values of a token are projections of its hidden state.  A recurrent layer comes after every attention
    layer but the last."""

    def __init__(self, layers=2, heads=8, kv_heads=2, dim=64, vocab=1000, device="cuda:0", dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device=device).manual_seed(seed)
        self.layers, self.heads, self.kv_heads, self.dim, self.hidden, self.vocab = layers, heads, kv_heads, dim, heads * dim, vocab
        draw = lambda wide: (torch.randn(self.hidden, wide, device=device, generator=g) / self.hidden ** 0.5).to(dtype)  # noqa: E731
        self.proj = [draw((heads + 2 * kv_heads) * dim) for _ in range(layers)]
        self.recurrent = [draw(3 * heads * dim) for _ in range(layers - 1)]
        self.head = draw(vocab)
        self.embedding = torch.randn(vocab, self.hidden, device=device, generator=g).to(dtype)
        self.rates = torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], device=device)      # falls of the recurrent heads

    def _join(self, x, o):
        return torch.nn.functional.normalize(x.float() + o.reshape(x.shape).float(), dim=-1).mul(self.hidden ** 0.5).to(x.dtype)

    def run(self, x, kv: ICPagedKV, states: ICStates, seqs, starts=None, trace=None):
        """x [tokens, hidden]: the newest tokens of `seqs`, already reserved.  One extend (or, without starts, decode) per layer."""
        for layer, w in enumerate(self.proj):
            qkv = (x @ w).view(-1, self.heads + 2 * self.kv_heads, self.dim)
            q, k, v = qkv.split([self.heads, self.kv_heads, self.kv_heads], dim=1)      # strided views: taken as they are
            q = kv.write_rotated(layer, q, k, v, seqs, starts)
            o = kv.decode(layer, q, seqs) if starts is None else kv.extend(layer, q, seqs, starts)
            if trace is not None:
                trace.append(("attention", layer, q, o))
            x = self._join(x, o)
            if layer < len(self.recurrent):
                q, k, v = (x @ self.recurrent[layer]).view(-1, 3 * self.heads, self.dim).split(self.heads, dim=1)
                o = states.decode(layer, q, k, v, self.rates, seqs) if starts is None else states.extend(layer, q, k, v, self.rates, seqs, starts)
                if trace is not None:
                    trace.append(("state", layer, q, k, v, o))
                x = self._join(x, o)
        return x


def serve(n_examples=40, n_requests=6, samples=2, steps=4, seed=0, check=None, watch=None):
    """Returns (kv, example of each request, hidden state of each sample after the last step, sequences of requests and samples).
    check(kv, layer, q, out, seqs, counts) is called after every attention; watch.state(states, layer, q, k, v, rates, out, seqs, counts) after every
    recurrent layer, watch.fork(parents, children) after every fork, watch.scores(logits, tokens, scores) after every score, watch.utility(ids, gains,
    store) at the end."""
    dev = "cuda:0"
    g = torch.Generator(device=dev).manual_seed(seed)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    model = Model(device=dev)
    dtype = torch.bfloat16

    def look(trace, seqs, counts):
        for kind, layer, *rest in trace:
            if kind == "attention" and check is not None:
                check(kv, layer, *rest, seqs, counts)
            if kind == "state" and watch is not None:
                watch.state(states, layer, *rest[:3], model.rates, rest[3], seqs, counts)

    def fork(parents, children):
        kv.fork(parents, children)
        states.fork(parents, children)
        if watch is not None:
            watch.fork(parents.tolist(), children.tolist())

    # the store: an embedding per example for retrieval, a sequence per example for its keys and values
    emb = torch.nn.functional.normalize(torch.randn(n_examples, 64, device=dev, generator=g), dim=-1).to(dtype)
    store = ICCache(64, n_examples)
    store.insert(emb, torch.arange(n_examples, device=dev))
    rows = n_examples + n_requests * (1 + samples)            # examples first, then requests, then samples
    kv = ICPagedKV(n_pages=1024, n_layers=model.layers, n_kv_heads=model.kv_heads, page_size=16, head_dim=model.dim, max_seqs=rows,
                   max_pages=32)
    kv.set_rotary(base=500000.0)
    states = ICStates(model.layers - 1, model.heads, model.dim, model.dim, rows)
    scores = ICTokenScores(model.vocab, dtype=dtype)
    lengths = torch.randint(20, 200, (n_examples,), generator=torch.Generator().manual_seed(seed)).tolist()
    which = list(range(n_examples))
    starts = ints([0] + torch.tensor(lengths).cumsum(0).tolist())
    kv.reserve(ints(which), ints(lengths))
    trace = []
    model.run(torch.randn(sum(lengths), model.hidden, device=dev, generator=g).to(dtype), kv, states, ints(which), starts, trace)
    look(trace, which, lengths)

    # requests: similar to some example each
    near = torch.randint(0, n_examples, (n_requests,), device=dev, generator=g)
    asked = torch.nn.functional.normalize(emb[near].float() + 0.05 * torch.randn(n_requests, 64, device=dev, generator=g), dim=-1).to(dtype)
    found, _ = store.query(asked, 1)                          # ids are the examples' sequence numbers, and stay on the device
    requests = [n_examples + i for i in range(n_requests)]
    fork(found[:, 0].to(torch.int32), ints(requests))
    fresh = [5 + 7 * i for i in range(n_requests)]
    kv.reserve(ints(requests), ints(fresh))
    trace = []
    x = model.run(torch.randn(sum(fresh), model.hidden, device=dev, generator=g).to(dtype), kv, states, ints(requests),
                  ints([0] + torch.tensor(fresh).cumsum(0).tolist()), trace)
    look(trace, requests, fresh)

    # samples: each request's are forks of it; the last token's state is where they begin
    drawn = [n_examples + n_requests + i for i in range(n_requests * samples)]
    fork(ints([r for r in requests for _ in range(samples)]), ints(drawn))
    last = torch.tensor(fresh, device=dev).cumsum(0) - 1
    x = x[last].repeat_interleave(samples, 0)
    liked = torch.zeros(len(drawn), device=dev)
    for _ in range(steps):
        logits = x @ model.head
        tokens = torch.multinomial(torch.softmax(logits.float(), -1), 1, generator=g)[:, 0].to(torch.int32)
        got = scores.score(logits, tokens, n_top=3)
        liked += got.log_probs
        if watch is not None:
            watch.scores(logits, tokens, got)
        kv.reserve(ints(drawn), ints([1] * len(drawn)))
        trace = []
        x = model.run(model.embedding[tokens.long()], kv, states, ints(drawn), None, trace)
        look(trace, drawn, [1] * len(drawn))
    # an example's gain: how likely the answers behind it were to the model, per token
    gains = (liked / steps).exp().view(n_requests, samples).mean(-1)
    store.utility_add(found[:, 0].cpu(), gains.cpu())
    if watch is not None:
        watch.utility(found[:, 0].cpu(), gains.cpu(), store)
    states.sync()
    scores.sync()
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
