"""Rotary positions, the paged cache, the state cache and the token scores in one run, as a server would call them: the example's, and one
captured into a graph."""
import math

import pytest
import torch

from kv_util import attention, close as close_attention
from paper_2501_12689_b200 import ICPagedKV, ICStates, ICTokenScores
from test_gpu_kv_example import _example
from test_gpu_kv_rotary import close as close_turned, turned
from test_gpu_states import close as close_state, draw, formula, ints, rates_of, starts_of
from test_gpu_token_scores import check as check_scores

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Watch:
    """Follows the states in 64 bits, along the forks.  The tolerance is that of one call: the state before a call is taken as it was, in 32 bits."""

    def __init__(self):
        self.pool, self.seen = None, dict(state=0, fork=0, scores=0, utility=0)

    def state(self, states, layer, q, k, v, rates, out, seqs, counts):
        now = states.pool.clone()
        before = torch.zeros_like(now) if self.pool is None else self.pool
        a = 0
        for s, c in zip(seqs, counts):
            part = slice(a, a + c)
            want = formula(q[part], k[part], v[part], rates, before[s, layer], 1.0 / math.sqrt(q.shape[-1]))
            close_state(out[part], now[s, layer], want, c, max(counts) > 1)
            a += c
        self.pool, self.seen["state"] = now, self.seen["state"] + 1

    def fork(self, parents, children):
        self.pool[children] = self.pool[parents]
        self.seen["fork"] += 1

    def scores(self, logits, tokens, got):
        want = check_scores(logits, 3, targets=tokens)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        self.seen["scores"] += 1

    def utility(self, ids, gains, store):
        held = dict(zip(*(x.tolist() for x in store.utility_read())))
        for i in set(ids.tolist()):
            assert held[i] == pytest.approx(float(gains[ids == i].double().sum()), rel=1e-5)      # (up to six additions in 32 bits)
        self.seen["utility"] += 1


def test_a_run_of_the_example():
    seen, watch = [], Watch()

    def check(kv, layer, q, out, seqs, counts):
        want, size = attention(kv, layer, q, seqs, counts)
        seen.append(close_attention(out, want, size))

    kv, found, x, used = _example().serve(check=check, watch=watch)
    assert len(seen) == 12 and watch.seen == dict(state=6, fork=2, scores=4, utility=1)
    assert torch.isfinite(x.float()).all()


def _caches(stream=None):
    kv = ICPagedKV(24, 1, 2, 16, 64, 4, 8, stream=stream)
    kv.set_rotary(48, base=10000.0)
    return kv, ICStates(1, 4, 64, 32, 4, stream=stream), ICTokenScores(1001, stream=stream)


def test_a_copied_example_moved_behind_an_instruction():
    """An example's copy goes behind 21 tokens of another sequence's positions, and its keys are as if they had been written there."""
    kv, states, _ = _caches()
    kv_, f = 2, [10000.0 ** (-2.0 * i / 48) for i in range(24)]
    k, v, q = draw(1, 70, kv_, 64), draw(2, 70, kv_, 64), draw(3, 70, 8, 64)
    kv.reserve(ints([0]), ints([70]))
    kv.write_rotated(0, q, k, v, ints([0]), starts_of([70]))
    kv.fork(ints([0]), ints([1]), copy=True)
    kv.shift(ints([1]), ints([21]))
    kv.reserve(ints([1]), ints([5]))
    fresh = [draw(4 + i, 5, h, 64) for i, h in enumerate((8, kv_, kv_))]
    at = torch.arange(91, 96, dtype=torch.int32, device=DEV)
    turned_q = kv.write_rotated(0, *fresh, ints([1]), starts_of([5]), positions=at)
    out = kv.extend(0, turned_q, ints([1]), starts_of([5]))
    kv.sync()
    close_turned(turned_q, *turned(fresh[0], at, f, 48, False))
    want, size = attention(kv, 0, turned_q, [1], [5])
    close_attention(out, want, size)
    # turned twice: the first rounding's errors, up to half a step of each of a pair, turn into up to sqrt(2) half steps of the pair's size
    held = torch.cat([kv.pool[p, 0, 0] for p in kv.tables[1, :5].long()], dim=1)[:, :70].transpose(0, 1).double()
    exact, length = turned(k, torch.arange(21, 91, device=DEV), f, 48, False)
    assert ((held - exact).abs() <= 2.0 ** -8 * (1.5 * length + exact.abs()) + 2.0 ** -18 * length).all()


def test_a_step_captured_and_replayed():
    """Positions, cache, states and scores of a decode step in one graph: replays do what eager calls do."""
    stream = torch.cuda.Stream()

    def step(c, x, seqs, tokens):
        kv, states, scores = c
        kv.reserve(seqs, torch.ones_like(seqs))
        q, k, v = x[:, :12].split([8, 2, 2], dim=1)
        o = kv.decode(0, kv.write_rotated(0, q, k, v, seqs), seqs)
        r = states.decode(0, x[:, 12:16], x[:, 16:20], x[:, 20:24, :32], rates, seqs)
        return o, r, scores.score(x.flatten(1)[:, :1001], tokens, n_top=7)

    rates = rates_of(4)
    seqs, tokens = ints([2, 0, 3]), ints([5, -1, 1000])
    xs = [draw(10 + i, 3, 24, 64) for i in range(4)]
    eager = _caches()
    wants = [step(eager, x, seqs, tokens) for x in xs]
    torch.cuda.synchronize()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        held = _caches(stream)
        x = xs[0].clone()
        first = step(held, x, seqs, tokens)                    # one eager step, then replays
        ones = torch.ones_like(seqs)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        held[0].reserve(seqs, ones)
        q, k, v = x[:, :12].split([8, 2, 2], dim=1)
        o = held[0].decode(0, held[0].write_rotated(0, q, k, v, seqs), seqs)
        r = held[1].decode(0, x[:, 12:16], x[:, 16:20], x[:, 20:24, :32], rates, seqs)
        s = held[2].score(x.flatten(1)[:, :1001], tokens, n_top=7)
    gots = [first]
    for i in range(1, 4):
        with torch.cuda.stream(stream):
            x.copy_(xs[i])
            graph.replay()
            gots.append((o.clone(), r.clone(), type(s)(*(y.clone() for y in s))))
    torch.cuda.synchronize()
    for c in held:
        c.sync()
    for got, want in zip(gots, wants):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert all(torch.equal(a, b) for a, b in zip(got[2], want[2]))
    assert torch.equal(held[1].pool, eager[1].pool)
