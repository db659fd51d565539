"""The state cache on the GPU: linear attention with a decay against its formula in 64 bits, forks, clears and refusals."""
import math
import random

import pytest
import torch

from kv_util import UNIT
from paper_2501_12689_b200 import IC_ERR_INVALID, ICCacheError, ICStates

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16 = torch.bfloat16, torch.float16
BLOCK = 64


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def starts_of(counts):
    s = [0]
    for c in counts:
        s.append(s[-1] + c)
    return ints(s)


def draw(seed, *shape, dtype=BF16, size=1.0):
    return (size * torch.randn(*shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed))).to(dtype)


def rates_of(heads, strong=1.0):
    return torch.tensor([strong * 2.0 ** (-8.0 * (i + 1) / heads) for i in range(heads)], device=DEV)


def formula(q, k, v, rates, state, scale):
    """One sequence in 64 bits, blocks of tokens at a time: (out, state, sizes of what may be rounded to 16 bits, sizes of the fp32 sums of
    out and of the state).  q, k [t, h, dk], v [t, h, dv], state [h, dk, dv]."""
    q, k, v = (x.double().transpose(0, 1) for x in (q, k, v))
    r, s = rates.double()[:, None, None], state.double().clone()
    h, t, _ = q.shape
    out = torch.zeros(h, t, v.shape[-1], dtype=torch.float64, device=DEV)
    rounded, summed, size = torch.zeros_like(out), torch.zeros_like(out), s.abs()
    fall = lambda steps: torch.exp(-torch.where(steps == 0, 0.0, r * steps))  # noqa: E731  (an infinite rate times no step is no fall)
    for a in range(0, t, BLOCK):
        x, y, z = q[:, a:a + BLOCK], k[:, a:a + BLOCK], v[:, a:a + BLOCK]
        n = x.shape[1]
        at = torch.arange(n, device=DEV, dtype=torch.float64)
        steps = (at[:, None] - at)[None]
        d = torch.where(steps < 0, 0.0, fall(steps.clamp(min=0)))
        to, left = fall((at + 1)[None, :, None]), fall((n - 1 - at)[None, :, None])
        p = (x @ y.transpose(-1, -2)) * d
        out[:, a:a + n] = p @ z + to * (x @ s)
        rounded[:, a:a + n] = p.abs() @ z.abs() + to * (x.abs() @ s.abs())
        summed[:, a:a + n] = ((x.abs() @ y.abs().transpose(-1, -2)) * d) @ z.abs() + to * (x.abs() @ size)
        whole = fall(torch.full((1, 1, 1), float(n), dtype=torch.float64, device=DEV))
        s = whole * s + (y * left).transpose(-1, -2) @ z
        size = whole * size + (y.abs() * left).transpose(-1, -2) @ z.abs()
    return tuple((f * x).transpose(0, 1) for f, x in ((scale, out), (abs(scale), rounded), (abs(scale), summed))) + (s, size)


def close(got, state, want, t, several):
    """The result is rounded once; in a call of several tokens the scores, or the states' copy for the queries, were before (once each:
    `several`).  fp32 sums: an element of the state is the sum of t products, each step with up to four roundings; the result sums key_dim of these,
    over lanes and warps or in a tensor core: half a unit an addition."""
    out, rounded, summed, s, size = want
    u = UNIT[got.dtype]
    steps = (4 * t + 64) * 2.0 ** -24
    bound = u * out.abs() + (1.01 * u * rounded if several else 0.0) + 2 * steps * summed + 2.0 ** -25
    off = (got.double() - out).abs()
    worst = (off / bound).max().item()
    assert worst <= 1.0, f"out: {worst:.2f} times the bound"
    off = (state.double() - s).abs()
    worst = (off / (steps * size + 1e-30)).max().item()
    assert worst <= 1.0, f"state: {worst:.2f} times the bound"
    # roundings are as often up as down: far from adding up
    for h in range(s.shape[0]):
        assert (state[h].double() - s[h]).norm() <= 2.0 ** -19 * s[h].norm() + 1e-30
        if t * out.shape[-1] >= 256:
            assert (got[:, h].double() - out[:, h]).norm() <= u * out[:, h].norm() + 2.0 ** -20 * summed[:, h].norm() + 0.6 * u * several * rounded[:, h].norm() / 8


def run(counts, *, heads=2, dk=64, dv=64, dtype=BF16, layers=2, layer=1, max_seqs=None, strong=1.0, single=False, strided=False, scale=None, seed=0,
        rates=None, states=None, order=None, shift=0.0):
    n, t = len(counts), sum(counts)
    s = states or ICStates(layers, heads, dk, dv, max_seqs or n, dtype=dtype, pool=draw(seed + 9, max_seqs or n, layers, heads, dk, dv, dtype=torch.float32))
    rates = rates_of(heads, strong) if rates is None else rates
    if strided:
        q, k, v = draw(seed, t, heads, 2 * dk + dv, dtype=dtype).split([dk, dk, dv], -1)
        out = torch.zeros(heads, t, dv + 8, dtype=dtype, device=DEV).transpose(0, 1)[..., :dv]
    else:
        q, k, v = draw(seed, t, heads, dk, dtype=dtype), draw(seed + 1, t, heads, dk, dtype=dtype) + shift, draw(seed + 2, t, heads, dv, dtype=dtype) + shift
        k, v = k.to(dtype), v.to(dtype)
        out = None
    seqs = list(range(n)) if order is None else order
    before = s.pool.clone()
    if single:
        got = s.decode(layer, q, k, v, rates, ints(seqs), scale=scale, out=out)
    else:
        got = s.extend(layer, q, k, v, rates, ints(seqs), starts_of(counts), scale=scale, out=out)
    s.sync()
    a = 0
    for c, x in zip(counts, seqs):
        if c:
            part = slice(a, a + c)
            want = formula(q[part], k[part], v[part], rates, before[x, layer], 1.0 / math.sqrt(dk) if scale is None else scale)
            close(got[part], s.pool[x, layer], want, c, max(counts) > 1)
        else:
            assert torch.equal(s.pool[x], before[x])
        a += c
    rest = [x for x in range(s.max_seqs) if x not in seqs]
    assert torch.equal(s.pool[rest], before[rest])
    others = [x for x in range(s.n_layers) if x != layer]
    assert torch.equal(s.pool[:, others], before[:, others])
    return s, got


DIMS = [(64, 64), (128, 128), (8, 8), (16, 32), (80, 72), (96, 256), (128, 256), (24, 136), (128, 8), (8, 248), (72, 128), (40, 200)]
LONG = [1, 0, 2, 63, 64, 65, 127, 128, 129, 255, 257, 500]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dk,dv", DIMS)
def test_single_tokens(dk, dv, dtype):
    run([1] * 5, heads=3, dk=dk, dv=dv, dtype=dtype, single=True, max_seqs=7, order=[6, 0, 3, 2, 5])
    run([1] * 90, heads=8, dk=dk, dv=dv, dtype=dtype, single=True, seed=20)         # wide slices


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dk,dv", DIMS)
def test_few_tokens(dk, dv, dtype):
    run([3, 0, 1, 7, 16, 2], heads=3, dk=dk, dv=dv, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("dk,dv", DIMS)
def test_prompts(dk, dv, dtype):
    run(LONG, heads=3, dk=dk, dv=dv, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("counts,heads", [([3000], 1), ([2500, 1], 2), ([5001], 5), ([700] * 40, 4), ([64 * 30, 64 * 30 + 1, 64 * 31 - 1], 3)])
def test_long_prompts(counts, heads, dtype):
    """More chunks than one CTA takes: the work is split over the length."""
    run(counts, heads=heads, dk=64, dv=128, dtype=dtype, layers=1, layer=0)
    run(counts, heads=heads, dk=128, dv=128, dtype=dtype, layers=1, layer=0, seed=5, strong=0.01)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("strong", [0.0, 1e-3, 8.0, 100.0, 1e30, math.inf])
@pytest.mark.parametrize("counts,single", [([1] * 3, True), ([5, 2, 9], False), ([200, 70, 1], False)])
def test_decays(strong, counts, single, dtype):
    run(counts, heads=4, dk=64, dv=64, dtype=dtype, single=single, rates=torch.full((4,), strong, device=DEV))


@pytest.mark.parametrize("counts", [[1, 4], [100, 300]])
@pytest.mark.parametrize("scale", [0.0, -1.0, 3.0])
def test_scales_and_strides(scale, counts):
    run(counts, heads=3, dk=64, dv=72, scale=scale, strided=True)


@pytest.mark.parametrize("size", [1e-4, 1e-2, 30.0])
@pytest.mark.parametrize("counts", [[3], [300]])
def test_small_and_large_values_in_fp16(size, counts):
    """Scores of up to 1e6 and values far below one: neither leaves fp16's range."""
    t, heads, d = sum(counts), 2, 64
    s = ICStates(1, heads, d, d, 1, dtype=F16)
    q, k, v = (draw(i, t, heads, d, dtype=F16, size=size) for i in range(3))
    rates = rates_of(heads)
    got = s.extend(0, q, k, v, rates, ints([0]), starts_of(counts), scale=1.0 / size)
    s.sync()
    out, rounded, summed, st, sz = formula(q, k, v, rates, torch.zeros(heads, d, d, device=DEV), 1.0 / size)
    u, steps = 2.0 ** -11, (4 * t + 64) * 2.0 ** -24
    bound = u * out.abs() + 1.01 * u * rounded + 2 * steps * summed + 2.0 ** -25
    beyond = (out.abs() + bound >= 65504) & (got.double() == out.sign() * math.inf)       # the result itself has no place in fp16
    assert (beyond | ((got.double() - out).abs() <= bound)).all()
    assert (s.pool[0, 0].double() - st).norm() <= 2.0 ** -19 * st.norm()


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_values_with_a_mean(dtype):
    """Sums that grow with the length: nothing averages out."""
    run([600, 77], heads=2, dk=64, dv=64, dtype=dtype, shift=1.0, rates=torch.tensor([0.0, 0.01], device=DEV))


def test_shared_heads_by_a_stride_of_zero():
    t, heads = 130, 4
    s = ICStates(1, heads, 64, 64, 1)
    q, k, v = draw(1, t, heads, 64), draw(2, t, 1, 64).expand(t, heads, 64), draw(3, t, heads, 64)
    got = s.extend(0, q, k, v, rates_of(heads), ints([0]), starts_of([t]))
    s.sync()
    close(got, s.pool[0, 0], formula(q, k, v, rates_of(heads), torch.zeros(heads, 64, 64, device=DEV), 0.125), t, True)


@pytest.mark.parametrize("n", [256, 257, 1000])
@pytest.mark.parametrize("kind", ["single", "few", "prompts"])
def test_many_sequences(n, kind):
    rng = random.Random(n)
    order = list(range(n))
    rng.shuffle(order)
    counts = [1] * n if kind == "single" else [rng.choice([0, 1, 3]) for _ in range(n)] if kind == "few" else [rng.choice([0, 1, 30, 70]) for _ in range(n)]
    run(counts, heads=1, dk=16, dv=16, layers=1, layer=0, single=kind == "single", order=order, max_seqs=n + 3)


def test_pieces_and_wholes_agree():
    """A prompt in one call, in two, and token by token: the same sequence of states."""
    t, heads, rates = 300, 2, rates_of(2)
    q, k, v = draw(1, t, heads, 64), draw(2, t, heads, 64), draw(3, t, heads, 64)
    s = ICStates(1, heads, 64, 64, 3)
    whole = s.extend(0, q, k, v, rates, ints([0]), starts_of([t]))
    a = s.extend(0, q[:133], k[:133], v[:133], rates, ints([1]), starts_of([133]))
    b = s.extend(0, q[133:], k[133:], v[133:], rates, ints([1]), starts_of([t - 133]))
    c = torch.cat([s.decode(0, q[i:i + 1], k[i:i + 1], v[i:i + 1], rates, ints([2])) for i in range(t)])
    s.sync()
    want = formula(q, k, v, rates, torch.zeros(heads, 64, 64, device=DEV), 0.125)
    for got, x in ((whole, 0), (torch.cat([a, b]), 1), (c, 2)):
        close(got, s.pool[x, 0], want, t, x < 2)


@pytest.mark.parametrize("counts", [[1] * 3, [4, 1, 2], [90, 300, 1]])
def test_repeatable_on_other_streams_and_in_graphs(counts):
    t, heads = sum(counts), 3
    start = draw(9, 3, 1, heads, 64, 64, dtype=torch.float32)
    q, k, v, rates = draw(1, t, heads, 64), draw(2, t, heads, 64), draw(3, t, heads, 64), rates_of(heads)
    s = ICStates(1, heads, 64, 64, 3, pool=start.clone())
    seqs, starts = ints([2, 0, 1]), starts_of(counts)
    a = s.extend(0, q, k, v, rates, seqs, starts)
    s.sync()
    pool = s.pool.clone()
    s.pool.copy_(start)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b = s.extend(0, q * 1.0, k, v, rates, seqs, starts)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(s.pool, pool)
    s.set_stream(side)
    out = torch.empty_like(a)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        s.extend(0, q, k, v, rates, seqs, starts, out=out)
    for _ in range(2):
        s.pool.copy_(start)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, a) and torch.equal(s.pool, pool)


@pytest.mark.parametrize("n", [1, 5, 300])
def test_fork_and_clear(n):
    rng = random.Random(n)
    rows = 2 * n + 2
    s = ICStates(2, 3, 24, 40, rows, pool=draw(4, rows, 2, 3, 24, 40, dtype=torch.float32))
    before = s.pool.clone()
    children = rng.sample(range(rows), n)
    parents = [rng.randrange(rows) for _ in children]
    s.fork(ints(parents), ints(children))
    s.sync()
    want = before.clone()
    want[children] = before[parents]
    assert torch.equal(s.pool, want)
    # all of them exchanged, in place
    order = list(range(rows))
    rng.shuffle(order)
    s.fork(ints(order), ints(list(range(rows))))
    s.clear(ints([order[0], order[-1], order[0]]))
    s.sync()
    want = want[order]
    want[[order[0], order[-1]]] = 0
    assert torch.equal(s.pool, want)
    s.fork(ints([]), ints([]))
    s.clear(ints([]))
    s.sync()


@pytest.mark.parametrize("bad", ["twice", "range", "negative", "starts", "end", "first", "rate", "nan", "many", "many twice"])
@pytest.mark.parametrize("long", [False, True])
def test_refused_on_the_device_changes_nothing(bad, long):
    n = 300 if bad.startswith("many") else 3
    c = 80 if long else 2
    t, heads = c * n, 2
    s = ICStates(1, heads, 16, 16, n + 1, pool=draw(1, n + 1, 1, heads, 16, 16, dtype=torch.float32))
    q, k, v, rates = draw(1, t, heads, 16), draw(2, t, heads, 16), draw(3, t, heads, 16), rates_of(heads)
    seqs, starts = list(range(n)), [c * i for i in range(n + 1)]
    good, ok, all_rates = ints(seqs), ints(starts), rates.clone()
    if bad in ("twice", "many twice"):
        seqs[-1] = seqs[0]
    elif bad in ("range", "many"):
        seqs[1] = n + 1
    elif bad == "negative":
        seqs[2] = -1
    elif bad == "starts":
        starts[1] = starts[2] + 1
    elif bad == "end":
        starts[-1] = t + 1
    elif bad == "first":
        starts[0] = 1
    elif bad == "rate":
        rates[1] = -0.5
    else:
        rates[0] = float("nan")
    before, out = s.pool.clone(), torch.zeros_like(v)
    s.extend(0, q, k, v, rates, ints(seqs), ints(starts), out=out)
    with pytest.raises(ICCacheError) as e:
        s.sync()
    assert e.value.status == IC_ERR_INVALID
    assert torch.equal(s.pool, before) and not out.any()
    s.extend(0, q, k, v, all_rates, good, ok, out=out)
    s.sync()
    assert out.any()


def test_refused_forks_and_clears():
    s = ICStates(1, 1, 8, 8, 4, pool=draw(1, 4, 1, 1, 8, 8, dtype=torch.float32))
    before = s.pool.clone()
    for parents, children in (([0, 1], [2, 2]), ([4], [1]), ([0], [-1]), ([-1], [0])):
        s.fork(ints(parents), ints(children))
        torch.cuda.synchronize()
        with pytest.raises(ICCacheError):
            s.fork(ints([0]), ints([1]))
        with pytest.raises(ICCacheError):
            s.sync()
        assert torch.equal(s.pool, before)
    s.clear(ints([1, 4, -1, 2]))
    with pytest.raises(ICCacheError):
        s.sync()
    assert not s.pool[1:3].any() and torch.equal(s.pool[[0, 3]], before[[0, 3]])


def test_host_refusals():
    s = ICStates(1, 2, 16, 24, 3)
    q, k, v, r, one = draw(1, 2, 2, 16), draw(2, 2, 2, 16), draw(3, 2, 2, 24), rates_of(2), ints([0, 1])
    for call in (lambda: s.decode(1, q, k, v, r, one), lambda: s.decode(-1, q, k, v, r, one), lambda: s.decode(0, q, k, v, r, one, scale=math.nan),
                 lambda: s.extend(0, q[:0], k[:0], v[:0], r, ints([0] * 4), ints([0] * 5)), lambda: s.fork(ints([0] * 4), ints([0] * 4)),
                 lambda: s.decode(0, q, k, v, r, one, out=v[:1].expand(2, 2, 24))):
        with pytest.raises(ICCacheError):
            call()
    for call in (lambda: s.decode(0, q, k, v, r, ints([0])), lambda: s.decode(0, q.half(), k, v, r, one), lambda: s.decode(0, q, k[:1], v, r, one),
                 lambda: s.decode(0, q, k, v[..., :16], r, one), lambda: s.decode(0, q, k, v, r.double(), one), lambda: s.decode(0, q, k, v, r[:1], one),
                 lambda: s.extend(0, q, k, v, r, one, ints([0, 2])), lambda: s.fork(ints([0]), ints([0, 1]))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        ICStates(1, 2, 16, 24, 3, pool=torch.zeros(3, 1, 2, 16, 16, device=DEV))
    with pytest.raises(ICCacheError):
        ICStates(1, 2, 16, 24, 3, workspace=torch.empty(16, dtype=torch.uint8, device=DEV))
    assert s.decode(0, q[:0], k[:0], v[:0], r, ints([])).shape == (0, 2, 24)
    s.sync()
    s.close()
    with pytest.raises(ValueError):
        s.clear(one)


def test_rows_behind_the_last_sequence_stay():
    """A padded batch: starts that end before the rows do are refused, empty sequences at the end are not."""
    s, _ = run([5, 0, 0], heads=1, dk=16, dv=16)
    q = draw(1, 8, 1, 16)
    out = torch.full((8, 1, 16), 7.0, dtype=BF16, device=DEV)
    s.extend(0, q, q, q, rates_of(1), ints([0, 1]), ints([0, 5, 5]), out=out)
    with pytest.raises(ICCacheError):
        s.sync()
    assert (out == 7).all()


@pytest.mark.parametrize("counts", [[9000], [700, 30, 2500]])
def test_two_handles_at_once(counts):
    """Calls of two handles on two streams, not waited for in between: CTAs of one wait for the states that others of the same call publish."""
    n, t = len(counts), sum(counts)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    q, k, v = (draw(30 + i, t, 2, 64) for i in range(3))
    rates, seqs, starts = rates_of(2), ints(list(range(n))), starts_of(counts)
    alone = ICStates(1, 2, 64, 64, n)
    wants = [alone.extend(0, q, k, v, rates, seqs, starts) for _ in range(4)]
    alone.sync()
    torch.cuda.synchronize()
    held = []
    for s in streams:
        with torch.cuda.stream(s):
            held.append(ICStates(1, 2, 64, 64, n, stream=s))
    torch.cuda.synchronize()
    gots = [[], []]
    for _ in range(4):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                gots[i].append(held[i].extend(0, q, k, v, rates, seqs, starts))
    torch.cuda.synchronize()
    for i in range(2):
        held[i].sync()
        assert torch.equal(held[i].pool, alone.pool)
        assert all(torch.equal(a, b) for a, b in zip(gots[i], wants))


@pytest.mark.parametrize("counts", [[8192], [64 * 31, 64 * 33 + 1], [4000, 1, 0, 17]])
@pytest.mark.parametrize("heads", [1, 3])
def test_parts_of_an_item(counts, heads):
    """Few heads and long sequences: an item is divided among fewer CTAs than there are."""
    run(counts, heads=heads, dk=128, dv=64, layers=1, layer=0, seed=40)


@pytest.mark.parametrize("each", [8, 9, 16, 17, 32, 33])
def test_around_the_change_of_kernels(each):
    run([each], heads=4, seed=50)
    run([each] * 3, heads=2, dk=72, dv=136, dtype=F16, seed=51)
    run([each] * 40, heads=16, dk=16, dv=16, seed=52)


@pytest.mark.parametrize("bad", [0, 33, 100, 199])
@pytest.mark.parametrize("each", [1, 30])
def test_refused_calls_of_many_ctas(each, bad):
    """Some CTAs begin when others have already reported the call: whole CTAs refuse it, wherever the bad number stands."""
    n, heads = 200, 16
    s = ICStates(1, heads, 16, 16, n, pool=draw(1, n, 1, heads, 16, 16, dtype=torch.float32))
    q, before = draw(2, n * each, heads, 16), s.pool.clone()
    seqs, starts = list(range(n)), starts_of([each] * n)
    good = ints(seqs)
    for number in (n, -1, (bad + 1) % n):
        seqs[bad] = number
        wrong = ints(seqs)
        for _ in range(5):
            out = torch.zeros_like(q)
            s.extend(0, q, q, q, rates_of(heads), wrong, starts, out=out)
            with pytest.raises(ICCacheError):
                s.sync()
            assert torch.equal(s.pool, before) and not out.any()
    s.extend(0, q, q, q, rates_of(heads), good, starts)
    s.sync()


@pytest.mark.parametrize("n,heads,dk", [(3, 1, 8), (2000, 32, 64), (8192, 1, 8)])
def test_a_bad_number_does_not_keep_the_others(n, heads, dk):
    """Bad numbers come first: the CTAs that begin after they have been met clear their sequences all the same."""
    s = ICStates(1, heads, dk, 16, n)
    for _ in range(3):
        s.pool.fill_(1.0)
        s.clear(ints([n, -1, 2 ** 31 - 1] + list(range(1, n))))
        with pytest.raises(ICCacheError) as e:
            s.sync()
        assert e.value.status == IC_ERR_INVALID
        assert not s.pool[1:].any() and (s.pool[0] == 1).all()
    s.clear(ints([0]))
    s.sync()
    assert not s.pool.any()


@pytest.mark.parametrize("counts,heads,dv", [([9000], 2, 64), ([3, 5000], 1, 128)])
def test_a_wait_that_runs_out_is_reported(counts, heads, dv):
    """A published state that nobody is told of (its word in the workspace is set to a number that it never leaves): the CTAs that wait for it give up after
    a second, the call is reported, and the handle goes on."""
    from paper_2501_12689_b200 import IC_ERR_TIMEOUT, ic_state_workspace_bytes
    n, t, words = len(counts), sum(counts), 64
    workspace = torch.empty(ic_state_workspace_bytes(1, heads, 64, dv, n), dtype=torch.uint8, device=DEV)
    s = ICStates(1, heads, 64, dv, n, workspace=workspace)
    s.sync()
    q, k, v, rates = draw(1, t, heads, 64), draw(2, t, heads, 64), draw(3, t, heads, dv), rates_of(heads)
    workspace.view(torch.int32)[words] = 1000          # of the first CTA
    s.extend(0, q, k, v, rates, ints(list(range(n))), starts_of(counts))
    with pytest.raises(ICCacheError) as e:
        s.sync()
    assert e.value.status == IC_ERR_TIMEOUT
    s.sync()
    s.clear(ints(list(range(n))))
    run(counts, heads=heads, dk=64, dv=dv, layers=1, layer=0, states=s)


@pytest.mark.parametrize("each", [6, 7, 8, 11, 12, 13])
def test_where_the_kernels_change(each):
    """7 | 8 tokens a sequence where there are many states, 12 | 13 where there are few."""
    run([each], heads=4, seed=60)
    run([each] * 3, heads=2, dk=72, dv=136, dtype=F16, seed=61)
    run([each] * 60, heads=4, dk=16, dv=16, seed=62)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("shared", ["q", "k", "v", "qkv"])
@pytest.mark.parametrize("counts,dk,dv", [([70, 3, 0, 200], 64, 64), ([1000, 130], 72, 136), ([3000], 128, 128)])
def test_rows_shared_among_the_tokens(counts, dk, dv, shared, dtype):
    """A stride of 0 between tokens, which no tensor map has: the rows come in 16-byte copies.  Whole items and cut ones, last chunks that are not full."""
    t, heads, n = sum(counts), 2, len(counts)
    s = ICStates(1, heads, dk, dv, n, dtype=dtype, pool=draw(9, n, 1, heads, dk, dv, dtype=torch.float32))
    rates = torch.tensor([0.5, 0.01], device=DEV)
    before = s.pool.clone()
    x = {name: draw(i, 1 if name in shared else t, heads, d, dtype=dtype).expand(t, heads, d) for i, (name, d) in enumerate((("q", dk), ("k", dk), ("v", dv)))}
    got = s.extend(0, x["q"], x["k"], x["v"], rates, ints(list(range(n))), starts_of(counts))
    s.sync()
    a = 0
    for i, c in enumerate(counts):
        part = slice(a, a + c)
        close(got[part], s.pool[i, 0], formula(*(x[name][part] for name in "qkv"), rates, before[i, 0], 1 / math.sqrt(dk)), c, True) if c else None
        a += c


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_what_lies_behind_a_short_chunk_is_not_read(dtype):
    """The rows behind a sequence's last token belong to another one, whose infinities and NaN stay its own; by tensor maps and by copies."""
    for shared in (False, True):
        counts = [70, 5, 100]
        t, heads = sum(counts), 2
        s = ICStates(1, heads, 64, 64, 3, dtype=dtype)
        q, k, v = (draw(i, t, heads, 64, dtype=dtype) for i in range(3))
        if shared:
            q = q[:1].expand(t, heads, 64)
        else:
            q[70:75] = math.nan
        k[70:75], v[70:75] = math.inf, math.nan
        got = s.extend(0, q, k, v, rates_of(heads), ints([0, 1, 2]), starts_of(counts))
        s.sync()
        for i, part in ((0, slice(0, 70)), (2, slice(75, 175))):
            close(got[part], s.pool[i, 0], formula(q[part], k[part], v[part], rates_of(heads), torch.zeros(heads, 64, 64, device=DEV), 0.125), part.stop - part.start, True)
        assert not got[70:75].isfinite().all()


MIXED = [[1] * 255 + [1500], [1] * 31 + [352], [0] * 10 + [70] + [1] * 10, [32, 33] + [1] * 20, [64] + [0] * 9, [65] + [0] * 9, [1] * 40 + [129, 31, 200] + [2] * 60,
         [1, 200, 1] * 3 + [1] * 300 + [500] + [3] * 20 + [33] + [0] * 30]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("which", range(len(MIXED)))
def test_a_prompt_among_single_tokens(which, dtype):
    """Calls whose mean is short and whose longest is not: each sequence by its own length."""
    counts = MIXED[which]
    run(counts, heads=2, dk=64, dv=64, dtype=dtype, layers=1, layer=0, seed=70)
    run(counts, heads=3, dk=72, dv=136, dtype=dtype, layers=1, layer=0, seed=71, order=random.Random(1).sample(range(len(counts) + 3), len(counts)),
        max_seqs=len(counts) + 3)


def test_many_prompts_among_many_single_tokens():
    """More long sequences than a launch takes."""
    counts = [1] * 2000 + [40, 33] * 150
    random.Random(2).shuffle(counts)
    run(counts, heads=1, dk=16, dv=16, layers=1, layer=0, seed=72)


@pytest.mark.parametrize("bad", ["range", "twice", "starts", "end", "rate"])
@pytest.mark.parametrize("n", [40, 300])
def test_refused_calls_of_mixed_lengths(n, bad):
    counts = [1] * (n - 1) + [120]
    t, heads = sum(counts), 2
    s = ICStates(1, heads, 16, 16, n, pool=draw(1, n, 1, heads, 16, 16, dtype=torch.float32))
    q, rates, seqs, starts = draw(2, t, heads, 16), rates_of(heads), list(range(n)), starts_of(counts).tolist()
    if bad == "range":
        seqs[5] = n
    elif bad == "twice":
        seqs[-1] = 0
    elif bad == "starts":
        starts[3] = 10 ** 9
    elif bad == "end":
        starts[-1] -= 1
    else:
        rates[1] = -1.0
    before, out = s.pool.clone(), torch.zeros_like(q)
    s.extend(0, q, q, q, rates, ints(seqs), ints(starts), out=out)
    with pytest.raises(ICCacheError) as e:
        s.sync()
    assert e.value.status == IC_ERR_INVALID
    assert torch.equal(s.pool, before) and not out.any()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("t,n,heads", [(3840, 30, 8), (16384, 12, 8)])
@pytest.mark.parametrize("rate", [0.0, 1e-6, 1e-5, 1e-4, 1e-3])
def test_slow_decays_over_many_chunks(rate, t, n, heads, dtype):
    """Items of many chunks that one CTA walks over: what a chunk leaves of the state is not off the same way every time.  fp32: a rounding a chunk of
    2^-24 of the state at most, as often up as down, so sqrt(chunks) 2^-24 of it or less, and each chunk's own sums, 2e-7 = 2^-22.2."""
    s = ICStates(1, heads, 64, 64, n, dtype=dtype)
    q, k, v = (draw(i, t, heads, 64, dtype=dtype) for i in range(3))
    rates = rate * torch.linspace(1.0, 1.7, heads, device=DEV)
    s.extend(0, *(x.repeat(n, 1, 1) for x in (q, k, v)), rates, ints(list(range(n))), starts_of([t] * n))
    s.sync()
    want = formula(q, k, v, rates, torch.zeros(heads, 64, 64, device=DEV), 0.125)[3]
    for i in (0, n // 2, n - 1):
        for h in range(heads):
            assert (s.pool[i, 0, h].double() - want[h]).norm() <= (math.sqrt(t / 64) * 2.0 ** -24 + 2.0 ** -22) * want[h].norm()
