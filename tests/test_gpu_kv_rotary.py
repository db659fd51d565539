"""Rotary positions over the paged cache on the GPU: rows against the formula in 64 bits, what is stored, moved and refused."""
import random

import pytest
import torch

from kv_util import UNIT
from paper_2501_12689_b200 import IC_ERR_INVALID, ICCacheError, ICPagedKV, rotary_frequencies

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16 = torch.bfloat16, torch.float16


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def starts_of(counts):
    return ints([0] + torch.tensor(counts).cumsum(0).tolist())


def draw(seed, *shape, dtype=BF16):
    return torch.randn(*shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed)).to(dtype)


def turned(x, position, f, dim, interleaved, magnitude=1.0):
    """(rows in 64 bits, size of the pair each element comes from)."""
    angle = position.double()[:, None] * torch.tensor(f, dtype=torch.float64, device=DEV)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    out, size = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device=DEV)
    one, two = (slice(0, dim, 2), slice(1, dim, 2)) if interleaved else (slice(0, dim // 2), slice(dim // 2, dim))
    a, b = out[..., one].clone(), out[..., two].clone()
    out[..., one], out[..., two] = magnitude * (a * c - b * s), magnitude * (a * s + b * c)
    size[..., one] = size[..., two] = magnitude * (a.abs() + b.abs())
    return out, size


def close(got, want, size):
    """One rounding to the type (half a step of the value; fp16's least step is 2**-24), and before it two products and a sum in fp32 of
    a sine and a cosine that are off by 2 units of 2**-23 at most, and an angle off by 2**-24 half turns (32-bit turns as a float):
    below 2**-20 of |a| + |b|."""
    bound = UNIT[got.dtype] * want.abs() + 2.0 ** -20 * size + 2.0 ** -25
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all() and (off <= bound).all(), f"{(off / bound).max().item():.2f} times the bound"


def make(had, counts, *, hkv=2, d=64, page=16, layers=2, dtype=BF16, max_seqs=None, extra=6):
    """A cache whose sequences hold `had` tokens (zeros) and have room reserved for `counts` more; NaN where nothing was written."""
    n = len(had)
    max_pages = max(1, -(-max(a + b for a, b in zip(had, counts)) // page)) + 1
    n_pages = sum(-(-(a + b) // page) for a, b in zip(had, counts)) + extra
    pool = torch.full((n_pages, layers, 2, hkv, page, d), float("nan"), dtype=dtype, device=DEV)
    kv = ICPagedKV(n_pages, layers, hkv, page, d, max_seqs or n, max_pages, dtype=dtype, pool=pool)
    order = list(range(n))
    random.Random(3).shuffle(order)
    kv.reserve(ints(order), ints([had[s] for s in order]))
    kv.reserve(ints(order), ints([counts[s] for s in order]))
    kv.sync()
    return kv


def check_write(kv, had, counts, hq, dim, interleaved, layer=1, positions=None, single=False, strided=False, inplace=False, magnitude=1.0, seed=1):
    n, t, d, hkv = len(had), sum(counts), kv.head_dim, kv.n_kv_heads
    f = rotary_frequencies(dim)
    kv.set_rotary(dim, interleaved=interleaved, magnitude=magnitude)
    if strided:
        q, k, v = draw(seed, t, hq + 2 * hkv, d, dtype=kv.dtype).split([hq, hkv, hkv], 1)
    else:
        q, k, v = (draw(seed + i, t, h, d, dtype=kv.dtype) for i, h in enumerate((hq, hkv, hkv)))
    at = torch.cat([torch.arange(a, a + c) for a, c in zip(had, counts)]).to(DEV)
    place = at if positions is None else positions
    before = kv.pool.clone()
    # the expected pool: NaN stays where no token of the call lies
    want_q, size_q = turned(q, place, f, dim, interleaved, magnitude)
    want_k, size_k = turned(k, place, f, dim, interleaved, magnitude)
    seqs = ints(list(range(n)))
    out = q if inplace else None
    got = kv.write_rotated(layer, q, k, v, seqs, None if single else starts_of(counts), positions=positions, out=out)
    kv.sync()
    if inplace:
        assert got.data_ptr() == q.data_ptr()
    close(got, want_q, size_q)
    rest = torch.ones_like(kv.pool, dtype=torch.bool)
    i = torch.repeat_interleave(torch.arange(n), torch.tensor(counts)).to(DEV)
    page = kv.tables[i, at // kv.page_size].long()
    slot = at % kv.page_size
    close(kv.pool[page, layer, 0, :, slot], want_k, size_k)
    assert torch.equal(kv.pool[page, layer, 1, :, slot], v)
    assert torch.equal(kv.pool[page, layer, 0, :, slot][..., dim:], k[..., dim:]) and torch.equal(got[..., dim:], (q if not inplace else got)[..., dim:])
    rest[page, layer, :, :, slot] = False
    raw = lambda x: x.view(torch.int16)  # noqa: E731
    assert torch.equal(raw(kv.pool)[rest], raw(before)[rest])


SHAPES = [(64, 64, False), (64, 64, True), (128, 128, False), (128, 32, False), (80, 80, False), (80, 20, False), (80, 20, True), (96, 38, False),
          (96, 38, True), (256, 256, False), (256, 102, False), (256, 256, True), (8, 8, False), (8, 2, False), (8, 4, True), (248, 240, False),
          (24, 16, False), (72, 72, False), (72, 70, True), (136, 136, False)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d,dim,interleaved", SHAPES)
def test_rows_of_every_shape(d, dim, interleaved, dtype):
    had, counts = [0, 17, 300, 5, 64], [1, 40, 0, 3, 130]
    kv = make(had, counts, hkv=2, d=d, dtype=dtype)
    check_write(kv, had, counts, 6, dim, interleaved)
    had, counts = [0, 15, 16, 100], [1] * 4
    kv = make(had, counts, hkv=3, d=d, page=8, dtype=dtype)
    check_write(kv, had, counts, 3, dim, interleaved, single=True, magnitude=1.25)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (32, 8), (7, 7), (130, 1), (16, 2)])
@pytest.mark.parametrize("tokens", [1, 2, 3, 5, 700])
def test_heads_and_lengths(hq, hkv, tokens):
    had, counts = [9], [tokens]
    kv = make(had, counts, hkv=hkv, d=64, page=32)
    check_write(kv, had, counts, hq, 64, False)


@pytest.mark.parametrize("n", [2, 255, 256, 257, 1500])
@pytest.mark.parametrize("most", [1, 4])
def test_many_sequences(n, most):
    rng = random.Random(n)
    had, counts = [rng.randint(0, 40) for _ in range(n)], [most if most == 1 else rng.randint(0, most) for _ in range(n)]
    kv = make(had, counts, hkv=1, d=64)
    check_write(kv, had, counts, 2, 64, False, single=most == 1)
    # few threads a CTA (three rows), more sequences than threads
    check_write(kv, had, counts, 1, 64, False, single=most == 1, seed=9)


@pytest.mark.parametrize("d,dim,interleaved", [(64, 64, False), (80, 20, False), (96, 38, True)])
@pytest.mark.parametrize("inplace", [False, True])
def test_strides_in_place_and_positions(d, dim, interleaved, inplace):
    had, counts = [3, 50], [70, 9]
    kv = make(had, counts, d=d)
    check_write(kv, had, counts, 4, dim, interleaved, strided=True, inplace=inplace)
    rng = random.Random(5)
    far = ints([rng.choice([0, -1, 1, 131071, -(2 ** 31), 2 ** 31 - 1, rng.randrange(2 ** 31)]) for _ in range(79)])
    check_write(kv, had, counts, 4, dim, interleaved, positions=far, inplace=inplace, seed=7)


def test_far_positions_are_exact():
    """Pairs that make whole turns: a frequency of 2 pi / 1024 comes back after 1024 tokens, at every distance."""
    import math
    kv = make([0], [1], d=8)
    kv.set_rotary(8, frequencies=[2 * math.pi / 1024] * 4)
    x = draw(1, 1, 1, 8)
    near = kv.rotate(x, ints([77]))
    for turns in (1, 1000, 2 ** 20):
        assert torch.equal(kv.rotate(x, ints([77 + 1024 * turns])), near)
        assert torch.equal(kv.rotate(x, ints([77 - 1024 * turns])), near)
    kv.sync()


def test_queries_alone_keys_alone_and_back():
    had, counts = [12, 0], [30, 7]
    kv = make(had, counts)
    kv.set_rotary(scaling="linear", factor=3.0)
    f = rotary_frequencies(64, scaling="linear", factor=3.0)
    k, v = draw(1, 37, 2, 64), draw(2, 37, 2, 64)
    assert kv.write_rotated(0, None, k, v, ints([0, 1]), starts_of(counts)) is None
    at = torch.cat([torch.arange(12, 42), torch.arange(7)]).to(DEV)
    x = draw(3, 37, 5, 64)
    y = kv.rotate(x, at.int())
    back = kv.rotate(y, at.int(), inverse=True)
    kv.sync()
    want, size = turned(x, at, f, 64, False)
    close(y, want, size)
    want, size = turned(y, -at, f, 64, False)
    close(back, want, size)
    i = torch.tensor([0] * 30 + [1] * 7, device=DEV)
    want, size = turned(k, at, f, 64, False)
    close(kv.pool[kv.tables[i, at // 16].long(), 0, 0, :, at % 16], want, size)
    # no tokens, no sequences
    kv.write_rotated(0, x[:0], k[:0], v[:0], ints([]), ints([0]))
    assert kv.rotate(x[:0], ints([])).shape == (0, 5, 64)
    kv.sync()


def test_other_streams_and_graphs():
    had, counts = [5, 20], [1, 1]
    kv = make(had, counts)
    kv.set_rotary()
    q, k, v = draw(1, 2, 4, 64), draw(2, 2, 2, 64), draw(3, 2, 2, 64)
    seqs = ints([0, 1])
    want = kv.write_rotated(1, q, k, v, seqs)
    kv.sync()
    pool = kv.pool.clone()
    kv.pool[:, 1] = 0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = kv.write_rotated(1, q * 1.0, k, v, seqs)
    torch.cuda.current_stream().wait_stream(side)
    i = torch.arange(2, device=DEV)
    where = kv.tables[i, kv.lengths.long().sub(1) // 16].long()
    slot = kv.lengths.long().sub(1) % 16
    assert torch.equal(got, want) and torch.equal(kv.pool[where, 1, :, :, slot], pool[where, 1, :, :, slot])
    # captured: the rotation is what it was when captured
    kv.set_stream(side)
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        kv.write_rotated(1, q, k, v, seqs, out=out)
        kv.shift(seqs, ints_3)
    kv.set_rotary(base=77.0)
    kv.pool[:, 1] = 0
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and torch.equal(kv.pool[where, 1, 1, :, slot], pool[where, 1, 1, :, slot])
    f = rotary_frequencies(64)
    w, size = turned(pool[where, 1, 0, :, slot], torch.full((2,), 3, device=DEV), f, 64, False)
    close(kv.pool[where, 1, 0, :, slot], w, size)


ints_3 = None


@pytest.fixture(autouse=True)
def _threes():
    global ints_3
    ints_3 = ints([3, 3])


@pytest.mark.parametrize("bad", ["sequence", "negative", "starts", "end", "length", "many"])
def test_bad_calls_store_and_turn_nothing(bad):
    n = 300 if bad == "many" else 3
    had, counts = [4] * n, [2] * n
    kv = make(had, counts)
    kv.set_rotary()
    t = 2 * n
    q, k, v = draw(1, t, 4, 64), draw(2, t, 2, 64), draw(3, t, 2, 64)
    seqs, starts = list(range(n)), [2 * i for i in range(n + 1)]
    if bad in ("sequence", "many"):
        seqs[-1] = n
    elif bad == "negative":
        seqs[0] = -1
    elif bad == "starts":
        starts[1] = 5
    elif bad == "end":
        starts[-1] = t - 1
    elif bad == "length":
        kv.lengths[1] = 1
    before, out = kv.pool.clone(), torch.zeros_like(q)
    kv.write_rotated(0, q, k, v, ints(seqs), ints(starts), out=out)
    with pytest.raises(ICCacheError) as e:
        kv.sync()
    assert e.value.status == IC_ERR_INVALID
    assert torch.equal(kv.pool.view(torch.int16), before.view(torch.int16)) and not out.any()
    if bad not in ("length",):
        kv.write_rotated(0, q, k, v, ints(list(range(n))), ints([2 * i for i in range(n + 1)]), out=out)
        kv.sync()
        assert out.any()


def test_a_bad_page_is_reported_and_the_others_are_written():
    kv = make([0, 0], [20, 20])
    kv.set_rotary()
    kv.tables[0, 1] = 10 ** 6
    k, v = draw(1, 40, 2, 64), draw(2, 40, 2, 64)
    kv.write_rotated(0, None, k, v, ints([0, 1]), starts_of([20, 20]))
    with pytest.raises(ICCacheError):
        kv.sync()
    assert torch.equal(kv.pool[int(kv.tables[1, 1]), 0, 1, :, :4].transpose(0, 1), v[36:])


def test_host_refusals():
    kv = make([0], [4])
    q, k, v, one = draw(1, 4, 4, 64), draw(2, 4, 2, 64), draw(3, 4, 2, 64), ints([0])
    for call in (lambda: kv.write_rotated(0, q, k, v, one, ints([0, 4])), lambda: kv.rotate(q, ints([0] * 4)), lambda: kv.shift(one, one)):
        with pytest.raises(ICCacheError, match="set_rotary"):
            call()
    with pytest.raises(ICCacheError):
        kv.set_rotary(66)
    with pytest.raises(ICCacheError):
        kv.set_rotary(63)
    with pytest.raises(ValueError):
        kv.set_rotary(64, frequencies=[1.0] * 31)
    with pytest.raises(ICCacheError):
        kv.set_rotary(64, frequencies=[float("inf")] * 32)
    kv.set_rotary()
    with pytest.raises(ICCacheError):
        kv.write_rotated(2, q, k, v, one, ints([0, 4]))
    with pytest.raises(ICCacheError):
        kv.write_rotated(0, q, k, v, one)                       # four tokens, one sequence, no starts
    with pytest.raises(ValueError):
        kv.write_rotated(0, q, k, v[:, :1], one, ints([0, 4]))
    with pytest.raises(ValueError):
        kv.write_rotated(0, q, k[:3], v[:3], one, ints([0, 4]))
    with pytest.raises(ValueError):
        kv.write_rotated(0, q, k, v, one, ints([0, 4]), positions=ints([0] * 3))
    with pytest.raises(ValueError):
        kv.rotate(q.float(), ints([0] * 4))
    with pytest.raises(ValueError):
        kv.rotate(q, ints([0] * 4), out=q[:, :2])
    with pytest.raises(ICCacheError):
        kv.rotate(q, ints([0] * 4), out=q[:1].expand(4, 4, 64))     # rows of the result overlap
    kv.sync()


# ---------------------------------------------------------------- shift
def filled(lens, *, hkv=2, d=64, page=16, layers=2, dtype=BF16, max_seqs=None):
    kv = make([0] * len(lens), lens, hkv=hkv, d=d, page=page, layers=layers, dtype=dtype, max_seqs=max_seqs, extra=sum(-(-x // page) for x in lens) + 4)
    for x in range(layers):
        k, v = draw(10 + x, sum(lens), hkv, d, dtype=dtype), draw(50 + x, sum(lens), hkv, d, dtype=dtype)
        kv.write(x, k, v, ints(list(range(len(lens)))), starts_of(lens))
    kv.sync()
    return kv


def check_shift(kv, seqs, by, f, dim, interleaved):
    before, lens = kv.pool.clone(), kv.lengths.tolist()
    kv.shift(ints(seqs), ints(by))
    kv.sync()
    rest = torch.ones_like(before, dtype=torch.bool)
    for s, d in zip(seqs, by):
        at = torch.arange(lens[s], device=DEV)
        page, slot = kv.tables[s, at // kv.page_size].long(), at % kv.page_size
        was, now = (x[page, :, 0, :, slot].flatten(1, 2) for x in (before, kv.pool))
        want, size = turned(was, torch.full_like(at, d), f, dim, interleaved)
        close(now, want, size)
        assert torch.equal(now[..., dim:], was[..., dim:])
        rest[page, :, 0, :, slot] = False
    assert torch.equal(kv.pool.view(torch.int16)[rest], before.view(torch.int16)[rest])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d,dim,interleaved", SHAPES)
def test_shift_shapes(d, dim, interleaved, dtype):
    kv = filled([33, 0, 16, 1, 100], d=d, dtype=dtype, layers=3)
    kv.set_rotary(dim, interleaved=interleaved, magnitude=1.5)
    check_shift(kv, [4, 0, 1, 3], [7, -19, 5, 100000], rotary_frequencies(dim), dim, interleaved)


@pytest.mark.parametrize("hkv,page,layers,n", [(1, 8, 9, 5), (8, 128, 1, 3), (3, 256, 2, 2), (1, 16, 1, 1100)])
def test_shift_sizes(hkv, page, layers, n):
    rng = random.Random(n)
    kv = filled([rng.randint(0, 200) for _ in range(n)], hkv=hkv, page=page, layers=layers)
    kv.set_rotary()
    seqs = list(range(n))
    rng.shuffle(seqs)
    check_shift(kv, seqs, [rng.randint(-5000, 5000) for _ in seqs], rotary_frequencies(64), 64, False)


def test_shift_by_nothing_and_of_nothing():
    kv = filled([40, 0])
    kv.set_rotary()
    before = kv.pool.clone()
    kv.shift(ints([0, 1]), ints([0, 9]))
    kv.shift(ints([]), ints([]))
    kv.sync()
    assert torch.equal(kv.pool.view(torch.int16), before.view(torch.int16))


@pytest.mark.parametrize("n", [3, 1200])
@pytest.mark.parametrize("bad", ["shared", "twice", "range", "page"])
def test_shift_refused_on_the_device_changes_nothing(n, bad):
    kv = filled([40] * n, hkv=1, max_seqs=n + 1)
    kv.set_rotary()
    seqs = list(range(n))
    if bad == "shared":
        kv.fork(ints([n - 1]), ints([n]))
    elif bad == "twice":
        seqs[-1] = 0
    elif bad == "range":
        seqs[1] = n + 1
    else:
        kv.tables[n - 1, 2] = -1
    before = kv.pool.clone()
    kv.shift(ints(seqs), ints([3] * n))
    with pytest.raises(ICCacheError) as e:
        kv.sync()
    assert e.value.status == IC_ERR_INVALID
    assert torch.equal(kv.pool.view(torch.int16), before.view(torch.int16))
    if bad == "shared":
        kv.fork(ints([n]), ints([n]), copy=True)               # a copy of its own: the tail was its own already
        kv.shift(ints(seqs), ints([3] * n))
        kv.sync()
        assert not torch.equal(kv.pool.view(torch.int16), before.view(torch.int16))


def test_a_copied_example_behind_another_one():
    """Keys written at 0 .. and moved by 100 are those written at 100 .., but for a rounding more; attention through them agrees with attention
    of queries that are as far away."""
    lens = [50]
    kv = make([0, 0], [50, 50], d=64, page=16)
    kv.set_rotary()
    k, v = draw(1, 50, 2, 64), draw(2, 50, 2, 64)
    kv.write_rotated(1, None, k, v, ints([0]), starts_of(lens))
    kv.write_rotated(1, None, k, v, ints([1]), starts_of(lens), positions=torch.arange(100, 150, device=DEV, dtype=torch.int32))
    kv.shift(ints([0]), ints([100]))
    q = draw(3, 2, 4, 64)
    kv.rotate(q, ints([160, 160]), out=q)
    q[1] = q[0]
    out = kv.decode(1, q, ints([0, 1]))
    kv.sync()
    at = torch.arange(50, device=DEV)
    a, b = (kv.pool[kv.tables[s, at // 16].long(), 1, 0, :, at % 16].double() for s in (0, 1))
    assert (a - b).abs().max() <= 3 * 2.0 ** -8 * b.abs().max()
    assert (out[0].float() - out[1].float()).abs().max() < 0.06


@pytest.mark.parametrize("n", [40, 300])
def test_bad_pages_among_many_tokens(n):
    """Entries that name no page all over the call: CTAs report them while others begin.  A token is stored and turned as a whole or not at all, and
    nothing else is touched."""
    counts = [50] * n
    f = rotary_frequencies(64)
    q, k, v = draw(1, 50 * n, 4, 64), draw(2, 50 * n, 2, 64), draw(3, 50 * n, 2, 64)
    at = torch.arange(50, device=DEV).repeat(n)
    want_q, size_q = turned(q, at, f, 64, False)
    want_k, size_k = turned(k, at, f, 64, False)
    for seed in range(5):
        kv = make([0] * n, counts)
        kv.set_rotary()
        rng = random.Random(seed)
        i = torch.repeat_interleave(torch.arange(n), 50).to(DEV)
        page = kv.tables[i, at // 16].long()
        bad = torch.zeros(n, 4, dtype=torch.bool, device=DEV)
        for s in rng.sample(range(n), n // 8):
            col = rng.randrange(4)
            bad[s, col] = True
            kv.tables[s, col] = rng.choice([-1, 10 ** 6, 2 ** 31 - 1])
        before, out = kv.pool.clone(), torch.zeros_like(q)
        kv.write_rotated(1, q, k, v, ints(list(range(n))), starts_of(counts), out=out)
        with pytest.raises(ICCacheError):
            kv.sync()
        slot = at % 16
        stored = ~kv.pool[page, 1, 0, :, slot].isnan().flatten(1).any(1)
        assert not (stored & bad[i, at // 16]).any()
        close(kv.pool[page, 1, 0, :, slot][stored], want_k[stored], size_k[stored])
        assert torch.equal(kv.pool[page, 1, 1, :, slot][stored], v[stored])
        done = (out != 0).flatten(1).any(1)
        assert not (stored & ~done).any()
        close(out[done], want_q[done], size_q[done])
        rest = torch.ones_like(before, dtype=torch.bool)
        rest[page[stored], 1, :, :, slot[stored]] = False
        raw = lambda x: x.view(torch.int16)  # noqa: E731
        assert torch.equal(raw(kv.pool)[rest], raw(before)[rest])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d,dim,interleaved", SHAPES + [(16, 6, True), (16, 10, False), (256, 250, True), (40, 2, True)])
@pytest.mark.parametrize("what", [float("inf"), float("nan"), -0.0])
def test_elements_that_do_not_turn_are_left_as_they_are(d, dim, interleaved, dtype, what):
    """Bit for bit, next to infinities, NaN and zeros of either sign; and what turns does not meet them."""
    had, counts = [0, 17], [1, 40]
    for single in (False, True):
        kv = make(had, [1, 1] if single else counts, d=d, dtype=dtype)
        kv.set_rotary(dim, interleaved=interleaved)
        t = 2 if single else 41
        q, k, v = (draw(i, t, h, d, dtype=dtype) for i, h in enumerate((4, 2, 2)))
        for x in (q, k, v):
            x[..., dim::2] = what
            x[..., dim + 1::4] = 0.0
        raw = lambda x: x.contiguous().view(torch.int16)  # noqa: E731
        at = torch.tensor([0, 17] if single else [0] + list(range(17, 57)), device=DEV)
        seqs = ints([0, 1])
        got = kv.write_rotated(1, q, k, v, seqs, None if single else starts_of(counts))
        inplace = q.clone()
        kv.rotate(inplace, at.int(), out=inplace)
        kv.sync()
        i = ints([0, 1] if single else [0] + [1] * 40).long()
        page, slot = kv.tables[i, at // 16].long(), at % 16
        f = rotary_frequencies(dim)
        stored = kv.pool[page, 1, 0, :, slot]
        for now, was in ((got, q), (inplace, q), (stored, k)):
            assert torch.equal(raw(now[..., dim:]), raw(was[..., dim:]))
            want, size = turned(was[..., :dim], at, f, dim, interleaved)
            close(now[..., :dim], want, size)
        assert torch.equal(raw(kv.pool[page, 1, 1, :, slot]), raw(v))
        # the cached keys moved
        kv.pool.nan_to_num_(nan=1.0) if what == what else None
        before = kv.pool.clone()
        kv.shift(seqs, ints([5, -3]))
        kv.sync()
        assert torch.equal(raw(kv.pool[..., dim:]), raw(before[..., dim:])) and torch.equal(raw(kv.pool[:, :, 1]), raw(before[:, :, 1]))
        want, size = turned(before[page, 1, 0, :, slot][..., :dim], torch.where(i == 0, 5, -3), f, dim, interleaved)
        close(kv.pool[page, 1, 0, :, slot][..., :dim], want, size)
