"""The paged key-value cache on the GPU: page operations against a plain model, attention against its formula in 64 bits."""
import random

import pytest
import torch

import kv_util
from kv_util import Model, attention, close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16 = torch.bfloat16, torch.float16


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def starts_of(counts):
    s = [0]
    for c in counts:
        s.append(s[-1] + c)
    return ints(s)


def make(lens, *, hkv=2, d=64, page=16, layers=2, dtype=BF16, layer=1, spare=5, seed=0, max_seqs=None, poison=True):
    """A cache whose sequences have these lengths, written through reserve and write in ragged pieces; every slot that holds no
    token is NaN."""
    from paper_2501_12689_b200 import ICPagedKV
    g = torch.Generator(device=DEV).manual_seed(seed)
    rng = random.Random(seed)
    n = len(lens)
    max_pages = max(1, -(-max(lens + [0]) // page)) + 2
    n_pages = sum(-(-x // page) for x in lens) + spare
    pool = torch.full((n_pages, layers, 2, hkv, page, d), float("nan") if poison else 0.0, dtype=dtype, device=DEV)
    kv = ICPagedKV(n_pages, layers, hkv, page, d, max_seqs or n, max_pages, dtype=dtype, pool=pool)
    # in two pieces, the second in another order, so that the tables are not in order
    first = [rng.randint(0, x) for x in lens]
    order = list(range(n))
    rng.shuffle(order)
    for who, counts in ((list(range(n)), first), (order, [lens[s] - first[s] for s in order])):
        total = sum(counts)
        kv.reserve(ints(who), ints(counts))
        for x in range(layers):
            k, v = (torch.randn(total, hkv, d, device=DEV, generator=g).to(dtype) for _ in range(2))
            if x == layer:
                k = k * 1.5
            kv.write(x, k, v, ints(who), starts_of(counts))
    kv.sync()
    return kv


def query(rows, hq, d, dtype, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (2.0 * torch.randn(rows, hq, d, device=DEV, generator=g)).to(dtype)


def check(kv, seqs, counts, hq, window=0, sinks=0, layer=1, decode=False, scale=None, seed=1):
    q = query(sum(counts), hq, kv.head_dim, kv.dtype, seed)
    if decode:
        got = kv.decode(layer, q, ints(seqs), window=window, sinks=sinks, scale=scale)
    else:
        got = kv.extend(layer, q, ints(seqs), starts_of(counts), window=window, sinks=sinks, scale=scale)
    kv.sync()
    want, size = attention(kv, layer, q, seqs, counts, window, sinks, scale)
    return close(got, want, size)


# ---------------------------------------------------------------- attention of one new token
LENGTHS = [1, 0, 2, 7, 15, 16, 17, 31, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 2049]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hq,hkv,d,page", [
    (8, 2, 64, 16), (2, 2, 128, 16), (8, 1, 128, 8), (6, 2, 80, 32), (5, 1, 8, 64), (16, 1, 256, 16), (12, 4, 96, 128),
    (20, 1, 64, 256), (40, 1, 128, 16), (128, 1, 72, 16), (14, 2, 248, 64), (7, 7, 136, 32), (136, 2, 64, 16)])
def test_decode_heads_and_sizes(hq, hkv, d, page, dtype):
    kv = make(LENGTHS, hkv=hkv, d=d, page=page, dtype=dtype)
    check(kv, list(range(len(LENGTHS))), [1] * len(LENGTHS), hq, decode=True)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 0), (16, 4), (64, 4), (64, 64), (63, 65), (100, 17), (1000, 4), (4000, 4), (3, 500)])
@pytest.mark.parametrize("page", [16, 128])
def test_decode_window_and_sinks(window, sinks, page):
    kv = make(LENGTHS, hkv=2, d=64, page=page)
    check(kv, list(range(len(LENGTHS))), [1] * len(LENGTHS), 8, window, sinks, decode=True)


@pytest.mark.parametrize("n", [1, 3, 150, 700, 1100])
def test_decode_batches(n):
    rng = random.Random(n)
    lens = [rng.choice([0, 1, 40, 100, 333]) for _ in range(n)]
    kv = make(lens, hkv=2, d=64, page=16)
    order = list(range(n))
    rng.shuffle(order)
    check(kv, order, [1] * n, 6, decode=True)
    check(kv, order, [1] * n, 6, 50, 3, decode=True)


@pytest.mark.parametrize("hq,hkv,d", [(8, 1, 128), (32, 4, 128), (4, 4, 256), (3, 1, 64)])
def test_decode_long(hq, hkv, d):
    """A few long sequences: the work is split over their length and joined."""
    kv = make([40001, 5, 20000], hkv=hkv, d=d, page=16)
    check(kv, [0, 1, 2], [1, 1, 1], hq, decode=True)
    check(kv, [0], [1], hq, decode=True)
    check(kv, [2, 0], [1, 1], hq, 9000, 4, decode=True)


@pytest.mark.parametrize("hq,hkv,d,page,dtype", [(8, 1, 128, 64, F16), (8, 1, 64, 128, BF16), (16, 2, 64, 16, F16), (16, 1, 192, 32, BF16),
                                                 (4, 1, 256, 128, BF16), (16, 1, 256, 64, F16), (16, 1, 128, 16, BF16)])
def test_decode_many_tiles_per_cta(hq, hkv, d, page, dtype):
    """Enough key tiles for every stage of the ring to go round many times in each CTA."""
    kv = make([120_011, 60_000], hkv=hkv, d=d, page=page, dtype=dtype, layers=1, layer=0)
    check(kv, [0, 1], [1, 1], hq, layer=0, decode=True)
    check(kv, [1, 0], [1, 1], hq, 40_000, 70, layer=0, decode=True)


def test_decode_same_sequence_twice_and_repeatable():
    kv = make([3000, 17], hkv=2, d=128)
    q = query(4, 8, 128, BF16)
    a = kv.decode(1, q, ints([0, 0, 1, 0]))
    b = kv.decode(1, q, ints([0, 0, 1, 0]))
    kv.sync()
    assert torch.equal(a, b)            # nothing depends on the order in which the parts finish
    want, size = attention(kv, 1, q, [0, 0, 1, 0], [1] * 4)
    close(a, want, size)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), 3e38])
@pytest.mark.parametrize("decode", [True, False])
def test_hidden_values_have_no_influence(value, decode):
    """Keys and values that no query sees may hold anything: outside the window, past the end, in free pages."""
    lens, window, sinks = [500, 129, 64, 1], 70, 3
    kv = make(lens, hkv=2, d=64, page=16)
    counts = [1] * 4 if decode else [20, 1, 33, 1]
    for s, (n, c) in enumerate(zip(lens, counts)):
        first = max(sinks, n - c - window + 1)
        for j in range(sinks, first):
            p = int(kv.tables[s, j // 16])
            kv.pool[p, 1, :, :, j % 16] = value
    check(kv, [0, 1, 2, 3], counts, 8, window, sinks, decode=decode)


@pytest.mark.parametrize("hq,d,counts", [(8, 64, [40, 3]), (2, 128, [200, 100]), (4, 256, [30, 20]), (1, 64, [1, 1])])
def test_a_nan_key_reaches_the_queries_that_see_it_and_no_others(hq, d, counts):
    lens, at = [300, 150], [280, 120]
    kv = make(lens, hkv=1, d=d)
    q = query(sum(counts), hq, d, BF16)
    want, size = attention(kv, 1, q, [0, 1], counts)
    for s, j in enumerate(at):
        kv.pool[int(kv.tables[s, j // 16]), 1, 0, :, j % 16, 1] = float("nan")
    got = kv.extend(1, q, ints([0, 1]), starts_of(counts))
    kv.sync()
    t = 0
    for n, f, j in zip(lens, counts, at):
        pos = torch.arange(n - f, n, device=DEV)
        mine = slice(t, t + f)
        assert got[mine][pos >= j].isnan().all()
        close(got[mine][pos < j], want[mine][pos < j], size[mine][pos < j])
        t += f


@pytest.mark.parametrize("counts", [[1, 1], [50, 60]])
def test_infinite_scores(counts):
    """A score of plus infinity makes NaN of its rows as the formula does; one of minus infinity takes its key out."""
    kv = make([100, 90], hkv=1, d=64)
    kv.pool[int(kv.tables[0, 1]), 1, 0, :, 3] = torch.tensor(3e38, dtype=BF16, device=DEV)      # key 19 of sequence 0
    q = query(sum(counts), 4, 64, BF16).abs()
    q[:, 2:] = -q[:, 2:]
    got = kv.extend(1, q, ints([0, 1]), starts_of(counts))
    kv.sync()
    a = counts[0]
    assert got[:a, :2].isnan().all()
    keep = torch.ones(100, dtype=torch.bool, device=DEV)
    keep[19] = False
    k, v = kv_util.gathered(kv, 1, 0, 100)
    for t in range(a):
        n = 100 - a + t + 1
        w = torch.softmax((q[t, 2:].double() @ k[:n, 0].T / 8.0).masked_fill(~keep[:n], float("-inf")), -1)
        close(got[t:t + 1, 2:], (w @ v[:n, 0])[None], (w @ v[:n, 0].abs())[None])
    want, size = attention(kv, 1, q[a:], [1], counts[1:])
    close(got[a:], want, size)


def test_large_scores_and_scale():
    kv = make([700, 90], hkv=1, d=128)
    check(kv, [0, 1], [1, 1], 8, decode=True, scale=1.0)       # one key takes nearly all the weight
    check(kv, [0, 1], [33, 2], 8, scale=-0.3)
    check(kv, [0, 1], [1, 1], 8, decode=True, scale=0.0)       # all keys alike


# ---------------------------------------------------------------- attention of several new tokens
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hq,hkv,d,page", [(8, 2, 64, 16), (2, 2, 128, 16), (8, 1, 128, 8), (6, 2, 80, 32), (5, 1, 8, 64), (16, 1, 256, 16),
                                           (28, 4, 128, 128), (130, 1, 64, 16), (4, 4, 248, 64)])
def test_extend_heads_and_sizes(hq, hkv, d, page, dtype):
    lens = [1, 5, 16, 64, 129, 300, 700, 0, 128, 513]
    counts = [1, 5, 3, 64, 128, 1, 257, 0, 128, 200]
    kv = make(lens, hkv=hkv, d=d, page=page, dtype=dtype)
    check(kv, list(range(len(lens))), counts, hq)


@pytest.mark.parametrize("hq", [2, 6, 8, 32])
@pytest.mark.parametrize("counts", [[1, 1, 1], [2, 3, 1], [9, 0, 17], [40, 33, 64], [100, 127, 128], [300, 129, 1], [0, 0, 5]])
def test_extend_counts(hq, counts):
    kv = make([901, 130, 333], hkv=2, d=128)
    check(kv, [2, 1, 0], [min(c, x) for c, x in zip(counts, (333, 130, 901))], hq)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (16, 4), (127, 1), (128, 128), (129, 0), (300, 17), (5000, 4)])
@pytest.mark.parametrize("hq,d", [(8, 64), (4, 128)])
def test_extend_window_and_sinks(window, sinks, hq, d):
    kv = make([1000, 129, 400], hkv=2, d=d, page=16)
    check(kv, [0, 1, 2], [1000, 129, 70], hq, window, sinks)
    check(kv, [2, 0], [7, 3], hq, window, sinks)


@pytest.mark.parametrize("lens,counts,hq,hkv,d", [([5000], [5000], 8, 2, 128), ([9000, 100], [50, 100], 16, 2, 128), ([20000], [7], 8, 1, 64),
                                                  ([3000, 2000, 1000, 1], [3000, 100, 1000, 1], 4, 1, 64), ([2500], [2500], 2, 2, 256)])
def test_extend_long(lens, counts, hq, hkv, d):
    kv = make(lens, hkv=hkv, d=d)
    check(kv, list(range(len(lens))), counts, hq)
    check(kv, list(range(len(lens))), counts, hq, 700, 5)


@pytest.mark.parametrize("d,page,dtype", [(136, 16, BF16), (192, 64, F16), (200, 8, F16), (256, 128, BF16)])
def test_extend_wide_heads(d, page, dtype):
    kv = make([3001, 1, 64, 65, 700, 0, 128], hkv=2, d=d, page=page, dtype=dtype)
    seqs = list(range(7))
    check(kv, seqs, [500, 1, 64, 65, 700, 0, 127], 4)                # odd and even numbers of 64 keys, whole items and pieces
    check(kv, seqs, [2, 1, 3, 4, 129, 0, 128], 34, 100, 5)
    check(kv, [0], [9], 8)
    check(kv, [3, 4], [33, 300], 8, 1, 0)


@pytest.mark.parametrize("d", [128, 256])
@pytest.mark.parametrize("total", [63, 64, 65, 1023, 1024, 1025, 1100, 2049])
def test_items_about_the_length_that_is_cut(total, d):
    lens = [total] * 41 + [7 * total]                               # decode with 1 row a sequence, extend with 20
    kv = make(lens, hkv=1, d=d, page=64)
    seqs = list(range(42))
    check(kv, seqs, [1] * 42, 1, decode=True)
    check(kv, seqs, [5] * 42, 4)


def test_extend_many_sequences():
    rng = random.Random(5)
    lens = [rng.randint(0, 90) for _ in range(1300)]
    counts = [rng.randint(0, x) for x in lens]
    kv = make(lens, hkv=1, d=64)
    check(kv, list(range(1300)), counts, 4)


def test_extend_is_repeatable():
    kv = make([3000, 1700], hkv=2, d=128)
    q = query(3700, 8, 128, BF16)
    a = kv.extend(1, q, ints([0, 1]), starts_of([2500, 1200]))
    b = kv.extend(1, q, ints([0, 1]), starts_of([2500, 1200]))
    kv.sync()
    assert torch.equal(a, b)


def test_decode_is_extend_of_one():
    kv = make([3000, 17, 260], hkv=2, d=128)
    q = query(3, 8, 128, BF16)
    assert torch.equal(kv.decode(1, q, ints([0, 1, 2])), kv.extend(1, q, ints([0, 1, 2]), starts_of([1, 1, 1])))


# ---------------------------------------------------------------- layouts, streams, graphs
def test_strided_and_misaligned_arguments():
    kv = make([100, 33], hkv=2, d=64)
    both = query(2, 24, 64, BF16)                      # q, k and v of one projection, side by side
    q = both[:, :8]
    out = torch.zeros(2, 16, 64, dtype=BF16, device=DEV)
    kv.decode(1, q, ints([0, 1]), out=out[:, 4:12])
    want, size = attention(kv, 1, q, [0, 1], [1, 1])
    close(out[:, 4:12], want, size)
    assert not out[:, :4].any() and not out[:, 12:].any()
    odd = torch.zeros(2 * 8 * 64 + 1, dtype=BF16, device=DEV)[1:].view(2, 8, 64).copy_(q)      # 2-byte aligned
    assert torch.equal(kv.decode(1, odd, ints([0, 1])), kv.decode(1, q, ints([0, 1])))
    turned = q.permute(1, 0, 2).contiguous().permute(1, 0, 2)                                  # heads outermost
    assert torch.equal(kv.decode(1, turned, ints([0, 1])), kv.decode(1, q, ints([0, 1])))
    columns = q.permute(2, 0, 1).contiguous().permute(1, 2, 0)                                 # values of a row apart
    odd_out = torch.zeros(2 * 8 * 64 + 1, dtype=BF16, device=DEV)[1:].view(2, 8, 64)
    kv.decode(1, columns, ints([0, 1]), out=odd_out)
    assert torch.equal(odd_out, kv.decode(1, q, ints([0, 1])))


def test_strided_writes():
    from paper_2501_12689_b200 import ICPagedKV
    kv = ICPagedKV(8, 1, 2, 16, 64, 2, 4)
    kv.reserve(ints([1, 0]), ints([20, 3]))
    x = query(23, 8, 64, BF16)
    kv.write(0, x[:, 2:4], x[:, 6:8], ints([1, 0]), ints([0, 20, 23]))
    k, v = kv_util.gathered(kv, 0, 1, 20)
    assert torch.equal(k, x[:20, 2:4].double()) and torch.equal(v, x[:20, 6:8].double())
    odd = torch.zeros(2 * 2 * 64 + 1, dtype=BF16, device=DEV)[1:].view(2, 2, 64).copy_(x[:2, :2])
    kv.write(0, odd, x[:2, 3:5], ints([0, 1]))         # one token each: the newest
    k, v = kv_util.gathered(kv, 0, 0, 3)
    assert torch.equal(k[2], x[0, :2].double()) and torch.equal(v[2], x[0, 3:5].double()) and torch.equal(k[1], x[21, 2:4].double())
    kv.sync()


def test_other_streams():
    kv = make([2000, 100], hkv=2, d=128)
    q = query(2, 8, 128, BF16)
    want = kv.decode(1, q, ints([0, 1]))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    seqs = ints([0, 1])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        late = torch.zeros_like(q)
        torch.cuda._sleep(20_000_000)
        late.copy_(q)
        got = kv.decode(1, late, seqs)                 # waits for the copy on `side`
        del late
        again = got.clone()                            # and `side` waits for the result
    torch.cuda.synchronize()
    assert torch.equal(again, want)
    kv.set_stream(side)
    with torch.cuda.stream(side):
        assert torch.equal(kv.decode(1, q, seqs), want)
    kv.sync()


def test_step_in_a_graph():
    """reserve, write, decode and a beam reorder captured once and replayed: the lengths live on the device."""
    kv = make([40, 17, 30, 16], hkv=2, d=64, spare=60)
    model = Model(kv.n_pages, 16, 4, kv.max_pages)
    model.lens, model.refs = kv.lengths.tolist(), kv.refs.tolist()
    model.rows = [kv.tables[s, :-(-n // 16)].tolist() for s, n in enumerate(model.lens)]
    seqs, ones, parents = ints([0, 1, 2, 3]), ints([1, 1, 1, 1]), ints([0, 0, 3, 2])
    k, v, q = query(4, 2, 64, BF16, 3), query(4, 2, 64, BF16, 4), query(4, 8, 64, BF16, 5)
    side = torch.cuda.Stream()
    kv.set_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        kv.fork(parents, seqs)
        kv.reserve(seqs, ones)
        kv.write(1, k, v, seqs)
        out = kv.decode(1, q, seqs)
    for step in range(6):
        before = kv.pool.clone()
        graph.replay()
        torch.cuda.synchronize()
        moves = model.fork([0, 0, 3, 2], [0, 1, 2, 3])
        assert moves is not None and model.reserve([0, 1, 2, 3], [1] * 4)
        model.check(kv)
        want, size = attention(kv, 1, q, [0, 1, 2, 3], [1] * 4)
        close(out, want, size)
        for a, b in moves:                                     # copied pages are copies, but for the new token's slot
            same = (kv.pool[b, 0] == before[a, 0]) | (kv.pool[b, 0].isnan() & before[a, 0].isnan())
            assert same.all()
    kv.sync()


def test_offsets_beyond_32_bits():
    """A pool of more than 2**32 bytes and more than 2**31 elements, read, written and copied at its far end."""
    from paper_2501_12689_b200 import ICPagedKV
    n_pages, layers, hkv, page, d = 4200, 4, 8, 128, 128          # 2.2e9 elements, 8.8 GB
    kv = ICPagedKV(n_pages * 2, layers, hkv, page, d, 4, n_pages)
    assert kv.pool.numel() > 2 ** 32
    kv.reserve(ints([0]), ints([(2 * n_pages - 40) // 2 * page]))   # all but some pages are taken
    kv.reserve(ints([1]), ints([(2 * n_pages - 40 - (2 * n_pages - 40) // 2) * page]))
    kv.reserve(ints([2]), ints([1000]))
    k, v = query(1000, hkv, d, BF16, 7), query(1000, hkv, d, BF16, 8)
    kv.write(3, k, v, ints([2]), ints([0, 1000]))
    kv.sync()
    assert int(kv.tables[2, 0]) == 2 * n_pages - 40
    check(kv, [2], [1], 16, layer=3, decode=True)
    check(kv, [2], [1000], 8, layer=3)
    kv.fork(ints([2]), ints([3]), copy=True)
    kv.free(ints([2, 0]))
    kv.sync()
    a, b = kv_util.gathered(kv, 3, 3, 1000)
    assert torch.equal(a, k.double()) and torch.equal(b, v.double())
    kv.free(ints([1]))
    kv.compact()
    kv.sync()
    assert kv.tables[3, :8].tolist() == list(range(8))
    a, b = kv_util.gathered(kv, 3, 3, 1000)
    assert torch.equal(a, k.double()) and torch.equal(b, v.double())
    check(kv, [3], [1], 16, layer=3, decode=True)


# ---------------------------------------------------------------- page operations against the model
class Driver:
    """Runs the same calls on the library and on the model, with pool contents that name the page they were written for."""

    def __init__(self, n_pages, page, max_seqs, max_pages, layers=2, hkv=1, d=8):
        from paper_2501_12689_b200 import ICPagedKV
        pool = (torch.arange(n_pages, device=DEV) % 2048).view(-1, 1, 1, 1, 1, 1).expand(n_pages, layers, 2, hkv, page, d).to(F16).contiguous()
        self.kv = ICPagedKV(n_pages, layers, hkv, page, d, max_seqs, max_pages, dtype=F16, pool=pool)
        self.model = Model(n_pages, page, max_seqs, max_pages)
        self.stamp = [float(p % 2048) for p in range(n_pages)]       # whole numbers that fp16 holds

    def reserve(self, seqs, counts):
        fits = self.model.reserve(seqs, counts)
        self.kv.reserve(ints(seqs), ints(counts))
        return fits

    def fork(self, *a, **k):
        moves = self.model.fork(*a, **k)
        self.kv.fork(ints(a[0]), ints(a[1]), ints(a[2]) if len(a) > 2 and a[2] is not None else None, copy=k.get("copy", False))
        for x, y in moves or []:
            self.stamp[y] = self.stamp[x]
        return moves is not None

    def free(self, seqs):
        self.model.free(seqs)
        self.kv.free(ints(seqs))

    def compact(self):
        old = list(self.stamp)
        for x, y in self.model.compact():
            self.stamp[y] = old[x]
        self.kv.compact()

    def check(self):
        self.kv.sync()
        self.model.check(self.kv)
        got = self.kv.pool.float().flatten(1)
        want = torch.tensor(self.stamp, device=DEV)[:, None]
        assert (got == want).all()


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("n_pages,page,max_seqs,max_pages", [(61, 8, 9, 12), (300, 16, 40, 30), (1030, 32, 70, 64)])
def test_random_operations(seed, n_pages, page, max_seqs, max_pages):
    rng = random.Random(seed)
    d = Driver(n_pages, page, max_seqs, max_pages)
    for step in range(40):
        op = rng.choice(["reserve", "reserve", "fork", "beams", "copy", "free", "compact", "upto"])
        m = d.model
        live = [s for s in range(max_seqs) if m.lens[s]]
        if op == "reserve":
            who = rng.sample(range(max_seqs), rng.randint(1, max_seqs // 2))
            counts = [rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, 3 * page)]) for _ in who]
            if not Model.reserve(_copy(m), who, counts):
                continue
            assert d.reserve(who, counts)
        elif op == "free":
            d.free(rng.sample(range(max_seqs), rng.randint(1, max_seqs // 2)))
        elif op == "compact":
            d.compact()
        elif live:
            if op == "beams":
                who = rng.sample(live, rng.randint(1, len(live)))
                a = ([rng.choice(who) for _ in who], who)
            else:
                kids = rng.sample(range(max_seqs), rng.randint(1, max_seqs // 2))
                a = ([rng.choice(live) for _ in kids], kids)
            if op == "upto":
                a += ([rng.randint(0, m.lens[p]) for p in a[0]],)
            if Model.fork(_copy(m), *a, copy=op == "copy") is None:
                continue
            assert d.fork(*a, copy=op == "copy")
        if step % 5 == 4:
            d.check()
    d.check()


def _copy(m):
    c = Model(len(m.refs), m.page, len(m.lens), m.max_pages)
    c.refs, c.rows, c.lens = list(m.refs), [list(r) for r in m.rows], list(m.lens)
    return c


@pytest.mark.parametrize("n_pages,held", [(40000, 33000), (70001, 69990)])
def test_large_pools(n_pages, held):
    """More pages than one round of the planning kernels looks at, and more sequences than it has threads."""
    d = Driver(n_pages, 8, 1500, 3000, layers=1)
    rng = random.Random(n_pages)
    share = [8 * (held // 1100) - rng.randint(0, 7) for _ in range(1100)]
    assert d.reserve(list(range(1100)), share)
    d.check()
    d.free([s for s in range(1100) if s % 3 == 0])
    d.compact()
    d.check()
    assert d.fork([rng.choice(range(1, 1100, 3)) for _ in range(300)], list(range(1100, 1400)))
    assert d.reserve(list(range(0, 1400)), [rng.choice([0, 0, 1, 9]) for _ in range(1400)])
    d.check()


def test_zero_work():
    d = Driver(16, 8, 4, 4)
    none = ints([])
    d.kv.reserve(none, none)
    d.kv.free(none)
    d.kv.fork(none, none)
    d.kv.write(0, torch.empty(0, 1, 8, dtype=F16, device=DEV), torch.empty(0, 1, 8, dtype=F16, device=DEV), none)
    assert d.kv.decode(0, torch.empty(0, 4, 8, dtype=F16, device=DEV), none).shape == (0, 4, 8)
    assert d.kv.extend(0, torch.empty(0, 4, 8, dtype=F16, device=DEV), ints([1, 2]), ints([0, 0, 0])).shape == (0, 4, 8)
    d.compact()
    d.reserve([0, 1], [0, 5])
    d.fork([0, 2], [1, 3])              # empty parents: the children become empty
    d.compact()
    d.check()
    assert d.kv.lengths.tolist() == [0, 0, 0, 0]


# ---------------------------------------------------------------- refusals
def test_a_full_pool_changes_nothing_until_sync():
    from paper_2501_12689_b200 import IC_ERR_FULL, ICCacheError
    d = Driver(10, 8, 4, 8)
    assert d.reserve([0, 1], [30, 25])                 # 8 of 10 pages
    d.check()
    assert not d.reserve([2, 3], [8, 16])              # three more do not fit: neither gets any
    try:
        d.kv.free(ints([0]))                           # does nothing: either refused here or ignored on the device
    except ICCacheError as e:
        assert e.status == IC_ERR_FULL
    with pytest.raises(ICCacheError) as e:
        d.kv.sync()
    assert e.value.status == IC_ERR_FULL
    d.check()
    assert d.fork([0, 1], [2, 3])                      # two tails: the last pages
    d.check()
    assert not d.fork([0], [0], None, copy=True)       # its own pages would have to stand beside the copies
    with pytest.raises(ICCacheError) as e:
        d.kv.sync()
    assert e.value.status == IC_ERR_FULL
    d.check()
    d.free([1])
    d.check()


def test_a_full_row():
    from paper_2501_12689_b200 import IC_ERR_FULL, ICCacheError
    d = Driver(20, 8, 2, 3)
    assert d.reserve([0], [24])
    assert not d.reserve([1, 0], [1, 1])
    with pytest.raises(ICCacheError) as e:
        d.kv.sync()
    assert e.value.status == IC_ERR_FULL
    d.check()


@pytest.mark.parametrize("call", [
    lambda kv: kv.reserve(ints([0, 0]), ints([1, 1])),
    lambda kv: kv.reserve(ints([1, 4]), ints([1, 1])),
    lambda kv: kv.reserve(ints([1, -1]), ints([1, 1])),
    lambda kv: kv.reserve(ints([1]), ints([-1])),
    lambda kv: kv.fork(ints([0, 0]), ints([2, 2])),
    lambda kv: kv.fork(ints([7]), ints([2])),
    lambda kv: kv.fork(ints([0]), ints([9])),
    lambda kv: kv.fork(ints([0]), ints([2]), ints([13])),
    lambda kv: kv.fork(ints([0]), ints([2]), ints([-1])),
    lambda kv: kv.write(0, torch.zeros(1, 1, 8, dtype=F16, device=DEV), torch.zeros(1, 1, 8, dtype=F16, device=DEV), ints([5])),
    lambda kv: kv.write(0, torch.zeros(1, 1, 8, dtype=F16, device=DEV), torch.zeros(1, 1, 8, dtype=F16, device=DEV), ints([3])),
    lambda kv: kv.write(0, torch.zeros(3, 1, 8, dtype=F16, device=DEV), torch.zeros(3, 1, 8, dtype=F16, device=DEV), ints([0, 1]), ints([0, 1, 2])),
    lambda kv: kv.free(ints([3, 4])),
])
def test_bad_device_arguments_change_nothing(call):
    from paper_2501_12689_b200 import IC_ERR_INVALID, ICCacheError
    d = Driver(20, 8, 4, 4)
    assert d.reserve([0, 1], [12, 8])
    before = [x.clone() for x in (d.kv.tables, d.kv.lengths, d.kv.refs)]
    d.kv.sync()
    call(d.kv)
    with pytest.raises(ICCacheError) as e:
        d.kv.sync()
    assert e.value.status == IC_ERR_INVALID
    for a, b in zip(before, (d.kv.tables, d.kv.lengths, d.kv.refs)):
        assert torch.equal(a, b)
    assert d.reserve([2], [3])                         # the handle stays usable
    d.kv.sync()
    d.model.check(d.kv)


def test_bad_sequences_in_attention_are_reported():
    from paper_2501_12689_b200 import IC_ERR_INVALID, ICCacheError
    kv = make([100, 33], hkv=2, d=64)
    q = query(3, 8, 64, BF16)
    good = kv.decode(1, q[:1], ints([1]))
    got = kv.decode(1, q, ints([1, 2, -1]))
    with pytest.raises(ICCacheError) as e:
        kv.sync()
    assert e.value.status == IC_ERR_INVALID
    assert torch.equal(got[:1], good) and not got[1:].any()


def test_refused_arguments():
    from paper_2501_12689_b200 import IC_ERR_INVALID, IC_ERR_NOMEM, ICCacheError, ICPagedKV, ic_kv_workspace_bytes
    kv = make([20], hkv=2, d=64)
    q, s = query(1, 8, 64, BF16), ints([0])
    bad = [lambda: kv.decode(1, q.float(), s), lambda: kv.decode(1, q.to(F16), s), lambda: kv.decode(1, q[..., :32], s),
           lambda: kv.decode(1, q.cpu(), s), lambda: kv.decode(1, q, s.long()), lambda: kv.decode(1, q, s.cpu()),
           lambda: kv.decode(1, q, ints([0, 0])), lambda: kv.extend(1, q, s, ints([0])), lambda: kv.decode(1, q, s, out=q[:0]),
           lambda: kv.reserve(s, ints([1, 2])), lambda: kv.fork(s, ints([0, 1])), lambda: kv.write(1, q, q, s),
           lambda: kv.write(1, q[:, :2], q[:, :1], s)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"case {i} was accepted")
    for f in (lambda: kv.decode(2, q, s), lambda: kv.decode(-1, q, s), lambda: kv.decode(1, q[:, :3], s), lambda: kv.decode(1, q, s, window=-1),
              lambda: kv.decode(1, q, s, window=4, sinks=-1), lambda: kv.decode(1, q, s, scale=float("nan")),
              lambda: kv.write(2, q[:, :2], q[:, :2], s)):
        with pytest.raises(ICCacheError) as e:
            f()
        assert e.value.status == IC_ERR_INVALID
    for n_pages, layers, hkv, page, d, seqs, row in ((0, 1, 1, 16, 64, 1, 1), (1, 0, 1, 16, 64, 1, 1), (1, 1, 1, 12, 64, 1, 1),
                                                     (1, 1, 1, 16, 63, 1, 1), (1, 1, 1, 16, 264, 1, 1), (1, 1, 1, 16, 64, 0, 1),
                                                     (1, 1, 1, 16, 64, 1, 0), (1, 1, 1, 512, 64, 1, 1), (1, 1, 1, 16, 64, 20000, 1)):
        with pytest.raises(ICCacheError):
            ICPagedKV(n_pages, layers, hkv, page, d, seqs, row)
    with pytest.raises(TypeError):
        ICPagedKV(1, 1, 1, 16, 64, 1, 1, dtype=torch.float32)
    with pytest.raises(ValueError):
        ICPagedKV(4, 1, 1, 16, 64, 1, 1, refs=torch.zeros(5, dtype=torch.int32, device=DEV))
    need = ic_kv_workspace_bytes(4, 1, 1, 16, 64, 2, 2)
    with pytest.raises(ICCacheError) as e:
        ICPagedKV(4, 1, 1, 16, 64, 2, 2, workspace=torch.empty(need - 256, dtype=torch.uint8, device=DEV))
    with ICPagedKV(4, 1, 1, 16, 64, 2, 2, workspace=torch.empty(need, dtype=torch.uint8, device=DEV)) as lent:
        lent.reserve(ints([0, 1]), ints([17, 5]))
        lent.sync()
        assert lent.lengths.tolist() == [17, 5] and lent.tables[:, 0].tolist() == [0, 2]
    assert IC_ERR_NOMEM and kv.launch_count > 0
    kv.close()
    with pytest.raises(ValueError):
        kv.compact()


def test_borrowed_state_is_taken_over():
    from paper_2501_12689_b200 import ICPagedKV
    kv = make([100, 33], hkv=2, d=64)
    q = query(2, 8, 64, BF16)
    want = kv.decode(1, q, ints([0, 1]))
    kv.sync()
    other = ICPagedKV(kv.n_pages, 2, 2, 16, 64, 2, kv.max_pages, pool=kv.pool.clone(), tables=kv.tables.clone(), lengths=kv.lengths.clone(),
                      refs=kv.refs.clone())
    assert torch.equal(other.decode(1, q, ints([0, 1])), want)
    other.reserve(ints([1]), ints([40]))
    other.sync()
    assert len(set(other.tables[0, :7].tolist() + other.tables[1, :5].tolist())) == 12
