"""The paged key-value cache where calls go wrong or reach the ends of a type's range: refused and reported calls leave no trace,
small weights keep their value, and calls of mixed lengths, in place, on other streams and in graphs agree with the formula."""
import ctypes

import pytest
import torch

import kv_util
from kv_util import attention, close
from test_gpu_paged_kv import BF16, DEV, F16, check, ints, make, query, starts_of

pytestmark = pytest.mark.gpu


def reported(kv):
    """The error that the kernels found, cleared."""
    from paper_2501_12689_b200 import ICCacheError
    with pytest.raises(ICCacheError) as e:
        kv.sync()
    return e.value.status


# ---------------------------------------------------------------- lent books that are not a cache's
class Lent:
    """A small cache in lent tensors, each in the middle of a larger one: what surrounds them must stay.  Sequences 0, 1 and 2 of 12, 8
    and 27 tokens, sequence 3 empty; max_pages decides how many launches a fork of three takes."""

    def __init__(self, max_pages):
        from paper_2501_12689_b200 import ICPagedKV
        n_pages, layers, page, d, rows, edge = 24, 2, 8, 8, 4, 1024
        self.cap = max_pages * page
        self.all = {"tables": torch.full((rows * max_pages + 2 * edge,), -77, dtype=torch.int32, device=DEV),
                    "lengths": torch.full((rows + 2 * edge,), -77, dtype=torch.int32, device=DEV),
                    "refs": torch.full((n_pages + 2 * edge,), -77, dtype=torch.int32, device=DEV)}
        inner = {name: t[edge:-edge].zero_() for name, t in self.all.items()}
        around = torch.randn(n_pages + 16, layers, 2, 1, page, d, device=DEV, generator=torch.Generator(device=DEV).manual_seed(5)).to(F16)
        self.all["pool"] = around
        self.kv = ICPagedKV(n_pages, layers, 1, page, d, rows, max_pages, dtype=F16, pool=around[8:-8], tables=inner["tables"].view(rows, max_pages),
                            lengths=inner["lengths"], refs=inner["refs"])
        self.kv.reserve(ints([0, 1, 2]), ints([12, 8, 27]))
        self.kv.fork(ints([2]), ints([3]), ints([16]))          # pages 3 and 4 twice
        self.kv.free(ints([3]))
        self.kv.sync()
        self.keep()

    def keep(self):
        self.before = {name: t.clone() for name, t in self.all.items()}

    def unchanged(self):
        return all(torch.equal(t, self.before[name]) for name, t in self.all.items())


LENT = pytest.mark.parametrize("max_pages", [4, 4096])          # (a fork of three rows in two launches, and in three)


@LENT
@pytest.mark.parametrize("length", [1, -1, 2 ** 31 - 1, -2 ** 31])
def test_lengths_that_no_row_holds(max_pages, length):
    from paper_2501_12689_b200 import IC_ERR_INVALID
    x = Lent(max_pages)
    kv = x.kv
    kv.lengths[1] = length = x.cap + 1 if length == 1 else length
    x.keep()
    one = torch.ones(1, 1, 8, dtype=F16, device=DEV)
    for call in (lambda: kv.reserve(ints([1]), ints([1])), lambda: kv.reserve(ints([0, 1]), ints([1, 0])),
                 lambda: kv.fork(ints([1]), ints([3])), lambda: kv.fork(ints([1]), ints([3]), ints([3])), lambda: kv.fork(ints([0]), ints([1])),
                 lambda: kv.fork(ints([0, 1, 2]), ints([2, 3, 0])), lambda: kv.fork(ints([0, 2, 0]), ints([0, 1, 3]), copy=True),
                 lambda: kv.compact(), lambda: kv.free(ints([1])), lambda: kv.free(ints([1, 1])), lambda: kv.write(0, one, one, ints([1])),
                 lambda: kv.decode(0, one, ints([1])), lambda: kv.extend(0, one.expand(20, 1, 8), ints([1]), ints([0, 20]))):
        call()
        assert reported(kv) == IC_ERR_INVALID
        assert x.unchanged()
    kv.free(ints([1, 0]))                                       # the others are given back
    assert reported(kv) == IC_ERR_INVALID
    assert kv.lengths.tolist() == [0, length, 27, 0] and kv.refs[:3].tolist() == [0, 0, 1] and kv.refs[3:7].tolist() == [1] * 4
    kv.lengths[1] = 8                                           # as it was: all is well again
    kv.free(ints([1]))
    kv.compact()
    kv.sync()
    assert kv.lengths.tolist() == [0, 0, 27, 0] and kv.tables[2, :4].tolist() == [3, 0, 1, 2]


ENTRIES = pytest.mark.parametrize("entry", [-1, 24, 2 ** 31 - 1, -2 ** 31])


@LENT
@ENTRIES
@pytest.mark.parametrize("at", [0, 1, 3])                       # shared pages of sequence 2, and its last one, which is copied
def test_a_fork_of_entries_that_name_no_page(max_pages, entry, at):
    from paper_2501_12689_b200 import IC_ERR_INVALID
    x = Lent(max_pages)
    kv = x.kv
    right = int(kv.tables[2, at])
    kv.tables[2, at] = entry
    x.keep()
    for call in (lambda: kv.fork(ints([2]), ints([3])), lambda: kv.fork(ints([2]), ints([3]), copy=True),
                 lambda: kv.fork(ints([0, 2, 1]), ints([1, 3, 0])), lambda: kv.fork(ints([2, 2, 2]), ints([0, 1, 2]), copy=True),
                 lambda: kv.fork(ints([0]), ints([2])), lambda: kv.fork(ints([0, 0, 1]), ints([2, 3, 0]), copy=True),
                 lambda: kv.fork(ints([2]), ints([2]), ints([26]))):
        call()
        assert reported(kv) == IC_ERR_INVALID
        assert x.unchanged()
    kv.fork(ints([2, 2]), ints([3, 2]), ints([8 * at, 27]))     # what does not reach the entry is not concerned
    kv.sync()
    assert kv.lengths.tolist() == [12, 8, 27, 8 * at] and kv.tables[3, :at].tolist() == kv.tables[2, :at].tolist()
    kv.fork(ints([1]), ints([3]), ints([0]))
    kv.tables[2, at] = right
    kv.fork(ints([2]), ints([3]))
    kv.sync()
    a, b = kv_util.gathered(kv, 1, 2, 27), kv_util.gathered(kv, 1, 3, 27)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert torch.equal(x.all["pool"][:8], x.before["pool"][:8]) and torch.equal(x.all["pool"][-8:], x.before["pool"][-8:])


@LENT
@ENTRIES
def test_other_calls_on_entries_that_name_no_page(max_pages, entry):
    """free leaves such an entry alone, and write the token."""
    from paper_2501_12689_b200 import IC_ERR_INVALID
    x = Lent(max_pages)
    kv = x.kv
    kv.tables[2, 3] = entry
    x.keep()
    one = torch.ones(1, 1, 8, dtype=F16, device=DEV)
    kv.write(0, one, one, ints([2]))
    assert reported(kv) == IC_ERR_INVALID
    assert x.unchanged()
    kv.free(ints([2, 0]))
    assert reported(kv) == IC_ERR_INVALID
    assert kv.lengths.tolist() == [0, 8, 0, 0] and kv.refs.tolist() == [0, 0, 1, 0, 0, 0, 1] + [0] * 17


@LENT
@ENTRIES
@pytest.mark.parametrize("at", [0, 3])
def test_attention_over_entries_that_name_no_page(max_pages, entry, at):
    from paper_2501_12689_b200 import IC_ERR_INVALID
    x = Lent(max_pages)
    kv = x.kv
    kv.tables[2, at] = entry
    x.keep()
    one = torch.ones(1, 1, 8, dtype=F16, device=DEV)
    for call in (lambda: kv.decode(0, one, ints([2])), lambda: kv.extend(0, one.expand(27, 1, 8), ints([2]), ints([0, 27]))):
        call()
        assert reported(kv) == IC_ERR_INVALID
        assert x.unchanged()


@LENT
@pytest.mark.parametrize("entry", [-1, 24, 2 ** 31 - 1, -2 ** 31, 23])      # no page, and one that nobody holds
def test_compaction_of_entries_that_do_not_move(max_pages, entry):
    from paper_2501_12689_b200 import IC_ERR_INVALID
    x = Lent(max_pages)
    kv = x.kv
    kv.free(ints([0]))                                          # 0 and 1 are free: pages 5 and 6 move there
    kv.tables[1, 0] = entry
    pages = kv.pool.clone()
    kv.compact()
    assert reported(kv) == IC_ERR_INVALID
    assert kv.tables[1, 0] == entry and kv.tables[2, :4].tolist() == [3, 4, 0, 1] and kv.lengths.tolist() == [0, 8, 27, 0]
    assert kv.refs.tolist() == [1] * 5 + [0] * 19
    assert torch.equal(kv.pool[:2], pages[5:7]) and torch.equal(kv.pool[2:], pages[2:])
    for name, edge in (("tables", 1024), ("lengths", 1024), ("refs", 1024), ("pool", 8)):
        assert torch.equal(x.all[name][:edge], x.before[name][:edge]) and torch.equal(x.all[name][-edge:], x.before[name][-edge:])


# ---------------------------------------------------------------- after an error
@pytest.mark.parametrize("counts", [[1, 1], [9, 7]])    # either kernel
def test_an_error_that_is_cleared_leaves_nothing_in_the_scratch(counts):
    """A kernel that gives up in the middle leaves counts of arrived pieces behind (the words after the first 256 bytes of the
    workspace).  Once the error is reported and cleared, attention that is split over the length is right again: with counts
    that are too high nobody would join the pieces, and the result would not be written."""
    from paper_2501_12689_b200 import IC_ERR_INVALID, ICPagedKV, ic_kv_workspace_bytes
    made = make([30_000, 7], hkv=1, d=64)
    sizes = (made.n_pages, 2, 1, 16, 64, 2, made.max_pages)
    space = torch.zeros(ic_kv_workspace_bytes(*sizes), dtype=torch.uint8, device=DEV)
    kv = ICPagedKV(*sizes, pool=made.pool, tables=made.tables, lengths=made.lengths, refs=made.refs, workspace=space)
    space[256:256 + 2 * 160 * 4].view(torch.int32).fill_(1000)
    kv.reserve(ints([5]), ints([1]))                    # no such sequence
    assert reported(kv) == IC_ERR_INVALID
    q = query(sum(counts), 8, 64, BF16)
    out = torch.full_like(q, float("nan"))
    kv.extend(1, q, ints([0, 1]), starts_of(counts), out=out)
    kv.sync()
    want, size = attention(kv, 1, q, [0, 1], counts)
    close(out, want, size)


# ---------------------------------------------------------------- range of the weights
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("gap", [12.0, 15.0, 16.0, 17.0, 17.5, 18.0])
@pytest.mark.parametrize("group,count", [(2, 1), (16, 1), (4, 10)])
def test_one_key_far_above_many(group, count, gap, dtype):
    """A key whose score lies `gap` above 6,000 others and whose value is zero: the result is what the others add up to.  37
    sequences of 4 kv heads are an item per SM, so that no join gives the others a maximum of their own.

    The bound of `close` holds weights that are rounded once, to a unit roundoff of themselves.  In fp16 that takes a factor:
    18 is 26 powers of two, and a weight of 2**-26 is nothing.  With 2**15, as single tokens have it, it is off by 2**-14 of
    itself at most.  With 2**7 it stands at 2**-19, 32 steps of 2**-24, and is off by up to 2**-6, but each by its own share: the
    spread of 0.3 nats goes over ten steps, and the mean of 6,000 such errors is 2**-6 / sqrt(3 * 6000) = 1.2e-4, a tenth of
    the bound of 2 u + 2e-4."""
    n, hkv, d = 6000, 4, 64
    kv = make([n] * 37, hkv=hkv, d=d, page=64, layers=1, layer=0, dtype=dtype, poison=False)
    g = torch.Generator(device=DEV).manual_seed(3)
    kv.pool[:, 0, 0] = 0.0
    kv.pool[:, 0, 0, :, :, 1] = (0.3 * torch.randn(kv.n_pages, hkv, 64, device=DEV, generator=g)).to(dtype)
    kv.pool[:, 0, 1] = (0.5 + torch.rand(kv.n_pages, hkv, 64, d, device=DEV, generator=g)).to(dtype)
    first = kv.tables[:, 0].long()
    kv.pool[first, 0, 0, :, 0, 0] = gap
    kv.pool[first, 0, 1, :, 0] = 0.0
    seqs, counts = list(range(37)), [count] * 37
    q = torch.zeros(37 * count, hkv * group, d, dtype=dtype, device=DEV)
    q[..., :2] = 1.0
    if count == 1:
        got = kv.decode(0, q, ints(seqs), scale=1.0)
    else:
        got = kv.extend(0, q, ints(seqs), starts_of(counts), scale=1.0)
    kv.sync()
    want, size = attention(kv, 0, q, seqs, counts, scale=1.0)
    close(got, want, size)


# ---------------------------------------------------------------- starts that do not cover the tokens
@pytest.mark.parametrize("n", [2, 300])                 # (one launch, and two)
@pytest.mark.parametrize("group", [1, 40])              # either kernel
@pytest.mark.parametrize("wrong", ["begin", "end", "past"])
def test_starts_that_do_not_cover_the_tokens_are_reported(n, group, wrong):
    from paper_2501_12689_b200 import IC_ERR_INVALID
    kv = make([5] * n, hkv=1, d=64)
    starts = starts_of([1] * n)
    q = query(n, group, 64, BF16)
    good = kv.extend(1, q, ints(list(range(n))), starts)
    kv.sync()
    if wrong == "begin":
        starts[0] = 1
    elif wrong == "end":
        starts[n] = n - 1
    else:
        starts[n] = n + 1
    got = kv.extend(1, q, ints(list(range(n))), starts)
    assert reported(kv) == IC_ERR_INVALID
    assert torch.equal(got[1:n - 1], good[1:n - 1])
    assert torch.equal(kv.extend(1, q, ints(list(range(n))), starts_of([1] * n)), good)
    kv.sync()


def test_more_tokens_than_32_bits_are_refused():
    from paper_2501_12689_b200 import IC_ERR_INVALID, paged_kv
    kv = make([5], hkv=1, d=64)
    q, seqs, starts = query(1, 4, 64, BF16), ints([0]), ints([0, 1])
    a = paged_kv.ic_kv_attend_t()
    a.struct_size = ctypes.sizeof(a)
    a.layer, a.n, a.n_heads, a.n_tokens, a.scale = 1, 1, 4, 1 << 62, 1.0       # times 4 heads: 0 in 64 bits
    a.q = a.out = q.data_ptr()
    a.q_token_stride = a.out_token_stride = 256
    a.q_head_stride = a.out_head_stride = 64
    a.seqs, a.starts = seqs.data_ptr(), starts.data_ptr()
    assert kv._lib.ic_kv_attend(kv._h, ctypes.byref(a)) == IC_ERR_INVALID
    a.n_tokens = 1
    assert kv._lib.ic_kv_attend(kv._h, ctypes.byref(a)) == 0
    kv.sync()


# ---------------------------------------------------------------- a write that is refused on the device
@pytest.mark.parametrize("seqs,starts", [
    ([0, 5, 1], [0, 8, 20, 40]),            # no such sequence
    ([0, -1, 1], [0, 8, 20, 40]),
    ([0, 3, 1], [0, 8, 20, 40]),            # an empty sequence has no 12 tokens
    ([0, 1, 2], [0, 8, 20, 39]),            # a token too few
    ([0, 1, 2], [0, 8, 20, 41]),            # and too many
    ([0, 1, 2], [1, 8, 20, 40]),
    ([0, 1, 2], [0, 20, 8, 40]),
    ([0, 1, 2], [0, -8, 20, 40]),
    ([0, 1, 2], [0, 31, 31, 40]),           # more than sequence 0 has
])
@pytest.mark.parametrize("many", [1, 40])
def test_a_write_that_is_reported_stores_nothing(seqs, starts, many):
    """`many`: how often the 40 tokens are repeated, each time in sequences of their own; the fault is in the last ones."""
    from paper_2501_12689_b200 import IC_ERR_INVALID, ICPagedKV
    rows = 3 * many + 1
    kv = ICPagedKV(rows * 8, 2, 2, 8, 16, rows, 8, dtype=F16, pool=torch.zeros(rows * 8, 2, 2, 2, 8, 16, dtype=F16, device=DEV))
    kv.reserve(ints(list(range(rows - 1))), ints([30] * (rows - 1)))
    good_seqs = [3 * i + s for i in range(many) for s in (0, 1, 2)]
    good_starts = [0]
    for c in [8, 12, 20] * many:
        good_starts.append(good_starts[-1] + c)
    base, at = 3 * (many - 1), 40 * (many - 1)
    bad_seqs = good_seqs[:-3] + [base + s if 0 <= s < 3 else (rows - 1 if s == 3 else (rows + 1 if s > 0 else s)) for s in seqs]
    bad_starts = good_starts[:-4] + [at + s for s in starts]
    if many > 1 and starts[0] == 1:
        bad_starts = [1] + good_starts[1:]              # the first of all starts
    elif many > 1 and starts[1] < 0:
        bad_starts[-3] = at - 8                         # below the start before it
    k, v = query(40 * many, 2, 16, F16, 7) + 9.0, query(40 * many, 2, 16, F16, 8) - 9.0
    kv.write(1, k, v, ints(bad_seqs), ints(bad_starts))
    assert reported(kv) == IC_ERR_INVALID
    assert not kv.pool.any()
    kv.write(1, k, v, ints(good_seqs), ints(good_starts))
    kv.sync()
    for s in (0, 1, 2, base, base + 2):
        i = good_seqs.index(s)
        c = good_starts[i + 1] - good_starts[i]
        a, b = kv_util.gathered(kv, 1, s, 30)
        assert torch.equal(a[30 - c:], k[good_starts[i]:good_starts[i + 1]].double()) and not a[:30 - c].any()
        assert torch.equal(b[30 - c:], v[good_starts[i]:good_starts[i + 1]].double()) and not b[:30 - c].any()


@pytest.mark.parametrize("n", [1, 700, 5000])
def test_a_write_of_single_tokens_that_is_reported_stores_nothing(n):
    from paper_2501_12689_b200 import IC_ERR_INVALID, ICPagedKV
    kv = ICPagedKV(n + 1, 1, 1, 8, 16, n + 1, 1, dtype=F16, pool=torch.zeros(n + 1, 1, 2, 1, 8, 16, dtype=F16, device=DEV))
    kv.reserve(ints(list(range(n))), ints([1] * n))
    k = query(n, 1, 16, F16) + 9.0
    for last in (n, n + 1, -7):                         # an empty sequence, and none
        kv.write(0, k, k, ints(list(range(n - 1)) + [last]))
        assert reported(kv) == IC_ERR_INVALID
        assert not kv.pool.any()
    kv.write(0, k, k, ints(list(range(n))))
    kv.sync()
    at = kv.tables[:n, 0].long()
    assert torch.equal(kv.pool[at, 0, 0, 0, 0], k[:, 0]) and torch.equal(kv.pool[at, 0, 1, 0, 0], k[:, 0])


@pytest.mark.parametrize("n", [255, 257, 600, 4099])
def test_writes_of_many_ragged_sequences(n):
    from paper_2501_12689_b200 import ICPagedKV
    g = torch.Generator().manual_seed(n)
    counts = torch.randint(0, 4, (n,), generator=g)
    counts[n // 2] = 45
    seqs = torch.randperm(n, generator=g)
    kv = ICPagedKV(7 * n, 1, 1, 8, 8, n, 8, dtype=F16)
    had = torch.randint(0, 12, (n,), generator=g)
    kv.reserve(ints(list(range(n))), ints(had.tolist()))
    kv.reserve(ints(seqs.tolist()), ints(counts.tolist()))
    k, v = query(int(counts.sum()), 1, 8, F16, 7), query(int(counts.sum()), 1, 8, F16, 8)
    kv.write(0, k, v, ints(seqs.tolist()), starts_of(counts.tolist()))
    kv.sync()
    who = seqs.repeat_interleave(counts).to(DEV)
    first = (counts.cumsum(0) - counts).repeat_interleave(counts)
    pos = had[who.cpu()].to(DEV) + (torch.arange(len(who)) - first).to(DEV)
    page = kv.tables[who, pos // 8].long()
    assert torch.equal(kv.pool[page, 0, 0, 0, pos % 8], k[:, 0]) and torch.equal(kv.pool[page, 0, 1, 0, pos % 8], v[:, 0])


# ---------------------------------------------------------------- where results go
@pytest.mark.parametrize("size,stride", [
    ((3, 8, 64), (0, 64, 1)), ((3, 8, 64), (512, 0, 1)), ((3, 8, 64), (512, 32, 1)), ((3, 8, 64), (64, 64, 1)), ((3, 8, 64), (448, 64, 1)),
    ((3, 8, 64), (64, 128, 1)), ((3, 8, 64), (192, 136, 1))])
def test_results_that_overlap_are_refused(size, stride):
    from paper_2501_12689_b200 import IC_ERR_INVALID, ICCacheError
    kv = make([100, 33, 5], hkv=2, d=64)
    q = query(3, 8, 64, BF16)
    out = torch.zeros(5000, dtype=BF16, device=DEV).as_strided(size, stride)
    with pytest.raises(ICCacheError) as e:
        kv.decode(1, q, ints([0, 1, 2]), out=out)
    assert e.value.status == IC_ERR_INVALID
    kv.sync()


@pytest.mark.parametrize("stride", [(64, 192, 1), (512, 64, 1), (192, 576, 1), (128, 448, 1), (256, 64 * 12 + 128, 1)])
def test_results_that_interleave_are_taken(stride):
    """Heads outermost, or tokens and heads in turn, with no value in common."""
    kv = make([100, 33, 5], hkv=2, d=64)
    q = query(3, 8, 64, BF16)
    out = torch.zeros(9000, dtype=BF16, device=DEV).as_strided((3, 8, 64), stride)
    kv.decode(1, q, ints([0, 1, 2]), out=out)
    assert torch.equal(out, kv.decode(1, q, ints([0, 1, 2])))
    kv.sync()


def test_results_of_one_token_or_head_may_have_any_stride():
    kv = make([100], hkv=1, d=64)
    q = query(1, 4, 64, BF16)
    out = torch.zeros(256, dtype=BF16, device=DEV).as_strided((1, 4, 64), (0, 64, 1))
    kv.decode(1, q, ints([0]), out=out)
    assert torch.equal(out, kv.decode(1, q, ints([0])))
    one = torch.zeros(64, dtype=BF16, device=DEV).as_strided((1, 1, 64), (0, 0, 1))
    kv.decode(1, q[:, :1], ints([0]), out=one)
    assert torch.equal(one, kv.decode(1, q[:, :1], ints([0])))
    kv.sync()


@pytest.mark.parametrize("lens,counts,hq,hkv,d", [([3000, 17, 700], [1, 1, 1], 8, 2, 128), ([40_001, 5], [1, 1], 8, 1, 64),
                                                  ([3000, 170, 700], [300, 160, 7], 8, 2, 128), ([9000, 100], [50, 100], 16, 2, 256)])
def test_results_in_the_place_of_the_queries(lens, counts, hq, hkv, d):
    kv = make(lens, hkv=hkv, d=d)
    seqs = ints(list(range(len(lens))))
    q = query(sum(counts), hq, d, BF16)
    want = kv.extend(1, q, seqs, starts_of(counts))
    got = kv.extend(1, q, seqs, starts_of(counts), out=q)
    kv.sync()
    assert got is q and torch.equal(q, want)


# ---------------------------------------------------------------- many handles
def test_many_handles_at_once():
    """More than a thousand caches; an error stays with the one that met it."""
    from paper_2501_12689_b200 import IC_ERR_FULL, ICPagedKV, ic_kv_workspace_bytes
    sizes = (2, 1, 1, 8, 8, 1, 2)
    space = torch.empty(ic_kv_workspace_bytes(*sizes), dtype=torch.uint8, device=DEV)      # lent to all, as they are used in turn
    all_of = [ICPagedKV(*sizes, dtype=F16, workspace=space) for _ in range(2100)]
    for i in (0, 1023, 1024, 2099):
        all_of[i].reserve(ints([0]), ints([9]))
        all_of[i].sync()
        all_of[i].reserve(ints([0]), ints([9]))
        assert reported(all_of[i]) == IC_ERR_FULL
    for i in (1, 1022, 1025, 2098):
        all_of[i].sync()
    for kv in all_of:
        kv.close()
    with ICPagedKV(*sizes, dtype=F16, workspace=space) as kv:
        kv.reserve(ints([0]), ints([9]))
        kv.sync()


def test_a_scale_that_leaves_the_range_is_refused():
    """The softmax works in powers of two: scale * log2(e) has to be a finite number."""
    from paper_2501_12689_b200 import IC_ERR_INVALID, ICCacheError
    kv = make([40], hkv=1, d=64)
    q = torch.zeros(1, 4, 64, dtype=BF16, device=DEV)
    for scale in (2.5e38, -3e38):
        with pytest.raises(ICCacheError) as e:
            kv.decode(1, q, ints([0]), scale=scale)
        assert e.value.status == IC_ERR_INVALID
    got = kv.decode(1, q, ints([0]), scale=2e38)        # scores of zero, whatever the scale: the mean of the values
    want, size = attention(kv, 1, q, [0], [1], scale=2e38)
    kv.sync()
    close(got, want, size)


# ---------------------------------------------------------------- calls of many kinds
@pytest.mark.parametrize("singles,prompt,hq,hkv,d", [(255, 512, 8, 2, 128), (60, 1500, 8, 2, 64), (3, 900, 4, 1, 256), (300, 40, 8, 2, 128)])
def test_single_tokens_and_a_prompt_in_one_call(singles, prompt, hq, hkv, d):
    """A serving step: what a sequence gets does not depend on the others beyond the rounding of its weights."""
    rng = torch.Generator().manual_seed(singles)
    lens = torch.randint(1, 700, (singles,), generator=rng).tolist()
    at = singles // 2
    lens.insert(at, prompt + 100)
    counts = [1] * (singles + 1)
    counts[at] = prompt
    kv = make(lens, hkv=hkv, d=d)
    seqs = list(range(singles + 1))
    check(kv, seqs, counts, hq)
    check(kv, seqs, counts, hq, 200, 4)


def test_a_token_by_either_kernel():
    """One token alone, and in a call whose average takes the other kernel."""
    kv = make([3000, 500], hkv=2, d=128)
    q = query(201, 8, 128, BF16)
    alone = kv.decode(1, q[:1], ints([0]))
    among = kv.extend(1, q, ints([0, 1]), ints([0, 1, 201]))[:1]
    kv.sync()
    want, size = attention(kv, 1, q[:1], [0], [1])
    close(alone, want, size)
    close(among, want, size)


@pytest.mark.parametrize("hq,hkv,d,n", [(32, 1, 128, 40_001), (128, 1, 64, 30_000), (64, 2, 256, 20_011), (24, 1, 192, 131_071)])
def test_decode_of_many_heads_over_a_long_cache(hq, hkv, d, n):
    kv = make([n, 300], hkv=hkv, d=d, layers=1, layer=0, page=64)
    check(kv, [0, 1], [1, 1], hq, layer=0, decode=True)
    check(kv, [1, 0], [1, 1], hq, 9000, 4, layer=0, decode=True)


def test_extend_on_another_stream():
    kv = make([2000, 100], hkv=2, d=128)
    q, seqs, starts = query(90, 8, 128, BF16), ints([0, 1]), ints([0, 70, 90])
    want = kv.extend(1, q, seqs, starts)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        late = torch.zeros_like(q)
        torch.cuda._sleep(20_000_000)
        late.copy_(q)
        got = kv.extend(1, late, seqs, starts)
        del late
        again = got.clone()
    torch.cuda.synchronize()
    assert torch.equal(again, want)
    kv.sync()


def test_extend_in_a_graph():
    """Drafted tokens: reserve, write and extend captured once and replayed, the lengths growing on the device."""
    kv = make([400, 17, 3000], hkv=2, d=64, spare=60)
    seqs, counts, starts = ints([0, 1, 2]), ints([9, 9, 9]), ints([0, 9, 18, 27])
    k, v, q = query(27, 2, 64, BF16, 3), query(27, 2, 64, BF16, 4), query(27, 8, 64, BF16, 5)
    side = torch.cuda.Stream()
    kv.set_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        kv.reserve(seqs, counts)
        kv.write(1, k, v, seqs, starts)
        out = kv.extend(1, q, seqs, starts)
    for step in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert kv.lengths.tolist() == [400 + 9 * (step + 1), 17 + 9 * (step + 1), 3000 + 9 * (step + 1)]
        want, size = attention(kv, 1, q, [0, 1, 2], [9, 9, 9])
        close(out, want, size)
    kv.sync()
