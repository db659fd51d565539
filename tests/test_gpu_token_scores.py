"""Log-probabilities, entropy and top alternatives on the GPU against their formulas in 64 bits."""
import math

import pytest
import torch

from paper_2501_12689_b200 import IC_ERR_INVALID, ICCacheError, ICTokenScores, IC_SCORE_MAX_TOP

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
INF = math.inf


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def draw(rows, vocab, dtype, seed=0, banned=0.0, spread=2.5):
    x = spread * torch.randn(rows, vocab, device=DEV, generator=gen(seed))
    if banned:
        x.masked_fill_(torch.rand(rows, vocab, device=DEV, generator=gen(seed + 1)) < banned, -INF)
    return x.to(dtype)


def check(x, n_top, scale=1.0, targets="some", scores=None, seed=0):
    rows, vocab = x.shape
    s = scores or ICTokenScores(vocab, dtype=x.dtype)
    t = torch.randint(-1, vocab, (rows,), device=DEV, generator=gen(seed + 7), dtype=torch.int32) if isinstance(targets, str) else targets
    got = s.score(x, t, n_top=n_top, scale=scale)
    s.sync()
    y = x.double() * torch.tensor(scale, dtype=F32).double().item()
    top = y.amax(-1, keepdim=True)
    m = torch.where(top == -INF, 0.0, top)
    e = (y - m).exp()
    total = e.sum(-1, keepdim=True)
    log_total = torch.where(total == 0, 0.0, total.log())
    far = torch.where(e == 0, 0.0, e * (m - y)).sum(-1) / torch.where(total == 0, 1.0, total)[:, 0]       # the mean distance from the maximum
    entropy = log_total[:, 0] + far
    # fp32: y and y - max are off by half a unit each; every exponential by 2^-22 and, from its argument, by 2^-23 of its distance from the
    # maximum; a thread's chain of additions by half a unit each, and as much again in joining threads, warps and pieces; log and the
    # last differences by a unit each.  The entropy has its second sum's error as well.
    chain = (vocab // 512 + 64) * 2.0 ** -24
    sums = 2.0 ** -21 * (1 + far) + chain
    tol_e = 2 * sums * (1 + far) + 2.0 ** -22 * (log_total[:, 0].abs() + far)
    assert ((got.entropy.double() - entropy).abs() <= tol_e).all()

    def logs(values, out):
        want = values - m - log_total
        tol = sums[:, None] + 2.0 ** -22 * (torch.where(values == -INF, 0.0, values).abs() + m.abs() + log_total)
        ok = ((out.double() - want).abs() <= tol) | (want == out.double())
        assert ok.all(), (out[~ok], want[~ok])
    if t is not None:
        none = t < 0
        values = y.gather(1, t.clamp(min=0).long()[:, None])
        logs(values[~none], got.log_probs[~none][:, None]) if none.sum() == 0 else None
        keep = ~none
        want = (values - m - log_total)[:, 0]
        tol = sums + 2.0 ** -22 * (torch.where(values == -INF, 0.0, values).abs() + m.abs() + log_total)[:, 0]
        off = (got.log_probs.double() - want).abs()
        assert ((off <= tol) | (got.log_probs.double() == want))[keep].all()
        assert (got.log_probs[none] == 0).all()
    if n_top:
        ids = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :n_top]
        assert torch.equal(got.top_ids.long(), ids)
        logs(y.gather(1, ids), got.top_log_probs)
    else:
        assert got.top_ids is None and got.top_log_probs is None
    return got


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 8, 9, 31, 33, 101, 255, 1000, 1023, 4096, 8191, 8193, 32001, 50021])
def test_vocabularies(vocab, dtype):
    for rows, n in ((1, 1), (3, 5), (5, 32), (2, 0)):
        check(draw(rows, vocab, dtype, vocab + n), min(n, vocab))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 2, 14, 65, 150, 443, 445, 1000])
def test_rows(rows, dtype):
    """Split rows, and rows that are not."""
    check(draw(rows, 20011, dtype, rows), 8)
    check(draw(rows, 20011, dtype, rows, banned=0.5), 20, scale=1.43)


@pytest.mark.parametrize("n", [1, 2, 8, 20, 31, IC_SCORE_MAX_TOP])
def test_number_of_alternatives(n):
    check(draw(9, 128256, BF16, n), n)
    check(draw(500, 5003, F16, n, banned=0.99), n)


@pytest.mark.parametrize("rows", [3, 600])
@pytest.mark.parametrize("kind", ["equal", "banned", "one", "few", "rising", "falling", "lowest", "zeros", "two values", "huge", "tiny scale"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_are_not_normal(kind, dtype, rows):
    vocab = 9001
    x = torch.zeros(rows, vocab, dtype=dtype, device=DEV)
    scale = 1.0
    ramp = torch.arange(vocab, device=DEV).to(F32)
    if kind == "equal":
        x[:] = 3.25
    elif kind == "banned":
        x[:] = -INF
    elif kind == "one":
        x[:] = -INF
        x[torch.arange(rows), (torch.arange(rows) * 37) % vocab] = -77.0
    elif kind == "few":
        x[:] = -INF
        x[:, 8990:] = 1.0
        x[:, 5] = 1.0
        x[:, 4000] = 2.0
    elif kind == "rising":
        x[:] = (ramp / 256).to(dtype)
    elif kind == "falling":
        x[:] = (-ramp / 256).to(dtype)
    elif kind == "lowest":      # masked with the type's lowest value instead of minus infinity
        x[:] = torch.finfo(dtype).min
        x[:, ::1000] = draw(rows, 10, dtype, 3)
        x[0] = torch.finfo(dtype).min
    elif kind == "zeros":
        x[:, ::2] = -0.0
    elif kind == "two values":
        x[:, ::3] = 1.0
    elif kind == "huge":
        x[:] = draw(rows, vocab, dtype, 3, spread=1e4)
    else:
        x[:] = draw(rows, vocab, dtype, 4)
        scale = 1e-20
    got = check(x, 20, scale)
    if kind == "banned":
        assert (got.entropy == 0).all() and (got.top_log_probs == -INF).all()
    if kind == "one":
        assert (got.entropy == 0).all() and (got.top_log_probs[:, 0] == 0).all() and (got.top_log_probs[:, 1:] == -INF).all()


@pytest.mark.parametrize("bad", [float("nan"), INF])
@pytest.mark.parametrize("rows", [1, 600])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_a_nan_or_infinite_logit_spoils_its_row_and_no_other(bad, rows, dtype):
    x = draw(rows + 1, 5001, dtype, 1)
    for at in (0, 5000, 2500, 17):
        y = x.clone()
        y[rows // 2, at] = bad
        s = ICTokenScores(5001, dtype=dtype)
        t = torch.zeros(rows + 1, dtype=torch.int32, device=DEV)
        got, good = s.score(y, t, n_top=3), s.score(x, t, n_top=3)
        s.sync()
        spoiled = torch.zeros(rows + 1, dtype=torch.bool, device=DEV)
        spoiled[rows // 2] = True
        assert (got.top_ids[spoiled] == -1).all()
        for a, b in zip(got, good):
            assert torch.equal(a[~spoiled], b[~spoiled])
            assert a.dtype == torch.int32 or a[spoiled].isnan().all()


def test_a_scale_that_leaves_the_type():
    x = torch.full((2, 300), -3e38, device=DEV)
    x[1, 7] = 3e38
    s = ICTokenScores(300, dtype=F32)
    got = s.score(x, torch.zeros(2, dtype=torch.int32, device=DEV), n_top=1, scale=4.0)
    s.sync()
    assert got.log_probs[0] == -INF and got.entropy[0] == 0          # every y is minus infinity: banned
    assert got.log_probs[1].isnan() and got.top_ids[1, 0] == -1      # the largest y is plus infinity


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_strides_and_alignment(dtype):
    base = draw(40, 3000 + 50, dtype, 2)
    for first in range(9):
        check(base[:, first:first + 2900], 5)
    check(base[::3, 11:2011], 5)
    check(base[:1, 3:1003].expand(7, 1000), 5)
    check(base[:, :2000:2], 5)                                # copied
    check(base.t().contiguous().t()[:, :500], 5)              # copied


def test_what_is_not_asked_for():
    x = draw(3, 1000, F32)
    s = ICTokenScores(1000, dtype=F32)
    r = s.score(x, entropy=False, n_top=2)
    assert r.log_probs is None and r.entropy is None and r.top_ids.shape == (3, 2)
    full = check(x, 2, scores=s)
    assert torch.equal(r.top_log_probs, full.top_log_probs)
    assert s.score(x).entropy.equal(full.entropy)
    empty = s.score(x[:0], torch.empty(0, dtype=torch.int32, device=DEV), n_top=4)
    assert empty.log_probs.shape == (0,) and empty.top_ids.shape == (0, 4)
    s.sync()


@pytest.mark.parametrize("rows", [2, 700])
def test_repeatable_and_on_other_streams(rows):
    x, t = draw(rows, 30001, BF16, 5), torch.arange(rows, dtype=torch.int32, device=DEV)
    s = ICTokenScores(30001)
    a = s.score(x, t, n_top=9)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        b = s.score(x, t, n_top=9)
    torch.cuda.current_stream().wait_stream(side)
    s.set_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c = s.score(x, t, n_top=9)
    for _ in range(3):
        graph.replay()
    s.sync()
    torch.cuda.synchronize()
    for u, v, w in zip(a, b, c):
        assert torch.equal(u, v) and torch.equal(u, w)
    assert s.launch_count == 3


def test_targets_outside_the_vocabulary():
    x = draw(4, 500, F16)
    s = ICTokenScores(500, dtype=F16)
    t = torch.tensor([1, 500, -1, -2], dtype=torch.int32, device=DEV)
    got = s.score(x, t)
    with pytest.raises(ICCacheError) as e:
        s.sync()
    assert e.value.status == IC_ERR_INVALID
    assert got.log_probs[0] < 0 and got.log_probs[1].isnan() and got.log_probs[2] == 0 and got.log_probs[3].isnan()
    s.score(x, t[:1].expand(4).contiguous())
    s.sync()
    s.score(x, t)
    torch.cuda.synchronize()
    with pytest.raises(ICCacheError):
        s.score(x, t)
    with pytest.raises(ICCacheError):
        s.sync()
    s.sync()


def test_refusals():
    x = draw(4, 500, F16)
    s = ICTokenScores(500, dtype=F16)
    for bad in (dict(n_top=33), dict(n_top=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=INF), dict(scale=float("nan")), dict(entropy=False)):
        with pytest.raises(ICCacheError):
            s.score(x, **bad)
    for call in (lambda: s.score(x.float()), lambda: s.score(x[:, :499]), lambda: s.score(x[0]), lambda: s.score(x.cpu()),
                 lambda: s.score(x, torch.zeros(4, dtype=torch.int64, device=DEV)), lambda: s.score(x, torch.zeros(3, dtype=torch.int32, device=DEV))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ICCacheError):
        ICTokenScores(5, dtype=F32).score(draw(2, 5, F32), n_top=6)
    with pytest.raises(ICCacheError):
        ICTokenScores(500, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError):
        ICTokenScores(500, workspace=torch.empty(1 << 20, dtype=torch.uint8))
    s.close()
    with pytest.raises(ValueError):
        s.score(x)


def test_more_than_two_to_the_32_bytes():
    """Rows far behind the first, and every row of them."""
    rows, vocab = 20001, 131072
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("not enough memory")
    x = torch.empty(rows, vocab, dtype=BF16, device=DEV).normal_(generator=gen(1))
    s = ICTokenScores(vocab)
    t = torch.randint(0, vocab, (rows,), device=DEV, dtype=torch.int32)
    got = s.score(x, t, n_top=2)
    s.sync()
    for a in (0, rows - 100):
        part = check(x[a:a + 100], 2, targets=t[a:a + 100].contiguous(), scores=s)
        assert torch.equal(part.top_ids, got.top_ids[a:a + 100])
        assert (part.log_probs - got.log_probs[a:a + 100]).abs().max() < 1e-5


@pytest.mark.parametrize("kind", ["drawn", "banned", "rising", "falling", "two values"])
@pytest.mark.parametrize("rows,vocab,dtype", [(1, 16777216, BF16), (600, 262145, BF16), (3, 1500001, F32), (600, 130001, F32)])
def test_rows_of_many_blocks(rows, vocab, dtype, kind):
    """Rows so long that a thread's blocks are put together in groups, whole and split, with 32 alternatives."""
    x = torch.empty(rows, vocab, dtype=dtype, device=DEV)
    ramp = torch.arange(vocab, device=DEV).to(F32) / vocab
    if kind == "drawn":
        x[:] = draw(rows, vocab, dtype, 5)
    elif kind == "banned":          # fewer left than are asked for
        x[:] = -INF
        x[:, vocab // 3:: vocab // 7] = 1.5
        x[:, -1] = 2.5
    elif kind == "rising":
        x[:] = (8 * ramp).to(dtype)
    elif kind == "falling":
        x[:] = (-8 * ramp).to(dtype)
    else:
        x[:] = 0
        x[:, 7:: max(1, vocab // 40)] = 1.0
    s = ICTokenScores(vocab, dtype=dtype)
    t = torch.randint(-1, vocab, (rows,), device=DEV, generator=gen(8), dtype=torch.int32)
    got = s.score(x, t, n_top=32)
    s.sync()
    for a in range(0, rows, 100):       # (a part at a time: 64 bits a logit)
        part = x[a:a + 100]
        assert torch.equal(got.top_ids[a:a + 100].long(), torch.sort(part, dim=-1, descending=True, stable=True).indices[:, :32])
    last = x[-1:].contiguous()
    again = check(last, 32, targets=t[-1:].contiguous(), scores=ICTokenScores(vocab, dtype=dtype))
    assert torch.equal(again.top_ids[0], got.top_ids[-1])
    # (another division into pieces: the same sums in another order, each within the bound that check() holds)
    assert torch.allclose(again.entropy[0], got.entropy[-1], rtol=2.0 ** -10, atol=2.0 ** -10)


@pytest.mark.parametrize("scale", [0.7, 0.9, 1 / 1.3, 1.1, 1.4])
@pytest.mark.parametrize("mask", ["lowest", -1e30, -1e10])
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_masked_rows_at_a_temperature(dtype, mask, scale):
    """Rows masked with large finite numbers, all but a few tokens (row 0: all of them), where scale * x is not exact."""
    vocab, rows = 9001, 5
    mask = torch.finfo(dtype).min if mask == "lowest" else max(mask, torch.finfo(dtype).min)
    x = torch.full((rows, vocab), mask, dtype=dtype, device=DEV)
    for r in range(1, rows):
        x[r, 37 * r::900] = draw(1, 10, dtype, r)[0]
    finite = mask * scale > -torch.finfo(F32).max       # (otherwise y of a masked token is minus infinity in fp32)
    check(x[1:], 10, scale, targets=torch.tensor([37 * r for r in range(1, rows)], dtype=torch.int32, device=DEV))
    if finite:
        check(x[1:], 20, scale)
    s = ICTokenScores(vocab, dtype=dtype)
    got = s.score(x, ints_of(rows, 8000), n_top=20, scale=scale)
    s.sync()
    assert torch.equal(got.top_ids[0], torch.arange(20, dtype=torch.int32, device=DEV))
    if finite:
        # every weight is 1 and the sum the exact vocab: what is left is the logarithm's error and a rounding, 2 units
        want = math.log(vocab)
        for value in (-got.log_probs[0], got.entropy[0], *-got.top_log_probs[0]):
            assert abs(float(value) - want) <= 2.0 ** -22 * want
    else:           # banned
        assert got.log_probs[0] == -INF and got.entropy[0] == 0


def ints_of(n, value):
    return torch.full((n,), value, dtype=torch.int32, device=DEV)


@pytest.mark.parametrize("rows", [2, 700])
def test_logits_far_apart(rows):
    """Differences beyond fp32's largest number, brought back by the scale, and the largest scale there is."""
    x = draw(rows, 3001, F32, 6)
    x[:, 5], x[:, 9], x[:, 11] = 3e38, -3e38, 2.9e38
    s = ICTokenScores(3001, dtype=F32)
    got = s.score(x, ints_of(rows, 9), scale=1e-36)
    s.sync()
    want = (-6e38 * 1e-36) - math.log(1 + math.exp(-10.0) + 0.0)          # (the others are e^-300 and less)
    assert (got.log_probs.double() - want).abs().max() <= 2.0 ** -22 * abs(want)
    with pytest.raises(ICCacheError):
        s.score(x, scale=3e38)          # times log2(e) not finite
    got = s.score(torch.tensor([0.0, -1e-30], device=DEV).repeat(rows, 1501)[:, :3001].contiguous(), ints_of(rows, 1), scale=1e30)
    s.sync()
    want = -1.0 - math.log(1501 + 1500 * math.exp(-1.0))
    assert (got.log_probs.double() - want).abs().max() <= 2.0 ** -18 * abs(want)      # (seven additions a thread, and those of threads and warps)
