"""The paged key-value cache's operators: what is measured, with each operator's plain form and its values in 64 bits.

A case names an operator ("op"), its shapes, and "mix", the number from which the ragged lengths are made; the values
come from the seed.  The pool is [pages, layers, 2 (K, V), kv heads, page size, head dim]; tables, lengths and refs are the
page tables, the sequence lengths and the pages' reference counts, all on the device.  The operators:

  decode   attention of one new token per sequence over its pages
  extend   attention of the last `fresh` tokens of every sequence over its pages, causal
  append   slots for new tokens (lowest free pages), and their K and V written into one layer's pages
  fork     children become copies of a prefix of their parents: full pages shared, or every page copied
  compact  finished sequences give their pages back, and the live pages move to the front of the pool

A query at position p sees the keys j <= p with j > p - window (window 0: all) or j < sinks.
"""
import math
import random

import torch

own = False

LAYER = 1   # the layer that the attention reads and the append writes


def listed():
    return [
        # the second token of a short request on a small model: latency
        dict(name="decode_token", op="decode", n=1, hq=8, hkv=2, d=64, page=16, layers=2, dtype="bf16", longest=37, shortest=37, window=0, sinks=0, mix=1),
        # one step of a serving batch, ragged lengths
        dict(name="decode_batch", op="decode", n=64, hq=32, hkv=8, d=128, page=16, layers=2, dtype="bf16", longest=8192, shortest=900, window=0, sinks=0, mix=2),
        # one long conversation: the work has to be split over its length
        dict(name="decode_long", op="decode", n=1, hq=32, hkv=4, d=128, page=64, layers=2, dtype="fp16", longest=131071, shortest=131071, window=0, sinks=0, mix=3),
        # short requests behind cached examples
        dict(name="extend_request", op="extend", n=4, hq=32, hkv=8, d=128, page=16, layers=2, dtype="bf16", longest=6001, shortest=2500, fresh=57, fresh_least=9, window=0, sinks=0, mix=4),
        # whole prompts, nothing cached before them
        dict(name="extend_prompts", op="extend", n=8, hq=32, hkv=8, d=128, page=16, layers=2, dtype="bf16", longest=4096, shortest=1500, fresh=4096, fresh_least=1500, window=0, sinks=0, mix=5),
        # a long document under a sliding window with four sink tokens
        dict(name="extend_window", op="extend", n=1, hq=16, hkv=4, d=64, page=32, layers=2, dtype="fp16", longest=12289, shortest=12289, fresh=12289, fresh_least=12289, window=1024, sinks=4, mix=6),
        # the new token of every sequence of a serving batch
        dict(name="append_token", op="append", n=64, hkv=8, d=128, page=16, layers=2, dtype="bf16", longest=1500, shortest=1, fresh=1, fresh_least=1, mix=7),
        # whole prompts behind short cached prefixes
        dict(name="append_prompts", op="append", n=8, hkv=8, d=128, page=16, layers=2, dtype="bf16", longest=700, shortest=0, fresh=6000, fresh_least=2001, mix=8),
        # a beam search's reordering in place
        dict(name="fork_beams", op="fork", n=8, hkv=4, d=64, page=16, layers=4, dtype="fp16", longest=501, shortest=170, fresh=0, copy=False, beams=True, mix=9),
        # examples copied for requests that will rewrite them
        dict(name="fork_examples", op="fork", n=48, hkv=8, d=128, page=16, layers=8, dtype="bf16", longest=700, shortest=100, fresh=0, copy=True, beams=False, mix=10),
        # a small pool after a few requests have ended
        dict(name="compact_small", op="compact", n=12, hkv=2, d=64, page=16, layers=2, dtype="bf16", longest=300, shortest=1, mix=11),
        # a large pool after half of its sequences have ended
        dict(name="compact_large", op="compact", n=96, hkv=8, d=128, page=16, layers=4, dtype="bf16", longest=1000, shortest=100, mix=12),
    ]


def _spread(rng, low, high):
    """A size between the two, even over the logarithm; odd nearly always, a power of two now and then."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    v = 1 << (v.bit_length() - 1) if rng.random() < 0.2 else v | 1
    return max(low, min(high, v))


def draw(rng):
    op = rng.choice(["decode", "decode", "extend", "extend", "append", "fork", "compact"])
    d = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
    hkv = rng.choice([1, 2, 4, 8])
    c = dict(op=op, hkv=hkv, d=d, page=rng.choice([16, 16, 32, 64, 128]), layers=2, dtype=rng.choice(["bf16", "bf16", "fp16"]), mix=rng.randrange(1 << 30))
    if op in ("decode", "extend"):
        c["hq"] = hkv * rng.choice([1, 2, 3, 4, 5, 7, 8] + [16] * (hkv <= 4))
        windowed = rng.random() < 0.4
        c["window"] = _spread(rng, 1, 8192) if windowed else 0
        c["sinks"] = rng.choice([0, 1, 4, 4, 17, 64]) if windowed else 0
    if op == "decode":
        c["n"] = _spread(rng, 1, 128)
        # no more cached tokens in all than the largest listed case holds bytes for
        most = min(131071, 64 * 4500 * 8 * 128 // (c["n"] * hkv * d))
        c["longest"] = _spread(rng, 1, most)
        c["shortest"] = _spread(rng, 1, c["longest"])
    elif op == "extend":
        c["n"] = _spread(rng, 1, 16)
        most = int(min(12289, math.sqrt(8 * 32 * 4096 * 4096 * 0.9 / (c["n"] * c["hq"]))))
        c["longest"] = _spread(rng, 1, most)
        c["shortest"] = _spread(rng, 1, c["longest"])
        c["fresh"] = _spread(rng, 1, c["longest"])
        c["fresh_least"] = _spread(rng, 1, c["fresh"])
    elif op == "append":
        c["n"] = _spread(rng, 1, 128)
        c["longest"] = _spread(rng, 1, 1500)
        c["shortest"] = rng.choice([0, 1, c["longest"]])
        c["fresh"] = _spread(rng, 1, max(1, 24000 * 8 * 128 // (c["n"] * hkv * d) // 2))
        c["fresh_least"] = rng.choice([0, 1, c["fresh"]])
    elif op == "fork":
        c["n"] = _spread(rng, 1, 64)
        c["layers"] = rng.choice([2, 3, 8])
        c["longest"] = _spread(rng, 1, max(1, 48 * 400 * 8 * 8 * 128 // (c["n"] * c["layers"] * hkv * d) // 2))
        c["shortest"] = _spread(rng, 1, c["longest"])
        c["fresh"] = 0
        c["beams"] = rng.random() < 0.5
        c["copy"] = rng.random() < 0.4
    else:
        c["n"] = _spread(rng, 2, 128)
        c["longest"] = _spread(rng, 1, max(1, 96 * 550 * 4 * 8 * 128 // (c["n"] * c["layers"] * hkv * d) // 2))
        c["shortest"] = _spread(rng, 1, c["longest"])
    return c


# ---------------------------------------------------------------- shapes that follow from a case
def _pages(tokens, page):
    return -(-tokens // page)


def _shape(case):
    """Lengths as they are when the call begins, tokens of the call per sequence, slots, parents and pages of the pool."""
    rng = random.Random(case["mix"])
    n, page, op = case["n"], case["page"], case["op"]
    lens = [case["longest"]] + [rng.randint(case["shortest"], case["longest"]) for _ in range(n - 1)]
    rng.shuffle(lens)
    fresh = [0] * n
    if op in ("extend", "append"):
        fresh = [rng.randint(case["fresh_least"], case["fresh"]) for _ in range(n)]
        if op == "extend":
            if case["fresh"] == case["longest"] and case["fresh_least"] == case["shortest"]:
                fresh = list(lens)
            fresh = [min(f, x) for f, x in zip(fresh, lens)]
    s = dict(lens=lens, fresh=fresh, n=n, max_seqs=n, held=list(lens))
    if op == "append":
        most = max(a + b for a, b in zip(lens, fresh))
        need = sum(_pages(a + b, page) for a, b in zip(lens, fresh))
    elif op == "fork":
        if case["beams"]:
            s["parents"], s["children"] = [rng.randrange(n) for _ in range(n)], list(range(n))
            s["upto"] = [lens[p] for p in s["parents"]]
            need = 2 * sum(_pages(x, page) for x in lens) + n * _pages(max(lens), page) * case["copy"] + n
        else:
            # slots 0 .. n-1 hold examples, n .. 2n-1 are the requests' and empty
            s["max_seqs"], s["held"] = 2 * n, lens + [0] * n
            s["parents"], s["children"] = [rng.randrange(n) for _ in range(n)], [n + i for i in range(n)]
            s["upto"] = [rng.randint((lens[p] + 1) // 2, lens[p]) for p in s["parents"]]
            need = sum(_pages(x, page) for x in lens) + sum(_pages(x, page) for x in s["upto"])
        most = max(lens)
    else:
        most, need = max(lens), sum(_pages(x, page) for x in lens)
    s["ended"] = sorted(rng.sample(range(n), n // 2)) if op == "compact" else []
    s["max_pages"] = max(4, -(-_pages(most, page) // 4) * 4)
    s["n_pages"] = -(-(need + need // 16 + 2) // 64) * 64 + 7
    return s


def _type(case):
    return torch.float16 if case["dtype"] == "fp16" else torch.bfloat16


def prepare(case, seed):
    s, dev = _shape(case), "cuda"
    g = torch.Generator(device=dev).manual_seed(seed)
    n_pages, page, n = s["n_pages"], case["page"], s["n"]
    pool = torch.randn(n_pages, case["layers"], 2, case["hkv"], page, case["d"], dtype=_type(case), device=dev, generator=g)
    # a pool that has been in use: the sequences' pages lie anywhere in it
    order = torch.randperm(n_pages, device=dev, generator=g).to(torch.int32)
    # pages tables, lengths and reference counts in one block, so that a pass can put them back with one copy
    r64 = lambda x: -(-x // 64) * 64  # noqa: E731
    a, b = r64(n_pages), r64(s["max_seqs"] * s["max_pages"])
    book = torch.zeros(a + b + r64(s["max_seqs"]), dtype=torch.int32, device=dev)
    refs, tables, lengths = book[:n_pages], book[a:a + s["max_seqs"] * s["max_pages"]].view(s["max_seqs"], -1), book[a + b:a + b + s["max_seqs"]]
    held = torch.tensor(s["held"], device=dev)
    owned = torch.arange(s["max_pages"], device=dev)[None, :] < ((held + page - 1) // page)[:, None]
    names = order[:int(owned.sum())]
    tables[owned] = names
    refs[names.long()] = 1
    lengths.copy_(held)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    starts = [0]
    for f in s["fresh"]:
        starts.append(starts[-1] + f)
    st = dict(case=case, pool=pool, book=book, refs=refs, tables=tables, lengths=lengths, seqs=ints(list(range(n))), copied=case.get("copy", False),
              counts=ints(s["fresh"]), starts=ints(starts), most_fresh=max(s["fresh"]), window=case.get("window", 0), sinks=case.get("sinks", 0))
    if case["op"] in ("append", "fork", "compact"):
        st["saved"] = book.clone()
    rows = n if case["op"] == "decode" else starts[-1]
    if case["op"] in ("decode", "extend"):
        st["q"] = (2.0 * torch.randn(rows, case["hq"], case["d"], device=dev, generator=g)).to(_type(case))
    elif case["op"] == "append":
        st["k"], st["v"] = (torch.randn(rows, case["hkv"], case["d"], dtype=_type(case), device=dev, generator=g) for _ in range(2))
    elif case["op"] == "fork":
        st["parents"], st["children"], st["upto"] = ints(s["parents"]), ints(s["children"]), ints(s["upto"])
    else:
        st["ended"] = ints(s["ended"])
    if own:
        from paper_2501_12689_b200 import ICPagedKV
        st["kv"] = ICPagedKV(n_pages, case["layers"], case["hkv"], page, case["d"], s["max_seqs"], s["max_pages"], dtype=_type(case),
                             pool=pool, tables=tables, lengths=lengths, refs=refs)
    return st


def run(st):
    op = st["case"]["op"]
    if op in ("append", "fork", "compact"):
        st["book"].copy_(st["saved"])       # the state before the call; page contents that a call overwrites lie in free pages
    if own:
        kv = st["kv"]
        if op == "decode":
            return kv.decode(LAYER, st["q"], st["seqs"], window=st["window"], sinks=st["sinks"])
        if op == "extend":
            return kv.extend(LAYER, st["q"], st["seqs"], st["starts"], window=st["window"], sinks=st["sinks"])
        if op == "append":
            kv.reserve(st["seqs"], st["counts"])
            kv.write(LAYER, st["k"], st["v"], st["seqs"], st["starts"])
        elif op == "fork":
            kv.fork(st["parents"], st["children"], st["upto"], copy=st["copied"])
        else:
            kv.free(st["ended"])
            kv.compact()
    elif op == "decode":
        return _plain_attention(st, st["q"], st["seqs"].long(), torch.arange(st["seqs"].numel(), device="cuda"), torch.zeros_like(st["seqs"]).long(), torch.ones_like(st["counts"]), 1)
    elif op == "extend":
        # one row per token: which sequence of the batch it belongs to, and the how-manieth of its tokens it is
        i = torch.repeat_interleave(torch.arange(st["seqs"].numel(), device="cuda"), st["counts"].long(), output_size=st["q"].shape[0])
        return _plain_attention(st, st["q"], st["seqs"].long(), i, torch.arange(i.numel(), device="cuda") - st["starts"].long()[i], st["counts"], st["most_fresh"])
    elif op == "append":
        _plain_append(st)
    elif op == "fork":
        _plain_fork(st)
    else:
        _plain_compact(st)
    return dict(tables=st["tables"], lengths=st["lengths"], refs=st["refs"], pool=st["pool"])


# ---------------------------------------------------------------- the plain forms
def _plain_attention(st, q, seqs, i, t, counts, most):
    """Attention of ragged tokens (token x is the t[x]-th new one of sequence i[x] of the batch) over gathered pages, padded to the longest."""
    pool = st["pool"]
    _, _, _, hkv, page, d = pool.shape
    n, g = seqs.numel(), q.shape[1] // hkv
    lens = st["lengths"].long()[seqs]
    cols = torch.arange(st["tables"].shape[1], device="cuda")
    rows = torch.where(cols < ((lens + page - 1) // page)[:, None], st["tables"][seqs].long(), 0)
    kv = pool[rows, LAYER].float()                                                     # [n, pages, 2, hkv, page, d]
    k, v = (kv[:, :, x].permute(0, 2, 1, 3, 4).reshape(n, hkv, 1, -1, d) for x in (0, 1))
    padded = torch.zeros(n, hkv, g, most, d, device="cuda")
    padded[i, :, :, t] = q.float().view(-1, hkv, g, d)
    at = lens[:, None] - counts.long()[:, None] + torch.arange(most, device="cuda")     # a query's position
    j = torch.arange(k.shape[3], device="cuda")
    seen = (j <= at[..., None]) & (j < lens[:, None, None])
    if st["window"]:
        seen &= (j > at[..., None] - st["window"]) | (j < st["sinks"])
    v = torch.where((j < lens[:, None])[:, None, None, :, None], v, 0.0)
    s = (padded.reshape(n, hkv, 1, g * most, d) @ k.transpose(-1, -2)).view(n, hkv, g, most, -1)
    s = s.mul_(d ** -0.5).masked_fill_(~seen[:, None, None], float("-inf"))
    top = s.amax(-1, keepdim=True)
    p = s.sub_(torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(n, hkv, 1, g * most, -1) @ v).view(n, hkv, g, most, d) / torch.where(total == 0, 1.0, total)
    return o[i, :, :, t].reshape(q.shape).to(q.dtype)


def _plain_append(st):
    pool, tables, lengths, refs, seqs, counts = st["pool"], st["tables"], st["lengths"], st["refs"], st["seqs"].long(), st["counts"].long()
    page, total = pool.shape[4], st["k"].shape[0]
    had = lengths.long()[seqs]
    before, after = (had + page - 1) // page, (had + counts + page - 1) // page
    free = torch.argsort((refs > 0).to(torch.int8), stable=True)                        # free pages first, lowest first
    begin = torch.cumsum(after - before, 0) - (after - before)
    cols = torch.arange(tables.shape[1], device="cuda")
    new = (cols >= before[:, None]) & (cols < after[:, None])
    name = free[torch.where(new, begin[:, None] + cols - before[:, None], 0)]
    tables[seqs] = torch.where(new, name.to(torch.int32), tables[seqs])
    refs.index_add_(0, name.view(-1), new.view(-1).to(torch.int32))
    lengths.index_add_(0, seqs, counts.to(torch.int32))
    i = torch.repeat_interleave(torch.arange(seqs.numel(), device="cuda"), counts, output_size=total)
    at = had[i] + torch.arange(total, device="cuda") - st["starts"].long()[i]
    where = tables[seqs[i], at // page].long()
    pool[where, LAYER, 0, :, at % page] = st["k"]
    pool[where, LAYER, 1, :, at % page] = st["v"]


def _plain_fork(st):
    pool, tables, lengths, refs = st["pool"], st["tables"], st["lengths"], st["refs"]
    parents, children, upto, copied = st["parents"].long(), st["children"].long(), st["upto"].long(), st["copied"]
    page = pool.shape[4]
    source, target, had = tables[parents].long(), tables[children].long(), lengths.long()[children]
    pages = (upto + page - 1) // page
    shared = torch.zeros_like(pages) if copied else torch.where((parents == children) & (upto == had), pages, upto // page)
    free = torch.argsort((refs > 0).to(torch.int8), stable=True)
    begin = torch.cumsum(pages - shared, 0) - (pages - shared)
    cols = torch.arange(tables.shape[1], device="cuda")
    kept, new = cols < shared[:, None], (cols >= shared[:, None]) & (cols < pages[:, None])
    name = torch.where(new, free[torch.where(new, begin[:, None] + cols - shared[:, None], 0)], torch.where(kept, source, target))
    held, left = kept | new, cols < ((had + page - 1) // page)[:, None]
    pool[name[new]] = pool[source[new]]
    refs.index_add_(0, torch.where(held, name, 0).view(-1), held.view(-1).to(torch.int32))
    refs.index_add_(0, torch.where(left, target, 0).view(-1), -left.view(-1).to(torch.int32))
    tables[children] = name.to(torch.int32)
    lengths[children] = upto.to(torch.int32)


def _plain_compact(st):
    pool, tables, lengths, refs, ended = st["pool"], st["tables"], st["lengths"], st["refs"], st["ended"].long()
    page = pool.shape[4]
    cols = torch.arange(tables.shape[1], device="cuda")
    left = cols < ((lengths.long()[ended] + page - 1) // page)[:, None]
    refs.index_add_(0, torch.where(left, tables[ended], 0).view(-1), -left.view(-1).to(torch.int32))
    lengths[ended] = 0
    alive = refs > 0
    below = torch.arange(refs.numel(), device="cuda") < alive.sum()
    to, come = torch.nonzero(below & ~alive).view(-1), torch.nonzero(~below & alive).view(-1)
    pool[to] = pool[come]
    refs[to] = refs[come]
    refs[come] = 0
    moved = torch.arange(refs.numel(), dtype=torch.int32, device="cuda")
    moved[come] = to.to(torch.int32)
    held = cols < ((lengths.long() + page - 1) // page)[:, None]
    tables.copy_(torch.where(held, moved[torch.where(held, tables, 0).long()], tables))


# ---------------------------------------------------------------- what the path cannot do without
def _seen(p, window, sinks):
    """How many keys a query at position p sees."""
    if not window or window > p:
        return p + 1
    return window + min(sinks, p + 1 - window)


def work(case):
    s = _shape(case)
    token = case["hkv"] * case["d"] * 2 * 2                      # bytes of one token's K and V in one layer
    whole = token * case["page"] * case["layers"]                # bytes of a page
    page, op = case["page"], case["op"]
    if op in ("decode", "extend"):
        fresh = [1] * s["n"] if op == "decode" else s["fresh"]
        pairs = cached = 0
        for x, f in zip(s["lens"], fresh):
            w, k = case["window"], case["sinks"]
            # sum of _seen over the positions x - f .. x - 1
            ramp = lambda e: e * (e + 1) // 2  # noqa: E731
            if not w:
                pairs += ramp(x) - ramp(x - f)
            else:
                pairs += sum(_seen(p, w, k) for p in range(x - f, x))
            first = max(0, x - f - w + 1) if w else 0            # the first key in any query's window
            cached += (x - first + min(k, first)) if f else 0
        return dict(bytes=cached * token + 2 * sum(fresh) * case["hq"] * case["d"] * 2, flops=4 * pairs * case["hq"] * case["d"])
    if op == "append":
        return dict(bytes=2 * sum(s["fresh"]) * token + 8 * s["n"], flops=0)
    if op == "fork":
        moved = 0
        for a, b, x in zip(s["parents"], s["children"], s["upto"]):
            moved += _pages(x, page) if case["copy"] else (0 if a == b and x == s["held"][a] else int(x % page > 0))
        entries = sum(_pages(x, page) for x in s["upto"])
        return dict(bytes=2 * moved * whole + 12 * entries + 12 * s["n"], flops=0)
    gone = sum(_pages(s["lens"][i], page) for i in s["ended"])
    live = sum(_pages(x, page) for x in s["lens"]) - gone
    # the pages lie anywhere: a hole below n_live is as likely as an unused page anywhere
    moved = live * (s["n_pages"] - live) / s["n_pages"]
    return dict(bytes=2 * moved * whole + 8 * (live + gone) + 4 * s["n_pages"], flops=0)


# ---------------------------------------------------------------- the operators' values, from their definitions
def exact(case, seed):
    st = prepare(case, seed)
    page, op = case["page"], case["op"]
    if op in ("decode", "extend"):
        if work(case)["flops"] > 4e12:
            return None
        return _exact_attention(case, st)
    pool, lens, refs = st["pool"].clone(), st["lengths"].tolist(), st["refs"].tolist()
    rows = st["tables"].tolist()
    vacant = [p for p, r in enumerate(refs) if r == 0]
    if op == "append":
        start = 0
        for s, f in zip(st["seqs"].tolist(), st["counts"].tolist()):
            for col in range(_pages(lens[s], page), _pages(lens[s] + f, page)):
                rows[s][col] = vacant.pop(0)
                refs[rows[s][col]] = 1
            done = 0
            while done < f:                        # page by page
                at = lens[s] + done
                some = min(page - at % page, f - done)
                part = slice(start + done, start + done + some)
                for x, new in ((0, st["k"]), (1, st["v"])):
                    pool[rows[s][at // page], LAYER, x, :, at % page:at % page + some] = new[part].transpose(0, 1)
                done += some
            start += f
            lens[s] += f
    elif op == "fork":
        before, had = [list(r) for r in rows], list(lens)
        for a, b, x in zip(st["parents"].tolist(), st["children"].tolist(), st["upto"].tolist()):
            if not case["copy"] and a == b and x == had[a]:
                continue
            for col in range(_pages(x, page)):
                name = before[a][col]
                if case["copy"] or (col + 1) * page > x:
                    name = vacant.pop(0)
                    pool[name] = st["pool"][before[a][col]]
                rows[b][col] = name
                refs[name] += 1
            for col in range(_pages(had[b], page)):
                refs[before[b][col]] -= 1
            lens[b] = x
    else:
        for s in st["ended"].tolist():
            for col in range(_pages(lens[s], page)):
                refs[rows[s][col]] -= 1
            lens[s] = 0
        live = [p for p, r in enumerate(refs) if r > 0]
        holes = [p for p in range(len(live)) if refs[p] == 0]
        name = {a: b for a, b in zip([p for p in live if p >= len(live)], holes)}
        for a, b in name.items():
            pool[b] = st["pool"][a]
            refs[b], refs[a] = refs[a], 0
        rows = [[name.get(p, p) if col < _pages(lens[s], page) else p for col, p in enumerate(r)] for s, r in enumerate(rows)]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return dict(tables=ints(rows), lengths=ints(lens), refs=ints(refs), pool=pool)


def _exact_attention(case, st):
    """Sequence by sequence, kv head by kv head, block of tokens by block of tokens, in 64 bits."""
    page, hkv, g, window, sinks = case["page"], case["hkv"], case["hq"] // case["hkv"], case["window"], case["sinks"]
    q, rows, lens = st["q"].double(), st["tables"].tolist(), st["lengths"].tolist()
    fresh = [1] * case["n"] if case["op"] == "decode" else st["counts"].tolist()
    out, start = torch.zeros_like(q), 0
    for s, f in enumerate(fresh):
        x = lens[s]
        both = st["pool"][rows[s][:_pages(x, page)], LAYER].double()               # [pages, 2, hkv, page, d]
        for h in range(hkv):
            k, v = (both[:, w, h].reshape(-1, case["d"])[:x] for w in (0, 1))
            for a in range(0, f, 2048):
                b = min(f, a + 2048)
                p = torch.arange(x - f + a, x - f + b, device="cuda")[:, None, None]
                j = torch.arange(x, device="cuda")
                hidden = (j > p) | ((j <= p - window) & (j >= sinks)) if window else j > p
                w = torch.einsum("tgd,jd->tgj", q[start + a:start + b, h * g:(h + 1) * g], k) / math.sqrt(case["d"])
                w = torch.softmax(w.masked_fill(hidden, -math.inf), -1)
                out[start + a:start + b, h * g:(h + 1) * g] = torch.einsum("tgj,jd->tgd", w, v)
        start += f
    return out
