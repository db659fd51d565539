"""Operators around the paged cache and the example store: what is measured, with each one's plain form and its values in 64 bits.

A case names an operator ("op"), its shapes, and "mix", the number from which ragged lengths are made; the values come from
the seed.  Index lists are int32 on the device.  The operators:

  rotate   rotary positions of new tokens: queries rotated, keys rotated into one layer's pages, values written beside them
  shift    the cached keys of sequences, in all layers, moved by a number of positions each
  score    log-probabilities of given tokens, entropy and top alternatives of rows of logits
  state    linear attention with a decay per head over states kept by sequence: one token or several per sequence

Rotation: pair i of a head at position p turns by p * f_i, f_i = base^(-2i / rotary_dim), scaled as the case says; the pair is
elements (i, i + rotary_dim / 2), or (2i, 2i + 1) where it says interleaved; elements from rotary_dim on stay.
State: S <- exp(-rate) S + k v^T, out = scale * q S, token by token, S [key dim, value dim] in 32 bits.
"""
import math
import random

import torch

own = False

LAYER = 0   # the layer that rotate writes and state reads


def listed():
    return [
        # the next token of a request on a small model: latency
        dict(name="rotate_token", op="rotate", n=1, hq=8, hkv=2, d=64, rotary=64, interleaved=False, scaling="none", page=16, layers=2, dtype="bf16", had=37, had_least=37, fresh=1, fresh_least=1, mix=1),
        # whole prompts behind short cached examples
        dict(name="rotate_prompts", op="rotate", n=8, hq=32, hkv=8, d=128, rotary=128, interleaved=False, scaling="none", page=16, layers=2, dtype="bf16", had=700, had_least=0, fresh=6000, fresh_least=2001, mix=2),
        # a part of the head, neighbours paired, frequencies stretched: requests at the far end of long contexts
        dict(name="rotate_partial", op="rotate", n=5, hq=32, hkv=8, d=80, rotary=32, interleaved=True, scaling="bands", page=32, layers=1, dtype="fp16", had=120001, had_least=90001, fresh=901, fresh_least=17, mix=3),
        # one copied example that stands behind another one now
        dict(name="shift_request", op="shift", n=1, hkv=4, d=64, rotary=64, interleaved=False, scaling="none", page=16, layers=4, dtype="bf16", had=333, had_least=333, mix=4),
        # examples copied for a batch of requests
        dict(name="shift_examples", op="shift", n=48, hkv=8, d=128, rotary=128, interleaved=False, scaling="linear", page=16, layers=8, dtype="bf16", had=701, had_least=100, mix=5),
        # the token that was just drawn
        dict(name="score_token", op="score", rows=1, vocab=32001, top=5, scale=1.0, banned=0.0, given=True, dtype="bf16", mix=6),
        # one step of a batch, logits in 32 bits with tokens banned by a grammar, at a temperature
        dict(name="score_batch", op="score", rows=65, vocab=50021, top=20, scale=1.25, banned=0.3, given=True, dtype="fp32", mix=7),
        # whole answers, scored for the utility of the examples in front of them
        dict(name="score_answers", op="score", rows=4001, vocab=128256, top=5, scale=1.0, banned=0.0, given=True, dtype="bf16", mix=8),
        # the next token of a request on a small model
        dict(name="state_token", op="state", n=1, heads=4, dk=64, dv=64, dtype="bf16", fresh=1, fresh_least=1, strength=1.0, mix=9),
        # one step of a serving batch
        dict(name="state_batch", op="state", n=64, heads=32, dk=128, dv=128, dtype="bf16", fresh=1, fresh_least=1, strength=1.0, mix=10),
        # whole prompts
        dict(name="state_prompts", op="state", n=8, heads=32, dk=128, dv=128, dtype="bf16", fresh=4096, fresh_least=1500, strength=1.0, mix=11),
        # one long document on a model of few heads: the work has to be split over its length
        dict(name="state_long", op="state", n=1, heads=8, dk=64, dv=128, dtype="fp16", fresh=30011, fresh_least=30011, strength=1.0, mix=12),
    ]


def _spread(rng, low, high):
    """A size between the two, even over the logarithm; odd nearly always, a power of two now and then."""
    v = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    v = 1 << (v.bit_length() - 1) if rng.random() < 0.2 else v | 1
    return max(low, min(high, v))


def draw(rng):
    op = rng.choice(["rotate", "rotate", "shift", "score", "score", "state", "state", "state"])
    mix = rng.randrange(1 << 30)
    if op == "score":
        c = dict(op=op, rows=_spread(rng, 1, 4001), top=rng.choice([0, 1, 3, 5, 8, 20, 32]), scale=rng.choice([1.0, 1.0, 0.5, 1.43]),
                 banned=rng.choice([0.0, 0.0, 0.3, 0.999]), given=rng.random() < 0.8, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), mix=mix)
        most = 4001 * 128256 // (c["rows"] * (2 if c["dtype"] == "fp32" else 1))
        c["vocab"] = _spread(rng, 101, min(262144, most))
        return c
    if op == "state":
        c = dict(op=op, n=_spread(rng, 1, 64), heads=rng.choice([1, 2, 4, 5, 8, 16, 32]), dk=rng.choice([16, 32, 64, 64, 80, 96, 128, 128]),
                 dv=rng.choice([32, 64, 64, 72, 128, 128, 256]), dtype=rng.choice(["bf16", "bf16", "fp16"]), mix=mix)
        c["strength"] = rng.choice([1.0, 1.0, 8.0])
        most = min(30011, 8 * 32 * 2798 * 128 * 128 // (c["n"] * c["heads"] * c["dk"] * c["dv"]))
        c["fresh"] = 1 if rng.random() < 0.25 else _spread(rng, 1, max(1, most))
        c["fresh_least"] = _spread(rng, 1, c["fresh"])
        return c
    d = rng.choice([64, 64, 80, 96, 128, 128, 128, 256])
    hkv = rng.choice([1, 2, 4, 8])
    c = dict(op=op, hkv=hkv, d=d, rotary=rng.choice([d, d, d // 2, d // 4, 2 * (d // 5)]), interleaved=rng.random() < 0.4,
             scaling=rng.choice(["none", "linear", "base", "bands"]), page=rng.choice([16, 16, 32, 64, 128]), layers=2,
             dtype=rng.choice(["bf16", "bf16", "fp16"]), mix=mix)
    if op == "rotate":
        c["hq"] = hkv * rng.choice([1, 2, 3, 4, 5, 7, 8] + [16] * (hkv <= 4))
        c["n"] = _spread(rng, 1, 128)
        c["had"] = _spread(rng, 1, min(120001, 400000000 // (c["n"] * hkv * d)))
        c["had_least"] = rng.choice([0, 1, c["had"]])
        c["fresh"] = _spread(rng, 1, max(1, min(262144 // c["n"], 8 * 4000 * (2 * 32 + 4 * 8) * 128 // (c["n"] * (2 * c["hq"] + 4 * hkv) * d))))
        c["fresh_least"] = rng.choice([0, 1, c["fresh"]])
        c["layers"] = 1
    else:
        c["n"] = _spread(rng, 1, 64)
        c["layers"] = rng.choice([1, 2, 3, 8])
        c["had"] = _spread(rng, 1, max(1, min(262144 // c["n"], 48 * 400 * 8 * 8 * 128 // (c["n"] * c["layers"] * hkv * d))))
        c["had_least"] = _spread(rng, 1, c["had"])
    return c


# ---------------------------------------------------------------- shapes that follow from a case
def _pages(tokens, page):
    return -(-tokens // page)


def _shape(case):
    """Tokens of each sequence that are in the cache before the call, and tokens of the call."""
    rng = random.Random(case["mix"])
    n = case["n"]
    had, fresh = [0] * n, [0] * n
    if "had" in case:
        had = [case["had"]] + [rng.randint(case["had_least"], case["had"]) for _ in range(n - 1)]
    if "fresh" in case:
        fresh = [case["fresh"]] + [rng.randint(case["fresh_least"], case["fresh"]) for _ in range(n - 1)]
    rng.shuffle(had)
    rng.shuffle(fresh)
    return had, fresh


def _by(case):
    """By how many positions each sequence moves."""
    rng = random.Random(case["mix"] + 1)
    return [rng.choice([-1, 1]) * rng.randint(0, 9000) for _ in range(case["n"])]


def _scaling(case):
    """How the case's frequencies are scaled: the arguments of set_rotary."""
    return {"none": {}, "linear": dict(factor=4.0), "base": dict(factor=8.0), "bands": dict(factor=16.0, low=1.0, high=32.0, original=8192, magnitude=1.2772588722239782)}[case["scaling"]]


def _type(case):
    return {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}[case["dtype"]]


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    op, kind = case["op"], _type(case)
    st = dict(case=case)
    if op == "score":
        rows, vocab = case["rows"], case["vocab"]
        x = torch.empty(rows, vocab, dtype=kind, device="cuda")
        for a in range(0, rows, 512):
            b = min(rows, a + 512)
            part = normal(b - a, vocab) * 2.5
            if case["banned"]:
                part.masked_fill_(torch.rand(b - a, vocab, device="cuda", generator=g) < case["banned"], float("-inf"))
            x[a:b] = part
        # most rows are sure of some token, which is most rows' target
        likely = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
        sure = torch.rand(rows, device="cuda", generator=g) < 0.7
        at = torch.arange(rows, device="cuda")
        x[at, likely] = torch.where(sure, (8 + 3 * normal(rows)).to(kind), x[at, likely])
        other = torch.randint(0, vocab, (rows,), device="cuda", generator=g)
        st.update(logits=x, targets=torch.where(torch.rand(rows, device="cuda", generator=g) < 0.8, likely, other).to(torch.int32) if case["given"] else None)
        if own:
            from paper_2501_12689_b200 import ICTokenScores
            st["scores"] = ICTokenScores(vocab, dtype=kind)
        return st
    had, fresh = _shape(case)
    n, tokens = case["n"], sum(fresh)
    starts = [0]
    for f in fresh:
        starts.append(starts[-1] + f)
    st.update(seqs=_ints(list(range(n))), counts=_ints(fresh), starts=_ints(starts), most=max(fresh), single=case.get("fresh") == 1 and min(fresh) == 1)
    if op == "state":
        h, dk, dv = case["heads"], case["dk"], case["dv"]
        # sequences with a past, and new ones
        old = torch.rand(n, 1, 1, 1, 1, device="cuda", generator=g) < 0.6
        st["pool"] = torch.where(old, 2.0 * normal(n, 1, h, dk, dv), 0.0)
        st["q"], st["k"] = (torch.nn.functional.silu(1.5 * normal(tokens, h, dk)).to(kind) for _ in range(2))
        st["v"] = normal(tokens, h, dv).to(kind)
        st["rates"] = torch.tensor([case["strength"] * 2.0 ** (-8.0 * (i + 1) / h) for i in range(h)], device="cuda")
        if own:
            from paper_2501_12689_b200 import ICStates
            st["states"] = ICStates(1, h, dk, dv, n, dtype=kind, pool=st["pool"])
        return st
    page, hkv, d = case["page"], case["hkv"], case["d"]
    lens = [a + b for a, b in zip(had, fresh)]
    max_pages = max(4, -(-_pages(max(lens), page) // 4) * 4)
    need = sum(_pages(x, page) for x in lens)
    n_pages = -(-(need + need // 16 + 2) // 64) * 64 + 7
    # a pool that has been in use: the sequences' pages lie anywhere in it
    st["pool"] = torch.randn(n_pages, case["layers"], 2, hkv, page, d, dtype=kind, device="cuda", generator=g)
    order = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)
    st["tables"] = torch.zeros(n, max_pages, dtype=torch.int32, device="cuda")
    st["lengths"] = _ints(lens)
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    owned = torch.arange(max_pages, device="cuda")[None, :] < ((st["lengths"] + page - 1) // page)[:, None]
    st["tables"][owned] = order[:need]
    refs[order[:need].long()] = 1
    if op == "rotate":
        st["q"] = normal(tokens, case["hq"], d).to(kind)
        st["k"], st["v"] = (normal(tokens, hkv, d).to(kind) for _ in range(2))
    else:
        st["by"] = _ints(_by(case))
    st["f"], st["magnitude"] = _plain_frequencies(case)
    if own:
        from paper_2501_12689_b200 import ICPagedKV
        st["kv"] = ICPagedKV(n_pages, case["layers"], hkv, page, d, n, max_pages, dtype=kind, pool=st["pool"], tables=st["tables"], lengths=st["lengths"], refs=refs)
        st["kv"].set_rotary(case["rotary"], base=10000.0, interleaved=case["interleaved"], scaling=case["scaling"], **_scaling(case))
    return st


def run(st):
    op = st["case"]["op"]
    if op == "rotate":
        starts = None if st["single"] else st["starts"]
        if own:
            out = st["kv"].write_rotated(LAYER, st["q"], st["k"], st["v"], st["seqs"], starts)
        else:
            out = _plain_rotate(st)
        return dict(q=out, pool=st["pool"])
    if op == "shift":
        if own:
            st["kv"].shift(st["seqs"], st["by"])
        else:
            _plain_shift(st)
        return dict(pool=st["pool"])
    if op == "score":
        c = st["case"]
        if own:
            r = st["scores"].score(st["logits"], st["targets"], n_top=c["top"], scale=c["scale"])
            r = dict(log_probs=r.log_probs, entropy=r.entropy, top_ids=r.top_ids, top_log_probs=r.top_log_probs)
        else:
            r = _plain_score(st["logits"], st["targets"], c["top"], c["scale"])
        return {k: v for k, v in r.items() if v is not None}
    if own:
        if st["single"]:
            out = st["states"].decode(LAYER, st["q"], st["k"], st["v"], st["rates"], st["seqs"])
        else:
            out = st["states"].extend(LAYER, st["q"], st["k"], st["v"], st["rates"], st["seqs"], st["starts"])
    else:
        out = _plain_state(st)
    return dict(out=out, pool=st["pool"])


# ---------------------------------------------------------------- the plain forms
def _plain_frequencies(case):
    """Radians per token of each pair, in 64 bits, and the factor of the result."""
    s, dim = _scaling(case), case["rotary"]
    i = torch.arange(dim // 2, dtype=torch.float64, device="cuda")
    base = 10000.0
    if case["scaling"] == "base" and dim > 2:
        base *= s["factor"] ** (dim / (dim - 2))
    f = base ** (-2.0 * i / dim)
    if case["scaling"] == "linear":
        f = f / s["factor"]
    if case["scaling"] == "bands":
        turns = s["original"] * f / (2 * math.pi)
        kept = ((turns - s["low"]) / (s["high"] - s["low"])).clamp(0.0, 1.0)
        f = kept * f + (1.0 - kept) * f / s["factor"]
    return f, s.get("magnitude", 1.0)


def _plain_turn(st, x, position, scaled=True):
    """x [tokens, heads, d] at these positions; angles in 64 bits (a position is far from the first), the rest in 32."""
    case = st["case"]
    dim = case["rotary"]
    angle = position.double()[:, None] * st["f"]
    m = st["magnitude"] if scaled else 1.0
    cos, sin = (angle.cos() * m).float()[:, None], (angle.sin() * m).float()[:, None]
    out = x.float()
    a, b = (out[..., 0:dim:2], out[..., 1:dim:2]) if case["interleaved"] else (out[..., :dim // 2], out[..., dim // 2:dim])
    a, b = a * cos - b * sin, a * sin + b * cos
    out = torch.cat([torch.stack([a, b], -1).flatten(-2) if case["interleaved"] else torch.cat([a, b], -1), out[..., dim:]], -1)
    return out.to(x.dtype)


def _plain_rotate(st):
    pool, page, total = st["pool"], st["case"]["page"], st["q"].shape[0]
    counts = st["counts"].long()
    i = torch.repeat_interleave(torch.arange(counts.numel(), device="cuda"), counts, output_size=total)
    at = st["lengths"].long()[i] - counts[i] + torch.arange(total, device="cuda") - st["starts"].long()[i]
    where = st["tables"][i, at // page].long()
    pool[where, LAYER, 0, :, at % page] = _plain_turn(st, st["k"], at)
    pool[where, LAYER, 1, :, at % page] = st["v"]
    return _plain_turn(st, st["q"], at)


def _plain_shift(st):
    pool, page = st["pool"], st["case"]["page"]
    total = sum(_shape(st["case"])[0])
    lens = st["lengths"].long()
    i = torch.repeat_interleave(torch.arange(lens.numel(), device="cuda"), lens, output_size=total)
    at = torch.arange(total, device="cuda") - (torch.cumsum(lens, 0) - lens)[i]
    where = st["tables"][i, at // page].long()
    keys = pool[where, :, 0, :, at % page]                       # [tokens, layers, heads, d]
    pool[where, :, 0, :, at % page] = _plain_turn(st, keys.flatten(1, 2), st["by"][i], scaled=False).view(keys.shape)


def _plain_score(logits, targets, top, scale):
    x = logits.float() * scale
    best = x.amax(-1, keepdim=True)
    best = torch.where(best == float("-inf"), 0.0, best)
    e = (x - best).exp()
    total = e.sum(-1, keepdim=True)
    total = torch.where(total == 0, 1.0, total)                  # a row that bans every token: nothing has a probability
    log_total = total.log()
    entropy = log_total[:, 0] - torch.where(e == 0, 0.0, e * (x - best)).sum(-1) / total[:, 0]
    r = dict(log_probs=None, entropy=entropy, top_ids=None, top_log_probs=None)
    if targets is not None:
        r["log_probs"] = (x.gather(1, targets.long()[:, None]) - best - log_total)[:, 0]
    if top:
        # the logits as whole numbers in their order, the lowest index first among equals
        bits = (logits.float() + 0.0).view(torch.int32).long()
        key = torch.where(bits < 0, -(bits & 0x7fffffff) - 1, bits) * (1 << 32) - torch.arange(x.shape[1], device="cuda")
        ids = key.topk(top, -1).indices
        r["top_ids"], r["top_log_probs"] = ids.to(torch.int32), x.gather(1, ids) - best - log_total
    return r


def _plain_state(st, chunk=128):
    """Chunks of tokens: within a chunk as masked products, between chunks by the states at their borders."""
    case, pool = st["case"], st["pool"]
    n, h, dk, dv = case["n"], case["heads"], case["dk"], case["dv"]
    counts, total = st["counts"].long(), st["q"].shape[0]
    i = torch.repeat_interleave(torch.arange(n, device="cuda"), counts, output_size=total)
    t = torch.arange(total, device="cuda") - st["starts"].long()[i]
    chunk = min(chunk, st["most"])
    c = -(-st["most"] // chunk)
    padded = lambda x: torch.zeros(n, c * chunk, h, x.shape[-1], device="cuda").index_put_((i, t), x.float()).transpose(1, 2)  # noqa: E731
    q, k, v = (padded(st[x]) for x in "qkv")
    rate, old = st["rates"].double()[:, None], pool[:, LAYER].clone()
    decay = lambda steps: torch.where(steps < 0, 0.0, torch.exp(-rate.view(-1, *[1] * steps.dim()) * steps.clamp(min=0))).float()  # noqa: E731
    split = lambda x: x.reshape(n, h, c, chunk, -1)  # noqa: E731
    at = torch.arange(chunk, device="cuda")
    # what each chunk adds, and with that the state in front of each chunk
    added = (split(k) * decay(chunk - 1 - at)[:, None, :, None]).transpose(-1, -2) @ split(v)            # [n, h, c, dk, dv]
    many = torch.arange(c, device="cuda")
    before = (decay((many[:, None] - 1 - many) * chunk) @ added.flatten(-2)).view(added.shape)
    before += decay(many * chunk)[:, :, None, None] * old[:, :, None]
    p = (split(q) @ split(k).transpose(-1, -2)) * decay(at[:, None] - at)[:, None]
    out = p @ split(v) + decay(at + 1)[:, None, :, None] * (split(q) @ before)
    left = counts[:, None, None] - 1 - torch.arange(c * chunk, device="cuda")                            # [n, 1, tokens]
    weight = torch.where(left < 0, 0.0, torch.exp(-rate * left.clamp(min=0))).float()
    pool[:, LAYER] = (k * weight[..., None]).transpose(-1, -2) @ v + torch.exp(-rate * counts[:, None, None]).float()[..., None] * old
    return (out.view(n, h, -1, dv)[i, :, t] * dk ** -0.5).to(st["q"].dtype)


# ---------------------------------------------------------------- what the path cannot do without
def work(case):
    op = case["op"]
    if op == "score":
        wide = 4 if case["dtype"] == "fp32" else 2
        return dict(bytes=case["rows"] * (case["vocab"] * wide + 12 + 8 * case["top"]), flops=0)
    had, fresh = _shape(case)
    if op == "rotate":
        return dict(bytes=sum(fresh) * (case["hq"] + 2 * case["hkv"]) * case["d"] * 2 * 2, flops=0)
    if op == "shift":
        return dict(bytes=sum(had) * case["layers"] * case["hkv"] * case["rotary"] * 2 * 2, flops=0)
    tokens, h, dk, dv = sum(fresh), case["heads"], case["dk"], case["dv"]
    return dict(bytes=tokens * h * (2 * dk + 2 * dv) * 2 + case["n"] * h * dk * dv * 4 * 2, flops=4 * tokens * h * dk * dv)


# ---------------------------------------------------------------- the operators' values, from their definitions
def _exact_turned(case, x, position, magnitude):
    """x [..., d] in 64 bits as complex numbers, one a pair, times e^(i angle)."""
    s, dim = _scaling(case), case["rotary"]
    f = []
    for i in range(dim // 2):
        b = 10000.0 * (s["factor"] ** (dim / (dim - 2.0)) if case["scaling"] == "base" and dim > 2 else 1.0)
        w = 1.0 / b ** (2.0 * i / dim)
        if case["scaling"] == "linear":
            w /= s["factor"]
        elif case["scaling"] == "bands":
            turns = s["original"] / (2.0 * math.pi / w)
            part = min(1.0, max(0.0, (turns - s["low"]) / (s["high"] - s["low"])))
            w = part * w + (1.0 - part) * w / s["factor"]
        f.append(w)
    turn = torch.polar(torch.full((), magnitude, dtype=torch.float64, device="cuda"), position.double()[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda"))
    out = x.double().clone()
    pairs = (slice(0, dim, 2), slice(1, dim, 2)) if case["interleaved"] else (slice(0, dim // 2), slice(dim // 2, dim))
    z = torch.complex(out[..., pairs[0]], out[..., pairs[1]]) * turn[:, None]
    out[..., pairs[0]], out[..., pairs[1]] = z.real, z.imag
    return out


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "score":
        return _exact_score(case, st)
    if op == "state":
        return _exact_state(case, st)
    had, fresh = _shape(case)
    page, pool = case["page"], st["pool"].double()
    m = _scaling(case).get("magnitude", 1.0)
    if op == "shift":
        by = _by(case)
        for s, x in enumerate(had):
            row = st["tables"][s, :_pages(x, page)].long()
            keys = pool[row, :, 0]                               # [pages, layers, heads, slots, d]
            turned = _exact_turned(case, keys.view(1, -1, case["d"]), _ints([by[s]]), 1.0).view(keys.shape)
            turned[-1, :, :, x - (len(row) - 1) * page:] = keys[-1, :, :, x - (len(row) - 1) * page:]
            pool[row, :, 0] = turned
        return dict(pool=pool)
    q, start = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda"), 0
    rows = st["tables"].tolist()
    for s, f in enumerate(fresh):
        part = slice(start, start + f)
        at = torch.arange(had[s], had[s] + f, device="cuda")
        q[part] = _exact_turned(case, st["q"][part], at, m)
        keys = _exact_turned(case, st["k"][part], at, m)
        done = 0
        while done < f:                                          # page by page
            a = had[s] + done
            some = min(page - a % page, f - done)
            for x, new in ((0, keys), (1, st["v"][part].double())):
                pool[rows[s][a // page], LAYER, x, :, a % page:a % page + some] = new[done:done + some].transpose(0, 1)
            done += some
        start += f
    return dict(q=q, pool=pool)


def _exact_score(case, st):
    got = dict(log_probs=[], entropy=[], top_ids=[], top_log_probs=[])
    for a in range(0, case["rows"], 256):
        x = st["logits"][a:a + 256]
        y = x.double() * case["scale"]
        size = torch.logsumexp(y, -1, keepdim=True)
        y = y - torch.where(size == -math.inf, 0.0, size)
        got["entropy"].append(-torch.where(y == -math.inf, 0.0, y.exp() * y).sum(-1))
        if case["given"]:
            got["log_probs"].append(y[torch.arange(len(y), device="cuda"), st["targets"][a:a + 256].long()])
        if case["top"]:
            ids = torch.sort(x, stable=True, dim=-1, descending=True).indices[:, :case["top"]]      # equal ones stay in their order
            got["top_ids"].append(ids.to(torch.int32))
            got["top_log_probs"].append(y.gather(1, ids))
    return {k: torch.cat(v) for k, v in got.items() if v}


def _exact_state(case, st):
    """Every output as a sum over all earlier tokens, sequence by sequence and head by head."""
    _, fresh = _shape(case)
    h, dk, dv = case["heads"], case["dk"], case["dv"]
    if sum(f * f for f in fresh) * h * (dk + dv) > 8e12:
        return None
    out = torch.zeros(st["v"].shape, dtype=torch.float64, device="cuda")
    pool, start = st["pool"].double(), 0
    for s, f in enumerate(fresh):
        for x in range(h):
            r = float(st["rates"][x])
            q, k, v = (st[y][start:start + f, x].double() for y in "qkv")
            old = pool[s, LAYER, x].clone()
            at = torch.arange(f, dtype=torch.float64, device="cuda")
            for a in range(0, f, 2048):
                b = min(f, a + 2048)
                steps = at[a:b, None] - at[None, :b]
                w = torch.where(steps < 0, 0.0, torch.exp(-r * steps.clamp(min=0))) * (q[a:b] @ k[:b].T)
                out[start + a:start + b, x] = (w @ v[:b] + torch.exp(-r * (at[a:b] + 1))[:, None] * (q[a:b] @ old)) / math.sqrt(dk)
            pool[s, LAYER, x] = (k * torch.exp(-r * (f - 1 - at))[:, None]).T @ v + math.exp(-r * f) * old
        start += f
    return dict(out=out, pool=pool)
