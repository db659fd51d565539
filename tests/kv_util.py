"""Shared helpers of the paged-cache tests: a plain model of the page operations and attention in 64 bits, written from the
definitions in include/ic_kv.h and sharing nothing with the library."""
from __future__ import annotations

import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # unit roundoff


class Model:
    """Page tables, lengths and reference counts as Python lists; `moves` collects the page copies of a call."""

    def __init__(self, n_pages, page, max_seqs, max_pages):
        self.page, self.max_pages = page, max_pages
        self.refs = [0] * n_pages
        self.rows = [[] for _ in range(max_seqs)]
        self.lens = [0] * max_seqs

    def _pages(self, tokens):
        return -(-tokens // self.page)

    def _vacant(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def reserve(self, seqs, counts):
        """True, or False with nothing changed where pages or a row run out."""
        new = [self._pages(self.lens[s] + c) - self._pages(self.lens[s]) for s, c in zip(seqs, counts)]
        vacant = self._vacant()
        if sum(new) > len(vacant) or any(self._pages(self.lens[s] + c) > self.max_pages for s, c in zip(seqs, counts)):
            return False
        for s, c, x in zip(seqs, counts, new):
            for _ in range(x):
                p = vacant.pop(0)
                self.rows[s].append(p)
                self.refs[p] = 1
            self.lens[s] += c
        return True

    def fork(self, parents, children, upto=None, copy=False):
        """The list of (from, to) page copies, or None with nothing changed."""
        rows, lens, refs = [list(r) for r in self.rows], list(self.lens), list(self.refs)
        vacant, moves, drop = self._vacant(), [], []
        for i, (a, b) in enumerate(zip(parents, children)):
            x = self.lens[a] if upto is None else upto[i]
            if a == b and x == self.lens[a] and not copy:
                continue
            row = []
            for c in range(self._pages(x)):
                if not copy and (c + 1) * self.page <= x:
                    row.append(self.rows[a][c])
                    refs[row[-1]] += 1
                else:
                    if not vacant:
                        return None
                    p = vacant.pop(0)
                    moves.append((self.rows[a][c], p))
                    refs[p] = 1
                    row.append(p)
            drop += self.rows[b]
            rows[b] = row
            lens[b] = x
        for p in drop:
            refs[p] -= 1
        self.rows, self.lens, self.refs = rows, lens, refs
        return moves

    def free(self, seqs):
        for s in seqs:
            for p in self.rows[s]:
                self.refs[p] -= 1
            self.rows[s], self.lens[s] = [], 0

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r]
        n = len(live)
        holes = [p for p in range(n) if self.refs[p] == 0]
        to = dict(zip([p for p in live if p >= n], holes))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.rows = [[to.get(p, p) for p in r] for r in self.rows]
        return list(to.items())

    def check(self, kv):
        """The device state is this model's, and the counts are those of the rows."""
        lens, refs, tables = kv.lengths.cpu().tolist(), kv.refs.cpu().tolist(), kv.tables.cpu().tolist()
        assert lens == self.lens
        assert refs == self.refs
        for s, r in enumerate(self.rows):
            assert tables[s][:len(r)] == r, f"row {s}"
        count = [0] * len(self.refs)
        for r in self.rows:
            for p in r:
                count[p] += 1
        assert count == self.refs


def gathered(kv, layer, s, length):
    """Keys and values [length, n_kv_heads, head_dim] of a sequence, in 64 bits."""
    row = kv.tables[s, :-(-length // kv.page_size)].long()
    x = kv.pool[row, layer].double()                                  # [pages, 2, heads, page, dim]
    x = x.permute(1, 0, 3, 2, 4).reshape(2, -1, kv.n_kv_heads, kv.head_dim)[:, :length]
    return x[0], x[1]


def attention(kv, layer, q, seqs, counts, window=0, sinks=0, scale=None):
    """(out, sum of weight * |v|) in 64 bits, token by token block; zeros where nothing is visible."""
    scale = 1.0 / math.sqrt(kv.head_dim) if scale is None else scale
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    size = torch.zeros_like(out)
    g, t0 = q.shape[1] // kv.n_kv_heads, 0
    for s, f in zip(seqs, counts):
        length = int(kv.lengths[s])
        k, v = gathered(kv, layer, s, length)
        for a in range(0, f, 512):
            b = min(f, a + 512)
            p = torch.arange(length - f + a, length - f + b, device=q.device)[:, None]
            j = torch.arange(length, device=q.device)[None]
            seen = j <= p
            if window:
                seen &= (j > p - window) | (j < sinks)
            # keys that nobody sees may hold anything
            anyone = seen.any(0)
            kk, vv, ss = k[anyone], v[anyone], seen[:, anyone]
            x = q[t0 + a:t0 + b].double().view(b - a, kv.n_kv_heads, g, kv.head_dim)
            w = torch.einsum("thgd,jhd->thgj", x, kk) * scale
            w = w.masked_fill(~ss[:, None, None], -math.inf)
            top = w.amax(-1, keepdim=True) if w.shape[-1] else w.new_full(w.shape[:-1] + (1,), -math.inf)
            w = torch.exp(w - torch.where(top == -math.inf, 0.0, top))
            total = w.sum(-1, keepdim=True)
            w = w / torch.where(total == 0, 1.0, total)
            for to, vals in ((out, vv), (size, vv.abs())):
                to[t0 + a:t0 + b] = torch.einsum("thgj,jhd->thgd", w, vals).reshape(b - a, q.shape[1], kv.head_dim)
        t0 += f
    return out, size


def close(got, want, size):
    """got rounds a weighted sum whose weights may have been rounded once: half a unit in the last place of the result, twice
    the unit roundoff of the weights (rounded weight, and their sum against the rounded ones), and the fp32 scores' error:
    a score of magnitude up to ~100 off by 2**-24 * 100 * a few, below 1e-4 of relative weight, above and below the line."""
    u = UNIT[got.dtype]
    bound = u * want.abs() + (2 * u + 2e-4) * size + 2.0 ** -24
    off = (got.double() - want).abs()
    assert torch.isfinite(got).all(), "not finite"
    worst = (off / bound).max().item() if got.numel() else 0.0
    assert worst <= 1.0, f"{worst:.2f} times the bound"
    return worst
