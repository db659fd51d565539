"""The example that runs retrieval and the paged cache together, with every attention in it against the formula in 64 bits."""
import importlib.util
import os

import pytest
import torch

from kv_util import attention, close

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("serve_with_examples", os.path.join(ROOT, "examples", "serve_with_examples.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_requests_behind_shared_examples():
    seen = []

    def check(kv, layer, q, out, seqs, counts):
        # (later layers have been written by now; a layer's own keys and values are as the call saw them)
        want, size = attention(kv, layer, q, seqs, counts)
        seen.append(close(out, want, size))

    kv, found, x, used = _example().serve(check=check)
    assert len(seen) == 2 * 2 + 4 * 2 and torch.isfinite(x.float()).all()
    assert (kv.refs > 1).any()
    before = [kv.pool[kv.tables[s, :2].long()].clone() for s in range(3)]
    held = kv.lengths.clone()
    kv.free(torch.tensor(used, dtype=torch.int32, device=kv.device))
    kv.compact()
    kv.sync()
    live = int((kv.refs > 0).sum())
    assert (kv.refs[:live] == 1).all() and not kv.refs[live:].any()
    assert torch.equal(kv.lengths[:40], held[:40]) and not kv.lengths[40:].any()
    for s, b in enumerate(before):
        n = min(2, -(-int(held[s]) // kv.page_size))
        rest = int(held[s]) - (n - 1) * kv.page_size
        now = kv.pool[kv.tables[s, :n].long()]
        assert torch.equal(now[: n - 1], b[: n - 1]) and torch.equal(now[n - 1, ..., :min(rest, kv.page_size), :], b[n - 1, ..., :min(rest, kv.page_size), :])
