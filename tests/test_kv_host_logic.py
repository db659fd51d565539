"""CPU-only checks of the paged cache's ABI: exported symbols, header constants, refused options, and hand-worked cases that pin
the plain model the GPU tests compare with."""
import ctypes
import os
import re

import pytest
import torch

import paper_2501_12689_b200 as pkg
from kv_util import Model
from paper_2501_12689_b200 import paged_kv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _header():
    text = open(os.path.join(ROOT, "include", "ic_kv.h")).read()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_library_exports_every_declared_symbol():
    from paper_2501_12689_b200.build import build
    names = sorted(set(re.findall(r"\b(ic_kv_[a-z_]+)\s*\(", _header())))
    assert "ic_kv_create" in names and len(names) == len(paged_kv.SIGNATURES)
    for lib in (ctypes.CDLL(build()), ctypes.CDLL(build(debug_checks=True))):
        for name in names:
            assert hasattr(lib, name) and name in paged_kv.SIGNATURES, name


def test_header_constants_match_binding():
    text = _header()
    for name in ("IC_KV_MAX_HEAD_DIM", "IC_KV_MAX_PAGE", "IC_KV_MAX_SEQS"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(pkg, name)
    assert re.search(r"IC_KV_BF16 = 0, IC_KV_F16 = 1", text) and (pkg.IC_KV_BF16, pkg.IC_KV_F16) == (0, 1)


def test_struct_layouts_match_the_header():
    """Fields in the header's order; sizes as the C compiler lays them out."""
    text = _header()
    for name, struct in (("ic_kv_opts", paged_kv.ic_kv_opts_t), ("ic_kv_attend", paged_kv.ic_kv_attend_t)):
        body = re.search(rf"typedef struct {name} {{(.*?)}} {name}_t;", text, re.S).group(1)
        fields = re.findall(r"(\w+)\s*;", body)
        assert fields == [f for f, _ in struct._fields_]
    assert ctypes.sizeof(paged_kv.ic_kv_opts_t) == 40 + 7 * 8
    assert ctypes.sizeof(paged_kv.ic_kv_attend_t) == 16 + 8 + 16 + 8 * 8


@pytest.mark.parametrize("change", [dict(n_pages=0), dict(n_layers=0), dict(n_kv_heads=0), dict(page_size=12), dict(page_size=4),
                                    dict(page_size=512), dict(head_dim=0), dict(head_dim=20), dict(head_dim=264), dict(max_seqs=0),
                                    dict(max_seqs=16385), dict(max_pages=0), dict(max_pages=1 << 28), dict(n_pages=1 << 30)])
def test_invalid_sizes(change):
    sizes = dict(n_pages=100, n_layers=2, n_kv_heads=8, page_size=16, head_dim=128, max_seqs=64, max_pages=32)
    assert pkg.ic_kv_workspace_bytes(**sizes) > 0
    assert pkg.ic_kv_workspace_bytes(**{**sizes, **change}) == 0
    assert pkg.ic_cache_last_error()


def test_null_handles_and_options():
    lib = paged_kv._library()
    assert lib.ic_kv_create(None) is None
    assert lib.ic_kv_reserve(None, None, None, 1) == pkg.IC_ERR_INVALID
    assert lib.ic_kv_attend(None, None) == pkg.IC_ERR_INVALID
    assert lib.ic_kv_sync(None) == pkg.IC_ERR_INVALID and lib.ic_kv_compact(None) == pkg.IC_ERR_INVALID
    lib.ic_kv_destroy(None)
    if not torch.cuda.is_available():
        o = paged_kv._options(4, 1, 1, 16, 64, 1, 1, torch.bfloat16)
        assert lib.ic_kv_create(ctypes.byref(o)) is None and "no CPU fallback" in pkg.ic_cache_last_error()


def test_model_pins():
    m = Model(8, 4, 4, 6)
    assert m.reserve([1, 0], [5, 4])
    assert m.rows == [[2], [0, 1], [], []] and m.lens == [4, 5, 0, 0] and m.refs == [1, 1, 1, 0, 0, 0, 0, 0]
    assert not m.reserve([0, 1], [16, 8])                      # 4 + 2 pages of 5
    assert m.fork([1, 1, 0], [2, 3, 0]) == [(1, 3), (1, 4)]     # the full page shared, the tail copied; 0 stays
    assert m.rows == [[2], [0, 1], [0, 3], [0, 4]] and m.refs == [3, 1, 1, 1, 1, 0, 0, 0]
    assert m.fork([1, 2], [2, 1], [4, 2]) == [(0, 5)]          # both from the rows before the call
    assert m.rows == [[2], [5], [0], [0, 4]] and m.refs == [2, 0, 1, 0, 1, 1, 0, 0] and m.lens == [4, 2, 4, 5]
    m.free([0, 0])
    assert m.refs == [2, 0, 0, 0, 1, 1, 0, 0]
    assert m.compact() == [(4, 1), (5, 2)]
    assert m.rows == [[], [2], [0], [0, 1]] and m.refs == [2, 1, 1, 0, 0, 0, 0, 0]
    assert m.fork([3], [3], [5], copy=True) == [(0, 3), (1, 4)] and m.refs == [1, 0, 1, 1, 1, 0, 0, 0]
