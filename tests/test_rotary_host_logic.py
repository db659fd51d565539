"""CPU-only checks of rotary positions: the frequencies against their formulas, refused options, struct layouts."""
import ctypes
import math
import os
import re

import pytest

import paper_2501_12689_b200 as pkg
from paper_2501_12689_b200 import paged_kv, rotary_frequencies

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layouts_match_the_header():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ic_kv.h")).read(), flags=re.S)
    for name, struct in (("ic_kv_rotary", paged_kv.ic_kv_rotary_t), ("ic_kv_rotate", paged_kv.ic_kv_rotate_t)):
        body = re.search(rf"typedef struct {name} {{(.*?)}} {name}_t;", text, re.S).group(1)
        assert re.findall(r"(\w+)\s*;", body) == [f for f, _ in struct._fields_]
    assert ctypes.sizeof(paged_kv.ic_kv_rotary_t) == 16 + 7 * 8
    assert ctypes.sizeof(paged_kv.ic_kv_rotate_t) == 16 + 8 + 8 + 13 * 8
    assert [s.upper() for s in paged_kv.ROTARY_SCALINGS] == re.findall(r"IC_KV_ROTARY_(NONE|LINEAR|BASE|BANDS) = \d", text)


@pytest.mark.parametrize("dim", [2, 4, 20, 64, 256])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 0.5])
def test_frequencies(dim, base):
    f = [base ** (-2.0 * i / dim) for i in range(dim // 2)]
    close = lambda got, want: all(abs(a - b) <= 1e-14 * abs(b) for a, b in zip(got, want)) and len(got) == len(want)  # noqa: E731
    assert close(rotary_frequencies(dim, base=base), f)
    assert close(rotary_frequencies(dim, base=base, scaling="linear", factor=8.0), [x / 8.0 for x in f])
    wide = base * 8.0 ** (dim / (dim - 2.0)) if dim > 2 else base
    assert close(rotary_frequencies(dim, base=base, scaling="base", factor=8.0), [wide ** (-2.0 * i / dim) for i in range(dim // 2)])
    want = []
    for x in f:
        w = min(1.0, max(0.0, (4096 * x / (2 * math.pi) - 1.0) / (32.0 - 1.0)))
        want.append(w * x + (1.0 - w) * x / 8.0)
    assert close(rotary_frequencies(dim, base=base, scaling="bands", factor=8.0, low=1.0, high=32.0, original=4096), want)


@pytest.mark.parametrize("change", [dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=258), dict(base=-1.0), dict(base=math.inf),
                                    dict(factor=-2.0), dict(factor=math.nan), dict(scaling="bands", original=0.0),
                                    dict(scaling="bands", original=10.0, low=2.0, high=2.0), dict(scaling="bands", original=10.0, low=-1.0)])
def test_refused_options(change):
    args = {**dict(rotary_dim=64), **change}
    with pytest.raises(pkg.ICCacheError) as e:
        rotary_frequencies(**args)
    assert e.value.status == pkg.IC_ERR_INVALID


def test_refused_arguments():
    with pytest.raises(ValueError):
        rotary_frequencies(64, scaling="other")
    with pytest.raises(ValueError):
        rotary_frequencies(64, base=0.0)
    lib = paged_kv._library()
    assert lib.ic_kv_set_rotary(None, None) == pkg.IC_ERR_INVALID
    assert lib.ic_kv_rotate(None, None) == pkg.IC_ERR_INVALID
    assert lib.ic_kv_shift(None, None, None, 1) == pkg.IC_ERR_INVALID
    r = paged_kv._rotary(64, 1e4, False, "none", 1.0, 1.0, 32.0, 0.0, 1.0, None)
    assert lib.ic_kv_rotary_frequencies(ctypes.byref(r), None) == pkg.IC_ERR_INVALID
    r.struct_size = 1000
    assert lib.ic_kv_rotary_frequencies(ctypes.byref(r), (ctypes.c_double * 32)()) == pkg.IC_ERR_INVALID


def test_a_result_without_queries_is_refused():
    """Before anything is stored."""
    import torch
    kv = object.__new__(pkg.ICPagedKV)
    kv._r, kv._h = paged_kv.ic_kv_rotate_t(), None
    rows, one = torch.zeros(1, 2, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="there is no q"):
        kv.write_rotated(0, None, rows, rows, one, out=rows)
