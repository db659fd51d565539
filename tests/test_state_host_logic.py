"""CPU-only checks of the state cache's ABI: exported symbols, header constants, struct layouts, refused options."""
import ctypes
import os
import re

import pytest
import torch

import paper_2501_12689_b200 as pkg
from paper_2501_12689_b200 import states

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ic_state.h")).read(), flags=re.S)


def test_library_exports_every_declared_symbol():
    from paper_2501_12689_b200.build import build
    names = sorted(set(re.findall(r"\b(ic_state_[a-z_]+)\s*\(", _header())))
    assert "ic_state_attend" in names and len(names) == len(states.SIGNATURES)
    for lib in (ctypes.CDLL(build()), ctypes.CDLL(build(debug_checks=True))):
        for name in names:
            assert hasattr(lib, name) and name in states.SIGNATURES, name


def test_constants_and_structs_match_the_header():
    text = _header()
    for name in ("IC_STATE_MAX_KEY_DIM", "IC_STATE_MAX_VALUE_DIM", "IC_STATE_MAX_SEQS"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(pkg, name)
    assert re.search(r"IC_STATE_BF16 = 0, IC_STATE_F16 = 1", text) and (pkg.IC_STATE_BF16, pkg.IC_STATE_F16) == (0, 1)
    for name, struct in (("ic_state_opts", states.ic_state_opts_t), ("ic_state_attend", states.ic_state_attend_t)):
        body = re.search(rf"typedef struct {name} {{(.*?)}} {name}_t;", text, re.S).group(1)
        assert re.findall(r"(\w+)\s*;", body) == [f for f, _ in struct._fields_]
    assert ctypes.sizeof(states.ic_state_opts_t) == 32 + 4 * 8
    assert ctypes.sizeof(states.ic_state_attend_t) == 16 + 8 + 12 * 8 + 3 * 8


@pytest.mark.parametrize("change", [dict(n_layers=0), dict(n_layers=1025), dict(n_heads=0), dict(n_heads=1025), dict(key_dim=0), dict(key_dim=12),
                                    dict(key_dim=136), dict(value_dim=0), dict(value_dim=20), dict(value_dim=264), dict(max_seqs=0),
                                    dict(max_seqs=8193)])
def test_invalid_sizes(change):
    sizes = dict(n_layers=2, n_heads=8, key_dim=128, value_dim=128, max_seqs=64)
    assert pkg.ic_state_workspace_bytes(**sizes) > 0
    assert pkg.ic_state_workspace_bytes(**{**sizes, **change}) == 0 and pkg.ic_cache_last_error()
    with pytest.raises(pkg.ICCacheError):
        pkg.ICStates(**{**sizes, **change})


def test_null_handles_and_types():
    lib = states._library()
    assert lib.ic_state_create(None) is None
    assert lib.ic_state_attend(None, None) == pkg.IC_ERR_INVALID
    assert lib.ic_state_fork(None, None, None, 1) == pkg.IC_ERR_INVALID and lib.ic_state_clear(None, None, 1) == pkg.IC_ERR_INVALID
    assert lib.ic_state_sync(None) == pkg.IC_ERR_INVALID
    lib.ic_state_destroy(None)
    with pytest.raises(TypeError):
        pkg.ic_state_workspace_bytes(1, 1, 8, 8, 1, torch.float32)
    if not torch.cuda.is_available():
        o = states._options(1, 1, 8, 8, 1, torch.bfloat16)
        assert lib.ic_state_create(ctypes.byref(o)) is None and "no CPU fallback" in pkg.ic_cache_last_error()
