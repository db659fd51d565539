"""CPU-only checks of the token scores' ABI: exported symbols, header constants, struct layouts, refused options."""
import ctypes
import os
import re

import pytest
import torch

import paper_2501_12689_b200 as pkg
from paper_2501_12689_b200 import token_scores

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ic_score.h")).read(), flags=re.S)


def test_library_exports_every_declared_symbol():
    from paper_2501_12689_b200.build import build
    names = sorted(set(re.findall(r"\b(ic_score_[a-z_]+)\s*\(", _header())))
    assert "ic_score_tokens" in names and len(names) == len(token_scores.SIGNATURES)
    for lib in (ctypes.CDLL(build()), ctypes.CDLL(build(debug_checks=True))):
        for name in names:
            assert hasattr(lib, name) and name in token_scores.SIGNATURES, name


def test_constants_and_structs_match_the_header():
    text = _header()
    for name in ("IC_SCORE_MAX_TOP", "IC_SCORE_MAX_VOCAB"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(pkg, name)
    assert re.search(r"IC_SCORE_BF16 = 0, IC_SCORE_F16 = 1, IC_SCORE_F32 = 2", text)
    assert (pkg.IC_SCORE_BF16, pkg.IC_SCORE_F16, pkg.IC_SCORE_F32) == (0, 1, 2)
    for name, struct in (("ic_score_opts", token_scores.ic_score_opts_t), ("ic_score_args", token_scores.ic_score_args_t)):
        body = re.search(rf"typedef struct {name} {{(.*?)}} {name}_t;", text, re.S).group(1)
        assert re.findall(r"(\w+)\s*;", body) == [f for f, _ in struct._fields_]
    assert ctypes.sizeof(token_scores.ic_score_opts_t) == 16 + 3 * 8
    assert ctypes.sizeof(token_scores.ic_score_args_t) == 8 + 8 + 8 + 7 * 8


def test_invalid_options_and_null_handles():
    assert pkg.ic_score_workspace_bytes(32000) > 0
    for vocab in (0, -1, pkg.IC_SCORE_MAX_VOCAB + 1):
        assert pkg.ic_score_workspace_bytes(vocab) == 0 and pkg.ic_cache_last_error()
    with pytest.raises(TypeError):
        pkg.ic_score_workspace_bytes(100, torch.float64)
    with pytest.raises(pkg.ICCacheError):
        pkg.ICTokenScores(0)
    lib = token_scores._library()
    assert lib.ic_score_create(None) is None
    assert lib.ic_score_tokens(None, None) == pkg.IC_ERR_INVALID
    assert lib.ic_score_sync(None) == pkg.IC_ERR_INVALID and lib.ic_score_set_stream(None, None) == pkg.IC_ERR_INVALID
    lib.ic_score_destroy(None)
    if not torch.cuda.is_available():
        assert lib.ic_score_create(ctypes.byref(token_scores._options(100, torch.float32))) is None
        assert "no CPU fallback" in pkg.ic_cache_last_error()
