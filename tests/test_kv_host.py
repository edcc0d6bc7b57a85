"""Host side of the cached-history calls: its C++ functions that are not part of the C ABI,
sizes that have to pass or to be refused, and what the binding does around a call."""
import ctypes
import os

import numpy as np
import pytest

import paper_2609_34144_amd as cast
from test_abi import _HAS_GPU
from test_kv_abi import A, append, cache, rope, seqs

HIP = 6                          # what a launch gives without a GPU


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cast.LIB_PATH):
        pytest.skip("libcast.so not built (run __graft_entry__.build())")
    return cast.load()


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_loads_of_a_tile_of_codes_stay_inside_it(lib, dh):
    """The rows that the four waves' loads cover are those of the 64-key tile, each once: rows
    behind them may lie behind the cache."""
    first = lib._ZN4cast17kv_attn_code_rowsEiii
    rows = []
    for wave in range(4):
        for i in range(4):
            at = first(dh, wave, i)
            if at >= 0:
                rows += range(at, at + 1024 // dh)            # 64 lanes, dh / 16 of them to a row
    assert sorted(rows) == list(range(64))


def test_pages_far_longer_than_the_call_are_taken(lib):
    """The work of an append goes by the call's tokens, not by what its pages could hold: 2048 (page,
    head) pieces of 200 tokens in pages of 524288 pass every check (and find no GPU to run on)."""
    if _HAS_GPU:
        pytest.skip("calls with fake pointers run GPU-less only")
    c = cache(dtype=2, k_exp=A, v_exp=A, page=1 << 19, H=8, dh=128, pages=64)
    s = seqs(n_seq=64, n_tok=12800, max_pages=2)
    for r in (False, rope(rot_dim=128), rope(rot_dim=30)):
        assert append(lib, c, s, r, ks=1024, vs=1024) == HIP, lib.cast_last_error_detail()
