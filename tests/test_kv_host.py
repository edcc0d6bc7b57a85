"""Host code of the cached history that is not part of the C ABI, through the library's own
C++ symbols."""
import ctypes
import os

import numpy as np
import pytest

import paper_2609_34144_amd as cast


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
