"""Forms of the cached-history calls that lie next to a limit: the last page of a cache,
other streams, extreme values and exponents, long pages."""
import numpy as np
import pytest
import torch

from kv_util import Batch, bf16
from test_gpu_kv_attn import MASKS, run

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("page", [32, 64])
@pytest.mark.parametrize("causal,window,sinks", MASKS)
def test_narrow_heads_up_to_the_last_page(cast_lib, bits, page, causal, window, sinks):
    """32-wide heads in pages of whole runs, many rows; a sequence ends with the cache's last row,
    another in a page whose rows behind it belong to no token."""
    rng = np.random.default_rng(page)
    b = Batch(rng, [40, 70, 130], [2 * page, 70, 130 + page], page, 3, 32, bits, extra_pages=0)
    last = np.argwhere(b.table == b.pages - 1)[0]
    b.table[tuple(last)], b.table[0, 1] = b.table[0, 1], b.pages - 1
    run(cast_lib, b, bf16(rng, b.n, 6, 32, scale=2.0), 0.2, causal, window, sinks, "narrow")
