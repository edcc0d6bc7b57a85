"""The routed attention on scores of which one half of each group of eight keys (the half that
one half-wave holds) lies far above the other, against the float64 reference."""
import numpy as np
import pytest
import torch

from kv_util import bf16, f64
from oracle import attn as OA

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("half", [0, 4])
@pytest.mark.parametrize("gap", [12.0, 60.0, 200.0])
def test_scores_of_one_half_far_above_the_other(cast_lib, dh, half, gap):
    """Keys half .. half + 3 of every eight score `gap` above the rest: the running maximum has to be
    over both halves, else the exponentials of one are up to e^gap."""
    rng = np.random.default_rng(dh + half)
    n_a, S, H, M, Bv = 1, 100, 2, 5, 64
    q = torch.zeros((n_a, S, H, dh))
    q[..., 0] = 8.0
    q[..., 1:] = bf16(rng, n_a, S, H, dh - 1, scale=0.25).float()
    k = bf16(rng, M, Bv, H, dh, scale=0.25).float()
    up = (np.arange(Bv) % 8 // 4) == half // 4
    k[:, up, :, 0], k[:, ~up, :, 0] = gap / 8.0, 0.0
    q, k, v = q.to(torch.bfloat16), k.to(torch.bfloat16), bf16(rng, M, Bv, H, dh)
    idx = torch.arange(M, dtype=torch.int32).repeat(n_a, H, 1).contiguous()
    scale = 1.0
    print(f"[scores] dh {dh} half {half} gap {gap}", flush=True)
    out, lse = cast_lib.cast_anchor_attn(q.to(DEV), k.to(DEV), v.to(DEV), idx.to(DEV), M, scale, want_lse=True)
    want, wl = OA.anchor_attention(f64(q), f64(k), f64(v), idx.numpy(), scale)
    got, gl = f64(out), f64(lse)
    assert np.isfinite(got).all() and np.isfinite(gl).all()
    # probabilities rounded to bf16 (2^-8 of sum p |v|, at most of max |v|), the output once more, and
    # logits in fp32: dh roundings of 2^-24 of sum |q k|, which moves a probability by as much, twice
    logit = dh * 2.0 ** -24 * (np.abs(f64(q)).max((0, 1, 2)) * np.abs(f64(k)).max((0, 1, 2))).sum()
    top = np.abs(f64(v)).max()
    assert np.all(np.abs(got - want) <= top * (2.0 ** -8 + 2 * logit + 2.0 ** -20) + 2.0 ** -8 * np.abs(want) * 1.01)
    assert np.all(np.abs(gl - wl) <= logit + 2.0 ** -20 * (1 + np.abs(wl)))
