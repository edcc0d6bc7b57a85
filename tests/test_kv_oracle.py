"""Pins of the float64 reference of the cached-history operators (oracle/kv.py): each
property is checked against a computation of another kind than the one that made it."""
import math

import numpy as np
import pytest
import torch

from oracle import kv as O


def test_e4m3_codes_match_torch():
    codes = torch.arange(256, dtype=torch.uint8)
    v = codes.view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.nan_to_num(v, nan=1e9), np.nan_to_num(O.E4M3, nan=1e9))
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=4000) * 10.0 ** rng.integers(-4, 3, 4000), O.E4M3[:127],
                        (O.E4M3[:126] + O.E4M3[1:127]) / 2])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    got = O.e4m3_code(x.astype(np.float64))
    assert np.array_equal(O.E4M3[got], O.E4M3[want])


def test_need_exp_is_least():
    for top in (448.0, 448.0001, 1.0, 0.875, 0.8751, 3.3e38, 1e-30, 0.0):
        e = O.need_exp(np.array([top, -top / 2, math.nan, math.inf]))
        assert top <= 448.0 * 2.0 ** e
        assert e == -117 or top > 448.0 * 2.0 ** (e - 1)


def test_rope_is_a_complex_product_and_depends_on_distance_only():
    rng = np.random.default_rng(1)
    turns, _ = O.frequencies([16])
    x = rng.normal(size=(5, 2, 24))
    pos = rng.integers(0, 1000, (5, 1))
    for inter in (False, True):
        y = O.rope(x, pos, turns, inter=inter)
        z = x[..., 0:16:2] + 1j * x[..., 1:16:2] if inter else x[..., :8] + 1j * x[..., 8:16]
        w = z * np.exp(2j * math.pi * pos[:, None, :] * turns)
        got = y[..., 0:16:2] + 1j * y[..., 1:16:2] if inter else y[..., :8] + 1j * y[..., 8:16]
        assert np.allclose(got, w, atol=1e-11) and np.array_equal(y[..., 16:], x[..., 16:])
        # q at p + s against k at p' + s: the same score for every s
        dots = [(O.rope(x, pos + s, turns, inter=inter)[0] * O.rope(x, pos + s, turns, inter=inter)[1]).sum()
                for s in (0, 77)]
        assert abs(dots[0] - dots[1]) < 1e-10


def test_frequencies_parts():
    plain, _ = O.frequencies([64])
    t, _ = O.frequencies([64], scaling="parts", factor=4.0, orig_len=4096)
    assert np.allclose(t[4096 * plain > 32], plain[4096 * plain > 32])          # fast pairs keep their frequency
    assert np.allclose(t[4096 * plain < 1], plain[4096 * plain < 1] / 4.0)     # slow ones are stretched
    assert np.all(np.diff(t) < 0)


def test_attention_against_torch_dense():
    rng = np.random.default_rng(2)
    page, H, g, dh, L, n = 4, 2, 3, 8, 13, 5
    k, v = rng.normal(size=(2, L, H, dh))
    q = rng.normal(size=(n, H * g, dh))
    table = np.array([[3, 0, 2, 1]])
    kv, vv = np.zeros((2, 4, page, H, dh))
    for j in range(L):
        kv[table[0, j // page], j % page], vv[table[0, j // page], j % page] = k[j], v[j]
    for causal, window, sinks in ((True, 0, 0), (False, 0, 0), (True, 3, 2), (False, 4, 1)):
        out, lse, _ = O.attention(q, kv, vv, [0, n], [L], table, page, 0.4, causal, window, sinks)
        s = np.einsum("nhd,jhd->hnj", q, np.repeat(k, g, axis=1)) * 0.4
        i, j = np.arange(L - n, L)[:, None], np.arange(L)[None, :]
        ok = np.ones((n, L), bool)
        if causal:
            ok &= j <= i
        if window:
            ok &= (j > i - window) | (j < sinks)
        s = torch.from_numpy(np.where(ok[None], s, -np.inf))
        want = torch.einsum("hnj,jhd->nhd", torch.softmax(s, -1), torch.from_numpy(np.repeat(v, g, axis=1)))
        assert np.allclose(out, want.numpy(), atol=1e-12)
        assert np.allclose(lse, torch.logsumexp(s, -1).numpy().T, atol=1e-12)


def test_append_in_steps_equals_append_at_once_but_for_subnormals():
    rng = np.random.default_rng(3)
    page, H, dh, n = 8, 2, 8, 13
    x = rng.normal(size=(n, H, dh)) * 4.0 ** rng.integers(-2, 3, (n, 1, 1))
    table = np.array([[1, 0]])

    def fresh():
        return {"k": np.zeros((2, page, H, dh), np.uint8), "v": np.zeros((2, page, H, dh), np.uint8),
                "k_exp": np.zeros((2, H), np.uint8), "v_exp": np.zeros((2, H), np.uint8)}
    once, steps = fresh(), fresh()
    O.append(once, [0, n], [n], table, x, -x)
    at = 0
    for m in (1, 3, 4, 5):
        O.append(steps, [0, m], [at + m], table, x[at:at + m], -x[at:at + m])
        at += m
    assert np.array_equal(once["k_exp"], steps["k_exp"])
    a, b = O.values(once["k"], once["k_exp"]), O.values(steps["k"], steps["k_exp"])
    step = 2.0 ** (once["k_exp"].astype(float) - 127 - 9)[:, None, :, None]      # one subnormal step
    assert np.all(np.abs(a - b) <= step)
    assert np.array_equal(O.values(once["v"], once["v_exp"]), -a)


@pytest.mark.parametrize("bad", [(-1,), (2,)])
def test_append_drops_missing_pages(bad):
    cache = {"k": np.zeros((2, 2, 1, 4)), "v": np.zeros((2, 2, 1, 4))}
    O.append(cache, [0, 4], [4], np.array([[bad[0], 1]]), np.ones((4, 1, 4)), np.ones((4, 1, 4)))
    assert cache["k"][0].sum() == 0 and cache["k"][1].sum() == 8
