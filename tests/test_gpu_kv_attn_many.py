"""Attention over the paged cache with many rows of 128 channels, against the float64
reference: few heads run as tiles of 128 rows, many heads (enough to fill the card) as
pairs of 256, whole and in pieces."""
import numpy as np
import pytest
import torch

from kv_util import Batch, bf16, check_attn, f64
from oracle import kv as O
from test_gpu_kv_attn import DEV, MASKS

pytestmark = pytest.mark.gpu
HEADS = [2, 64]          # tiles, pairs
DH = 128


def some(H):
    """The KV heads that are compared: of many, the first, the last and two between."""
    return list(range(H)) if H <= 8 else [0, 1, H // 2 + 1, H - 1]


def run(cast, b, q, scale, causal=True, window=0, sinks=0, what="", **kw):
    cache, seqs = b.device(cast)
    print(f"[kv_attn {what}] n {b.n} lens {b.lens.tolist()[:8]} page {b.page} H {b.H} Hq {q.shape[1]} dh {b.dh} bits {b.bits} "
          f"causal {causal} window {window} sinks {sinks}", flush=True)
    out = torch.full((b.n, q.shape[1], b.dh), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((b.n, q.shape[1]), 7.0, device=DEV)
    cast.cast_kv_attn(q.to(DEV), cache, seqs, scale, causal, window, sinks, out=out, lse_out=lse, **kw)
    rows = int(b.cu[-1])
    assert bool((out[rows:] == 7.0).all()) and bool((lse[rows:] == 7.0).all())      # rows of no sequence
    hs, g = some(b.H), q.shape[1] // b.H
    hq = [h * g + i for h in hs for i in range(g)]
    check_attn(out[:, hq], lse[:, hq], q[:, hq], b, scale, causal, window, sinks, what, kv=[x[:, :, hs] for x in b.values()])
    return out, lse


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,page", [(2, 16), (2, 37), (64, 16), (64, 37)])
@pytest.mark.parametrize("causal,window,sinks", MASKS)
def test_ragged(cast_lib, bits, H, page, causal, window, sinks):
    """Chunks behind a history, more key tiles than one lookup takes, an empty sequence, a few rows."""
    rng = np.random.default_rng(H + window)
    b = Batch(rng, [300, 0, 257, 3], [300, 9, 650, 70], page, H, DH, bits, spare=1)
    run(cast_lib, b, bf16(rng, b.n, H, DH, scale=2.0), DH ** -0.5, causal, window, sinks, "ragged")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,g", [(3, 2), (32, 2), (24, 1)])
def test_pieces(cast_lib, bits, H, g):
    """Long key ranges with few row tiles, cut along the keys: causal, and a window with sinks whose
    pieces hold nothing for some rows."""
    rng = np.random.default_rng(H)
    b = Batch(rng, [130, 170], [2600, 2300], 64, H, DH, bits)
    q = bf16(rng, b.n, H * g, DH, scale=2.0)
    run(cast_lib, b, q, DH ** -0.5, True, 0, 0, f"H {H} g {g}")
    run(cast_lib, b, q, DH ** -0.5, True, 700, 130, f"H {H} g {g}")
    run(cast_lib, b, q, DH ** -0.5, False, 1100, 0, f"H {H} g {g}", split=False)


@pytest.mark.parametrize("H", HEADS)
@pytest.mark.parametrize("bits", [16, 8])
def test_every_single_visible_key(cast_lib, bits, H):
    """A window of one: row p sees key p alone, so out = V_p, at every place of a tile."""
    rng = np.random.default_rng(41)
    b = Batch(rng, [260, 300, 200], [260, 333, 200], 16, H, DH, bits)
    out, _ = run(cast_lib, b, bf16(rng, b.n, H, DH, scale=2.0), 0.1, True, 1, 0, "one key")
    vv, got = b.values()[1], f64(out)
    for r, s, t in O.tokens(b.cu, b.lens, 3):
        want = vv[b.table[s, t // 16], t % 16]
        assert np.all(np.abs(got[r] - want) <= 2.0 ** -8 * np.abs(want))


@pytest.mark.parametrize("H", HEADS)
@pytest.mark.parametrize("bits", [16, 8])
def test_holes(cast_lib, bits, H):
    rng = np.random.default_rng(42)
    b = Batch(rng, [200, 260, 200], [900, 700, 300], 16, H, DH, bits)
    b.table[0, 3:47] = -1                                   # whole key tiles and parts of them
    b.table[1, ::2] = b.pages
    b.table[2, :] = -1
    q = bf16(rng, b.n, H, DH, scale=2.0)
    out, lse = run(cast_lib, b, q, 0.1, True)
    assert bool(torch.isneginf(lse[460:]).all()) and bool((out[460:] == 0).all())
    run(cast_lib, b, q, 0.1, True, 20, 5)
    run(cast_lib, b, q, 0.1, False, 100, 0)


@pytest.mark.parametrize("H", HEADS)
@pytest.mark.parametrize("bad", [["nan"], ["inf"], ["-inf"], ["inf", "-inf"]])
def test_infinities_at_invisible_places(cast_lib, H, bad):
    """Infinities and NaN behind the sequence, before the window and after the row leave the rows
    that do not see them as they are; a row that sees an infinite or NaN value gets it."""
    rng = np.random.default_rng(43)
    bad = [float(x) for x in bad]
    L, new, page, w = 500, 300, 16, 9
    b = Batch(rng, [new] * 3, [L] * 3, page, H, DH, 16)
    clean = (f64(b.k), f64(b.v))
    q = bf16(rng, b.n, H, DH, scale=2.0)
    first = L - 64 - len(bad)                               # tokens that are not finite in channel 5
    for s in range(3):
        place = lambda t: (b.table[s, t // page], t % page)  # noqa: E731
        p, r = place(L - 1)
        b.k[p, r + 1:], b.v[p, r + 1:] = float("nan"), float("nan")
        for i, x in enumerate(bad):
            pp, rr = place(first + i)
            b.v[pp, rr, :, 5] = x
        for t in range(0, L - new - w + 1):
            pp, rr = place(t)
            b.k[pp, rr], b.v[pp, rr] = float("nan"), float("inf")
    cache, seqs = b.device(cast_lib)
    out, lse = cast_lib.cast_kv_attn(q.to(DEV), cache, seqs, 0.1, True, w, 0, want_lse=True)
    hs = some(H)
    want, wl, mag = O.attention(f64(q[:, hs]), *[x[:, :, hs] for x in clean], b.cu, b.lens, b.table, page, 0.1, True, w, 0)
    got, lse = f64(out[:, hs]), lse[:, hs]
    tol = mag * 2.0 ** -7.9 + 2.0 ** -8 * np.abs(want) + 1e-5
    others = [c for c in range(DH) if c != 5]
    assert np.all(np.abs(got - want)[..., others] <= tol[..., others])
    assert np.all(np.abs(f64(lse) - wl) <= 1e-4)
    for row in range(b.n):
        t = L - new + row % new
        seen = [x for i, x in enumerate(bad) if t - w < first + i <= t]
        if not seen:
            assert np.all(np.abs(got - want)[row, :, 5] <= tol[row, :, 5]), t
            continue
        ref, g = sum(seen), got[row, :, 5]
        assert np.all(np.isnan(g)) if np.isnan(ref) else np.all(g == ref), (t, g[:4])


@pytest.mark.parametrize("H", HEADS)
@pytest.mark.parametrize("bits", [16, 8])
def test_large_and_one_sided_scores(cast_lib, bits, H):
    """Logits of hundreds, the largest in one half of a tile only, in a late tile, and all far below zero."""
    rng = np.random.default_rng(45)
    for sign, hot in ((1.0, lambda t: t % 8 == 4), (1.0, lambda t: t % 8 == 0), (1.0, lambda t: t == 290),
                      (-1.0, lambda t: t % 8 == 5), (-1.0, lambda t: True)):
        b = Batch(rng, [150] * 3, [400] * 3, 16, H, DH, bits, spread=False)
        q = torch.full((b.n, H, DH), 8.0 * sign).to(torch.bfloat16)
        if bits == 8:
            b.ke.fill_(127)
        one, quarter = (1.0, 0.25) if bits == 16 else (56, 40)
        for s in range(3):
            for t in range(400):
                b.k[b.table[s, t // 16], t % 16] = one if hot(t) else quarter
        run(cast_lib, b, q, 1.0, True, what=f"sign {sign}")


@pytest.mark.parametrize("H", HEADS)
def test_many_sequences(cast_lib, H):
    """More sequences than one lookup step of 64 counts, empty ones among them; row tiles that end
    exactly with a sequence and past it."""
    rng = np.random.default_rng(46)
    sizes = [0, 128, 256, 129, 300, 1, 257]
    new = [sizes[i % 7] if H == 2 or i % 9 == 0 else sizes[2 * (i % 2)] for i in range(70)]
    b = Batch(rng, new, [n + int(x) for n, x in zip(new, rng.integers(0, 30, 70))], 16, H if H == 2 else 8, DH, 16)
    run(cast_lib, b, bf16(rng, b.n, b.H * (2 if H == 2 else 1), DH), 0.1)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H", [1, 2, 3, 6, 8])
def test_few_rows_of_any_number_of_heads(cast_lib, bits, H):
    """Waves take 4, 2 or 1 heads; 16 rows and 17."""
    rng = np.random.default_rng(47)
    for dh, new in ((64, [16, 16]), (128, [8, 8]), (32, [5, 12]), (64, [17, 17])):
        g = 2 if dh == 128 else 1
        b = Batch(rng, new, [900, 1500], 16, H, dh, bits)
        run(cast_lib, b, bf16(rng, b.n, H * g, dh, scale=2.0), 0.1, True, what="few")


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_many_pieces(cast_lib, dh):
    """Short row tiles over a long range: more pieces than one thread joins; rows of no sequence, and
    rows that see nothing in most pieces or at all."""
    rng = np.random.default_rng(48)
    b = Batch(rng, [20, 0, 40, 30], [4000, 100, 2500, 30], 16, 3, dh, 16, spare=3)
    b.table[3, :] = -1
    q = bf16(rng, b.n, 3, dh, scale=2.0)
    run(cast_lib, b, q, 0.1, True, what="pieces")
    run(cast_lib, b, q, 0.1, True, 3900, 60, what="pieces")


def test_workspace_of_a_longer_bound_serves_shorter_ones(cast_lib):
    """The workspace does not fall as max_len grows, whichever way the rows are cut."""
    z = lambda *s, d=torch.int32: torch.zeros(s, dtype=d, device=DEV)  # noqa: E731
    for H, g in ((1, 1), (2, 4), (8, 1), (24, 1), (64, 1)):
        for dh in (64, 128):
            kv = z(1, 16, H, dh, d=torch.bfloat16)
            cache = cast_lib.KvCache(kv, kv)
            for n_seq in (1, 3, 40):
                seqs = cast_lib.KvSeqs(z(n_seq + 1), z(n_seq), z(n_seq, 2048))
                for mean in (1, 20, 130, 200, 257, 600):
                    q = z(mean * n_seq, H * g, 1, d=torch.bfloat16)
                    for window in (0, 500):
                        b = [cast_lib.cast_kv_attn_workspace_bytes(q, cache, seqs, max_len=m, window=window)
                             for m in (1, 64, 300, 512, 513, 800, 1024, 1500, 2100, 4000, 9000, 32000)]
                        assert b == sorted(b), (H, g, dh, n_seq, mean, window, b)
