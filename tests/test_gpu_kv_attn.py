"""Attention over the paged cache on the GPU against the float64 reference: ragged
batches, grouped heads, causal rows, windows with sinks, holes in the table, both cache
types and both kernels (few and many rows), whole and in pieces."""
import numpy as np
import pytest
import torch

from kv_util import Batch, bf16, check_attn, f64
from oracle import kv as O

pytestmark = pytest.mark.gpu
DEV = "cuda"


def run(cast, b, q, scale, causal=True, window=0, sinks=0, what="", **kw):
    cache, seqs = b.device(cast)
    print(f"[kv_attn {what}] n {b.n} lens {b.lens.tolist()[:8]} page {b.page} H {b.H} Hq {q.shape[1]} dh {b.dh} bits {b.bits} "
          f"causal {causal} window {window} sinks {sinks}", flush=True)
    out = torch.full((b.n, q.shape[1], b.dh), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((b.n, q.shape[1]), 7.0, device=DEV)
    cast.cast_kv_attn(q.to(DEV), cache, seqs, scale, causal, window, sinks, out=out, lse_out=lse, **kw)
    check_attn(out, lse, q, b, scale, causal, window, sinks, what)
    rows = int(b.cu[-1])
    assert bool((out[rows:] == 7.0).all()) and bool((lse[rows:] == 7.0).all())      # rows of no sequence
    return out, lse


MASKS = [(True, 0, 0), (False, 0, 0), (True, 17, 0), (True, 40, 3), (False, 33, 65)]


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("causal,window,sinks", MASKS)
def test_tokens(cast_lib, bits, dh, causal, window, sinks):
    """Single tokens (and two, and none) on ragged lengths; lengths of 0 and 1; in pieces and whole."""
    rng = np.random.default_rng(dh + window)
    for g, page in ((1, 16), (4, 37), (7, 1), (33, 64)):
        b = Batch(rng, [1, 1, 0, 2, 1, 1, 1], [1, 200, 9, 65, 0, 33, 700], page, 2, dh, bits, spare=2)
        q = bf16(rng, b.n, 2 * g, dh, scale=2.0)
        o1, l1 = run(cast_lib, b, q, dh ** -0.5, causal, window, sinks, f"pieces g{g}")
        o2, l2 = run(cast_lib, b, q, dh ** -0.5, causal, window, sinks, f"whole g{g}", split=False)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("causal,window,sinks", MASKS)
def test_prompts(cast_lib, bits, dh, causal, window, sinks):
    """Many rows: whole prompts, chunks behind a history, more rows than tokens, lengths past a tile."""
    rng = np.random.default_rng(dh * 2 + window)
    for g, page in ((1, 16), (3, 29)):
        b = Batch(rng, [150, 1, 90, 40], [150, 70, 333, 30], page, 2, dh, bits, spare=1)
        q = bf16(rng, b.n, 2 * g, dh, scale=2.0)
        run(cast_lib, b, q, dh ** -0.5, causal, window, sinks, f"g{g}")


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new,rows", [(1, "few"), (130, "many")])
def test_every_single_visible_key(cast_lib, bits, new, rows):
    """A window of one: row p sees key p alone, so out = V_p and lse its logit, at every place of a tile."""
    rng = np.random.default_rng(21)
    lens = list(range(1, 71)) if new == 1 else [130, 141, 200]
    b = Batch(rng, [new] * len(lens), lens, 16, 1, 64, bits)
    q = bf16(rng, b.n, 1, 64, scale=2.0)
    out, _ = run(cast_lib, b, q, 0.125, True, 1, 0, rows)
    vv = b.values()[1]
    for r, s, t in O.tokens(b.cu, b.lens, len(lens)):
        want = vv[b.table[s, t // 16], t % 16, 0]
        assert np.all(np.abs(f64(out)[r, 0] - want) <= 2.0 ** -8 * np.abs(want))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("new", [2, 100])
def test_holes(cast_lib, bits, new):
    """Pages that left the cache are invisible; rows that see no other page give 0 and -inf."""
    rng = np.random.default_rng(22)
    b = Batch(rng, [new, new, new], [300, 300, 300], 16, 2, 64, bits)
    b.table[0, 3:7] = -1
    b.table[1, ::2] = b.pages
    b.table[2, :] = -1
    q = bf16(rng, b.n, 4, 64, scale=2.0)
    out, lse = run(cast_lib, b, q, 0.125, True)
    assert bool(torch.isneginf(lse[2 * new:]).all()) and bool((out[2 * new:] == 0).all())
    run(cast_lib, b, q, 0.125, True, 20, 5)


@pytest.mark.parametrize("new", [2, 100])
@pytest.mark.parametrize("what", ["nan", "inf", "-inf", "mixed"])
def test_infinities_at_invisible_places(cast_lib, new, what):
    """Keys and values behind the sequence, in holes' stand-ins, before the window and after the
    row hold infinities and NaN: rows that do not see them are as without them; a row that sees
    an infinite or NaN value gets it."""
    rng = np.random.default_rng(23)
    L, H, dh, page = 260, 1, 64, 16
    b = Batch(rng, [new], [L], page, H, dh, 16)
    clean = (b.k.clone(), b.v.clone())
    q = bf16(rng, b.n, 2, dh, scale=2.0)
    bad = {"nan": [float("nan")], "inf": [float("inf")], "-inf": [float("-inf")], "mixed": [float("inf"), float("-inf")]}[what]
    place = lambda t: (b.table[0, t // page], t % page)  # noqa: E731
    p, r = place(L - 1)
    b.k[p, r + 1:], b.v[p, r + 1:] = float("nan"), float("nan")      # rows behind the last token
    seen_from = L - 1                                       # the last token's value is not finite in channel 5
    for i, x in enumerate(bad):
        pp, rr = place(seen_from - i)
        b.v[pp, rr, 0, 5] = x
    for t in range(0, 150):                                 # everything before the windows
        pp, rr = place(t)
        b.k[pp, rr], b.v[pp, rr] = float("nan"), float("inf")
    cache, seqs = b.device(cast_lib)
    out, lse = cast_lib.cast_kv_attn(q.to(DEV), cache, seqs, 0.125, True, 9, 0, want_lse=True)
    kv, vv = f64(clean[0]), f64(clean[1])
    want, wl, mag = O.attention(f64(q), kv, vv, b.cu, b.lens, b.table, page, 0.125, True, 9, 0)
    got = f64(out)
    tol = mag * 2.0 ** -7.9 + 2.0 ** -8 * np.abs(want) + 1e-5
    first = seen_from - len(bad) + 1                        # the first token that is not finite
    for row in range(b.n):
        t = L - b.n + row
        chans = [c for c in range(dh) if not (c == 5 and t >= first)]
        assert np.all(np.abs(got[row][:, chans] - want[row][:, chans]) <= tol[row][:, chans]), (t, what)
        if t >= first:
            # values that the row sees; inf - inf and NaN give NaN
            ref = sum(bad[i] for i in range(len(bad)) if seen_from - i <= t)
            g = got[row][:, 5]
            assert np.all(np.isnan(g)) if np.isnan(ref) else np.all(g == ref), (t, what, g)
    assert np.all(np.abs(f64(lse) - wl) <= 1e-4)


def test_keys_before_the_window_in_a_shared_tile(cast_lib):
    """NaN keys that lie in the window's first tile but before it, for few and many rows."""
    rng = np.random.default_rng(24)
    for new in (1, 80):
        b = Batch(rng, [new], [333], 8, 2, 128, 16)
        q = bf16(rng, b.n, 2, 128)
        kv, vv = f64(b.k), f64(b.v)
        lo = 333 - new - 50 + 1
        for t in range(lo):
            b.k[b.table[0, t // 8], t % 8], b.v[b.table[0, t // 8], t % 8] = float("nan"), float("nan")
        cache, seqs = b.device(cast_lib)
        out, lse = cast_lib.cast_kv_attn(q.to(DEV), cache, seqs, 0.1, True, 50, 0, want_lse=True)
        check_attn(out, lse, q, b, 0.1, True, 50, 0, f"new {new}", kv=(kv, vv))


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("bits", [16, 8])
def test_large_and_one_sided_scores(cast_lib, bits, new):
    """Logits of hundreds, the largest in one half of a tile only, and all far below zero."""
    rng = np.random.default_rng(25)
    for sign, at in ((1.0, 4), (1.0, 0), (-1.0, 5), (-1.0, None)):
        b = Batch(rng, [new], [200], 16, 1, 64, bits, spread=False)
        q = torch.full((b.n, 1, 64), 16.0 * sign).to(torch.bfloat16)
        if bits == 16:
            b.k.fill_(1.0)
            for t in range(200):
                b.k[b.table[0, t // 16], t % 16] = 1.0 if at is None or t % 8 == at else 0.25
        else:
            b.k.fill_(56)                                   # 1.0
            b.ke.fill_(127)
            for t in range(200):
                b.k[b.table[0, t // 16], t % 16] = 56 if at is None or t % 8 == at else 40   # 0.25
        run(cast_lib, b, q, 1.0, True, what=f"sign {sign} at {at}")


def test_lowest_scores_are_still_scores(cast_lib):
    """Scores near the type's lowest value are visible: the softmax is over them, not empty."""
    b = Batch(np.random.default_rng(26), [1, 70], [40, 70], 16, 1, 32, 16)
    b.k.fill_(-2.0 ** 62)
    q = torch.full((b.n, 1, 32), 2.0 ** 58).to(torch.bfloat16)            # q.k = -2^125
    run(cast_lib, b, q, 0.25, True)


def test_expected_length_is_only_a_hint(cast_lib):
    rng = np.random.default_rng(27)
    b = Batch(rng, [1, 1], [900, 3], 16, 1, 64, 16)
    q = bf16(rng, b.n, 4, 64)
    for hint in (1, 40, 500, 10 ** 9):
        run(cast_lib, b, q, 0.125, max_len=hint, what=f"hint {hint}")
    b = Batch(rng, [100], [900], 16, 1, 64, 16)
    q = bf16(rng, b.n, 2, 64)
    for hint in (1, 400, None):
        run(cast_lib, b, q, 0.125, max_len=hint, what=f"hint {hint}")


def test_lengths_past_the_table_count_up_to_it(cast_lib):
    rng = np.random.default_rng(28)
    b = Batch(rng, [1, 2, 1], [64, 64, 20], 16, 1, 64, 16)
    b.lens = np.array([1000, 65, -4], dtype=np.int32)
    q = bf16(rng, b.n, 2, 64)
    run(cast_lib, b, q, 0.125)


def test_query_strides(cast_lib):
    rng = np.random.default_rng(29)
    b = Batch(rng, [3, 60], [50, 60], 16, 2, 64, 16)
    big = bf16(rng, b.n, 12, 64).to(DEV)
    cache, seqs = b.device(cast_lib)
    a = cast_lib.cast_kv_attn(big[:, 2:6], cache, seqs, 0.125)[0]
    assert torch.equal(a, cast_lib.cast_kv_attn(big[:, 2:6].contiguous(), cache, seqs, 0.125)[0])


def test_many_sequences(cast_lib):
    """More sequences than one lookup step of 64 finds, empty ones between them."""
    rng = np.random.default_rng(30)
    new = [int(x) for x in rng.integers(0, 3, 300)]
    lens = [n + int(x) for n, x in zip(new, rng.integers(0, 60, 300))]
    b = Batch(rng, new, lens, 8, 1, 32, 16, spare=2)
    run(cast_lib, b, bf16(rng, b.n, 2, 32), 0.2)
    big = Batch(rng, [40 if i % 50 == 7 else n for i, n in enumerate(new)], [x + 45 for x in lens], 8, 1, 32, 8)
    run(cast_lib, big, bf16(rng, big.n, 24, 32), 0.2)


def test_cache_past_4_gib(cast_lib):
    """Pages whose byte offsets pass 2^32 (and 2^31 elements)."""
    H, dh, page = 8, 128, 64
    pages = (5 << 30) // (page * H * dh * 2)
    k = torch.empty((pages, page, H, dh), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    used = torch.tensor([pages - 1, 0, pages // 2, pages - 2], device=DEV)
    k[used] = torch.randn((4, page, H, dh), device=DEV).bfloat16()
    v[used] = torch.randn((4, page, H, dh), device=DEV).bfloat16()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    for new in (1, 120):
        seqs = cast_lib.KvSeqs(i32([0, new]), i32([200]), i32([used.tolist()]))
        x, y = torch.randn((2, new, H, dh), device=DEV).bfloat16()
        cache = cast_lib.KvCache(k, v)
        cast_lib.cast_kv_append(cache, seqs, x, y)
        small = cast_lib.KvCache(k[used].contiguous(), v[used].contiguous())
        s2 = cast_lib.KvSeqs(i32([0, new]), i32([200]), i32([[0, 1, 2, 3]]))
        t = torch.arange(200 - new, 200, device=DEV)
        assert torch.equal(k[used[t // page], t % page], x) and torch.equal(v[used[t // page], t % page], y)
        q = torch.randn((new, 16, dh), device=DEV).bfloat16()
        assert torch.equal(cast_lib.cast_kv_attn(q, cache, seqs, 0.1)[0], cast_lib.cast_kv_attn(q, small, s2, 0.1)[0])
    kk, _ = cast_lib.cast_kv_read(cache, i32([pages - 1]), want_v=False)
    assert torch.equal(kk[0], k[pages - 1])


def test_workspace_refusals_and_growth(cast_lib):
    rng = np.random.default_rng(31)
    b = Batch(rng, [1, 1], [4000, 3000], 16, 2, 64, 16)
    cache, seqs = b.device(cast_lib)
    q = bf16(rng, b.n, 8, 64).to(DEV)
    sizes = [cast_lib.cast_kv_attn_workspace_bytes(q, cache, seqs, max_len=m) for m in (1, 100, 500, 1000, 2000, 4000)]
    assert sizes == sorted(sizes) and sizes[-1] > 0
    need = sizes[-1]
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    want = cast_lib.cast_kv_attn(q, cache, seqs, 0.125, max_len=4000)[0]
    ws.fill_(0xff)                                          # NaN in every part
    assert torch.equal(cast_lib.cast_kv_attn(q, cache, seqs, 0.125, max_len=4000, workspace=ws)[0], want)
    cast_lib.cast_kv_attn(q, cache, seqs, 0.125, max_len=700, workspace=ws)
    for w in (ws[:-256], ws[128:]):
        with pytest.raises(cast_lib.CastError) as e:
            cast_lib.cast_kv_attn(q, cache, seqs, 0.125, max_len=4000, workspace=w)
        assert e.value.status == 5


def test_repeats_are_bit_identical(cast_lib):
    rng = np.random.default_rng(32)
    b = Batch(rng, [1, 200, 3], [3000, 200, 900], 16, 2, 128, 8)
    cache, seqs = b.device(cast_lib)
    q = bf16(rng, b.n, 8, 128).to(DEV)
    first = cast_lib.cast_kv_attn(q, cache, seqs, 0.1, want_lse=True)
    for _ in range(5):
        again = cast_lib.cast_kv_attn(q, cache, seqs, 0.1, want_lse=True)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
