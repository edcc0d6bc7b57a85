"""Rotary positions, paged append and page read on the GPU against the float64 reference."""
import itertools

import numpy as np
import pytest
import torch

from kv_util import Batch, bf16, f64
from oracle import kv as O

pytestmark = pytest.mark.gpu
DEV = "cuda"


def make_rope(cast, rot, axes=None, **kw):
    r = cast.cast_rope_params_init(rot, axes=axes, **kw)
    return r, r.turns.cpu().numpy(), r.axis.cpu().numpy()


def rope_bound(x, want, turns, inter, amp, dtype):
    """|error| <= (|x| + |y|) a d + rounding: d = 8e-7 covers the angle (2^-26 revolutions of
    reduction, 9.4e-8 rad), sine and cosine (4 fp32 steps of 2^-24 each way from the function,
    2.4e-7), the amplitude and the two products and sum (4 roundings, 2.4e-7); the output's own
    rounding is half a step, 2^-8 (bf16) or 2^-24 of the value."""
    half = len(turns)
    pair = np.abs(np.array(x))
    s = np.zeros_like(pair)
    for j in range(half):
        c0, c1 = (2 * j, 2 * j + 1) if inter else (j, j + half)
        s[..., c0] = s[..., c1] = pair[..., c0] + pair[..., c1]
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    return s * abs(amp) * 8e-7 * (1 + step) + step * np.abs(want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dh,rot", [(128, 128), (128, 48), (64, 64), (64, 30), (32, 2), (32, 8), (32, 24), (32, 32)])
def test_rope(cast_lib, dtype, inter, dh, rot):
    rng = np.random.default_rng(rot + dh)
    for n, H in ((1, 1), (3, 5), (70, 3)):
        r, turns, _ = make_rope(cast_lib, rot, interleaved=inter, amplitude=1.3)
        x = torch.from_numpy(rng.standard_normal((n, H, dh)).astype(np.float32)).to(dtype)
        pos = rng.integers(-2 ** 31, 2 ** 31, n).astype(np.int32)
        pos[: n // 2] = rng.integers(0, 5000, n // 2)
        d, p = x.to(DEV), torch.from_numpy(pos).to(DEV)
        for tr in (False, True):
            want = O.rope(f64(x), pos, turns, inter=inter, amp=1.3, transpose=tr)
            got = f64(cast_lib.cast_rope(d, p, r, transpose=tr))
            # far positions: turns * 2^31 carries 2^31 * 2^-54 revolutions in fp64, 7.5e-7 rad
            far = np.abs(pos.astype(np.float64))[:, None, None] * 2.0 ** -53 * turns.max() * 2 * np.pi * 2
            bound = rope_bound(f64(x), want, turns, inter, 1.3, dtype)
            s = np.abs(f64(x)).max()
            assert np.all(np.abs(got - want) <= bound + far * 2 * s), (n, H, tr, (np.abs(got - want) / bound).max())
            assert np.array_equal(got[..., rot:], f64(x)[..., rot:])
        assert torch.equal(d.cpu(), x)
        y = cast_lib.cast_rope(d, p, r, out=d)             # in place
        assert y is d and np.array_equal(f64(d), f64(cast_lib.cast_rope(x.to(DEV), p, r)))


@pytest.mark.parametrize("layout", ["qkv", "head_major", "odd_offset", "odd_stride"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rope_strides(cast_lib, layout, dtype):
    rng = np.random.default_rng(5)
    n, H, dh = 9, 4, 64
    r, turns, _ = make_rope(cast_lib, 32)
    pos = torch.arange(100, 100 + n, dtype=torch.int32, device=DEV)
    if layout == "qkv":
        big = torch.from_numpy(rng.standard_normal((n, 3 * H, dh)).astype(np.float32)).to(dtype).to(DEV)
        x = big[:, H:2 * H]
    elif layout == "head_major":
        big = torch.from_numpy(rng.standard_normal((H, n, dh)).astype(np.float32)).to(dtype).to(DEV)
        x = big.transpose(0, 1)
    else:
        extra = 1 if layout == "odd_offset" else 3
        big = torch.from_numpy(rng.standard_normal(n * (H * dh + extra) + 1).astype(np.float32)).to(dtype).to(DEV)
        x = torch.as_strided(big, (n, H, dh), (H * dh + (extra if layout == "odd_stride" else 0), dh, 1), 1 if layout == "odd_offset" else 0)
    before, xc = big.clone(), x.cpu().clone()
    want = O.rope(f64(xc), pos.cpu().numpy(), turns)
    bound = rope_bound(f64(xc), want, turns, False, 1.0, dtype)
    got = cast_lib.cast_rope(x, pos, r)
    assert np.all(np.abs(f64(got) - want) <= bound) and torch.equal(big, before)
    cast_lib.cast_rope(x, pos, r, out=x)
    assert np.array_equal(f64(x), f64(got))
    # nothing but x changed
    x.copy_(xc.to(DEV))
    assert torch.equal(big, before)


def test_rope_axes_scaling_and_gradient(cast_lib):
    rng = np.random.default_rng(6)
    n, H, dh = 33, 3, 128
    r, turns, axis = make_rope(cast_lib, 128, axes=[44, 42, 42], interleaved=True, scaling="parts", factor=4.0, orig_len=64)
    x = torch.from_numpy(rng.standard_normal((n, H, dh)).astype(np.float32))
    pos = rng.integers(0, 90, (n, 3)).astype(np.int32)
    want = O.rope(f64(x), pos, turns, axis, inter=True)
    p = torch.from_numpy(pos).to(DEV)
    got = cast_lib.cast_rope(x.to(DEV), p, r)
    assert np.all(np.abs(f64(got) - want) <= rope_bound(f64(x), want, turns, True, 1.0, torch.float32))
    # gradient of sum(g * rope(x)): the transposed rotation of g, against central differences of
    # the float64 reference (linear in x, so they are exact to rounding)
    g = rng.standard_normal((n, H, dh))
    gx = f64(cast_lib.cast_rope(torch.from_numpy(g.astype(np.float32)).to(DEV), p, r, transpose=True))
    for _ in range(12):
        i = tuple(rng.integers(0, s) for s in (n, H, dh))
        e = np.zeros((n, H, dh))
        e[i] = 1e-3
        num = (g * (O.rope(f64(x) + e, pos, turns, axis, True) - O.rope(f64(x) - e, pos, turns, axis, True))).sum() / 2e-3
        assert abs(gx[i] - num) <= 8e-7 * 2 * np.abs(g).max() + 1e-9
    # a custom table: axis entries past n_axes - 1 count as the last
    ax = torch.full((64,), 200, dtype=torch.uint8, device=DEV)
    rc = cast_lib.RopeParams(r.turns, ax, 3, True)
    want = O.rope(f64(x), pos, turns, np.full(64, 2), inter=True)
    got = cast_lib.cast_rope(x.to(DEV), p, rc)
    assert np.all(np.abs(f64(got) - want) <= rope_bound(f64(x), want, turns, True, 1.0, torch.float32))


def test_rope_empty(cast_lib):
    r, _, _ = make_rope(cast_lib, 32)
    z = torch.zeros((0, 2, 32), device=DEV)
    assert cast_lib.cast_rope(z, torch.zeros((0, 1), dtype=torch.int32, device=DEV), r).shape == (0, 2, 32)


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------

def run_append(cast, b, k, v, rope=None, turns=None, axis=None, inter=False, amp=1.0, pos=None, q=None):
    """Kernel and reference side by side; returns the reference's rotated keys."""
    cache, seqs = b.device(cast)
    up = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    dq = up(q)
    qo = cast.cast_kv_append(cache, seqs, up(k), up(v), rope, None if pos is None else torch.from_numpy(pos).to(DEV), dq,
                             None if q is None else torch.full_like(dq, 7.0))
    kr, qr = f64(k), None if q is None else f64(q)
    if rope is not None:
        at = np.zeros((b.n, 1), dtype=np.int64)
        for r, s, t in O.tokens(b.cu, b.lens, len(b.lens)):
            at[r] = t
        at = at if pos is None else pos
        kr = O.rope(kr, at, turns, axis, inter, amp)
        qr = None if q is None else O.rope(qr, at, turns, axis, inter, amp)
    ref = b.host()
    O.append(ref, b.cu, b.lens, b.table, kr, f64(v))
    if q is not None:
        rows = int(b.cu[-1])
        got = f64(qo)
        assert np.all(np.abs(got - qr)[:rows] <= rope_bound(f64(q), qr, turns, inter, amp, torch.bfloat16)[:rows])
        assert np.all(got[rows:] == 7.0)                   # rows of no sequence: left alone
    return ref, kr


@pytest.mark.parametrize("page,H,dh", [(16, 2, 64), (1, 3, 32), (37, 1, 128), (64, 4, 128)])
@pytest.mark.parametrize("spare", [0, 5])
def test_append_bf16(cast_lib, page, H, dh, spare):
    rng = np.random.default_rng(page)
    # empty sequences, one token, a whole prompt, tokens in front of the sequence (length 3, 7 rows)
    b = Batch(rng, [0, 1, 70, 3, 0, 7, 33], [5, 100, 70, 40, 0, 3, 65], page, H, dh, 16, spare=spare)
    k, v, q = bf16(rng, b.n, H, dh), bf16(rng, b.n, H, dh), bf16(rng, b.n, 3 * H, dh)
    ref, _ = run_append(cast_lib, b, k, v)                   # no rotation: bit for bit
    assert np.array_equal(f64(b.dk), ref["k"]) and np.array_equal(f64(b.dv), ref["v"])
    for rot, inter in ((dh, False), (dh // 2, True), (dh - 6, False)):
        r, turns, _ = make_rope(cast_lib, rot, interleaved=inter, amplitude=0.8)
        ref, _ = run_append(cast_lib, b, k, v, r, turns, inter=inter, amp=0.8, q=q)
        want = ref["k"]
        # rows that were not written equal exactly; written ones within the rotation's bound, whose
        # |x| + |y| is at most twice the largest input
        bound = 2 * float(k.float().abs().max()) * 0.8 * 8e-7 * 1.01 + 2.0 ** -8 * np.abs(want)
        untouched = want == f64(b.k)
        assert np.all(np.where(untouched, f64(b.dk) == want, np.abs(f64(b.dk) - want) <= bound))
        assert np.array_equal(f64(b.dv), ref["v"])


def test_append_strides_axes_holes_and_in_place_queries(cast_lib):
    rng = np.random.default_rng(8)
    H, dh, page = 2, 64, 8
    b = Batch(rng, [20, 9], [30, 9], page, H, dh, 16)
    b.table[0, 2] = -1                                       # evicted page
    b.table[1, 0] = b.pages                                  # out of range
    r, turns, axis = make_rope(cast_lib, 48, axes=[16, 16, 16])
    pos = rng.integers(0, 60, (b.n, 3)).astype(np.int32)
    qkv = bf16(rng, b.n, 4 * H + 2 * H, dh).to(DEV)         # q, k, v of one projection
    q, k, v = qkv[:, :4 * H], qkv[:, 4 * H:5 * H], qkv[:, 5 * H:]
    cache, seqs = b.device(cast_lib)
    p = torch.from_numpy(pos).to(DEV)
    qo = cast_lib.cast_kv_append(cache, seqs, k, v, r, p, q)
    kr, qr = O.rope(f64(k), pos, turns, axis), O.rope(f64(q), pos, turns, axis)
    ref = b.host()
    O.append(ref, b.cu, b.lens, b.table, kr, f64(v))
    bound = 2 * float(qkv.float().abs().max()) * 8e-7 * 1.01
    assert np.all(np.abs(f64(b.dk) - ref["k"]) <= bound + 2.0 ** -8 * np.abs(ref["k"]))
    assert np.array_equal(f64(b.dv), ref["v"])
    assert np.all(np.abs(f64(qo) - qr) <= bound + 2.0 ** -8 * np.abs(qr))
    dense = q.contiguous()
    assert cast_lib.cast_kv_append(cache, seqs, k, v, r, p, dense, dense) is dense
    assert torch.equal(dense, qo)


@pytest.mark.parametrize("page,H,dh", [(16, 2, 64), (1, 2, 32), (37, 1, 128), (64, 3, 128), (700, 1, 64)])
def test_append_e4m3_values(cast_lib, page, H, dh):
    """Values take no arithmetic but the rounding: codes and exponents equal the reference's."""
    rng = np.random.default_rng(page + 1)
    b = Batch(rng, [0, 1, 70, 3, 0, 7, 633], [5, 100, 70, 40, 0, 3, 655], page, H, dh, 8, spare=3)
    size = torch.from_numpy((2.0 ** rng.integers(-8, 5, (b.n, 1, 1))).astype(np.float32))
    v = (bf16(rng, b.n, H, dh).float() * size).to(torch.bfloat16)
    # ties of the codes, whole rows of zeros, and the smallest and largest numbers
    v[1], v[2, 0], v[3, 0] = 0.0, 1.0 + 1.0 / 16, 2.0 ** -126
    v[5, 0, :8] = torch.tensor([3.0e38, -3.0e38, 1.0, 448.0, 449.0, 0.0, -0.0, 2.0 ** -130])
    v[74, 0, :2] = torch.tensor([float("nan"), float("inf")])
    ref, _ = run_append(cast_lib, b, v, v)
    for name, codes, exps in (("k", b.dk, b.dke), ("v", b.dv, b.dve)):
        assert np.array_equal(exps.cpu().numpy(), ref[name + "_exp"]), name
        got, want = codes.cpu().numpy(), ref[name]
        same = (got == want) | (np.isnan(O.E4M3[got]) & np.isnan(O.E4M3[want]))
        assert same.all(), (name, np.argwhere(~same)[:5])


@pytest.mark.parametrize("rot,inter,dh", [(64, False, 64), (48, False, 64), (64, True, 64), (30, True, 64), (20, False, 64), (30, False, 128)])
def test_append_e4m3_rotated(cast_lib, rot, inter, dh):
    rng = np.random.default_rng(rot)
    H, page = 2, 32
    b = Batch(rng, [1, 70, 40], [77, 90, 40], page, H, dh, 8)
    r, turns, _ = make_rope(cast_lib, rot, interleaved=inter)
    k, q = bf16(rng, b.n, H, dh), bf16(rng, b.n, 2 * H, dh)
    ref, kr = run_append(cast_lib, b, k, k, r, turns, inter=inter, q=q)
    # no page's largest key lies within 2^-16 of where the exponent changes, so exponents are equal
    assert np.array_equal(b.dke.cpu().numpy(), ref["k_exp"]) and np.array_equal(b.dve.cpu().numpy(), ref["v_exp"])
    got, want = O.values(b.dk.cpu().numpy(), b.dke.cpu().numpy()), O.values(ref["k"], ref["k_exp"])
    # the rotated key is off by at most 1e-5 (|x| + |y|) (v_sin, v_cos: 2^-18 at most), so its code
    # is the reference's or, next to a tie, the neighbour: one step is 2^-3 of the value
    off = got != want
    step = np.maximum(np.abs(want) * 2.0 ** -3, 2.0 ** (ref["k_exp"].astype(float) - 127 - 9)[:, None, :, None])
    assert np.all(np.abs(got - want) <= step * 1.0001)
    # ties are a share of at most 2 * 1e-5 * 4 * 2^4 (band over half a step) of values; x3
    assert off.mean() <= 4e-3, off.mean()
    assert np.array_equal(b.dv.cpu().numpy(), ref["v"])


def test_append_e4m3_token_by_token(cast_lib):
    """A page that fills up with growing values: its exponent grows and earlier codes follow."""
    rng = np.random.default_rng(12)
    H, dh, page, B = 2, 64, 8, 3
    b = Batch(rng, [1] * B, [20] * B, page, H, dh, 8)
    cache, seqs = b.device(cast_lib)
    ref = b.host()
    for t in range(20):
        x = (bf16(rng, B, H, dh).float() * 2.0 ** (t % 9 - 4)).to(torch.bfloat16)
        b.dlens.fill_(t + 1)
        cast_lib.cast_kv_append(cache, seqs, x.to(DEV), x.to(DEV))
        O.append(ref, b.cu, [t + 1] * B, b.table, f64(x), f64(x))
        assert np.array_equal(b.dke.cpu().numpy(), ref["k_exp"]), t
        assert np.array_equal(O.E4M3[b.dv.cpu().numpy()], O.E4M3[ref["v"]]), t
        assert np.array_equal(O.E4M3[b.dk.cpu().numpy()], O.E4M3[ref["k"]]), t


# ---------------------------------------------------------------------------
# read
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("page,H,dh", [(16, 2, 64), (1, 1, 32), (37, 3, 128), (1560, 5, 32)])
def test_read(cast_lib, bits, page, H, dh):
    rng = np.random.default_rng(page)
    b = Batch(rng, [1], [1], page, H, dh, bits, extra_pages=6)
    cache, _ = b.device(cast_lib)
    idx = np.array([3, 0, 3, -1, 6, b.pages, 2], dtype=np.int32)
    kv, vv = b.values()
    ok = (idx >= 0) & (idx < b.pages)
    pick = lambda x: np.where(ok[:, None, None, None], x[np.where(ok, idx, 0)], 0.0)  # noqa: E731
    di = torch.from_numpy(idx).to(DEV)
    k, v = cast_lib.cast_kv_read(cache, di)
    assert np.array_equal(f64(k), pick(kv)) and np.array_equal(f64(v), pick(vv))
    k, v = cast_lib.cast_kv_read(cache, di, want_v=False)
    assert v is None and np.array_equal(f64(k), pick(kv))
    k, v = cast_lib.cast_kv_read(cache, di, want_k=False)
    assert k is None and np.array_equal(f64(v), pick(vv))
    if bits == 8:
        # every exponent that append writes
        e = torch.arange(10, 248, dtype=torch.uint8, device=DEV).repeat_interleave(1)
        m = e.numel()
        codes = torch.arange(127, dtype=torch.uint8, device=DEV).repeat(m, 2)[:, :128].reshape(m, 4, 1, 32).contiguous()
        c2 = cast_lib.KvCache(codes, codes, e[:, None].contiguous(), e[:, None].contiguous())
        k, _ = cast_lib.cast_kv_read(c2, torch.arange(m, dtype=torch.int32, device=DEV))
        want = O.values(codes.cpu().numpy(), e[:, None].cpu().numpy())
        fits = np.abs(want) < 2.0 ** 128
        assert np.array_equal(f64(k)[fits], want[fits])


def test_rope_past_one_launch(cast_lib):
    """More tokens than the threads of one launch: the last ones equal a call of their own."""
    n, H, dh = (1 << 25) + 7, 1, 32
    rope = cast_lib.cast_rope_params_init(32)
    x = torch.empty((n, H, dh), dtype=torch.bfloat16, device="cuda")
    x[:100] = torch.randn((100, H, dh), device="cuda").bfloat16()
    x[-100:] = torch.randn((100, H, dh), device="cuda").bfloat16()
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    out = cast_lib.cast_rope(x, pos, rope)
    for part in (slice(0, 100), slice(n - 100, n)):
        assert torch.equal(out[part], cast_lib.cast_rope(x[part].clone(), pos[part].clone(), rope))


@pytest.mark.parametrize("rot,inter", [(128, False), (64, True), (50, False), (0, False)])
@pytest.mark.parametrize("page,H,new,lens", [(300, 2, [350, 1, 300, 0, 290], [400, 77, 300, 20, 640]),
                                             (16, 8, [40] * 64, [40 + i for i in range(64)])])
def test_append_e4m3_long_pages_and_many(cast_lib, rot, inter, page, H, new, lens):
    """Pages longer than a block keeps in registers, begun and continued, and calls with so many pages
    that two heads share their angles."""
    rng = np.random.default_rng(rot + page)
    b = Batch(rng, new, lens, page, H, 128, 8, spare=2)
    r, turns, _ = make_rope(cast_lib, rot, interleaved=inter) if rot else (None, None, None)
    k, v = bf16(rng, b.n, H, 128), bf16(rng, b.n, H, 128)
    ref, _ = run_append(cast_lib, b, k, v, r, turns, inter=inter)
    assert np.array_equal(b.dve.cpu().numpy(), ref["v_exp"]) and np.array_equal(b.dv.cpu().numpy(), ref["v"])
    exps = b.dke.cpu().numpy()
    # exponents differ only where the largest key lies within 1e-6 of where they change: a share of
    # at most 2e-6 / log(2) of the pages, none of these few hundred in 999 of 1000 draws
    assert np.array_equal(exps, ref["k_exp"])
    got, want = O.values(b.dk.cpu().numpy(), exps), O.values(ref["k"], ref["k_exp"])
    # a code is the reference's or, next to a tie, the neighbour
    off = got != want
    step = np.maximum(np.abs(want) * 2.0 ** -3, 2.0 ** (ref["k_exp"].astype(float) - 127 - 9)[:, None, :, None])
    assert np.all(np.abs(got - want) <= step * 1.0001) and off.mean() <= (4e-3 if rot else 0.0), off.mean()
