"""Forms of the cached-history calls that lie next to a limit: the last page of a cache,
other streams, extreme values and exponents, long pages."""
import numpy as np
import pytest
import torch

from kv_util import Batch, bf16, f64
from oracle import kv as O
from test_gpu_kv_attn import MASKS, run
from test_gpu_kv_attn_many import run as run_some
from test_gpu_kv_cache import make_rope, run_append

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


# ---------------------------------------------------------------------------
# append, e4m3: long pages, positions of several axes
# ---------------------------------------------------------------------------

def check_codes(cast, b, k, v, rot, inter=False, axes=None, pos=None, q=None):
    """The cache after an append against the reference's.  The kernel's rotated key is off by at most
    d = (|x| + |y|) 3e-7: cosine and sine by 7.5e-8, and four roundings of 2^-24 (amplitude, product,
    sum, and the angle's fp64 ones, which are far below).  So its exponents and codes lie between
    those of key - d and key + d; values, and rows that were there, equal the reference's."""
    r, turns, axis = make_rope(cast, rot, axes=axes, interleaved=inter) if rot else (None, None, None)
    ref, kr = run_append(cast, b, k, v, r, turns, axis, inter, 1.0, pos, q)
    d = np.zeros_like(kr)
    x = np.abs(f64(k))
    for j in range(rot // 2):
        c0, c1 = (2 * j, 2 * j + 1) if inter else (j, j + rot // 2)
        d[..., c0] = d[..., c1] = 3e-7 * (x[..., c0] + x[..., c1])
    lo, hi = b.host(), b.host()
    O.append(lo, b.cu, b.lens, b.table, kr - d, f64(v))
    O.append(hi, b.cu, b.lens, b.table, kr + d, f64(v))
    assert np.array_equal(b.dve.cpu().numpy(), ref["v_exp"]) and np.array_equal(b.dv.cpu().numpy(), ref["v"])
    exps, codes = b.dke.cpu().numpy(), b.dk.cpu().numpy()
    least, most = (f(lo["k_exp"], hi["k_exp"]) for f in (np.minimum, np.maximum))
    assert np.all((least <= exps) & (exps <= most))
    one = (least == most)[:, None, :, None]                  # else the codes have no common scale
    assert one.mean() > 0.9
    got = O.E4M3[codes]
    inside = (O.E4M3[lo["k"]] <= got) & (got <= O.E4M3[hi["k"]])
    assert np.all(inside | ~one), np.argwhere(~(inside | ~one))[:5]


LONG = [(128, 20, 300, [200, 150, 1, 300, 0, 250, 140, 180], [500, 150, 9, 300, 7, 256, 900, 301]),
        (64, 40, 700, [400, 300, 200, 350], [800, 300, 1500, 701]),
        (32, 76, 1100, [700, 600], [1500, 600]),
        (128, 3, 6000, [200, 140, 150], [6100, 140, 210])]


@pytest.mark.parametrize("dh,H,page,new,lens", LONG)
@pytest.mark.parametrize("layout", ["half", "interleaved", "any", "none"])
def test_append_e4m3_parts_of_long_pages(cast_lib, dh, H, page, new, lens, layout):
    """Pages that several blocks share, begun and continued, the same call's queries rotated: one and
    two heads of K to a block; calls that fill a small part of their pages."""
    rng = np.random.default_rng(page)
    b = Batch(rng, new, lens, page, H, dh, 8, spare=3)
    size = torch.from_numpy((2.0 ** rng.integers(-6, 5, (b.n, 1, 1))).astype(np.float32))
    k, v = ((bf16(rng, b.n, H, dh).float() * size).to(torch.bfloat16) for _ in range(2))
    rot, inter = {"half": (dh, False), "interleaved": (dh // 2, True), "any": (22, False), "none": (0, False)}[layout]
    check_codes(cast_lib, b, k, v, rot, inter, q=bf16(rng, b.n, H, dh) if rot else None)


@pytest.mark.parametrize("page,new,lens", [(16, [30, 1, 7], [40, 1, 100]), (300, [200, 150], [430, 150])])
@pytest.mark.parametrize("rot,inter,axes", [(64, False, None), (128, True, [44, 42, 42]), (96, False, [32, 32, 32]), (60, False, [20, 40])])
def test_append_e4m3_positions(cast_lib, page, new, lens, rot, inter, axes):
    """Positions that the call gives, of one axis and of several."""
    rng = np.random.default_rng(rot)
    b = Batch(rng, new, lens, page, 4, 128, 8, spare=1)
    pos = rng.integers(0, 5000, (b.n, len(axes or [1]))).astype(np.int32)
    check_codes(cast_lib, b, bf16(rng, b.n, 4, 128), bf16(rng, b.n, 4, 128), rot, inter, axes, pos, bf16(rng, b.n, 8, 128))


# ---------------------------------------------------------------------------
# other streams
# ---------------------------------------------------------------------------

def test_calls_on_two_streams_at_once(cast_lib):
    """Calls that cut long ranges, on two streams, with workspaces and outputs made in the call, while
    the current stream allocates: each gives what it gives alone."""
    rng = np.random.default_rng(60)
    sides = []
    for new, lens in (([1] * 4, [9000, 300, 7000, 4000]), ([40, 60], [9000, 5000])):
        b = Batch(rng, new, lens, 16, 2, 64, 16)
        cache, seqs = b.device(cast_lib)
        q = bf16(rng, b.n, 8, 64).to(DEV)
        assert cast_lib.cast_kv_attn_workspace_bytes(q, cache, seqs) > 0
        sides.append((q, cache, seqs, cast_lib.cast_kv_attn(q, cache, seqs, 0.125, want_lse=True)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for i in range(40):
        q, cache, seqs, _ = sides[i % 2]
        got.append((i % 2, cast_lib.cast_kv_attn(q, cache, seqs, 0.125, want_lse=True, stream=streams[(i // 2) % 2])))
        torch.full((1 << 20,), float("nan"), device=DEV)
    torch.cuda.synchronize()
    for i, (out, lse) in got:
        assert torch.equal(out, sides[i][3][0]) and torch.equal(lse, sides[i][3][1])


def test_outputs_are_not_memory_that_the_current_stream_still_uses(cast_lib):
    """Memory that was freed with work on the current stream pending does not become the output of a
    call on another stream."""
    rope = cast_lib.cast_rope_params_init(64)
    x = torch.randn((4096, 8, 64), device=DEV).bfloat16()
    pos = torch.arange(4096, dtype=torch.int32, device=DEV)
    want = cast_lib.cast_rope(x, pos, rope)
    busy = torch.randn((4096, 4096), device=DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(5):
        old = torch.empty_like(x)
        for _ in range(4):
            busy = torch.mm(busy, busy).clamp_(-1.0, 1.0)    # some milliseconds
        old.fill_(7.0)
        del old
        got = cast_lib.cast_rope(x, pos, rope, stream=s)
        torch.cuda.synchronize()
        assert torch.equal(got, want)


# ---------------------------------------------------------------------------
# attention: values up to the type's largest
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("H,dh,new,what", [(2, 64, [1, 2, 9], "rows"), (2, 64, [40, 70, 3], "tiles"), (3, 128, [200, 60, 130], "tiles"),
                                           (64, 128, [300, 200, 260], "pairs"), (1, 32, [1, 1, 1], "rows in pieces"),
                                           (2, 128, [60, 20, 40], "tiles in pieces")])
def test_the_largest_finite_values(cast_lib, bits, H, dh, new, what):
    """Values up to 2^127 under scores that rise by up to 10 (less than 2^16 in all) over the keys: a
    row's result is finite, whatever the sums on the way, and as exact as for small values."""
    rng = np.random.default_rng(61)
    lens = [700, 300, 520] if "pieces" not in what else [9000, 3000, 7000]
    b = Batch(rng, new, lens, 16, H, dh, bits, spread=False)
    # scores: q = 1 in one channel, the key's channel 0 rises with its index
    q = torch.zeros((b.n, H, dh))
    q[:, :, 0] = 1.0
    for s, L in enumerate(lens):
        t = np.arange(L)
        at, row = b.table[s, t // 16], t % 16
        rise = np.floor(10.0 * t / L * 16) / 16
        b.k[at, row] = 0
        if bits == 16:
            b.k[at, row, :, 0] = torch.from_numpy(rise.astype(np.float32)).to(torch.bfloat16)[:, None]
        else:
            code = torch.from_numpy(O.e4m3_code(rise))
            b.k[at, row, :, 0] = code[:, None]
    if bits == 16:
        b.v = (b.v.float().clamp(-1.9, 1.9) * 2.0 ** 126).to(torch.bfloat16)
    else:
        b.ke.fill_(127)
        b.v = torch.from_numpy(O.e4m3_code(rng.uniform(-240.0, 240.0, tuple(b.v.shape))))
        b.ve.fill_(127 + 119)                                # 240 * 2^119 < 2^127
    for causal, window in ((True, 0), (False, 250)):
        run_some(cast_lib, b, q.to(torch.bfloat16), 1.0, causal, window, 3, what)


def test_uniform_scores_over_the_largest_values(cast_lib):
    """Keys of one score whose values are all 2^127: their mean is that, their sum is not finite."""
    rng = np.random.default_rng(62)
    for new, dh, H in ((1, 64, 2), (50, 64, 2), (300, 128, 64)):
        b = Batch(rng, [new], [2000], 16, H, dh, 16)
        b.k.zero_()
        b.v.fill_(2.0 ** 127)
        out, _ = run_some(cast_lib, b, bf16(rng, b.n, H, dh), 0.1, False, what="uniform")
        assert bool(((out.float() / 2.0 ** 127 - 1.0).abs() <= 2.0 ** -7).all())


# ---------------------------------------------------------------------------
# every exponent byte
# ---------------------------------------------------------------------------

def all_bytes(cast, page=16, dh=32):
    """A cache with a page for each exponent byte, in which every code lies; its values as bf16
    (float64), rounded there once."""
    codes = torch.arange(page * dh).to(torch.uint8).reshape(1, page, 1, dh).repeat(256, 1, 1, 1)
    exps = torch.arange(256).to(torch.uint8)[:, None].contiguous()
    k, ones = torch.zeros_like(codes), torch.full_like(exps, 127)
    cache = cast.KvCache(k.to(DEV), codes.to(DEV), ones.to(DEV), exps.to(DEV))
    want = f64(torch.from_numpy(O.values(codes.numpy(), exps.numpy())).float().to(torch.bfloat16))
    return cache, want


def same(got, want):
    return (got == want) | (np.isnan(got) & np.isnan(want))


def test_every_exponent_byte_is_read(cast_lib):
    cache, want = all_bytes(cast_lib)
    idx = torch.arange(256, dtype=torch.int32, device=DEV)
    _, v = cast_lib.cast_kv_read(cache, idx, want_k=False)
    ok = same(f64(v), want)
    assert ok.all(), np.argwhere(~ok)[:5]
    assert np.isnan(f64(v)[255]).all()


@pytest.mark.parametrize("rows", ["few", "many"])
def test_every_exponent_byte_is_attended(cast_lib, rows):
    """A row that sees one key gives its value, as cast_kv_read does; what lies beside it, infinite or
    NaN, does not reach the row.  Terms below 2^-80 may be lost."""
    page, dh = 16, 32
    cache, want = all_bytes(cast_lib, page, dh)
    i32 = lambda x: torch.as_tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    if rows == "few":                                        # the last row of each page
        seqs = cast_lib.KvSeqs(i32(range(257)), i32([page] * 256), i32(range(256))[:, None].contiguous())
        want = want[:, -1]
    else:
        seqs = cast_lib.KvSeqs(i32([0, 256 * page]), i32([256 * page]), i32(range(256))[None].contiguous())
        want = want.reshape(256 * page, 1, dh)
    q = torch.ones((len(want), 1, dh), dtype=torch.bfloat16, device=DEV)
    got = f64(cast_lib.cast_kv_attn(q, cache, seqs, 0.1, True, 1, 0)[0])
    with np.errstate(invalid="ignore"):
        ok = same(got, want) | (np.abs(got - want) <= 2.0 ** -80)
    assert ok.all(), (np.argwhere(~ok)[:5], got[~ok][:5], want[~ok][:5])


@pytest.mark.parametrize("size", [2.0 ** 127, 1.0, 2.0 ** -120])
def test_every_exponent_byte_is_appended_to(cast_lib, size):
    """Tokens into pages that begin with any exponent: it only grows, earlier codes follow it."""
    rng = np.random.default_rng(63)
    b = Batch(rng, [3] * 256, [9] * 256, 16, 2, 32, 8)
    ex = np.arange(256)
    b.ke[b.table[:, 0]] = torch.from_numpy(np.stack([ex, ex[::-1]], 1).astype(np.uint8))
    b.ve[b.table[:, 0]] = torch.from_numpy(np.stack([(ex + 100) % 256, ex], 1).astype(np.uint8))
    x = torch.from_numpy(rng.uniform(-1.9, 1.9, (b.n, 2, 32)) * size).float().to(torch.bfloat16)
    ref, _ = run_append(cast_lib, b, x, x)
    for codes, exps, name in ((b.dk, b.dke, "k"), (b.dv, b.dve, "v")):
        assert np.array_equal(exps.cpu().numpy(), ref[name + "_exp"])
        ok = same(O.E4M3[codes.cpu().numpy()], O.E4M3[ref[name]])
        assert ok.all(), np.argwhere(~ok)[:5]
