"""Cached-history entry points without a GPU: refusals of every argument check of the C ABI
(each call has one invalid argument, so nothing is enqueued; addresses are never
dereferenced), empty calls, the host's frequency tables, the attention's workspace query,
and the refusals of the Python binding."""
import ctypes
import os

import numpy as np
import pytest
import torch
from hypothesis import given, settings, strategies as st

import paper_2609_34144_amd as cast
from oracle import kv as O
from test_abi import _HAS_GPU

pytestmark = pytest.mark.skipif(_HAS_GPU, reason="fake-pointer validation tests run GPU-less only")
OK, NULL, SHAPE, ANCHORS, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4, 5
A = 1 << 20


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(cast.LIB_PATH):
        pytest.skip("libcast.so not built (run __graft_entry__.build())")
    return cast.load()


def cache(**kw):
    f = dict(k=A, v=2 * A, k_exp=None, v_exp=None, dtype=1, pages=8, page=16, H=2, dh=64)
    f.update(kw)
    return cast.KvCacheStruct(f["k"], f["v"], f["k_exp"], f["v_exp"], f["dtype"], f["pages"], f["page"], f["H"], f["dh"])


def seqs(**kw):
    f = dict(cu=3 * A, len=4 * A, table=5 * A, n_seq=2, n_tok=5, max_pages=4)
    f.update(kw)
    return cast.KvSeqsStruct(f["cu"], f["len"], f["table"], f["n_seq"], f["n_tok"], f["max_pages"])


def rope(**kw):
    f = dict(rot_dim=32, interleaved=0, n_axes=1, amplitude=1.0, turns=6 * A, axis=None)
    f.update(kw)
    return cast.RopeStruct(f["rot_dim"], f["interleaved"], f["n_axes"], f["amplitude"], f["turns"], f["axis"])


NAN = float("nan")
BAD_CACHE = [(dict(dtype=0), SHAPE), (dict(dtype=3), SHAPE), (dict(dh=48), UNSUPPORTED), (dict(dh=256), UNSUPPORTED),
             (dict(pages=0), SHAPE), (dict(page=0), SHAPE), (dict(H=0), SHAPE), (dict(pages=1 << 30), UNSUPPORTED),
             (dict(H=5000), UNSUPPORTED), (dict(page=1 << 24, pages=1), UNSUPPORTED)]
BAD_CACHE_PTR = [(dict(k=None), NULL), (dict(v=None), NULL), (dict(k=A + 8), SHAPE), (dict(v=A + 2), SHAPE),
                 (dict(dtype=2), NULL), (dict(dtype=2, k_exp=A), NULL)]
BAD_SEQS = [(dict(n_seq=0), SHAPE), (dict(n_tok=-1), SHAPE), (dict(max_pages=0), SHAPE), (dict(n_seq=(1 << 20) + 1), UNSUPPORTED),
            (dict(n_tok=1 << 30), UNSUPPORTED), (dict(max_pages=1 << 26), UNSUPPORTED)]
BAD_SEQS_PTR = [(dict(cu=None), NULL), (dict(len=None), NULL), (dict(table=None), NULL), (dict(cu=A + 2), SHAPE),
                (dict(len=A + 1), SHAPE), (dict(table=A + 3), SHAPE)]
BAD_ROPE = [(dict(rot_dim=0), SHAPE), (dict(rot_dim=66), SHAPE), (dict(rot_dim=31), SHAPE), (dict(interleaved=2), SHAPE),
            (dict(n_axes=0), SHAPE), (dict(n_axes=4), SHAPE), (dict(amplitude=NAN), SHAPE), (dict(amplitude=float("inf")), SHAPE),
            (dict(turns=None), NULL), (dict(turns=A + 4), SHAPE)]


def r_rope(lib, p=None, **kw):
    f = dict(x=A, dtype=1, n=3, H=2, dh=64, xt=128, xh=64, pos=2 * A, tr=0, out=3 * A, yt=128, yh=64)
    f.update(kw)
    return lib.cast_rope(f["x"], f["dtype"], f["n"], f["H"], f["dh"], f["xt"], f["xh"], f["pos"],
                         None if p is False else ctypes.byref(p if p is not None else rope()), f["tr"], f["out"], f["yt"], f["yh"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(x=None), NULL), (dict(pos=None), NULL), (dict(out=None), NULL), (dict(dtype=2), SHAPE), (dict(n=-1), SHAPE),
    (dict(H=0), SHAPE), (dict(dh=96), UNSUPPORTED), (dict(tr=2), SHAPE), (dict(xt=63), SHAPE), (dict(xh=63), SHAPE), (dict(yt=-128), SHAPE),
    (dict(yt=64, yh=64), SHAPE), (dict(yt=100, yh=64), SHAPE), (dict(x=A + 1), SHAPE), (dict(out=A + 1), SHAPE), (dict(pos=A + 2), SHAPE),
    (dict(dtype=0, x=A + 2), SHAPE), (dict(out=A, xt=256), SHAPE), (dict(n=1 << 30, H=16, yt=1 << 20), UNSUPPORTED)])
def test_rope_refusals(lib, kw, want):
    assert r_rope(lib, **kw) == want, lib.cast_last_error_detail()


@pytest.mark.parametrize("kw,want", BAD_ROPE)
def test_rotation_refusals(lib, kw, want):
    assert r_rope(lib, rope(**kw)) == want
    assert append(lib, r=rope(**kw)) == want


def test_rope_null_params_and_empty(lib):
    assert r_rope(lib, False) == NULL
    assert r_rope(lib, n=0, x=None, pos=None, out=None) == OK


def append(lib, c=None, s=None, r=None, **kw):
    f = dict(k=7 * A, ks=128, v=8 * A, vs=128, pos=None, q=None, qs=256, Hq=4, qo=None)
    f.update(kw)
    ref = lambda x, d: None if x is False else ctypes.byref(x if x is not None else d)  # noqa: E731
    return lib.cast_kv_append(ref(c, cache()), ref(s, seqs()), f["k"], f["ks"], f["v"], f["vs"], ref(r, rope()), f["pos"], f["q"],
                              f["qs"], f["Hq"], f["qo"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(k=A + 8), SHAPE), (dict(v=A + 2), SHAPE), (dict(ks=120), SHAPE), (dict(vs=127), SHAPE),
    (dict(ks=132), SHAPE), (dict(ks=-128), SHAPE), (dict(q=9 * A), NULL), (dict(q=9 * A, qo=10 * A, Hq=0), SHAPE),
    (dict(q=9 * A, qo=10 * A, qs=255), SHAPE), (dict(q=9 * A, qo=10 * A + 4), SHAPE), (dict(q=9 * A, qo=9 * A, qs=264), SHAPE),
    (dict(q=9 * A, qo=10 * A, r=False), NULL), (dict(c=False), NULL), (dict(s=False), NULL), (dict(pos=A + 2), SHAPE),
    (dict(r=rope(n_axes=2, axis=A)), NULL)])
def test_append_refusals(lib, kw, want):
    assert append(lib, **kw) == want, lib.cast_last_error_detail()


def read(lib, c=None, **kw):
    f = dict(idx=3 * A, m=2, k=4 * A, v=5 * A)
    f.update(kw)
    return lib.cast_kv_read(None if c is False else ctypes.byref(c if c is not None else cache()), f["idx"], f["m"], f["k"], f["v"], None)


@pytest.mark.parametrize("kw,want", [(dict(idx=None), NULL), (dict(k=None, v=None), NULL), (dict(m=-1), SHAPE), (dict(idx=A + 1), SHAPE),
                                     (dict(k=A + 8), SHAPE), (dict(v=A + 8), SHAPE), (dict(c=False), NULL)])
def test_read_refusals(lib, kw, want):
    assert read(lib, **kw) == want


def attn(lib, c=None, s=None, **kw):
    f = dict(q=7 * A, qs=256, Hq=4, max_len=64, causal=1, window=0, sinks=0, scale=0.1, out=8 * A, lse=None, ws=None, wsb=0)
    f.update(kw)
    ref = lambda x, d: None if x is False else ctypes.byref(x if x is not None else d)  # noqa: E731
    return lib.cast_kv_attn(f["q"], f["qs"], f["Hq"], ref(c, cache()), ref(s, seqs()), f["max_len"], f["causal"], f["window"], f["sinks"],
                            f["scale"], f["out"], f["lse"], f["ws"], f["wsb"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), NULL), (dict(out=None), NULL), (dict(q=A + 8), SHAPE), (dict(out=A + 8), SHAPE), (dict(lse=A + 2), SHAPE),
    (dict(qs=248), SHAPE), (dict(qs=260), SHAPE), (dict(Hq=3), SHAPE), (dict(Hq=0), SHAPE), (dict(max_len=0), SHAPE),
    (dict(causal=2), SHAPE), (dict(window=-1), SHAPE), (dict(sinks=-1), SHAPE), (dict(scale=0.0), SHAPE), (dict(scale=-1.0), SHAPE),
    (dict(scale=NAN), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(ws=A + 64, wsb=1 << 30), WORKSPACE), (dict(c=False), NULL),
    (dict(s=False), NULL), (dict(s=seqs(n_tok=1 << 25), Hq=64, qs=4096), UNSUPPORTED)])
def test_attn_refusals(lib, kw, want):
    assert attn(lib, **kw) == want, lib.cast_last_error_detail()


@pytest.mark.parametrize("call", [append, read, attn])
@pytest.mark.parametrize("kw,want", BAD_CACHE + BAD_CACHE_PTR)
def test_cache_refusals(lib, call, kw, want):
    assert call(lib, cache(**kw)) == want, lib.cast_last_error_detail()


@pytest.mark.parametrize("call", [append, attn])
@pytest.mark.parametrize("kw,want", BAD_SEQS + BAD_SEQS_PTR)
def test_sequence_refusals(lib, call, kw, want):
    assert call(lib, s=seqs(**kw)) == want, lib.cast_last_error_detail()


def test_empty_calls(lib):
    """No rows, no pages: nothing is enqueued, no tensor is looked at."""
    none = cache(k=None, v=None)
    s = seqs(n_tok=0, cu=None, len=None, table=None)
    assert append(lib, none, s, k=None, v=None) == OK
    assert attn(lib, none, s, q=None, out=None) == OK
    assert read(lib, none, m=0, idx=None, k=None, v=None) == OK


@settings(max_examples=150, deadline=None)
@given(n_tok=st.integers(-2, 1 << 14), n_seq=st.integers(-1, 300), Hq=st.integers(-1, 200), H=st.integers(-1, 40),
       dh=st.sampled_from([32, 64, 128, 100]), page=st.integers(-1, 4000), max_len=st.integers(-1, 1 << 20), window=st.integers(-1, 1 << 16))
def test_attn_workspace_query_any_ints(n_tok, n_seq, Hq, H, dh, page, max_len, window):
    lib = cast.load()
    c, s = cache(H=H, dh=dh, page=page), seqs(n_tok=n_tok, n_seq=n_seq, max_pages=1 << 10)
    nb = lib.cast_kv_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(s), Hq, max_len, 1, window, 3)
    assert nb >= 0 and nb % 256 == 0


@pytest.mark.parametrize("scaling", ["none", "linear", "parts"])
@pytest.mark.parametrize("dims", [[128], [2], [44, 42, 42], [6, 26]])
def test_frequencies(lib, dims, scaling):
    t, a = cast.cast_rope_frequencies(dims, base=500000.0, scaling=scaling, factor=8.0, orig_len=8192, beta_fast=32.0, beta_slow=1.0)
    wt, wa = O.frequencies(dims, 500000.0, scaling, 8.0, 8192, 32.0, 1.0)
    assert np.allclose(t.numpy(), wt, rtol=1e-14, atol=0) and np.array_equal(a.numpy(), wa)


@pytest.mark.parametrize("kw", [dict(axis_dims=[]), dict(axis_dims=[2, 2, 2, 2]), dict(axis_dims=[0]), dict(axis_dims=[3]),
                                dict(axis_dims=[130]), dict(axis_dims=[64, 66]), dict(base=0.0), dict(base=NAN), dict(scaling="x"),
                                dict(scaling="linear", factor=0.5), dict(scaling="parts", factor=2.0, orig_len=0.0),
                                dict(scaling="parts", factor=2.0, orig_len=10.0, beta_fast=1.0, beta_slow=1.0)])
def test_frequency_refusals(lib, kw):
    f = dict(axis_dims=[64])
    f.update(kw)
    with pytest.raises(cast.CastError):
        cast.cast_rope_frequencies(**f)


def test_binding_refusals(lib):
    """What the C ABI cannot see: types, devices, shapes and density of the tensors."""
    bf, i32, u8 = torch.bfloat16, torch.int32, torch.uint8
    z = lambda *s, dtype=bf: torch.zeros(s, dtype=dtype)  # noqa: E731
    k = z(4, 16, 2, 64)
    c = cast.KvCache(k, k.clone())
    s = cast.KvSeqs(z(3, dtype=i32), z(2, dtype=i32), z(2, 4, dtype=i32))
    turns, axis = cast.cast_rope_frequencies([32])
    r = cast.RopeParams(turns, axis)
    kn, q = z(5, 2, 64), z(5, 4, 64)
    bad = [
        lambda: cast.KvCache(k.float(), k.float()), lambda: cast.KvCache(k, z(4, 16, 2, 32)), lambda: cast.KvCache(k[:, ::2], k[:, ::2]),
        lambda: cast.KvCache(k, k, z(4, 2, dtype=u8), None), lambda: cast.KvCache(z(4, 16, 2, 64, dtype=u8), z(4, 16, 2, 64, dtype=u8)),
        lambda: cast.KvCache(z(4, 16, 2, 64, dtype=u8), z(4, 16, 2, 64, dtype=u8), z(4, 3, dtype=u8), z(4, 2, dtype=u8)),
        lambda: cast.KvSeqs(z(3, dtype=torch.int64), z(2, dtype=i32), z(2, 4, dtype=i32)),
        lambda: cast.KvSeqs(z(2, dtype=i32), z(2, dtype=i32), z(2, 4, dtype=i32)),
        lambda: cast.RopeParams(turns.float(), axis), lambda: cast.RopeParams(turns, axis[:3]),
        lambda: cast.cast_kv_append(c, s, kn.float(), kn), lambda: cast.cast_kv_append(c, s, kn, z(4, 2, 64)),
        lambda: cast.cast_kv_append(c, s, z(5, 3, 64), kn), lambda: cast.cast_kv_append(c, s, kn, kn, pos=z(5, 1, dtype=i32)),
        lambda: cast.cast_kv_append(c, s, kn, kn, r, q=q, q_out=z(5, 3, 64)),
        lambda: cast.cast_kv_append(c, s, kn, z(5, 64, 2).transpose(1, 2)),
        lambda: cast.cast_kv_attn(q.float(), c, s, 0.1), lambda: cast.cast_kv_attn(z(5, 4, 32), c, s, 0.1),
        lambda: cast.cast_kv_attn(q, c, s, 0.1, out=z(5, 2, 64)), lambda: cast.cast_kv_attn(q, c, s, 0.1, lse_out=z(5, 4)),
        lambda: cast.cast_kv_read(c, z(2, dtype=torch.int64)), lambda: cast.cast_kv_read(c, z(2, dtype=i32), k_out=z(3, 16, 2, 64)),
        lambda: cast.cast_rope(z(5, 2, 64, dtype=torch.float16), z(5, dtype=i32), r), lambda: cast.cast_rope(kn, z(4, dtype=i32), r),
        lambda: cast.cast_rope(kn, z(5, dtype=torch.int64), r), lambda: cast.cast_rope(kn, z(5, dtype=i32), r, out=z(5, 2, 32)),
        lambda: cast.cast_kv_cache_alloc(4, 16, 2, 64, torch.float16, "cpu"),
        # right in everything but on the CPU
        lambda: cast.cast_kv_append(c, s, kn, kn, r), lambda: cast.cast_kv_attn(q, c, s, 0.1), lambda: cast.cast_kv_read(c, z(2, dtype=i32)),
        lambda: cast.cast_rope(kn, z(5, dtype=i32), r),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(cast.CastError):
            f()
            print("not refused:", i)


def test_refusals_of_sizes_that_no_launch_takes(lib):
    """More threads than a launch holds, and an output that is the query."""
    assert attn(lib, cache(H=4096, dh=32), seqs(n_seq=1 << 16, n_tok=1 << 16), Hq=4096, qs=4096 * 32) == UNSUPPORTED
    assert append(lib, cache(dtype=2, k_exp=A, v_exp=A, page=1, H=512, pages=8), seqs(n_tok=1 << 15), ks=512 * 64,
                  vs=512 * 64) == UNSUPPORTED
    assert append(lib, s=seqs(n_tok=(1 << 25) + 1)) == UNSUPPORTED
    assert attn(lib, out=A, q=A) == SHAPE


def test_binding_refuses_windows_past_int32():
    z = lambda *s, d=torch.int32: torch.zeros(s, dtype=d)  # noqa: E731
    kv = z(4, 16, 2, 64, d=torch.bfloat16)
    q, c, s = z(3, 2, 64, d=torch.bfloat16), cast.KvCache(kv, kv.clone()), cast.KvSeqs(z(2), z(1), z(1, 2))
    for kw in (dict(window=1 << 32), dict(window=8, sinks=1 << 31)):
        with pytest.raises(cast.CastError, match="below 2\\^31"):
            cast.cast_kv_attn(q, c, s, 0.1, **kw)
