"""Host side of the cached-history calls: its C++ functions that are not part of the C ABI,
sizes that have to pass or to be refused, and what the binding does around a call."""
import os
import subprocess
import sys
from types import SimpleNamespace

import pytest
import torch

import paper_2609_34144_amd as cast
from test_abi import _HAS_GPU
from test_kv_abi import A, SHAPE, append, attn, cache, rope, seqs

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


# ---------------------------------------------------------------------------
# the binding: what it allocates belongs to the stream of the call
# ---------------------------------------------------------------------------

class _AnyCall:
    """A library whose calls succeed without doing anything and want 256 bytes of workspace."""

    def __getattr__(self, name):
        return lambda *a: 256 if name.endswith("bytes") else 0


def _calls():
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    z = lambda *s, d=bf: torch.zeros(s, dtype=d)  # noqa: E731
    q, kv, frames = z(1, 8, 2, 64), z(3, 8, 2, 64), z(4, 8, 8, 2, d=f32)
    cache, seqs = cast.KvCache(z(4, 16, 2, 64), z(4, 16, 2, 64)), cast.KvSeqs(z(3, d=i32), z(2, d=i32), z(2, 4, d=i32))
    rope = cast.RopeParams(z(32, d=torch.float64), z(32, d=torch.uint8))
    k, qn, pos = z(5, 2, 64), z(5, 4, 64), z(5, d=i32)
    dp = cast.DiagParams(tile_h=8, tile_w=8, n_bands=2)
    return {
        "route_kv": (3, lambda s: cast.cast_route_kv(q, kv, 2, want_scores=True, stream=s)),
        "wo_gram": (1, lambda s: cast.cast_wo_gram(z(128, 128), 2, 64, stream=s)),
        "route_coupled": (3, lambda s: cast.cast_route_coupled(q, kv, kv, z(2, 64, 64, d=f32), [0], 4, 2, 1.0,
                                                               cast.CoupledParams(), want_u=True, stream=s)),
        "frame_select": (2, lambda s: cast.cast_frame_select(z(4, 8, 2), None, [0, 3], 2, z(4, d=i32), cast.SelectParams(), stream=s)),
        "spectral_diagnostics": (6, lambda s: cast.cast_spectral_diagnostics(frames, frames, [0, 3], dp, theta=frames,
                                                                             want_corrections=True, stream=s)),
        "phase_progress": (1, lambda s: cast.cast_phase_progress(frames, [0, 3], dp, stream=s)),
        "anchor_attn": (3, lambda s: cast.cast_anchor_attn(q, kv, kv, z(1, 2, 2, d=i32), 2, 1.0, want_lse=True, stream=s)),
        "par_reconstruct": (2, lambda s: cast.cast_par_reconstruct(frames, [0, 3], cast.ParParams(), stream=s)),
        "rope": (1, lambda s: cast.cast_rope(k, pos, rope, stream=s)),
        "kv_append": (1, lambda s: cast.cast_kv_append(cache, seqs, k, k, rope, q=qn, stream=s)),
        "kv_read": (2, lambda s: cast.cast_kv_read(cache, z(2, d=i32), stream=s)),
        "kv_attn": (3, lambda s: cast.cast_kv_attn(qn, cache, seqs, 0.1, want_lse=True, stream=s)),
    }


@pytest.mark.parametrize("name", ["route_kv", "wo_gram", "route_coupled", "frame_select", "spectral_diagnostics", "phase_progress",
                                  "anchor_attn", "par_reconstruct", "rope", "kv_append", "kv_read", "kv_attn"])
def test_allocations_belong_to_the_stream_of_the_call(lib, monkeypatch, name):
    """Outputs and workspaces of a call on another stream than the current one are that stream's:
    else the caching allocator would give a workspace to the current stream's next allocation while
    the call still runs (two calls on two streams would share one), or an output's memory would
    still be in use there."""
    count, call = _calls()[name]
    current, made = [], []

    class Under:
        def __init__(self, s):
            self.s = s

        def __enter__(self):
            current.append(self.s)

        def __exit__(self, *a):
            current.pop()

    def watch(f):
        def make(*a, **kw):
            made.append(current[-1] if current else None)
            return f(*a, **kw)
        return make

    stream = SimpleNamespace(cuda_stream=0x40, device_index=0)
    monkeypatch.setattr(cast, "_lib", _AnyCall())
    monkeypatch.setattr(cast, "_on", lambda device, s: 0)
    monkeypatch.setattr(torch.cuda, "stream", Under)
    for f in ("empty", "empty_like", "zeros", "zeros_like", "full"):
        monkeypatch.setattr(torch, f, watch(getattr(torch, f)))
    call(stream)
    assert made[-count:] == [stream] * count, made           # (inputs that the call's line makes come first)
    if name in ("rope", "kv_append", "kv_read", "kv_attn"):
        call(None)                                           # no stream: the current one, no switch
        assert made[-count:] == [None] * count


def test_a_stream_of_another_device_is_refused(lib, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    gpu = torch.device("cuda", 0)
    assert cast._on(gpu, SimpleNamespace(cuda_stream=0x40, device_index=0)) == 0x40
    for device, stream in ((gpu, SimpleNamespace(cuda_stream=0x40, device_index=1)),
                           (torch.device("cuda", 1), SimpleNamespace(cuda_stream=0x40, device_index=1))):
        with pytest.raises(cast.CastError):
            cast._on(device, stream)


def test_scales_whose_logarithmic_form_overflows_are_refused(lib):
    """The kernels take scale * log2(e), which must be finite."""
    if _HAS_GPU:
        pytest.skip("calls with fake pointers run GPU-less only")
    assert attn(lib, scale=2.5e38) == SHAPE and attn(lib, scale=2.0e38) == HIP and attn(lib, scale=1e-45) == HIP


@pytest.mark.parametrize("call", ["r_rope(lib, n=2 ** 31 - 1, H=1, dh=32, xt=32, xh=32, yt=32, yh=32)",
                                  "read(lib, cache(pages=1, page=1, H=1, dh=32), m=2 ** 31 - 1)"])
def test_launches_of_the_largest_counts_end(lib, call):
    """Tokens and pages next to 2^31 go in several launches, whose counter must not wrap."""
    if _HAS_GPU:
        pytest.skip("calls with fake pointers run GPU-less only")
    here = os.path.dirname(os.path.abspath(__file__))
    code = (f"import sys; sys.path[:0] = [{os.path.dirname(here)!r}, {here!r}]\n"
            "import paper_2609_34144_amd as cast\nlib = cast.load()\nfrom test_kv_abi import cache, r_rope, read\n"
            f"sys.exit({call})")
    assert subprocess.run([sys.executable, "-c", code], timeout=60).returncode == HIP


def test_the_current_stream_is_found_without_torchs_private_function():
    streams = {0: SimpleNamespace(cuda_stream=0x40), 1: SimpleNamespace(cuda_stream=0x50)}
    other = SimpleNamespace(_C=SimpleNamespace(), cuda=SimpleNamespace(current_stream=streams.get))
    assert [cast._current_raw_stream(other)(i) for i in (0, 1)] == [0x40, 0x50]
    other._C._cuda_getCurrentRawStream = lambda index: 0x60 + index
    assert cast._current_raw_stream(other)(1) == 0x61


# ---------------------------------------------------------------------------
# the binding: sizes that a C int does not hold
# ---------------------------------------------------------------------------

def test_sizes_past_32_bits_are_refused(lib):
    """ctypes would pass their low bits on: a window of -2^32 as none, 2^32 + 5 tokens as five."""
    z = lambda *s, d=torch.int32: torch.zeros(s, dtype=d)  # noqa: E731
    big = 1 << 32
    kv = z(4, 16, 2, 64, d=torch.bfloat16)
    q, c, s = z(3, 2, 64, d=torch.bfloat16), cast.KvCache(kv, kv.clone()), cast.KvSeqs(z(2), z(1), z(1, 2))
    rope = cast.RopeParams(z(32, d=torch.float64), None)
    many = kv[:1, :1].expand(big + 5, 1, 2, 64)
    bad = [lambda: cast.cast_kv_attn(q, c, s, 0.1, window=-big), lambda: cast.cast_kv_attn(q, c, s, 0.1, window=4, sinks=8 - big),
           lambda: cast.cast_kv_attn_workspace_bytes(q, c, s, window=big), lambda: cast.cast_kv_attn_workspace_bytes(q, c, s, sinks=-big),
           lambda: cast.cast_kv_attn_workspace_bytes(many[:, 0], c, s), lambda: cast.cast_kv_append(c, s, many[:, 0], many[:, 0]),
           lambda: cast.cast_rope(many[:, 0], z(1).expand(big + 5), rope), lambda: cast.cast_kv_read(c, z(1).expand(big + 5)),
           lambda: cast.KvCache(many, many)]
    for f in bad:
        with pytest.raises(cast.CastError, match="below 2\\^31"):
            f()
    for dims in ([big + 64], [1 << 40], [-big + 64]):
        with pytest.raises(cast.CastError):
            cast.cast_rope_frequencies(dims)
