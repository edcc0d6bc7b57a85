"""Python binding of libcast.so (the MI355X hot path of one CAST block step).

Argument marshalling only: every step of routing, anchor attention and PAR runs in
the library's HIP kernels.  Tensors are torch device tensors (torch supplies the
memory and the current HIP stream); the functions carry the C ABI names and
arguments of include/cast.h, plus small conveniences that allocate outputs and
workspaces with torch.  A call given `stream` does all of it as under
torch.cuda.stream(stream): inputs have to be ready there, and what it returns
belongs to that stream's memory.

There is no fallback: if libcast.so is missing or fails to load, every call
raises.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libcast.so")

CAST_OK = 0
STATUS_NAMES = {0: "CAST_OK", 1: "CAST_ERR_NULL", 2: "CAST_ERR_SHAPE", 3: "CAST_ERR_ANCHORS",
                4: "CAST_ERR_UNSUPPORTED", 5: "CAST_ERR_WORKSPACE", 6: "CAST_ERR_HIP"}

EXPORTED = ["cast_status_string", "cast_last_error_detail", "cast_abi_version",
            "cast_route_kv_workspace_bytes", "cast_route_kv", "cast_anchor_attn_workspace_bytes",
            "cast_anchor_attn",
            "cast_par_params_default", "cast_par_workspace_bytes", "cast_par_reconstruct",
            "cast_par_reconstruct_noalloc", "cast_par_static_scratch_bytes",
            "cast_coupled_params_default", "cast_wo_gram", "cast_route_coupled_workspace_bytes",
            "cast_route_coupled", "cast_select_params_default",
            "cast_frame_select_workspace_bytes", "cast_frame_select", "cast_diag_params_default",
            "cast_spectral_diagnostics_workspace_bytes", "cast_spectral_diagnostics",
            "cast_phase_progress", "cast_rope_frequencies", "cast_rope", "cast_kv_append",
            "cast_kv_read", "cast_kv_attn_workspace_bytes", "cast_kv_attn"]


class CastError(RuntimeError):
    def __init__(self, status: int, detail: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {detail}")
        self.status = status
        self.detail = detail


class ParParams(ctypes.Structure):
    """cast_par_params_t."""
    _fields_ = [("tile_h", ctypes.c_int), ("tile_w", ctypes.c_int),
                ("tau_low", ctypes.c_float), ("tau_high", ctypes.c_float),
                ("q", ctypes.c_float), ("T", ctypes.c_float),
                ("eta_rel", ctypes.c_float), ("eta_abs", ctypes.c_float),
                ("eps", ctypes.c_float), ("gate_mode", ctypes.c_int),
                ("accumulate", ctypes.c_int), ("update_anchors", ctypes.c_int)]


class CoupledParams(ctypes.Structure):
    """cast_coupled_params_t (include/cast.h)."""
    _fields_ = [("l_anc", ctypes.c_float), ("l_rec", ctypes.c_float),
                ("passes", ctypes.c_int), ("tol", ctypes.c_float), ("eps", ctypes.c_float)]


class SelectParams(ctypes.Structure):
    """cast_select_params_t (include/cast.h)."""
    _fields_ = [("lambda_cov", ctypes.c_float), ("eps", ctypes.c_float)]


class DiagParams(ctypes.Structure):
    """cast_diag_params_t (include/cast.h)."""
    _fields_ = [("tile_h", ctypes.c_int), ("tile_w", ctypes.c_int), ("n_bands", ctypes.c_int),
                ("band_edges", ctypes.c_float * 9), ("eps", ctypes.c_float)]


class RopeStruct(ctypes.Structure):
    """cast_rope_params_t (include/cast.h)."""
    _fields_ = [("rot_dim", ctypes.c_int), ("interleaved", ctypes.c_int), ("n_axes", ctypes.c_int),
                ("amplitude", ctypes.c_float), ("turns", ctypes.c_void_p), ("axis", ctypes.c_void_p)]


class KvCacheStruct(ctypes.Structure):
    """cast_kv_cache_t (include/cast.h)."""
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p),
                ("v_exp", ctypes.c_void_p), ("dtype", ctypes.c_int), ("pages", ctypes.c_int),
                ("page", ctypes.c_int), ("H", ctypes.c_int), ("dh", ctypes.c_int)]


class KvSeqsStruct(ctypes.Structure):
    """cast_kv_seqs_t (include/cast.h)."""
    _fields_ = [("cu", ctypes.c_void_p), ("len", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("n_seq", ctypes.c_int), ("n_tok", ctypes.c_int), ("max_pages", ctypes.c_int)]


_lib = None
_torch = _raw_stream = None       # set by load()
_c = ctypes
_ll = _c.c_longlong
_vp, _i, _f, _sz = _c.c_void_p, _c.c_int, _c.c_float, _c.c_size_t


def load(path: str = LIB_PATH):
    """Load libcast.so (after torch, so the library binds to torch's HIP runtime)."""
    global _lib
    if _lib is not None:
        return _lib
    import torch  # (loads the HIP runtime libcast.so must share)
    global _torch, _raw_stream
    _torch, _raw_stream = torch, _current_raw_stream(torch)
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is not built; run python -m paper_2609_34144_amd.build")
    lib = ctypes.CDLL(path, mode=ctypes.RTLD_LOCAL)
    lib.cast_status_string.restype = _c.c_char_p
    lib.cast_status_string.argtypes = [_i]
    lib.cast_last_error_detail.restype = _c.c_char_p
    lib.cast_last_error_detail.argtypes = []
    lib.cast_abi_version.restype = _i
    lib.cast_route_kv_workspace_bytes.restype = _sz
    lib.cast_route_kv_workspace_bytes.argtypes = [_i] * 6
    lib.cast_route_kv.restype = _i
    lib.cast_route_kv.argtypes = [_vp, _vp, _i, _i, _i, _i, _i, _i, _i, _f, _vp, _vp,
                                  _c.POINTER(_i), _vp, _sz, _vp]
    lib.cast_anchor_attn.restype = _i
    lib.cast_anchor_attn.argtypes = [_vp, _vp, _vp, _vp, _i, _vp, _vp, _i, _i, _i, _i, _i, _i,
                                     _i, _f, _vp, _vp, _vp, _sz, _vp]
    lib.cast_anchor_attn_workspace_bytes.restype = _sz
    lib.cast_anchor_attn_workspace_bytes.argtypes = [_i] * 7
    lib.cast_par_params_default.restype = None
    lib.cast_par_params_default.argtypes = [_c.POINTER(ParParams)]
    lib.cast_par_workspace_bytes.restype = _sz
    lib.cast_par_workspace_bytes.argtypes = [_i, _i, _i, _i, _i, _c.POINTER(ParParams)]
    lib.cast_par_reconstruct.restype = _i
    lib.cast_par_reconstruct.argtypes = [_vp, _c.POINTER(_i), _i, _i, _i, _i, _i,
                                         _c.POINTER(ParParams), _vp, _vp, _vp, _vp, _vp, _sz, _vp]
    lib.cast_par_reconstruct_noalloc.restype = _i
    lib.cast_par_reconstruct_noalloc.argtypes = [_vp, _c.POINTER(_i), _i, _i, _i, _i, _i,
                                                 _c.POINTER(ParParams), _vp, _vp, _vp, _vp, _vp]
    lib.cast_par_static_scratch_bytes.restype = _sz
    lib.cast_par_static_scratch_bytes.argtypes = []
    lib.cast_coupled_params_default.restype = None
    lib.cast_coupled_params_default.argtypes = [_c.POINTER(CoupledParams)]
    lib.cast_wo_gram.restype = _i
    lib.cast_wo_gram.argtypes = [_vp, _i, _i, _i, _vp, _vp]
    lib.cast_route_coupled_workspace_bytes.restype = _sz
    lib.cast_route_coupled_workspace_bytes.argtypes = [_i] * 6
    lib.cast_route_coupled.restype = _i
    lib.cast_route_coupled.argtypes = [_vp, _vp, _vp, _vp, _c.POINTER(_i), _i, _i, _i, _i, _i, _i,
                                       _i, _i, _f, _c.POINTER(CoupledParams), _vp, _vp,
                                       _c.POINTER(_i), _vp, _sz, _vp]
    lib.cast_select_params_default.restype = None
    lib.cast_select_params_default.argtypes = [_c.POINTER(SelectParams)]
    lib.cast_frame_select_workspace_bytes.restype = _sz
    lib.cast_frame_select_workspace_bytes.argtypes = [_i] * 3
    lib.cast_frame_select.restype = _i
    lib.cast_frame_select.argtypes = [_vp, _vp, _i, _i, _i, _i, _c.POINTER(_i), _i, _i,
                                      _c.POINTER(SelectParams), _vp, _vp, _vp, _vp, _vp, _sz, _vp]
    lib.cast_diag_params_default.restype = None
    lib.cast_diag_params_default.argtypes = [_c.POINTER(DiagParams)]
    lib.cast_spectral_diagnostics_workspace_bytes.restype = _sz
    lib.cast_spectral_diagnostics_workspace_bytes.argtypes = [_i, _i, _i, _i, _c.POINTER(DiagParams)]
    lib.cast_spectral_diagnostics.restype = _i
    lib.cast_spectral_diagnostics.argtypes = [_vp, _vp, _vp, _c.POINTER(_i), _i, _i, _i, _i, _i,
                                              _c.POINTER(DiagParams), _vp, _vp, _vp, _vp, _vp,
                                              _vp, _sz, _vp]
    lib.cast_phase_progress.restype = _i
    lib.cast_phase_progress.argtypes = [_vp, _c.POINTER(_i), _i, _i, _i, _i, _i,
                                        _c.POINTER(DiagParams), _vp, _vp]
    lib.cast_rope_frequencies.restype = _i
    lib.cast_rope_frequencies.argtypes = [_c.POINTER(_i), _i] + [_c.c_double, _i] + [_c.c_double] * 4 + [_vp, _vp]
    lib.cast_rope.restype = _i
    lib.cast_rope.argtypes = [_vp, _i, _i, _i, _i, _ll, _ll, _vp, _c.POINTER(RopeStruct), _i, _vp, _ll, _ll, _vp]
    lib.cast_kv_append.restype = _i
    lib.cast_kv_append.argtypes = [_c.POINTER(KvCacheStruct), _c.POINTER(KvSeqsStruct), _vp, _ll, _vp, _ll,
                                   _c.POINTER(RopeStruct), _vp, _vp, _ll, _i, _vp, _vp]
    lib.cast_kv_read.restype = _i
    lib.cast_kv_read.argtypes = [_c.POINTER(KvCacheStruct), _vp, _i, _vp, _vp, _vp]
    lib.cast_kv_attn_workspace_bytes.restype = _sz
    lib.cast_kv_attn_workspace_bytes.argtypes = [_c.POINTER(KvCacheStruct), _c.POINTER(KvSeqsStruct), _i, _i, _i, _i, _i]
    lib.cast_kv_attn.restype = _i
    lib.cast_kv_attn.argtypes = [_vp, _ll, _i, _c.POINTER(KvCacheStruct), _c.POINTER(KvSeqsStruct), _i, _i, _i, _i,
                                 _f, _vp, _vp, _vp, _sz, _vp]
    _lib = lib
    return lib


def _check(st: int):
    if st != CAST_OK:
        raise CastError(st, _lib.cast_last_error_detail().decode())


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _new(stream, make, *args, **kw):
    """make(...), with what it allocates (and the kernels that fill it) belonging to `stream`, where the
    call will use it.  Memory of the current stream would be handed out again there as soon as the
    call returns, or still be in use there by what had it before, with nothing to order the two."""
    if stream is None:
        return make(*args, **kw)
    import torch
    with torch.cuda.stream(stream):
        return make(*args, **kw)


def _ws(nbytes: int, device, workspace, stream=None):
    import torch
    if nbytes == 0:
        return None, 0
    if workspace is not None:
        return workspace, workspace.numel() * workspace.element_size()
    # torch's caching allocator returns >= 512-byte aligned blocks
    return _new(stream, torch.empty, nbytes, dtype=torch.uint8, device=device), nbytes


# ---------------------------------------------------------------------------
# C ABI mirrors
# ---------------------------------------------------------------------------

def cast_abi_version() -> int:
    return load().cast_abi_version()


def cast_route_kv_workspace_bytes(n_a, S, H, dh, M, Bv) -> int:
    return load().cast_route_kv_workspace_bytes(n_a, S, H, dh, M, Bv)


def cast_par_workspace_bytes(n_frames, n_anchor, Hg, Wg, D, params: ParParams) -> int:
    return load().cast_par_workspace_bytes(n_frames, n_anchor, Hg, Wg, D, ctypes.byref(params))


def cast_par_params_default(**overrides) -> ParParams:
    p = ParParams()
    load().cast_par_params_default(ctypes.byref(p))
    for k, v in overrides.items():
        setattr(p, k, v)
    return p


def cast_route_kv(q, k_hist, topk: int, scale: float = 1.0, scores_out=None, idx_out=None,
                  workspace=None, stream=None, want_scores: bool = False):
    """q bf16 [n_a, S, H, dh], k_hist bf16 [M, Bv, H, dh] (device).
    Returns (idx int32 [n_a, H, k_eff], k_eff, scores fp32 [n_a, H, M] or None)."""
    import torch
    lib = load()
    n_a, S, H, dh = q.shape
    M, Bv = k_hist.shape[0], k_hist.shape[1]
    k_eff_guess = min(topk, M)
    if idx_out is None and M > 0:
        idx_out = _new(stream, torch.empty, (n_a, H, k_eff_guess), dtype=torch.int32, device=q.device)
    if scores_out is None and want_scores and M > 0:
        scores_out = _new(stream, torch.empty, (n_a, H, M), dtype=torch.float32, device=q.device)
    ws, wsb = _ws(lib.cast_route_kv_workspace_bytes(n_a, S, H, dh, M, Bv), q.device, workspace, stream)
    k_eff = ctypes.c_int(-1)
    _check(lib.cast_route_kv(_ptr(q), _ptr(k_hist), n_a, S, H, dh, M, Bv, topk, scale,
                             _ptr(scores_out), _ptr(idx_out), ctypes.byref(k_eff), _ptr(ws), wsb,
                             _stream(stream)))
    return idx_out, k_eff.value, scores_out


def cast_coupled_params_default(**overrides) -> CoupledParams:
    p = CoupledParams()
    load().cast_coupled_params_default(ctypes.byref(p))
    for k, v in overrides.items():
        setattr(p, k, v)
    return p


def cast_route_coupled_workspace_bytes(n_a, S, H, dh, M, Bv) -> int:
    return load().cast_route_coupled_workspace_bytes(n_a, S, H, dh, M, Bv)


def cast_wo_gram(w_o, H: int, dh: int, gram_out=None, stream=None):
    """Gram matrices fp32 [H, dh, dh] of the head slices of w_o bf16 [D, D] (device)."""
    import torch
    lib = load()
    D = w_o.shape[0]
    if gram_out is None:
        gram_out = _new(stream, torch.empty, (H, dh, dh), dtype=torch.float32, device=w_o.device)
    _check(lib.cast_wo_gram(_ptr(w_o), D, H, dh, _ptr(gram_out), _stream(stream)))
    return gram_out


def cast_route_coupled(q, k_hist, v_hist, gram, anchors, n_frames: int, topk: int,
                       scale: float, params: CoupledParams | None = None, u_out=None,
                       idx_out=None, workspace=None, stream=None, want_u: bool = False):
    """Reconstruction-coupled routing.  q bf16 [n_a, S, H, dh]; k_hist, v_hist bf16
    [M, Bv, H, dh]; gram fp32 [H, dh, dh] (device); `anchors` the host frame index
    of each row of q.  Returns (idx int32 [n_a, H, k_eff], k_eff, u fp32 [n_a, H, M]
    or None)."""
    import torch
    lib = load()
    if params is None:
        params = cast_coupled_params_default()
    n_a, S, H, dh = q.shape
    M, Bv = k_hist.shape[0], k_hist.shape[1]
    if idx_out is None and M > 0:
        idx_out = _new(stream, torch.empty, (n_a, H, min(topk, M)), dtype=torch.int32, device=q.device)
    if u_out is None and want_u and M > 0:
        u_out = _new(stream, torch.empty, (n_a, H, M), dtype=torch.float32, device=q.device)
    anc = [int(a) for a in anchors]
    arr = (ctypes.c_int * max(len(anc), 1))(*anc)
    ws, wsb = _ws(lib.cast_route_coupled_workspace_bytes(n_a, S, H, dh, M, Bv), q.device, workspace, stream)
    k_eff = ctypes.c_int(-1)
    _check(lib.cast_route_coupled(_ptr(q), _ptr(k_hist), _ptr(v_hist), _ptr(gram), arr, n_a,
                                  n_frames, S, H, dh, M, Bv, topk, scale, ctypes.byref(params),
                                  _ptr(u_out), _ptr(idx_out), ctypes.byref(k_eff), _ptr(ws), wsb,
                                  _stream(stream)))
    return idx_out, k_eff.value, u_out


def cast_select_params_default(**overrides) -> SelectParams:
    p = SelectParams()
    load().cast_select_params_default(ctypes.byref(p))
    for k, v in overrides.items():
        setattr(p, k, v)
    return p


def cast_frame_select_workspace_bytes(n_cur: int, S: int, D: int) -> int:
    return load().cast_frame_select_workspace_bytes(n_cur, S, D)


def cast_frame_select(delta_cam, delta_act, anchors_prev, k_f: int, ages,
                      params: SelectParams | None = None, n_cur: int | None = None,
                      r_out=None, score_out=None, anchors_out=None, workspace=None, stream=None):
    """Control-aware frame selection.  delta_cam / delta_act: device [n_cur, S, D]
    (fp32 or bf16, the same dtype) or None; `anchors_prev` the host anchors the
    block ran with; `ages` device int32 [n_cur], updated in place.  Returns
    anchors_out (device int32 [k_f], ascending)."""
    import torch
    lib = load()
    if params is None:
        params = cast_select_params_default()
    given = [d for d in (delta_cam, delta_act) if d is not None]
    if given:
        n_cur, S, D = given[0].shape[0], given[0].shape[1], given[0].shape[2]
        dtype = 0 if given[0].dtype == torch.float32 else 1
        device = given[0].device
    else:
        n_cur, S, D, dtype, device = int(n_cur if n_cur is not None else ages.shape[0]), 1, 1, 0, ages.device
    if anchors_out is None:
        anchors_out = _new(stream, torch.empty, k_f, dtype=torch.int32, device=device)
    anc = [int(a) for a in anchors_prev]
    arr = (ctypes.c_int * max(len(anc), 1))(*anc)
    nb = lib.cast_frame_select_workspace_bytes(n_cur, S, D) if given else 0
    ws, wsb = _ws(nb, device, workspace, stream)
    _check(lib.cast_frame_select(_ptr(delta_cam), _ptr(delta_act), dtype, n_cur, S, D, arr,
                                 len(anc), k_f, ctypes.byref(params), _ptr(ages), _ptr(r_out),
                                 _ptr(score_out), _ptr(anchors_out), _ptr(ws), wsb,
                                 _stream(stream)))
    return anchors_out


def cast_diag_params_default(band_edges=None, **overrides) -> DiagParams:
    p = DiagParams()
    load().cast_diag_params_default(ctypes.byref(p))
    for k, v in overrides.items():
        setattr(p, k, v)
    if band_edges is not None:
        p.n_bands = len(band_edges) - 1
        for k, e in enumerate(band_edges):
            p.band_edges[k] = float(e)
    return p


def cast_spectral_diagnostics_workspace_bytes(n_frames, Hg, Wg, D, params: DiagParams) -> int:
    return load().cast_spectral_diagnostics_workspace_bytes(n_frames, Hg, Wg, D, ctypes.byref(params))


def cast_spectral_diagnostics(ref, approx, anchors, params: DiagParams | None = None, theta=None,
                              want_corrections: bool = False, workspace=None, stream=None):
    """Spectral diagnostics of the skipped frames.  ref, approx fp32 [n_frames, Hg,
    Wg, D] (device); theta: PAR's theta_out for the same anchors and tiling, or None.
    Returns dict(nrmse [n_frames], bands [n_frames, n_bands], phase_err [n_frames]
    or None, r_phase, r_mag [n_frames, Hg, Wg, D] or None)."""
    import torch
    lib = load()
    if params is None:
        params = cast_diag_params_default()
    n_frames, Hg, Wg, D = ref.shape
    dev = ref.device
    nrmse = _new(stream, torch.zeros, n_frames, dtype=torch.float32, device=dev)
    bands = _new(stream, torch.zeros, (n_frames, params.n_bands), dtype=torch.float32, device=dev)
    perr = _new(stream, torch.zeros, n_frames, dtype=torch.float32, device=dev) if theta is not None else None
    rp = _new(stream, torch.zeros_like, ref) if want_corrections else None
    rm = _new(stream, torch.zeros_like, ref) if want_corrections else None
    anc = [int(a) for a in anchors]
    arr = (ctypes.c_int * max(len(anc), 1))(*anc)
    nb = lib.cast_spectral_diagnostics_workspace_bytes(n_frames, Hg, Wg, D, ctypes.byref(params))
    ws, wsb = _ws(nb, dev, workspace, stream)
    _check(lib.cast_spectral_diagnostics(_ptr(ref), _ptr(approx), _ptr(theta), arr, len(anc),
                                         n_frames, Hg, Wg, D, ctypes.byref(params), _ptr(nrmse),
                                         _ptr(bands), _ptr(perr), _ptr(rp), _ptr(rm), _ptr(ws), wsb,
                                         _stream(stream)))
    return {"nrmse": nrmse, "bands": bands, "phase_err": perr, "r_phase": rp, "r_mag": rm}


def cast_phase_progress(ref, anchors, params: DiagParams | None = None, p_out=None, stream=None):
    """Phase progress of every coefficient over the interior frames of each anchor
    pair.  ref fp32 [n_frames, Hg, Wg, D] (device).  Returns p fp32 [n_frames,
    n_tiles, tile_h * (tile_w // 2 + 1), D]; entries the call does not write keep
    p_out's values (NaN when p_out is None)."""
    import torch
    lib = load()
    if params is None:
        params = cast_diag_params_default()
    n_frames, Hg, Wg, D = ref.shape
    nt = -(-Hg // params.tile_h) * -(-Wg // params.tile_w)
    if p_out is None:
        p_out = _new(stream, torch.full, (n_frames, nt, params.tile_h * (params.tile_w // 2 + 1), D),
                     float("nan"), dtype=torch.float32, device=ref.device)
    anc = [int(a) for a in anchors]
    arr = (ctypes.c_int * max(len(anc), 1))(*anc)
    _check(lib.cast_phase_progress(_ptr(ref), arr, len(anc), n_frames, Hg, Wg, D,
                                   ctypes.byref(params), _ptr(p_out), _stream(stream)))
    return p_out


def cast_anchor_attn_workspace_bytes(n_a, S, H, dh, k_eff, n0, Bv) -> int:
    return load().cast_anchor_attn_workspace_bytes(n_a, S, H, dh, k_eff, n0, Bv)


def cast_anchor_attn(q, k_hist, v_hist, idx, k_eff: int, scale: float, k_cur=None, v_cur=None,
                     out=None, lse_out=None, want_lse: bool = False, workspace=None,
                     split: bool = True, stream=None):
    """Routed block-sparse attention of the anchor frames; returns (out bf16, lse or None).
    split=True uses `workspace` (allocated here when None) to split the units of a
    last partial round along the keys; split=False runs every unit whole."""
    import torch
    lib = load()
    n_a, S, H, dh = q.shape
    M, Bv = k_hist.shape[0], k_hist.shape[1]
    n0 = 0 if k_cur is None else k_cur.shape[0]
    if out is None:
        out = _new(stream, torch.empty_like, q)
    if lse_out is None and want_lse:
        lse_out = _new(stream, torch.empty, (n_a, H, S), dtype=torch.float32, device=q.device)
    ws, wsb = None, 0
    if split:
        ws, wsb = _ws(lib.cast_anchor_attn_workspace_bytes(n_a, S, H, dh, k_eff, n0, Bv), q.device,
                      workspace, stream)
    _check(lib.cast_anchor_attn(_ptr(q), _ptr(k_hist), _ptr(v_hist), _ptr(idx), k_eff,
                                _ptr(k_cur), _ptr(v_cur), n0, n_a, S, H, dh, M, Bv, scale,
                                _ptr(out), _ptr(lse_out), _ptr(ws), wsb, _stream(stream)))
    return out, lse_out


def cast_par_reconstruct(resid, anchors, params: ParParams | None = None, out=None,
                         theta_out=None, gate_out=None, conf_out=None, workspace=None,
                         stream=None):
    """PAR over resid fp32 [n_frames, Hg, Wg, D] (device) with host `anchors`.
    Writes (or accumulates into) the skipped-frame slots of `out` (default: a new
    zero tensor) and returns it."""
    import torch
    lib = load()
    if params is None:
        params = cast_par_params_default()
    n_frames, Hg, Wg, D = resid.shape
    anc = [int(a) for a in anchors]
    arr = (ctypes.c_int * max(len(anc), 1))(*anc)
    if out is None:
        out = _new(stream, torch.zeros_like, resid)
    nbytes = lib.cast_par_workspace_bytes(n_frames, len(anc), Hg, Wg, D, ctypes.byref(params))
    ws, wsb = _ws(nbytes, resid.device, workspace, stream)
    _check(lib.cast_par_reconstruct(_ptr(resid), arr, len(anc), n_frames, Hg, Wg, D,
                                    ctypes.byref(params), _ptr(out), _ptr(theta_out),
                                    _ptr(gate_out), _ptr(conf_out), _ptr(ws), wsb,
                                    _stream(stream)))
    return out


def cast_par_reconstruct_noalloc(resid, anchors, params: ParParams | None = None, out=None,
                                 theta_out=None, gate_out=None, conf_out=None, stream=None):
    """cast_par_reconstruct with the library's static per-GPU scratch instead of a
    workspace (no device allocation in the call; `out` must be given)."""
    lib = load()
    if params is None:
        params = cast_par_params_default()
    n_frames, Hg, Wg, D = resid.shape
    anc = [int(a) for a in anchors]
    arr = (ctypes.c_int * max(len(anc), 1))(*anc)
    _check(lib.cast_par_reconstruct_noalloc(_ptr(resid), arr, len(anc), n_frames, Hg, Wg, D,
                                            ctypes.byref(params), _ptr(out), _ptr(theta_out),
                                            _ptr(gate_out), _ptr(conf_out), _stream(stream)))
    return out


def cast_par_static_scratch_bytes() -> int:
    return load().cast_par_static_scratch_bytes()


def par_debug_shapes(n_anchor, Hg, Wg, params: ParParams):
    """Shapes of the optional theta/gate ([pairs, tiles, bins]) and conf ([pairs, tiles])."""
    nt = -(-Hg // params.tile_h) * -(-Wg // params.tile_w)
    return (n_anchor - 1, nt, params.tile_h * (params.tile_w // 2 + 1)), (n_anchor - 1, nt)


# ---------------------------------------------------------------------------
# Cached history: rotary positions, paged append, page read, paged attention
# ---------------------------------------------------------------------------

ROPE_SCALING = {"none": 0, "linear": 1, "parts": 2}


def _bad(msg: str):
    raise CastError(2, msg)                        # CAST_ERR_SHAPE, before the library is asked


_INT_MAX = 0x7fffffff             # ctypes takes the low bits of what a C int does not hold


def _ints(what: str, *values):
    """Refuse sizes that a C int does not hold."""
    for v in values:
        if not 0 <= v <= _INT_MAX:
            _bad(f"{what} must be at least 0 and below 2^31, got {', '.join(str(x) for x in values)}")


def _want(name: str, t, dtypes, device=None, dense: bool = True):
    """The binding's checks of a tensor the C ABI sees as a bare pointer."""
    if t.dtype not in dtypes:
        _bad(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    if device is not None and t.device != device:
        _bad(f"{name} is on {t.device}, expected {device}")
    if dense and not t.is_contiguous():
        _bad(f"{name} must be contiguous")
    return t


def _rows(name, t, heads, dh, n, device):
    """Token stride of bf16 [n, heads, dh] with dense heads."""
    if t.dtype != _torch.bfloat16:
        _bad(f"{name} must be torch.bfloat16, got {t.dtype}")
    if t.device != device:
        _bad(f"{name} is on {t.device}, expected {device}")
    if t.shape != (n, heads, dh):
        _bad(f"{name} must be [{n}, {heads}, {dh}], got {list(t.shape)}")
    s = t.stride()
    if s[2] != 1 or (s[1] != dh and heads > 1):
        _bad(f"{name} must have dense heads")
    return s[0] if n > 1 else heads * dh


def _same(name, t, like, dtype):
    """A dense output of the shape and device of `like`."""
    if t.dtype != dtype or t.shape != like.shape or t.device != like.device or not t.is_contiguous():
        _bad(f"{name} must be a contiguous {dtype} {list(like.shape)} on {like.device}, got {t.dtype} "
             f"{list(t.shape)} on {t.device}")


def _current_raw_stream(torch):
    """Function of a device's index that gives the current stream's handle.  Small calls are bound by
    the host, so it is torch's own raw one (not public) where there is one."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw if raw is not None else lambda index: torch.cuda.current_stream(index).cuda_stream


def _on(device, stream):
    """The stream's handle, after checking that `device` is current (kernels run there)."""
    index = device.index
    if index is None or device.type != "cuda":
        _bad(f"tensors must be on a GPU, got {device}")
    if index != _torch.cuda.current_device():
        _bad(f"tensors are on {device}, the current device is cuda:{_torch.cuda.current_device()}")
    if stream is not None and stream.device_index != index:
        _bad(f"tensors are on {device}, the stream on cuda:{stream.device_index}")
    return _raw_stream(index) if stream is None else stream.cuda_stream


def cast_rope_frequencies(axis_dims, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                          orig_len: float = 0.0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """Host tables of a rotation: (turns float64 [rot/2], axis uint8 [rot/2]), CPU tensors."""
    import torch
    lib = load()
    dims = [int(d) for d in axis_dims]
    if scaling not in ROPE_SCALING:
        _bad(f"scaling must be one of {sorted(ROPE_SCALING)}, got {scaling!r}")
    n = max(min(sum(max(d, 0) for d in dims), 128) // 2, 1)      # (more are refused)
    turns = torch.zeros(n, dtype=torch.float64)
    axis = torch.zeros(n, dtype=torch.uint8)
    arr = (ctypes.c_int * max(len(dims), 1))(*(min(max(d, -1), 130) for d in dims))
    _check(lib.cast_rope_frequencies(arr, len(dims), base, ROPE_SCALING[scaling], factor, orig_len, beta_fast,
                                     beta_slow, _ptr(turns), _ptr(axis)))
    return turns, axis


class RopeParams:
    """cast_rope_params_t with its device tables (kept by a program once per model)."""

    def __init__(self, turns, axis, n_axes: int = 1, interleaved: bool = False, amplitude: float = 1.0):
        import torch
        _want("turns", turns, (torch.float64,))
        if turns.dim() != 1:
            _bad("turns must have one dimension")
        if axis is not None:
            _want("axis", axis, (torch.uint8,), turns.device)
            if axis.numel() != turns.numel():
                _bad("axis must have one entry for each of turns")
        self.turns, self.axis, self.n_axes, self.device = turns, axis, int(n_axes), turns.device
        self.struct = RopeStruct(2 * turns.numel(), int(bool(interleaved)), int(n_axes), amplitude, _ptr(turns),
                                 _ptr(axis))
        self.ref = ctypes.byref(self.struct)


def cast_rope_params_init(rot_dim: int, base: float = 10000.0, interleaved: bool = False, axes=None,
                          scaling: str = "none", factor: float = 1.0, orig_len: float = 0.0,
                          beta_fast: float = 32.0, beta_slow: float = 1.0, amplitude: float = 1.0,
                          device=None) -> RopeParams:
    """The rotation of the first rot_dim channels of a head, its tables on `device` (default:
    the current one).  axes: channels of each position component (default: one component)."""
    import torch
    dims = [int(rot_dim)] if axes is None else [int(d) for d in axes]
    if sum(dims) != rot_dim:
        _bad(f"axes {dims} do not add up to rot_dim {rot_dim}")
    turns, axis = cast_rope_frequencies(dims, base, scaling, factor, orig_len, beta_fast, beta_slow)
    if device is None:
        device = torch.device("cuda", torch.cuda.current_device())
    return RopeParams(turns.to(device), axis.to(device), len(dims), interleaved, amplitude)


def _pos(pos, n, rope, device):
    if pos.dtype != _torch.int32 or pos.device != device or not pos.is_contiguous():
        _bad(f"pos must be a contiguous torch.int32 tensor on {device}, got {pos.dtype} on {pos.device}")
    shape = pos.shape
    if shape != (n, rope.n_axes) and (rope.n_axes != 1 or shape != (n,)):
        _bad(f"pos must be [{n}, {rope.n_axes}], got {list(shape)}")
    return pos.data_ptr()


def cast_rope(x, pos, rope: RopeParams, transpose: bool = False, out=None, stream=None):
    """Rotary positions.  x [n, H, dh] fp32 or bf16 (device, any token and head strides); pos
    int32 [n, n_axes] (or [n]).  `out` may be x itself.  transpose: turn the other way (the
    gradient of the rotation).  Returns out."""
    lib = _lib or load()
    dtype, device, shape, xs = x.dtype, x.device, x.shape, x.stride()
    if dtype != _torch.bfloat16 and dtype != _torch.float32:
        _bad(f"x must be torch.float32 or torch.bfloat16, got {dtype}")
    if len(shape) != 3:
        _bad(f"x must be [n, H, dh], got {list(shape)}")
    n, H, dh = shape
    if n > _INT_MAX or H > _INT_MAX:
        _ints("tokens and heads", n, H)
    if out is None:
        out = _new(stream, _torch.empty_like, x, memory_format=_torch.contiguous_format)
        os_ = (H * dh, dh, 1)
    else:
        if out.dtype != dtype or out.device != device or out.shape != shape:
            _bad(f"out must be {dtype} {list(shape)} on {device}, got {out.dtype} {list(out.shape)} on {out.device}")
        os_ = out.stride()
    if (xs[2] != 1 or os_[2] != 1) and n > 0:
        _bad("the channels of x and out must be dense")
    if rope.device != device:
        _bad(f"the rotation's tables are on {rope.device}, x on {device}")
    if n < 2 or H < 2:                                 # torch gives any stride to a dimension of one
        fix = lambda s: (s[0] if n > 1 else max(s[0], H * dh), s[1] if H > 1 else dh)  # noqa: E731
        xs, os_ = fix(xs), fix(os_)
    pp = _pos(pos, n, rope, device)
    st = lib.cast_rope(x.data_ptr(), 1 if dtype == _torch.bfloat16 else 0, n, H, dh, xs[0], xs[1], pp, rope.ref,
                       1 if transpose else 0, out.data_ptr(), os_[0], os_[1], _on(device, stream))
    if st:
        _check(st)
    return out


class KvCache:
    """cast_kv_cache_t over tensors k, v [pages, page, H, dh]: bf16, or uint8 / float8_e4m3fn
    codes with exponent bytes k_exp, v_exp uint8 [pages, H]."""

    def __init__(self, k, v, k_exp=None, v_exp=None):
        import torch
        if k.dim() != 4 or v.shape != k.shape:
            _bad(f"k and v must be [pages, page, H, dh] alike, got {list(k.shape)} and {list(v.shape)}")
        _ints("pages, tokens of a page and heads", *k.shape[:3])
        codes = k.dtype != torch.bfloat16
        _want("k", k, (torch.uint8, torch.float8_e4m3fn) if codes else (torch.bfloat16,))
        _want("v", v, (k.dtype,), k.device)
        self.k, self.v, self.k_exp, self.v_exp, self.device = k, v, k_exp, v_exp, k.device
        self.pages, self.page, self.H, self.dh = k.shape
        if codes:
            for name, e in (("k_exp", k_exp), ("v_exp", v_exp)):
                if e is None:
                    _bad(f"an 8-bit cache needs {name}")
                _want(name, e, (torch.uint8,), k.device)
                if tuple(e.shape) != (self.pages, self.H):
                    _bad(f"{name} must be [{self.pages}, {self.H}], got {list(e.shape)}")
        elif k_exp is not None or v_exp is not None:
            _bad("a bf16 cache has no exponents")
        self.struct = KvCacheStruct(_ptr(k), _ptr(v), _ptr(k_exp), _ptr(v_exp), 2 if codes else 1, self.pages,
                                    self.page, self.H, self.dh)
        self.ref = ctypes.byref(self.struct)


def cast_kv_cache_alloc(pages: int, page: int, H: int, dh: int, dtype=None, device=None) -> KvCache:
    """A zeroed KvCache: dtype torch.bfloat16 (default) or torch.float8_e4m3fn."""
    import torch
    dtype = torch.bfloat16 if dtype is None else dtype
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    if dtype == torch.bfloat16:
        mk = lambda: torch.zeros((pages, page, H, dh), dtype=dtype, device=device)  # noqa: E731
        return KvCache(mk(), mk())
    if dtype != torch.float8_e4m3fn:
        _bad(f"a cache is bfloat16 or float8_e4m3fn, not {dtype}")
    mk = lambda *s: torch.zeros(s, dtype=torch.uint8, device=device)  # noqa: E731
    return KvCache(mk(pages, page, H, dh), mk(pages, page, H, dh), mk(pages, H), mk(pages, H))


class KvSeqs:
    """cast_kv_seqs_t over device int32 tensors cu [n_seq + 1], lens [n_seq] (WITH the call's
    tokens) and table [n_seq, max_pages].  The tensors may be updated in place between calls;
    the number of rows of a call is that of its tensors."""

    def __init__(self, cu, lens, table):
        import torch
        for name, t in (("cu", cu), ("lens", lens), ("table", table)):
            _want(name, t, (torch.int32,), cu.device)
        if table.dim() != 2 or lens.shape != table.shape[:1] or tuple(cu.shape) != (table.shape[0] + 1,):
            _bad(f"need cu [n_seq + 1], lens [n_seq], table [n_seq, max_pages], got {list(cu.shape)}, "
                 f"{list(lens.shape)}, {list(table.shape)}")
        _ints("sequences and pages of a sequence", *table.shape)
        self.cu, self.lens, self.table, self.device = cu, lens, table, cu.device
        self.max_pages = table.shape[1]
        self._structs = {}

    def ref(self, n_tok: int):
        r = self._structs.get(n_tok)
        if r is None:
            _ints("rows", n_tok)
            s = KvSeqsStruct(_ptr(self.cu), _ptr(self.lens), _ptr(self.table), self.table.shape[0], n_tok,
                             self.table.shape[1])
            if len(self._structs) >= 64:
                self._structs.clear()
            r = self._structs[n_tok] = ctypes.byref(s)
        return r


def cast_kv_append(cache: KvCache, seqs: KvSeqs, k, v, rope: RopeParams | None = None, pos=None, q=None,
                   q_out=None, stream=None):
    """Store k, v (bf16 [n, H, dh], heads dense, any token stride) into the cache's pages, keys
    rotated by `rope` (None: as they come) at pos (int32 [n, n_axes]; None: the token's index in
    its sequence), and rotate the queries q [n, Hq, dh].  Returns q_out, or None without q."""
    lib = _lib or load()
    n, dev, H, dh = k.shape[0], cache.device, cache.H, cache.dh
    if seqs.device != dev:
        _bad(f"the sequences are on {seqs.device}, the cache on {dev}")
    ks, vs = _rows("k", k, H, dh, n, dev), _rows("v", v, H, dh, n, dev)
    qs = hq = 0
    qp = op = rp = pp = None
    if q is not None:
        hq = q.shape[1] if q.dim() == 3 else 0
        qs = _rows("q", q, hq, dh, n, dev)
        if q_out is None:
            q_out = _new(stream, _torch.empty_like, q, memory_format=_torch.contiguous_format)
        else:
            _same("q_out", q_out, q, _torch.bfloat16)
        qp, op = q.data_ptr(), q_out.data_ptr()
    if rope is not None:
        if rope.device != dev:
            _bad(f"the rotation's tables are on {rope.device}, the cache on {dev}")
        rp = rope.ref
        if pos is not None:
            pp = _pos(pos, n, rope, dev)
    elif pos is not None:
        _bad("pos is given without a rotation")
    st = lib.cast_kv_append(cache.ref, seqs.ref(n), k.data_ptr(), ks, v.data_ptr(), vs, rp, pp, qp, qs, hq, op,
                            _on(dev, stream))
    if st:
        _check(st)
    return None if q is None else q_out


def cast_kv_read(cache: KvCache, pages, k_out=None, v_out=None, want_k: bool = True, want_v: bool = True,
                 stream=None):
    """The pages `pages` (int32 [m], device) as bf16 history blocks (k, v) [m, page, H, dh], the
    layout of cast_route_kv and cast_anchor_attn; None where not wanted."""
    lib = _lib or load()
    dev = cache.device
    m = pages.numel()
    if m > _INT_MAX:
        _ints("pages", m)
    if pages.dtype != _torch.int32 or pages.device != dev or not pages.is_contiguous():
        _bad(f"pages must be a contiguous torch.int32 tensor on {dev}, got {pages.dtype} on {pages.device}")
    shape = (m, cache.page, cache.H, cache.dh)
    for name, t in (("k_out", k_out), ("v_out", v_out)):
        if t is not None:
            _want(name, t, (_torch.bfloat16,), dev)
            if t.shape != shape:
                _bad(f"{name} must be {list(shape)}, got {list(t.shape)}")
    if k_out is None and want_k:
        k_out = _new(stream, _torch.empty, shape, dtype=_torch.bfloat16, device=dev)
    if v_out is None and want_v:
        v_out = _new(stream, _torch.empty, shape, dtype=_torch.bfloat16, device=dev)
    st = lib.cast_kv_read(cache.ref, pages.data_ptr(), m, _ptr(k_out), _ptr(v_out), _on(dev, stream))
    if st:
        _check(st)
    return k_out, v_out


def _max_len(cache, seqs, max_len):
    top = seqs.max_pages * cache.page
    return top if max_len is None else max(1, min(int(max_len), top))


def cast_kv_attn_workspace_bytes(q, cache: KvCache, seqs: KvSeqs, max_len=None, causal: bool = True,
                                 window: int = 0, sinks: int = 0) -> int:
    _ints("window and sinks", window, sinks)
    return load().cast_kv_attn_workspace_bytes(cache.ref, seqs.ref(q.shape[0]), q.shape[1],
                                               _max_len(cache, seqs, max_len), int(bool(causal)), window, sinks)


def cast_kv_attn(q, cache: KvCache, seqs: KvSeqs, scale: float, causal: bool = True, window: int = 0,
                 sinks: int = 0, max_len=None, out=None, lse_out=None, want_lse: bool = False, workspace=None,
                 split: bool = True, stream=None):
    """Attention of q (bf16 [n, Hq, dh], heads dense, any token stride) over the paged cache;
    returns (out bf16 [n, Hq, dh], lse fp32 [n, Hq] or None).  max_len: the longest length
    expected (default: what the table holds); split=True uses `workspace` (allocated here when
    None) to cut long key ranges into pieces, split=False runs every row tile whole."""
    lib = _lib or load()
    if q.dim() != 3:
        _bad(f"q must be [n, Hq, dh], got {list(q.shape)}")
    if not 0 <= window <= _INT_MAX or not 0 <= sinks <= _INT_MAX:
        _ints("window and sinks", window, sinks)
    n, hq, dh = q.shape
    dev = cache.device
    if seqs.device != dev:
        _bad(f"the sequences are on {seqs.device}, the cache on {dev}")
    qs = _rows("q", q, hq, cache.dh, n, dev)
    if out is None:
        out = _new(stream, _torch.empty_like, q, memory_format=_torch.contiguous_format)
    else:
        _same("out", out, q, _torch.bfloat16)
    lp = None
    if lse_out is not None:
        _want("lse_out", lse_out, (_torch.float32,), dev)
        if lse_out.shape != (n, hq):
            _bad(f"lse_out must be {[n, hq]}, got {list(lse_out.shape)}")
        lp = lse_out.data_ptr()
    elif want_lse:
        lse_out = _new(stream, _torch.empty, (n, hq), dtype=_torch.float32, device=dev)
        lp = lse_out.data_ptr()
    top, sref, causal = _max_len(cache, seqs, max_len), seqs.ref(n), 1 if causal else 0
    strm = _on(dev, stream)
    ws, wsb = None, 0
    if split:
        if workspace is not None:
            if workspace.device != dev or not workspace.is_contiguous():
                _bad(f"the workspace must be a contiguous tensor on {dev}, got one on {workspace.device}")
            ws, wsb = workspace.data_ptr(), workspace.nbytes
        else:
            wsb = lib.cast_kv_attn_workspace_bytes(cache.ref, sref, hq, top, causal, window, sinks)
            if wsb:
                workspace = _new(stream, _torch.empty, wsb, dtype=_torch.uint8, device=dev)
                ws = workspace.data_ptr()
    st = lib.cast_kv_attn(q.data_ptr(), qs, hq, cache.ref, sref, top, causal, window, sinks, scale, out.data_ptr(), lp,
                          ws, wsb, strm)
    if st:
        _check(st)
    return out, lse_out
