"""The cached-history operators of this framework as measurable cases: rotary positions,
appending to a paged cache with the rotation on the way, reading pages back as bf16
blocks, and attention over the paged cache.

`run` computes a case with elementary torch operations in fp32 (angles in fp64), or,
where `own` is set, with the calls a program makes of `paper_2609_34144_amd`.  `exact`
computes the same from the definitions in fp64.

`op` of a case:
  rope     cast_rope          append   cast_kv_append (8-bit caches: and cast_kv_read, which
  read     cast_kv_read                gives the values that the codes stand for)
  attn     cast_kv_attn

A batch of sequences is ragged: sequence b owns rows cu[b] .. cu[b + 1] of the call's
tokens, which are the last of its lens[b] tokens; its token t lies in page
table[b][t // page] of the cache at row t % page.  An 8-bit cache holds e4m3 codes and
one exponent byte per (page, head): value = code * 2^(byte - 127).
"""
import math

import torch

own = False
DEV = "cuda"
TWO_PI = 2.0 * math.pi


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _rope(**kw):
    c = dict(op="rope", n=8, H=24, dh=128, rot=128, inter=False, axes="", dtype="bf16", transpose=False,
             far=100000, base=10000.0, scaling="none", factor=1.0, orig_len=0, amplitude=1.0)
    c.update(kw)
    return c


def _append(**kw):
    c = dict(op="append", seqs=64, n=64, Hq=0, H=8, dh=128, page=16, bits=16, max_len=4096,
             rot=128, inter=False, base=10000.0, scaling="none", factor=1.0, orig_len=0, amplitude=1.0)
    c.update(kw)
    return c


def _read(**kw):
    c = dict(op="read", pages=64, take=40, page=64, H=24, dh=128, bits=8)
    c.update(kw)
    return c


def _attn(**kw):
    c = dict(op="attn", seqs=1, n=1, Hq=32, H=8, dh=128, page=16, bits=16, max_len=4096, min_len=1,
             causal=True, window=0, sinks=0, ragged=True)
    c.update(kw)
    return c


def listed():
    return [
        # the smallest rotation: queries of eight streams' next tokens, far into a scaled context
        _rope(name="rope_tokens", n=8, H=24, scaling="parts", factor=8.0, orig_len=8192, amplitude=1.2),
        # queries of eight 44x80 frames, three axes (frame, row, column) over interleaved pairs
        _rope(name="rope_frames", n=28160, H=24, axes="44,42,42", inter=True, far=80),
        # one token for each of 64 streams: keys and queries rotated, 16-token pages
        _append(name="append_tokens", seqs=64, n=64, Hq=32, H=8, page=16),
        # four chunks of 30x52-token frames enter the history, whose pages are frames
        _append(name="append_frames", seqs=4, n=24960, H=12, page=1560, max_len=12480),
        # ragged prompts into an 8-bit cache of 64-token pages, half of the head rotated
        _append(name="append8_prompts", seqs=24, n=15000, H=8, page=64, bits=8, max_len=2048, rot=64),
        # a routed selection of 8x8-token blocks of an 8-bit history, for the block step
        _read(name="read8_blocks", pages=390, take=78, page=64, H=24, dh=64),
        # a whole 8-bit history of 44x80 frames as the bf16 blocks the block step reads
        _read(name="read8_frames", pages=16, take=16, page=3520, H=24),
        # decoding: 16 streams, one token each, grouped heads, 16-token pages
        _attn(name="attn_tokens", seqs=16, n=16, Hq=32, H=8, page=16, max_len=8192),
        # decoding on few long contexts in 8 bits
        _attn(name="attn8_tokens_long", seqs=4, n=4, Hq=64, H=8, page=64, bits=8, max_len=131072, min_len=65536),
        # ragged causal prompts
        _attn(name="attn_prompts", seqs=4, n=13000, Hq=24, H=24, page=16, max_len=4096),
        # one 30x52 frame against an 8-bit history: all of the frame, a window of four frames
        # before it, and the first frame kept visible
        _attn(name="attn8_frame_window", seqs=1, n=1560, Hq=12, H=12, page=1560, bits=8, max_len=24960,
              min_len=24960, causal=False, window=7800, sinks=1560),
        # chunks of prompts on long contexts, 64-wide grouped heads, causal window and four sinks
        _attn(name="attn_chunks_dh64", seqs=6, n=3000, Hq=32, H=8, dh=64, page=32, max_len=16384,
              min_len=8192, window=4096, sinks=4),
    ]


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "append", "read", "attn", "attn", "attn", "attn"])
    dh = rng.choice([32, 64, 64, 128, 128, 128])
    page = rng.choice([_logint(rng, 5, 200), 16, 32, 64, 128, rng.randint(800, 3600)])
    rot = dh if rng.random() < 0.5 else 2 * rng.randint(1, dh // 2)
    scaling = rng.choice(["none", "linear", "parts"])
    scaled = dict(scaling=scaling, factor=1.0 if scaling == "none" else rng.uniform(1.5, 16.0),
                  orig_len=rng.choice([2048, 4096, 8192]), amplitude=rng.choice([1.0, rng.uniform(0.8, 1.4)]))
    if op == "rope":
        axes = ""
        if rot >= 6 and rng.random() < 0.4:
            a = 2 * rng.randint(1, rot // 2 - 2)
            b = 2 * rng.randint(1, (rot - a) // 2 - 1)
            axes = "%d,%d,%d" % (a, b, rot - a - b)
        return _rope(n=_logint(rng, 1, 20000), H=rng.randint(1, 32), dh=dh, rot=rot, inter=rng.random() < 0.5,
                     axes=axes, dtype=rng.choice(["bf16", "fp32"]), transpose=rng.random() < 0.3,
                     far=_logint(rng, 100, 1000000), base=rng.choice([10000.0, 500000.0]), **scaled)
    if op == "append":
        seqs = _logint(rng, 1, 96)
        H = rng.choice([1, 2, 3, 4, 5, 8, 12])
        n = seqs + (0 if rng.random() < 0.3 else _logint(rng, 1, 16000))
        return _append(seqs=seqs, n=n, Hq=rng.choice([0, H, H * rng.randint(1, 8)]), H=H, dh=dh, page=page,
                       bits=rng.choice([8, 16]), max_len=_logint(rng, 2 * n // seqs + 64, 2 * n // seqs + 4096),
                       rot=rot, inter=rng.random() < 0.5, base=rng.choice([10000.0, 500000.0]), **scaled)
    if op == "read":
        H = rng.randint(1, 24)
        pages = max(1, min(_logint(rng, 1, 2000), 60000000 // (page * H * dh)))
        return _read(pages=pages, take=rng.randint(1, pages), page=page, H=H, dh=dh, bits=rng.choice([8, 16]))
    H = rng.choice([1, 2, 3, 4, 8, 12])
    bits, form = rng.choice([8, 16]), rng.choice(["tokens", "tokens", "prompts", "chunks"])
    if form == "tokens":
        seqs = _logint(rng, 1, 64)
        return _attn(seqs=seqs, n=seqs, Hq=H * rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]), H=H, dh=dh, page=page, bits=bits,
                     max_len=max(2, min(_logint(rng, 2, 100000), 1500000 // (seqs * H))),
                     window=0 if rng.random() < 0.6 else _logint(rng, 1, 8192), sinks=rng.choice([0, 1, 4, 77]))
    g = rng.choice([1, 1, 2, 3, 4, 6])
    if form == "prompts":
        seqs = rng.randint(1, 5)
        n = seqs + _logint(rng, 16, 1500 * seqs)
        return _attn(seqs=seqs, n=n, Hq=H * g, H=H, dh=dh, page=page, bits=bits, max_len=max(2 * n // seqs, 64),
                     causal=rng.random() < 0.8, window=0 if rng.random() < 0.5 else _logint(rng, 8, 2048),
                     sinks=rng.choice([0, 1, 4, 77]))
    seqs = rng.randint(1, 4)
    n = seqs + _logint(rng, 1, 400 * seqs)
    return _attn(seqs=seqs, n=n, Hq=H * g, H=H, dh=dh, page=page, bits=bits, max_len=_logint(rng, 2 * n, 2 * n + 12000),
                 causal=rng.random() < 0.7, window=0 if rng.random() < 0.4 else _logint(rng, 8, 8192),
                 sinks=rng.choice([0, 1, 4, 77, 800]))


# ---------------------------------------------------------------------------
# the inputs
# ---------------------------------------------------------------------------

def _lengths(c):
    """Rows per sequence and lengths, from the sizes alone: ragged, every sequence at least one row."""
    seqs, n = c["seqs"], c["n"]
    rest = n - seqs
    w = [1.0 + 0.5 * math.sin(2.1 * b + 0.3) if c.get("ragged", True) else 1.0 for b in range(seqs)]
    new = [1 + int(rest * x / sum(w)) for x in w]
    new[0] += n - sum(new)
    lo, hi = c.get("min_len", 1), c["max_len"]
    lens = []
    for b, m in enumerate(new):
        f = 0.5 + 0.5 * math.sin(1.7 * b + 1.2)
        lens.append(max(m, int(round(lo + f * (hi - lo))) if hi > lo else hi))
    return new, lens


def _codes(shape, gen):
    """e4m3 codes of values with the spread that the largest of a page leaves them."""
    x = torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32)
    return (x * 100.0).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _cache(c, pages, gen):
    shape = (pages, c["page"], c["H"], c["dh"])
    if c["bits"] == 16:
        mk = lambda: torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)  # noqa: E731
        return {"k": mk(), "v": mk(), "k_exp": None, "v_exp": None}
    e = lambda: torch.randint(118, 123, (pages, c["H"]), generator=gen, device=DEV, dtype=torch.uint8)  # noqa: E731
    return {"k": _codes(shape, gen), "v": _codes(shape, gen), "k_exp": e(), "v_exp": e()}


def _frequencies(c):
    """Revolutions per position of each rotated pair (fp64), and the axis of each."""
    dims = [int(d) for d in c["axes"].split(",")] if c.get("axes") else [c["rot"]]
    turns, axis = [], []
    for a, d in enumerate(dims):
        for j in range(d // 2):
            t = c["base"] ** (-2.0 * j / d) / TWO_PI
            if c["scaling"] == "linear":
                t /= c["factor"]
            elif c["scaling"] == "parts":
                g = min(1.0, max(0.0, (c["orig_len"] * t - 1.0) / (32.0 - 1.0)))
                t *= g + (1.0 - g) / c["factor"]
            turns.append(t)
            axis.append(a)
    return turns, axis


def prepare(case, seed):
    c = case
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 7919 + 11)
    s = {"case": c}
    if c["op"] in ("rope", "append"):
        turns, axis = _frequencies(c)
        s["turns"] = torch.tensor(turns, dtype=torch.float64, device=DEV)
        s["axis"] = torch.tensor(axis, dtype=torch.int64, device=DEV)
    if c["op"] == "rope":
        dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        s["x"] = torch.randn((c["n"], c["H"], c["dh"]), generator=gen, device=DEV, dtype=dt)
        n_axes = len(c["axes"].split(",")) if c["axes"] else 1
        s["pos"] = torch.randint(0, c["far"], (c["n"], n_axes), generator=gen, device=DEV, dtype=torch.int32)
    elif c["op"] == "read":
        s.update(_cache(c, c["pages"], gen))
        s["pages"] = torch.randperm(c["pages"], generator=gen, device=DEV)[: c["take"]].to(torch.int32)
    else:
        new, lens = _lengths(c)
        per = [-(-x // c["page"]) for x in lens]
        total = sum(per)
        ids = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
        table = torch.full((c["seqs"], max(per)), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b, m in enumerate(per):
            table[b, :m] = ids[at : at + m]
            at += m
        s["table"] = table
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s["cu"] = torch.tensor([sum(new[:b]) for b in range(len(new) + 1)], dtype=torch.int32, device=DEV)
        s["max_new"], s["max_len"] = max(new), max(lens)
        s.update(_cache(c, total, gen))
        rnd = lambda h: torch.randn((c["n"], h, c["dh"]), generator=gen, device=DEV, dtype=torch.bfloat16)  # noqa: E731
        if c["op"] == "append":
            # channels and tokens of a real projection differ in size: a spread over a few octaves
            size = torch.exp2(torch.randint(-2, 3, (c["n"], 1, 1), generator=gen, device=DEV).to(torch.bfloat16))
            s["k_new"], s["v_new"] = rnd(c["H"]) * size, rnd(c["H"]) * size
            s["q"] = rnd(c["Hq"]) if c["Hq"] else None
            s["all_pages"] = torch.arange(total, dtype=torch.int32, device=DEV)
        else:
            s["q"] = rnd(c["Hq"]) * 2.0
            s["scale"] = 1.0 / math.sqrt(c["dh"])
    if own:
        _handles(s)
    return s


def _handles(s):
    """What a program that uses the framework keeps beside its tensors."""
    import paper_2609_34144_amd as cast
    c = s["case"]
    if c["op"] in ("rope", "append"):
        s["rope"] = cast.cast_rope_params_init(
            c["rot"], base=c["base"], interleaved=c["inter"],
            axes=[int(d) for d in c["axes"].split(",")] if c.get("axes") else None,
            scaling=c["scaling"], factor=c["factor"], orig_len=c["orig_len"], beta_fast=32.0, beta_slow=1.0,
            amplitude=c["amplitude"])
    if c["op"] != "rope":
        s["cache"] = cast.KvCache(s["k"], s["v"], s["k_exp"], s["v_exp"])
    if c["op"] in ("append", "attn"):
        s["seqs"] = cast.KvSeqs(s["cu"], s["lens"], s["table"])
    if c["op"] == "attn":
        nb = cast.cast_kv_attn_workspace_bytes(s["q"], s["cache"], s["seqs"], max_len=s["max_len"],
                                               causal=c["causal"], window=c["window"], sinks=c["sinks"])
        s["workspace"] = torch.empty(max(nb, 256), dtype=torch.uint8, device=DEV)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(state):
    return {"rope": _run_rope, "append": _run_append, "read": _run_read, "attn": _run_attn}[state["case"]["op"]](state)


def _angles(s, pos):
    """cos and sin of each (token, pair), fp32: the angle reduced to a revolution in fp64."""
    turns = pos.double()[:, s["axis"]] * s["turns"]
    a = (turns - torch.round(turns)) * TWO_PI
    amp = s["case"]["amplitude"]
    return (torch.cos(a) * amp).float(), (torch.sin(a) * amp).float()


def _rotate(x, cos, sin, rot, inter, transpose=False):
    """x [n, H, dh] in fp32, its first `rot` channels turned in pairs."""
    x = x.float()
    cos, sin = cos[:, None, :], sin[:, None, :]
    if transpose:
        sin = -sin
    r = x[..., :rot]
    a, b = (r[..., 0::2], r[..., 1::2]) if inter else (r[..., : rot // 2], r[..., rot // 2 :])
    p, q = a * cos - b * sin, a * sin + b * cos
    y = torch.stack((p, q), dim=-1).flatten(-2) if inter else torch.cat((p, q), dim=-1)
    return torch.cat((y, x[..., rot:]), dim=-1)


def _run_rope(s):
    c = s["case"]
    if own:
        import paper_2609_34144_amd as cast
        return cast.cast_rope(s["x"], s["pos"], s["rope"], transpose=c["transpose"])
    cos, sin = _angles(s, s["pos"])
    return _rotate(s["x"], cos, sin, c["rot"], c["inter"], c["transpose"]).to(s["x"].dtype)


def _where(s):
    """Sequence, index in it, page and row in the page of each new token."""
    n, page = s["case"]["n"], s["case"]["page"]
    row = torch.arange(n, device=DEV)
    b = torch.searchsorted(s["cu"][1:].long(), row, right=True)
    t = s["lens"].long()[b] - (s["cu"][b + 1].long() - row)
    return b, t, s["table"][b, t // page].long(), t % page


def _run_append(s):
    c = s["case"]
    if own:
        import paper_2609_34144_amd as cast
        q = cast.cast_kv_append(s["cache"], s["seqs"], s["k_new"], s["v_new"], rope=s["rope"], q=s["q"])
        k, v = (s["k"], s["v"]) if c["bits"] == 16 else cast.cast_kv_read(s["cache"], s["all_pages"])
        return {"k": k, "v": v, "q": q}
    b, t, page, row = _where(s)
    cos, sin = _angles(s, t[:, None])
    k = _rotate(s["k_new"], cos, sin, c["rot"], c["inter"])
    q = None if s["q"] is None else _rotate(s["q"], cos, sin, c["rot"], c["inter"]).to(torch.bfloat16)
    if c["bits"] == 16:
        s["k"][page, row] = k.to(torch.bfloat16)
        s["v"][page, row] = s["v_new"]
        return {"k": s["k"], "v": s["v"], "q": q}
    # rows of each page that held earlier tokens of the sequence
    first = s["lens"].long() - (s["cu"][1:] - s["cu"][:-1]).long()
    earlier = torch.zeros(s["k"].shape[0], dtype=torch.int64, device=DEV)
    earlier[page] = (first[b] - (t - row)).clamp(min=0)
    return {"k": _store8(s["k"], s["k_exp"], k, page, row, earlier),
            "v": _store8(s["v"], s["v_exp"], s["v_new"].float(), page, row, earlier), "q": q}


def _store8(codes, exps, x, page, row, earlier):
    """The new tokens x at (page, row) as codes under their page's exponent; the values of the whole cache."""
    top = torch.zeros(exps.shape, dtype=torch.float32, device=DEV)
    top.scatter_reduce_(0, page[:, None].expand(-1, exps.shape[1]), x.abs().amax(dim=-1), "amax")
    m, e = torch.frexp(top)                                     # top = m 2^e, m in [0.5, 1)
    need = torch.where(top > 0, e - 9 + (m > 0.875).to(e.dtype), -117).clamp(min=-117) + 127
    had, touched = earlier > 0, torch.zeros_like(earlier, dtype=torch.bool)
    touched[page] = True
    old = exps.int()
    new = torch.where(touched[:, None], torch.where(had[:, None], torch.maximum(old, need.int()), need.int()), old)
    is_old = (torch.arange(codes.shape[1], device=DEV)[None, :] < earlier[:, None])[:, :, None, None]
    f = codes.view(torch.float8_e4m3fn).float()
    f = torch.where(is_old, f * torch.exp2((old - new).float())[:, None, :, None], f)
    f[page, row] = x * torch.exp2((127 - new[page]).float())[:, :, None]
    codes.copy_(f.to(torch.float8_e4m3fn).view(torch.uint8))
    exps.copy_(new.to(torch.uint8))
    return _values(codes, exps)


def _values(codes, exps):
    x = codes.view(torch.float8_e4m3fn).float() * torch.exp2(exps.float() - 127.0)[:, None, :, None]
    return x.to(torch.bfloat16)


def _run_read(s):
    c = s["case"]
    if own:
        import paper_2609_34144_amd as cast
        return cast.cast_kv_read(s["cache"], s["pages"])
    at = s["pages"].long()
    if c["bits"] == 16:
        return s["k"][at], s["v"][at]
    return _values(s["k"][at], s["k_exp"][at]), _values(s["v"][at], s["v_exp"][at])


def _run_attn(s):
    c = s["case"]
    if own:
        import paper_2609_34144_amd as cast
        return cast.cast_kv_attn(s["q"], s["cache"], s["seqs"], s["scale"], causal=c["causal"], window=c["window"],
                                 sinks=c["sinks"], max_len=s["max_len"], want_lse=True, workspace=s["workspace"])
    B, H, dh, N, L = c["seqs"], c["H"], c["dh"], s["max_new"], s["max_len"]
    g = c["Hq"] // H
    b, t, _, _ = _where(s)
    # keys and values of each sequence side by side, rows past its end repeated (and masked)
    key = torch.arange(L, device=DEV)
    at = torch.minimum(key[None, :], s["lens"].long()[:, None] - 1)
    page, row = s["table"].gather(1, at // c["page"]).long(), at % c["page"]

    def wide(name):
        x = s[name][page, row]
        if c["bits"] == 8:
            x = x.view(torch.float8_e4m3fn).float() * torch.exp2(s[name + "_exp"][page].float() - 127.0)[..., None]
        return x.float().permute(0, 2, 1, 3).contiguous()       # [B, H, L, dh]

    # queries padded to the longest sequence's rows
    i = t - (s["lens"].long()[b] - (s["cu"][b + 1] - s["cu"][b]).long())
    q = torch.zeros((B, N, H, g, dh), dtype=torch.float32, device=DEV)
    q[b, i] = s["q"].view(-1, H, g, dh).float()
    p = torch.zeros((B, N), dtype=torch.int64, device=DEV)
    p[b, i] = t
    seen = key[None, None, :] < s["lens"].long()[:, None, None]
    if c["causal"]:
        seen = seen & (key[None, None, :] <= p[:, :, None])
    if c["window"]:
        seen = seen & ((key[None, None, :] > p[:, :, None] - c["window"]) | (key < c["sinks"])[None, None, :])
    x = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(B, H, N * g, dh), wide("k").transpose(2, 3).contiguous())
    x = (x * s["scale"]).view(B, H, N, g, L).masked_fill_(~seen[:, None, :, None, :].expand(B, 1, N, 1, L), -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    x = torch.exp(x - top)
    total = x.sum(dim=-1, keepdim=True)
    o = torch.matmul(x.view(B, H, N * g, L), wide("v")).view(B, H, N, g, dh)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    lse = (top + torch.log(total))[..., 0]
    return o[b, :, i].reshape(-1, c["Hq"], dh).to(torch.bfloat16), lse[b, :, i].reshape(-1, c["Hq"])


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    c = case
    if c["op"] == "rope":
        el = c["n"] * c["H"] * c["dh"]
        return {"bytes": 2 * el * (2 if c["dtype"] == "bf16" else 4), "flops": 3 * el}
    if c["op"] == "append":
        el, qel = 2 * c["n"] * c["H"] * c["dh"], c["n"] * c["Hq"] * c["dh"]
        new, lens = _lengths(c)
        # an 8-bit pass reads the values of the whole cache back
        back = 2 * 3 * sum(-(-x // c["page"]) for x in lens) * c["page"] * c["H"] * c["dh"] if c["bits"] == 8 else 0
        return {"bytes": el * (2 + c["bits"] // 8) + 4 * qel + back, "flops": 3 * (el // 2 + qel)}
    if c["op"] == "read":
        el = 2 * c["take"] * c["page"] * c["H"] * c["dh"]
        return {"bytes": el * (c["bits"] // 8 + 2), "flops": el}
    new, lens = _lengths(c)
    pairs = keys = 0
    for m, x in zip(new, lens):
        first = x - m
        lo = max(0, first - c["window"] + 1) if c["window"] else 0
        keys += x - lo + min(c["sinks"], lo)
        for p in range(first, x):
            hi = p + 1 if c["causal"] else x
            lo = min(max(0, p - c["window"] + 1), hi) if c["window"] else 0
            pairs += hi - lo + min(c["sinks"], lo)
    return {"bytes": 2 * keys * c["H"] * c["dh"] * (c["bits"] // 8) + 4 * c["n"] * c["Hq"] * c["dh"],
            "flops": 4 * pairs * c["Hq"] * c["dh"]}


# ---------------------------------------------------------------------------
# the definitions in fp64
# ---------------------------------------------------------------------------

def _turned64(x, pos, s, transpose):
    """y = R x per (token, pair), one pair of channels at a time."""
    c = s["case"]
    y, rot = x.double().clone(), c["rot"]
    turns, axis = s["turns"].tolist(), s["axis"].tolist()
    for j in range(rot // 2):
        u, w = (2 * j, 2 * j + 1) if c["inter"] else (j, j + rot // 2)
        angle = torch.remainder(pos[:, axis[j]].double() * turns[j], 1.0) * TWO_PI
        co, si = (c["amplitude"] * torch.cos(angle))[:, None], (c["amplitude"] * torch.sin(angle))[:, None]
        si = -si if transpose else si
        a, d = x[..., u].double(), x[..., w].double()
        y[..., u], y[..., w] = a * co - d * si, a * si + d * co
    return y


def _decode64(codes):
    """e4m3: sign, four exponent bits of bias 7, three of mantissa; subnormals of 2^-9."""
    v = codes.long()
    ex, man = (v >> 3) & 15, (v & 7).double()
    mag = torch.where(ex == 0, man * 2.0 ** -9, (8.0 + man) * torch.exp2(ex.double() - 10.0))
    return torch.where(v >= 128, -mag, mag)


def _round64(x):
    """To the nearest e4m3 value, ties to the even one (|x| <= 448)."""
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.clamp(x.abs(), min=1e-30))), min=-6.0) - 3.0)
    return torch.round(x / step) * step


def _stored64(codes, exps, x, s):
    """The values of the whole 8-bit cache after the new tokens x came in, page by page."""
    val, ex, page = _decode64(codes), exps.long() - 127, s["case"]["page"]
    cu, lens, table = s["cu"].tolist(), s["lens"].tolist(), s["table"].tolist()
    for b in range(len(lens)):
        first = lens[b] - (cu[b + 1] - cu[b])
        for g in range(first // page, (lens[b] - 1) // page + 1):
            lo, hi = max(first, g * page), min(lens[b], (g + 1) * page)
            new = x[cu[b] + lo - first : cu[b] + hi - first]                # [tokens, H, dh]
            top = new.abs().amax(dim=(0, 2)).clamp(min=448.0 * 2.0 ** -117)
            need = torch.ceil(torch.log2(top / 448.0) - 1e-12).long()
            need = torch.where(448.0 * torch.exp2(need.double()) < top, need + 1, need)
            at, had = table[b][g], lo - g * page
            if had:
                e = torch.maximum(ex[at], need)
                val[at, :had] = _round64(val[at, :had] * torch.exp2((ex[at] - e).double())[None, :, None])
            else:
                e = need
            ex[at] = e
            val[at, had : had + hi - lo] = _round64(new * torch.exp2(-e.double())[None, :, None])
    return val * torch.exp2(ex.double())[:, None, :, None]


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "rope":
        return _turned64(s["x"], s["pos"], s, c["transpose"])
    if c["op"] == "read":
        at = s["pages"].long()
        if c["bits"] == 16:
            return s["k"][at].double(), s["v"][at].double()
        return tuple(_decode64(s[x][at]) * torch.exp2(s[x + "_exp"][at].double() - 127.0)[:, None, :, None] for x in ("k", "v"))
    cu, lens, page = s["cu"].tolist(), s["lens"].tolist(), c["page"]
    if c["op"] == "append":
        index = torch.cat([torch.arange(n - (cu[b + 1] - cu[b]), n, device=DEV) for b, n in enumerate(lens)])[:, None]
        k = _turned64(s["k_new"], index, s, False)
        q = None if s["q"] is None else _turned64(s["q"], index, s, False)
        if c["bits"] == 8:
            return {"k": _stored64(s["k"], s["k_exp"], k, s), "v": _stored64(s["v"], s["v_exp"], s["v_new"].double(), s), "q": q}
        kc, vc = s["k"].double(), s["v"].double()
        of = torch.cat([torch.full((cu[b + 1] - cu[b],), b, device=DEV) for b in range(len(lens))])
        at = s["table"][of, index[:, 0] // page].long()
        kc[at, index[:, 0] % page], vc[at, index[:, 0] % page] = k, s["v_new"].double()
        return {"k": kc, "v": vc, "q": q}
    g = c["Hq"] // c["H"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        t = torch.arange(n, device=DEV)
        at, row = s["table"][b].long()[t // page], t % page
        p = torch.arange(n - (cu[b + 1] - cu[b]), n, device=DEV)[:, None]
        hidden = torch.zeros((p.shape[0], n), dtype=torch.bool, device=DEV)
        if c["causal"]:
            hidden |= t[None, :] > p
        if c["window"]:
            hidden |= (t[None, :] <= p - c["window"]) & (t[None, :] >= c["sinks"])
        for h in range(c["H"]):
            if c["bits"] == 8:
                k, v = (_decode64(s[x][at, row, h]) * torch.exp2(s[x + "_exp"][at, h].double() - 127.0)[:, None] for x in ("k", "v"))
            else:
                k, v = s["k"][at, row, h].double(), s["v"][at, row, h].double()
            for j in range(h * g, (h + 1) * g):
                z = (s["q"][cu[b] : cu[b + 1], j].double() @ k.t().contiguous()) * s["scale"]
                z.masked_fill_(hidden, -math.inf)
                lse[cu[b] : cu[b + 1], j] = torch.logsumexp(z, dim=-1)
                w = torch.nan_to_num(torch.softmax(z, dim=-1), nan=0.0)
                out[cu[b] : cu[b + 1], j] = w @ v
    return out, lse
