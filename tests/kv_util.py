"""Helpers of the cached-history tests: small ragged batches over a paged cache."""
import numpy as np
import torch

from oracle import kv as O


def f64(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def bf16(rng, *shape, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(torch.bfloat16)


class Batch:
    """Sequences with n new rows and lengths `lens`, pages shuffled over the cache; `spare` rows
    of the call's tensors belong to no sequence."""

    def __init__(self, rng, new, lens, page, H, dh, bits, extra_pages=2, spare=0, spread=True):
        self.new, self.page, self.H, self.dh, self.bits = list(new), page, H, dh, bits
        self.lens = np.array(lens, dtype=np.int32)
        self.cu = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        self.n = int(self.cu[-1]) + spare
        per = [max(1, -(-int(x) // page)) for x in lens]
        self.pages = sum(per) + extra_pages
        ids = rng.permutation(self.pages).astype(np.int32)
        self.table = np.full((len(lens), max(per)), -1, dtype=np.int32)
        at = 0
        for b, m in enumerate(per):
            self.table[b, :m] = ids[at:at + m]
            at += m
        shape = (self.pages, page, H, dh)
        if bits == 16:
            self.k, self.v, self.ke, self.ve = bf16(rng, *shape), bf16(rng, *shape), None, None
        else:
            # every finite code, exponents a few octaves apart
            mk = lambda: torch.from_numpy((rng.integers(0, 127, shape) + 128 * rng.integers(0, 2, shape)).astype(np.uint8))  # noqa: E731
            ex = lambda: torch.from_numpy(rng.integers(117, 121 if spread else 118, (self.pages, H)).astype(np.uint8))  # noqa: E731
            self.k, self.v, self.ke, self.ve = mk(), mk(), ex(), ex()

    def device(self, cast, dev="cuda"):
        up = lambda t: None if t is None else t.to(dev)  # noqa: E731
        self.dk, self.dv, self.dke, self.dve = up(self.k), up(self.v), up(self.ke), up(self.ve)
        self.dcu, self.dlens, self.dtable = (torch.from_numpy(a.copy()).to(dev) for a in (self.cu, self.lens, self.table))
        self.cache = cast.KvCache(self.dk, self.dv, self.dke, self.dve)
        self.seqs = cast.KvSeqs(self.dcu, self.dlens, self.dtable)
        return self.cache, self.seqs

    def host(self):
        """The cache as the oracle takes it."""
        if self.bits == 16:
            return {"k": f64(self.k), "v": f64(self.v)}
        return {"k": self.k.numpy().copy(), "v": self.v.numpy().copy(), "k_exp": self.ke.numpy().copy(),
                "v_exp": self.ve.numpy().copy()}

    def values(self):
        if self.bits == 16:
            return f64(self.k), f64(self.v)
        return O.values(self.k.numpy(), self.ke.numpy()), O.values(self.v.numpy(), self.ve.numpy())


def attn_bounds(q, kv, want, lse, mag, scale):
    """Elementwise bounds of cast_kv_attn's outputs, by arithmetic: probabilities rounded to bf16
    (half a step, 2^-8 of each: 2^-8 sum p |v|), the output rounded once (2^-8), logits summed in
    fp32 (dh roundings of 2^-24 of the largest sum of |q k|, which move every probability by that
    much relatively, twice: the numerator's and the sum's), and 2^-20 for the exponentials (a few
    fp32 steps of the exponent's argument, up to ~2^4 large) and sums."""
    dh = q.shape[-1]
    top = scale * np.abs(q).sum(-1).max() * np.nanmax(np.abs(np.where(np.isfinite(kv), kv, 0)))
    logit = dh * 2.0 ** -24 * top
    out = mag * (2.0 ** -8 + 2 * logit + 2.0 ** -20) + 2.0 ** -8 * np.abs(want) * 1.01 + 1e-30
    return out, logit + 2.0 ** -20 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0)))


def check_attn(got, got_lse, q, b, scale, causal, window, sinks, what="", kv=None):
    kvv, vv = b.values() if kv is None else kv
    want, lse, mag = O.attention(f64(q), kvv, vv, b.cu, b.lens, b.table, b.page, scale, causal, window, sinks)
    rows = int(b.cu[-1])
    ob, lb = attn_bounds(f64(q), kvv, want, lse, mag, scale)
    g, gl = f64(got)[:rows], f64(got_lse)[:rows]
    want, lse, ob, lb = want[:rows], lse[:rows], ob[:rows], lb[:rows]
    assert np.array_equal(np.isneginf(gl), np.isneginf(lse)), what
    fin = np.isfinite(lse)
    assert np.all(np.abs(gl[fin] - lse[fin]) <= lb[fin]), (what, np.abs(gl[fin] - lse[fin]).max())
    assert np.isfinite(g).all(), what
    bad = np.abs(g - want) > ob
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), (np.abs(g - want) / ob).max())
