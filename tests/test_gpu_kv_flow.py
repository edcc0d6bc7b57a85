"""The cached-history operators together, as a stream uses them: tokens appended and
attended step by step, an 8-bit history handed to the routed block step, captured graphs
that follow new lengths, and a stream of their own."""
import numpy as np
import pytest
import torch

from kv_util import Batch, bf16, check_attn, f64
from oracle import kv as O

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("bits", [16, 8])
def test_prompt_then_tokens(cast_lib, bits):
    """Prompts, then single tokens: every step's output against the reference over what the cache
    holds, queries and keys rotated by the same call."""
    rng = np.random.default_rng(40)
    H, g, dh, page, B = 2, 3, 64, 16, 3
    r = cast_lib.cast_rope_params_init(48)
    turns = r.turns.cpu().numpy()
    prompts = [50, 17, 33]
    b = Batch(rng, prompts, [x + 8 for x in prompts], page, H, dh, bits)
    cache, seqs = b.device(cast_lib)
    lens = np.array(prompts)
    for step in range(6):
        new = prompts if step == 0 else [1] * B
        if step:
            lens = lens + 1
        b.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        b.lens = lens.astype(np.int32)
        b.dcu.copy_(torch.from_numpy(b.cu))
        b.dlens.copy_(torch.from_numpy(b.lens))
        n = int(b.cu[-1])
        k, v, q = bf16(rng, n, H, dh), bf16(rng, n, H, dh), bf16(rng, n, H * g, dh)
        qr = cast_lib.cast_kv_append(cache, seqs, k.to(DEV), v.to(DEV), r, q=q.to(DEV))
        at = np.array([[t] for _, _, t in O.tokens(b.cu, b.lens, B)])
        kr = O.rope(f64(k), at, turns)
        held = (f64(b.dk), f64(b.dv)) if bits == 16 else tuple(O.values(c.cpu().numpy(), e.cpu().numpy()) for c, e in ((b.dk, b.dke), (b.dv, b.dve)))
        for row, s, t in O.tokens(b.cu, b.lens, B):          # the cache holds the rotated key
            kept = held[0][b.table[s, t // page], t % page]
            half = np.abs(kr[row]) * (2.0 ** -8 if bits == 16 else 2.0 ** -4)
            tiny = 1e-5 * np.abs(kr[row]).max() if bits == 16 else 2.0 ** -10 * np.abs(held[0]).max() / 256 + 1e-4
            assert np.all(np.abs(kept - kr[row]) <= half * 1.001 + tiny)
        out, lse = cast_lib.cast_kv_attn(qr, cache, seqs, 0.125, True, 20, 4, want_lse=True)
        b.n = n
        check_attn(out, lse, qr.cpu(), b, 0.125, True, 20, 4, f"step {step}", kv=held)


def test_8_bit_history_feeds_the_block_step(cast_lib):
    """Blocks of an 8-bit history, read back, give cast_route_kv and cast_anchor_attn what the
    values themselves give; pages of a bf16 cache serve as the history directly."""
    rng = np.random.default_rng(41)
    H, dh, page, M, S = 2, 64, 64, 6, 96
    b = Batch(rng, [M * page], [M * page], page, H, dh, 8, extra_pages=0)
    cache, seqs = b.device(cast_lib)
    k, v = bf16(rng, b.n, H, dh).to(DEV), bf16(rng, b.n, H, dh).to(DEV)
    cast_lib.cast_kv_append(cache, seqs, k, v)
    order = b.dtable[0].contiguous()
    kb, vb = cast_lib.cast_kv_read(cache, order)
    assert kb.shape == (M, page, H, dh)
    # half a step of e4m3, 2^-4 of the value; of subnormal codes 2^-10 * 2^e, and 2^e <= max / 224
    half = 2.0 ** -4 * np.abs(f64(k)) + 2.0 ** -10 * np.abs(f64(k)).max() / 224
    assert np.all(np.abs(f64(kb).reshape(-1, H, dh) - f64(k)) <= half)
    q = bf16(rng, 2, S, H, dh).to(DEV)
    idx, ke, _ = cast_lib.cast_route_kv(q, kb, 3, dh ** -0.5)
    out, lse = cast_lib.cast_anchor_attn(q, kb, vb, idx, ke, dh ** -0.5, want_lse=True)
    # the same attention through the cache: every (anchor, head) sees its routed pages; one head
    # and anchor at a time, the other pages taken out of the table
    for i in range(2):
        for h in range(H):
            table = torch.full((1, M), -1, dtype=torch.int32, device=DEV)
            sel = idx[i, h].long()
            table[0, sel] = order[sel]
            s2 = cast_lib.KvSeqs(torch.tensor([0, S], dtype=torch.int32, device=DEV), torch.tensor([M * page], dtype=torch.int32, device=DEV), table)
            o2, l2 = cast_lib.cast_kv_attn(q[i], cache, s2, dh ** -0.5, causal=False, want_lse=True)
            # both round probabilities and outputs to bf16: 2 (2^-8 sum p |v| + 2^-8 |o|); the mean of
            # |v| over N(0, 1) values is 0.8, over 192 of them or more below 1
            a, c = f64(out[i, :, h]), f64(o2[:, h])
            assert np.all(np.abs(a - c) <= 2 * 2.0 ** -8 * (1.0 + np.abs(a)))
            assert np.all(np.abs(f64(lse[i, h]) - f64(l2[:, h])) <= 1e-4)
    # bf16 pages in order are the history as they lie
    c16 = cast_lib.cast_kv_cache_alloc(M, page, H, dh)
    s16 = cast_lib.KvSeqs(b.dcu, b.dlens, torch.arange(M, dtype=torch.int32, device=DEV)[None].contiguous())
    cast_lib.cast_kv_append(c16, s16, k, v)
    assert torch.equal(c16.k.view(-1, H, dh), k) and torch.equal(c16.v.view(-1, H, dh), v)
    cast_lib.cast_route_kv(q, c16.k, 3, dh ** -0.5)


@pytest.mark.parametrize("bits", [16, 8])
def test_captured_step_follows_lengths(cast_lib, bits):
    """Append and attention captured once, replayed with the lengths and inputs of later steps and
    eager work between; two captured steps with workspaces of their own."""
    rng = np.random.default_rng(42)
    H, g, dh, page, B = 2, 2, 64, 16, 4
    b = Batch(rng, [1] * B, [900, 40, 1300, 5], page, H, dh, bits)
    eager = Batch(np.random.default_rng(42), [1] * B, [900, 40, 1300, 5], page, H, dh, bits)
    cache, seqs = b.device(cast_lib)
    ec, es = eager.device(cast_lib)
    b.dlens.sub_(4), eager.dlens.sub_(4)                    # room for the steps that follow
    r = cast_lib.cast_rope_params_init(64)
    k, v, q = (bf16(rng, B, h, dh).to(DEV) for h in (H, H, H * g))
    qr = torch.empty_like(q)
    outs, wss, graphs = [], [], []
    need = cast_lib.cast_kv_attn_workspace_bytes(q, cache, seqs)
    s = torch.cuda.Stream()
    for _ in range(2):
        out, ws = torch.empty_like(q), torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                cast_lib.cast_kv_append(cache, seqs, k, v, r, q=q, q_out=qr)
                cast_lib.cast_kv_attn(qr, cache, seqs, 0.125, True, 600, 4, out=out, workspace=ws)
        torch.cuda.synchronize()
        outs.append(out), wss.append(ws), graphs.append(graph)
    for step in range(4):
        for t in (k, v, q):
            t.copy_(torch.from_numpy(rng.standard_normal(tuple(t.shape)).astype(np.float32)).to(DEV))
        b.dlens.add_(1), eager.dlens.add_(1)
        graphs[step % 2].replay()
        qe = cast_lib.cast_kv_append(ec, es, k, v, r, q=q)
        want = cast_lib.cast_kv_attn(qe, ec, es, 0.125, True, 600, 4)[0]
        torch.cuda.synchronize()
        assert torch.equal(outs[step % 2], want), step
        assert torch.equal(b.dk, eager.dk) and torch.equal(b.dv, eager.dv)


def test_calls_on_a_stream_of_their_own(cast_lib):
    rng = np.random.default_rng(43)
    b = Batch(rng, [1, 64], [300, 64], 16, 2, 64, 16)
    cache, seqs = b.device(cast_lib)
    q = bf16(rng, b.n, 4, 64)
    dq = q.to(DEV)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(dq), torch.empty(b.n, 4, device=DEV)
    cast_lib.cast_kv_attn(dq, cache, seqs, 0.125, out=out, lse_out=lse, workspace=ws, stream=s)
    s.synchronize()
    check_attn(out, lse, q, b, 0.125, True, 0, 0)


def test_tensors_of_another_device_are_refused(cast_lib):
    """A CPU tensor among GPU ones is refused before anything runs."""
    b = Batch(np.random.default_rng(44), [2], [9], 16, 1, 32, 16)
    cache, seqs = b.device(cast_lib)
    x = torch.zeros((2, 1, 32), dtype=torch.bfloat16)
    for f in (lambda: cast_lib.cast_kv_append(cache, seqs, x, x.to(DEV)), lambda: cast_lib.cast_kv_attn(x, cache, seqs, 0.1),
              lambda: cast_lib.cast_kv_read(cache, torch.zeros(1, dtype=torch.int32)),
              lambda: cast_lib.cast_kv_attn(x.to(DEV), cache, seqs, 0.1, out=x)):
        with pytest.raises(cast_lib.CastError):
            f()
