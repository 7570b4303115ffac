"""The decode step over an 8-bit cache, and a run of the cache's calls together, as a program makes them."""
import math

import pytest
import torch

import cache_common as cc
import oracle
import paper_2508_19740_amd as sp
import workload as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
C = wl.CONFIGS
CASES = {
    "c1": C["C1"].scaled(n_tokens=600, topk=50, extra_tokens=7),
    "c2": C["C2"].scaled(n_q_heads=4, n_kv_heads=4, n_tokens=2000 + 37, topk=300, needles=5, extra_tokens=5),
    "gqa4": C["C4"].scaled(batch=2, n_q_heads=8, n_kv_heads=2, n_tokens=1500 + 13, topk=200, needles=3, extra_tokens=9),
    "gqa7_lin": C["Q7-128K"].scaled(n_q_heads=14, n_kv_heads=2, n_tokens=900, topk=100, needles=2, hidden=0, extra_tokens=9),
    "odd_words": C["C2"].scaled(n_q_heads=2, n_kv_heads=1, n_tokens=1200, topk=133, code_bits=96, hidden=64, needles=2, extra_tokens=4),
}


@pytest.mark.parametrize("name,code,block", [("c1", "e4m3", 16), ("c2", "i8", 64), ("gqa4", "e4m3", 32), ("gqa7_lin", "i8", 128),
                                             ("odd_words", "e4m3", 64)])
def test_prefill_then_decode_steps(name, code, block):
    """hash_rows and cache_write of a prompt, then decode steps: codes and indices are the oracle's, the cache is the tests' own,
    attention is that of the cache's values; a dense call over the same cache, as a layer with full attention makes it."""
    cfg = CASES[name]
    b, hq, hkv, n, k = cfg.batch, cfg.n_q_heads, cfg.n_kv_heads, cfg.n_tokens, cfg.topk
    w = wl.Workload(cfg)
    kv = {"bf16": torch.bfloat16, "f32": torch.float32}[cfg.kv_dtype]
    hK, hV = w.materialize("K", "cpu"), w.materialize("V", "cpu")
    hw = w.hash_weights()
    dw = tuple(None if t is None else t.to(DEV) for t in hw)
    wt = {"bf16": torch.bfloat16, "f32": torch.float32}[cfg.weight_dtype]
    ctx = sp.Spotlight(b, hq, hkv, cfg.code_bits, cfg.hidden, cfg.max_tokens, k, kv_dtype=kv, weight_dtype=wt, device=DEV)
    cache = ctx.new_cache(cc.CODES[code], block)
    host = cc.HostCache(b, hkv, cfg.max_tokens, block, code)
    codes = torch.zeros(b, hkv, cfg.max_tokens, cfg.words, dtype=torch.int32, device=DEV)
    prompt = n - 3
    K, V = (x[:, :, :prompt].contiguous() for x in (hK, hV))
    ctx.hash_rows(K.to(DEV), *dw, 0, codes)
    ctx.cache_write(cache, K.to(DEV), V.to(DEV))
    host.write(K, V)
    want_codes = torch.zeros(codes.shape, dtype=torch.int32)
    oracle.hash_keys(hK, *hw, cfg.code_bits, 0, prompt, want_codes)
    assert torch.equal(codes.cpu(), want_codes)
    for t in range(prompt, n):
        q = w.q if t % 2 else -w.q
        sink, local = ((4, 8), (0, 1), (0, 0))[t % 3]
        K, V = (x[:, :, t:t + 1].contiguous() for x in (hK, hV))
        idx, out = ctx.decode_step_cache(q.to(DEV), K.to(DEV), V.to(DEV), cache, *dw, codes, t + 1, k, sink, local)
        host.write(K, V, t)
        widx, _ = oracle.decode_step(q, hK, hV, *hw, want_codes, t + 1, k, sink, local, 1 / math.sqrt(128))
        assert torch.equal(codes.cpu(), want_codes)
        assert torch.equal(idx.cpu(), widx)
        for x in "kv":
            assert torch.equal(getattr(cache, x).cpu().double(), host.codes[x]) and torch.equal(getattr(cache, x + "_scale").cpu().double(), host.scale[x])
        # the same step as separate calls: the same bits
        again = ctx.sparse_decode_cache(q.to(DEV), cache, idx)
        assert torch.equal(again, out)
        dense = ctx.dense_decode_cache(q.to(DEV), cache, t + 1)
        for i in range(b):
            for h in range(hq):
                kk, vv = (host.values(x)[i, h // (hq // hkv)] for x in "kv")
                at = widx[i, h].long()
                for got, rows in ((out, at), (dense, torch.arange(t + 1))):
                    want, mag, size = cc.attention(q[i, h][None], kk[rows], vv[rows], torch.ones(1, rows.numel(), dtype=torch.bool), 1 / math.sqrt(128))
                    tol = cc.tolerance(mag, size, 64 + (t + 1) // 8, 2 if kv is torch.float32 else 1, 2.0 ** -20) + cc.split_floor(vv[rows])
                    assert bool(((got[i, h].cpu().double() - want).abs() <= tol).all()), (t, i, h)
    ctx.close()


def test_against_the_step_over_an_unquantised_cache():
    """Rows that the codes hold exactly (small integers): both steps select the same tokens and attend alike."""
    b, hq, hkv, n, k = 1, 4, 2, 700, 90
    g = torch.Generator().manual_seed(3)
    K, V = (torch.randint(-7, 8, (b, hkv, n, 128), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    q = torch.randn(b, hq, 128, generator=g).to(torch.bfloat16).to(DEV)
    w = wl.Workload(C["C2"].scaled(n_q_heads=hq, n_kv_heads=hkv, n_tokens=n, topk=k, needles=0))
    dw = tuple(t.to(DEV) for t in w.hash_weights())
    ctx = sp.Spotlight(b, hq, hkv, 128, 256, n, k, device=DEV)
    cache = ctx.new_cache(torch.float8_e4m3fn, 32)
    codes = [torch.zeros(b, hkv, n, 4, dtype=torch.int32, device=DEV) for _ in range(2)]
    ctx.hash_keys(K, *dw, 0, n - 1, codes[0])
    ctx.hash_rows(K[:, :, :n - 1].contiguous(), *dw, 0, codes[1])
    ctx.cache_write(cache, K[:, :, :n - 1].contiguous(), V[:, :, :n - 1].contiguous())
    idx, out = ctx.decode_step(q, K, V, *dw, codes[0], n, k, 4, 16)
    idx8, out8 = ctx.decode_step_cache(q, K[:, :, n - 1:].contiguous(), V[:, :, n - 1:].contiguous(), cache, *dw, codes[1], n, k, 4, 16)
    assert torch.equal(codes[0], codes[1]) and torch.equal(idx, idx8)
    # both within a few roundings of the same sums: 2 x (136 roundings of scores up to 128 x 7 x 4 / 11, 64 of sums)
    assert float((out - out8).abs().max()) <= 7 * 2 * 2.0 ** -24 * (136 * 330 + 2 * 64)
    ctx.close()


def test_a_captured_step():
    """The step replayed from a graph, with eager work between the replays, equals the eager step."""
    cfg = CASES["gqa4"]
    b, hq, hkv, n, k = cfg.batch, cfg.n_q_heads, cfg.n_kv_heads, cfg.n_tokens, cfg.topk
    w = wl.Workload(cfg)
    K, V = (w.materialize(x, torch.device(DEV)) for x in "KV")
    dw = tuple(t.to(DEV) for t in w.hash_weights())
    ctx = sp.Spotlight(b, hq, hkv, cfg.code_bits, cfg.hidden, cfg.max_tokens, k, device=DEV)
    ctx.prepack_weights(*dw)
    cache = ctx.new_cache(torch.int8, 64)
    codes = torch.zeros(b, hkv, cfg.max_tokens, cfg.words, dtype=torch.int32, device=DEV)
    k0, v0 = (x[:, :, :n - 1].contiguous() for x in (K, V))
    k1, v1 = (x[:, :, n - 1:n].contiguous() for x in (K, V))
    ctx.hash_rows(k0, *dw, 0, codes)
    ctx.cache_write(cache, k0, v0)
    q = w.q.to(DEV)
    idx, out = (torch.empty(b, hq, k, dtype=torch.int32, device=DEV), torch.empty(b, hq, 128, device=DEV))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.decode_step_cache(q, k1, v1, cache, *dw, codes, n, k, 4, 64, out_idx=idx, out=out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.decode_step_cache(q, k1, v1, cache, *dw, codes, n, k, 4, 64, out_idx=idx, out=out)
    for i in range(4):
        q.copy_(torch.roll(q, 1, 1))
        idx.fill_(-1)
        out.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        a, o = idx.clone(), out.clone()
        widx, wout = ctx.decode_step_cache(q, k1, v1, cache, *dw, codes, n, k, 4, 64)
        assert torch.equal(a, widx) and torch.equal(o, wout), i
        torch.cuda.synchronize()
    ctx.close()
