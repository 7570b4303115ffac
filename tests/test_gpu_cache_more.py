"""Calls of the 8-bit cache that are large, begin anywhere, or leave something out: writes of more rows than the last-level cache holds
over blocks that are continued, hashing of rows that lie by themselves at any position and in every size class, reading K or V alone."""
import math

import pytest
import torch

import cache_common as cc
import paper_2508_19740_amd as sp
import workload as wl

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("code,kv,block", [("e4m3", "bf16", 16), ("i8", "bf16", 64), ("i8", "f32", 32), ("e4m3", "f32", 128)])
def test_large_writes_equal_small_ones(code, kv, block):
    """Over 256 MB of rows in one call, with positions and counts of each sequence, rows before them in the first block, infinities
    and NaN: the same bytes as one call a sequence, which are written by the kernel that is tested against the definition."""
    b, hkv, n = 4, 4, 33001 if kv == "bf16" else 16501
    cap = n + 300
    assert 2 * b * hkv * n * cc.D * (2 if kv == "bf16" else 4) >= 256 << 20 > 2 * hkv * n * cc.D * (2 if kv == "bf16" else 4)
    g = torch.Generator(device=DEV).manual_seed(5)
    rows = [(torch.randn(b, hkv, n, cc.D, generator=g, device=DEV) * torch.exp(torch.randn(b, hkv, n, 1, generator=g, device=DEV))).to(cc.KV[kv]) for _ in "kv"]
    for i, x in enumerate(rows):
        x[0, 1, 2, 3], x[1, 0, n // 2, 5], x[3, 3, n - 1, 7] = math.inf, math.nan, -math.inf
        x[2, i, 5:40] *= 1000.0
    ctx = sp.Spotlight(b, hkv, hkv, 128, 256, cap, 1, kv_dtype=cc.KV[kv], device=DEV)
    one = sp.Spotlight(1, hkv, hkv, 128, 256, cap, 1, kv_dtype=cc.KV[kv], device=DEV)
    cache = ctx.new_cache(cc.CODES[code], block)
    # rows from before, of all sizes: some blocks' scales grow, some are kept
    before = [(torch.randn(b, hkv, 290, cc.D, generator=g, device=DEV) * torch.exp(3 * torch.randn(b, hkv, 290, 1, generator=g, device=DEV))).to(cc.KV[kv]) for _ in "kv"]
    ctx.cache_write(cache, *before)
    single = []
    for i in range(b):
        single.append(sp.Cache(*(getattr(cache, x)[i:i + 1].clone() for x in ("k", "v", "k_scale", "v_scale")), block))
    first = torch.tensor([7, block, 290 - block // 2, 299], dtype=torch.int32, device=DEV)
    count = torch.tensor([n, n - 1234, n, n + 99], dtype=torch.int32, device=DEV)
    ctx.cache_write(cache, *rows, 0, first, count)
    for i in range(b):
        one.cache_write(single[i], *(x[i:i + 1].contiguous() for x in rows), 0, first[i:i + 1].contiguous(), count[i:i + 1].contiguous())
        for x in ("k", "v"):
            assert torch.equal(getattr(cache, x)[i].view(torch.uint8), getattr(single[i], x)[0].view(torch.uint8)), (i, x)
            a, c = getattr(cache, x + "_scale")[i], getattr(single[i], x + "_scale")[0]
            assert torch.equal(torch.nan_to_num(a, nan=-1.0), torch.nan_to_num(c, nan=-1.0)), (i, x)
    ctx.close()
    one.close()


HASH = [  # batch, key-value heads, rows, t0, room behind, hidden, code bits, kv
    (1, 1, 1, 5, 0, 256, 128, "bf16"),
    (3, 2, 1, 1000, 7, 0, 128, "f32"),
    (1, 3, 5, 77, 3, 256, 128, "bf16"),
    (2, 2, 40, 31, 0, 64, 96, "bf16"),
    (1, 8, 700, 33, 12, 256, 128, "f32"),
    (1, 4, 3001, 4097, 64, 0, 256, "bf16"),
    (2, 4, 9001, 555, 1, 256, 128, "bf16"),                                       # enough for two passes
    (1, 2, 33003, 1, 70, 512, 128, "bf16"),
    (1, 2, 40000, 70001, 3, 256, 64, "bf16"),
]


@pytest.mark.parametrize("b,hkv,n,t0,behind,hidden,bits,kv", HASH)
def test_hash_rows_at_any_position(b, hkv, n, t0, behind, hidden, bits, kv):
    """The codes of hash_keys for the same rows in the whole cache, and no others touched."""
    cap = t0 + n + behind
    cfg = wl.CONFIGS["C2"].scaled(batch=b, n_q_heads=hkv, n_kv_heads=hkv, n_tokens=64, topk=1, needles=0, hidden=hidden, code_bits=bits)
    weights = tuple(None if t is None else t.to(DEV) for t in wl.Workload(cfg).hash_weights())
    wt = {"bf16": torch.bfloat16, "f32": torch.float32}[cfg.weight_dtype]
    ctx = sp.Spotlight(b, hkv, hkv, bits, hidden, cap, 1, kv_dtype=cc.KV[kv], weight_dtype=wt, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(n)
    K = torch.randn(b, hkv, cap, cc.D, generator=g, device=DEV).to(cc.KV[kv])
    want = torch.full((b, hkv, cap, bits // 32), -7, dtype=torch.int32, device=DEV)
    got = want.clone()
    ctx.hash_keys(K, *weights, t0, n, want)
    rows = K[:, :, t0:t0 + n].contiguous()
    ctx.hash_rows(rows, *weights, t0, got)
    assert torch.equal(got, want)
    assert bool((got[:, :, :t0] == -7).all()) and bool((got[:, :, t0 + n:] == -7).all())
    # in parts, as a long prompt arrives
    part = torch.full_like(want, -7)
    for a, e in ((0, n // 3), (n // 3, n // 3 + 1), (n // 3 + 1, n)):
        if e > a:
            ctx.hash_rows(rows[:, :, a:e].contiguous(), *weights, t0 + a, part)
    assert torch.equal(part[:, :, t0:t0 + n], want[:, :, t0:t0 + n])
    ctx.close()


@pytest.mark.parametrize("kv", ["bf16", "f32"])
def test_reading_keys_or_values_alone(kv):
    ctx = sp.Spotlight(2, 3, 3, 128, 256, 100, 1, kv_dtype=cc.KV[kv], device=DEV)
    cache = cc.random_cache(2, 3, 100, 32, "i8", 3).device()
    K, V = ctx.cache_read(cache, 50, 20)
    for skip in (0, 1):
        args = {"K": False} if skip == 0 else {"V": False}
        got = ctx.cache_read(cache, 50, 20, **args)
        assert got[skip] is None and torch.equal(got[1 - skip], (K, V)[1 - skip])
    out = torch.full_like(V, 9.0)
    k, v = ctx.cache_read(cache, 50, 20, K=False, V=out)
    assert k is None and v is out and torch.equal(out, V)
    k, v = ctx.cache_read(cache, 50, 20, V=out.fill_(9.0))
    assert torch.equal(k, K) and v is out and torch.equal(out, V)
    with pytest.raises(sp.SpotlightError) as e:
        ctx.cache_read(cache, 50, 20, K=False, V=False)
    assert e.value.rc == sp.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        ctx.cache_read(cache, 50, 20, K=False, V=out[:, :, :49])
    ctx.close()


def test_two_graphs_and_eager_calls_on_one_context():
    """Small calls of different group sizes, whose last workgroups join the parts, captured into two graphs that share a context's
    workspace and counters, replayed in turn with eager calls of other sizes between: every result is the eager one."""
    n = 4000
    host = cc.random_cache(2, 2, n, 64, "e4m3", 17)
    ctx, cache = sp.Spotlight(2, 4, 2, 128, 256, n, 600, device=DEV), host.device()
    g = torch.Generator().manual_seed(3)
    q = torch.randn(2, 4, 1, cc.D, generator=g).to(torch.bfloat16).to(DEV)
    lens = torch.tensor([n, 700], dtype=torch.int32, device=DEV)
    idx = torch.randint(0, n, (2, 4, 600), generator=g, dtype=torch.int32).to(DEV)
    calls = [lambda: ctx.dense_decode_cache(q, cache, n, lens), lambda: ctx.sparse_decode_cache(q[:, :, 0], cache, idx[:, :, :500].contiguous()),
             lambda: ctx.dense_decode_cache(q, cache, 1500), lambda: ctx.sparse_decode_cache(q[:, :, 0], cache, idx),
             lambda: ctx.dense_decode_cache(q, cache, n)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for c in calls:
            c()
    side.synchronize()
    want = [c().clone() for c in calls]
    torch.cuda.synchronize()
    graphs = []
    for pick in ((0, 1), (2, 3, 0)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = [calls[i]() for i in pick]
        graphs.append((graph, pick, out))
    for r in range(12):
        graph, pick, out = graphs[r % 2]
        for o in out:
            o.fill_(math.nan)
        graph.replay()
        e = calls[r % 5]()
        assert torch.equal(e, want[r % 5])
        for i, o in zip(pick, out):
            assert torch.equal(o, want[i]), (r, i)
        if r % 3 == 0:
            torch.cuda.synchronize()
    ctx.close()
