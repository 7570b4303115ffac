"""Writing rows into the 8-bit cache and reading them back, against the tests' own 64-bit cache: every code and every scale
the same bits, and every byte that a call has no business with as it was."""
import math

import pytest
import torch

import cache_common as cc
import paper_2508_19740_amd as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ctx(b, hkv, n, kv="bf16", group=1):
    return sp.Spotlight(b, hkv * group, hkv, 128, 256, n, 1, kv_dtype=cc.KV[kv], device=DEV)


def _rows(seed, *shape, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, cc.D, generator=g) * torch.exp(spread * torch.randn(*shape, 1, generator=g))
    return x


def _bits(cache):
    return {x: getattr(cache, x).view(torch.uint8).cpu() for x in "kv"}


def _same(host, cache):
    for x in "kv":
        codes, scale = getattr(cache, x).cpu(), getattr(cache, x + "_scale").cpu()
        want = host.codes[x].float().to(cc.CODES[host.code])
        nan = torch.isnan(host.codes[x])
        assert torch.equal(codes.float()[~nan], want.float()[~nan]), x          # -0 equals 0
        assert bool(torch.isnan(codes.float()[nan]).all()), x
        assert torch.equal(torch.nan_to_num(scale, nan=-1.0), torch.nan_to_num(host.scale[x].float(), nan=-1.0)), x


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_prompt_then_tokens(block, code, kv):
    """A prompt, then single tokens and short runs behind it, each larger than the last, so that scales grow."""
    b, hkv, n = 2, 3, 3 * block + 37
    ctx, host = _ctx(b, hkv, n, kv), cc.HostCache(b, hkv, n, block, code)
    cache = ctx.new_cache(cc.CODES[code], block)
    t = 0
    for i, rows in enumerate([block + 5, 1, 1, 2, 1, block, 1, 7, 1, 1]):
        K, V = (_rows(10 * i + j, b, hkv, rows).mul(1.0 + 0.7 * i).to(cc.KV[kv]) for j in (1, 2))
        ctx.cache_write(cache, K.to(DEV), V.to(DEV), t)
        host.write(K, V, t)
        _same(host, cache)
        t += rows
    assert t < n
    K, V = ctx.cache_read(cache, t)
    for x, got in (("k", K), ("v", V)):
        assert got.dtype is cc.KV[kv]
        assert torch.equal(got.cpu().double(), host.values(x)[:, :, :t])     # exact in both types
    ctx.close()


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_positions_and_counts_of_each_sequence(code):
    """Sequences of lengths of their own; rows before 0, behind the cache and behind a count are left out; other bytes stay."""
    b, hkv, n, block, rows = 6, 2, 150, 32, 20
    ctx, host = _ctx(b, hkv, n), cc.random_cache(b, hkv, n, block, code, 5)
    cache = host.device()
    first, count = [0, 13, n - 5, -3, n + 4, 96], [20, 7, 20, 20, 20, -2]
    K, V = (_rows(j, b, hkv, rows).mul(3.0).to(torch.bfloat16) for j in (1, 2))
    before = _bits(cache)
    f, c = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (first, count))
    ctx.cache_write(cache, K.to(DEV), V.to(DEV), 0, f, c)
    host.write(K, V, 0, first, count)
    _same(host, cache)
    after = _bits(cache)
    for i in range(b):
        lo, hi = max(first[i], 0), min(first[i] + min(max(count[i], 0), rows), n)
        lead = lo // block * block if hi > lo else n         # rows that a growing scale may round once more
        for x in "kv":
            assert torch.equal(after[x][i, :, :min(lead, n)], before[x][i, :, :min(lead, n)])
            assert torch.equal(after[x][i, :, max(hi, 0):], before[x][i, :, max(hi, 0):]) or hi <= lo
    # read with positions that leave the cache on both sides
    K, V = ctx.cache_read(cache, 40, 0, f)
    for x, got in (("k", K), ("v", V)):
        vals = host.values(x)
        for i in range(b):
            for r in range(40):
                t = first[i] + r
                want = vals[i, :, t] if 0 <= t < n else torch.zeros(hkv, cc.D, dtype=torch.float64)
                assert torch.equal(got[i, :, r].cpu().double(), want)
    # t0 and first add up
    a = ctx.cache_read(cache, 9, 4, f)[0]
    assert torch.equal(a, ctx.cache_read(cache, 9, 0, f + 4)[0])
    ctx.close()


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_values_at_the_edges(code, kv):
    """Zeros, the smallest and largest magnitudes, ties, infinities and NaN."""
    b, hkv, n, block = 1, 1, 16 * 9, 16
    ctx, host = _ctx(b, hkv, n, kv), cc.HostCache(b, hkv, n, block, code)
    cache = ctx.new_cache(cc.CODES[code], block)
    x = _rows(3, b, hkv, n)
    most = cc.MOST[code]
    x[0, 0, :16] = 0.0
    x[0, 0, 16:32] = 1e-38 * x[0, 0, 16:32]                                   # below binary32's normal range, some of it
    x[0, 0, 32:48] = x[0, 0, 32:48] * 2.0 ** 118
    x[0, 0, 48:64] = torch.randint(-448, 449, (16, cc.D), generator=torch.Generator().manual_seed(1)) * most / 448   # ties
    x[0, 0, 48, 0] = most
    x[0, 0, 64, 5], x[0, 0, 65, 6], x[0, 0, 66, 7] = math.inf, -math.inf, math.nan
    x[0, 0, 80, 0] = most * 4
    x[0, 0, 96:112] = math.nan
    K = x.to(cc.KV[kv])
    V = -K
    ctx.cache_write(cache, K.to(DEV), V.to(DEV))
    host.write(K, V)
    _same(host, cache)
    got = ctx.cache_read(cache, n)
    for name, y in zip("kv", got):
        want = host.values(name).to(cc.KV[kv])
        assert torch.equal(torch.isnan(y.cpu()), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(y.cpu()), torch.nan_to_num(want))
    # a token behind a block that holds NaN: only the integer code's block is lost, and a fresh write recovers it
    K1 = _rows(9, 1, 1, 1).to(cc.KV[kv])
    ctx.cache_write(cache, K1.to(DEV), K1.to(DEV), 70)
    host.write(K1, K1, 70)
    _same(host, cache)
    K2 = _rows(9, 1, 1, 16).to(cc.KV[kv])
    ctx.cache_write(cache, K2.to(DEV), K2.to(DEV), 64)
    host.write(K2, K2, 64)
    _same(host, cache)
    ctx.close()


def test_many_blocks_and_long_offsets():
    """A cache whose byte offsets pass 32 bits: rows at its end, and the neighbours of what is written."""
    n = (1 << 25) + 77                                                       # 4 GiB of codes a head
    ctx = _ctx(1, 1, n)
    cache = ctx.new_cache(torch.float8_e4m3fn, 128)
    K, V = (_rows(j, 1, 1, 300).to(torch.bfloat16) for j in (1, 2))
    ctx.cache_write(cache, K.to(DEV), V.to(DEV), n - 300)
    host = cc.HostCache(1, 1, 300 + (n - 300) % 128, 128, "e4m3")
    host.write(K, V, (n - 300) % 128)
    got = ctx.cache_read(cache, 300, n - 300)
    for x, y in zip("kv", got):
        assert torch.equal(y.cpu().double(), host.values(x)[:, :, (n - 300) % 128:])
    assert int(cache.k.view(torch.uint8)[0, 0, :n - 300].max()) == 0
    q = _rows(4, 1, 1).to(torch.bfloat16)
    idx = torch.arange(n - 40, n, dtype=torch.int32, device=DEV).view(1, 1, 40)
    ctx.close()
    ctx = sp.Spotlight(1, 1, 1, 128, 256, n, 40, device=DEV)
    out = ctx.sparse_decode_cache(q.to(DEV), cache, idx)
    v = host.values("v")[0, 0, -40:]
    want, mag, size = cc.attention(q[0], host.values("k")[0, 0, -40:], v, torch.ones(1, 40, dtype=torch.bool), 1 / math.sqrt(128))
    assert bool(((out[0].cpu().double() - want).abs() <= cc.tolerance(mag, size, 40)).all())
    # all of the cache: the rows before are zeros, with scores 0
    out = ctx.dense_decode_cache(q.to(DEV), cache, n)
    k = host.values("k")[0, 0, -300:]
    s = (q[0].double() @ k.T)[0] / math.sqrt(128)
    p = torch.exp(s)
    want = (p @ host.values("v")[0, 0, -300:]) / (p.sum() + n - 300)
    # 300 weighted rows among 2^25 equal weights: sums of up to 2^25 / 1024 / 32 steps a wavefront, and splits
    tol = (p @ host.values("v")[0, 0, -300:].abs()) / (p.sum() + n - 300) * 2 * (2.0 ** -20 + 2.0 ** -24 * (4 + 2048 + 136 * float(s.abs().max()) * 8))
    assert bool(((out[0, 0].cpu().double() - want).abs() <= tol).all())
    ctx.close()


def test_refusals_on_a_context():
    ctx = _ctx(2, 2, 100)
    cache = ctx.new_cache(torch.int8, 32)
    K = torch.zeros(2, 2, 3, 128, dtype=torch.bfloat16, device=DEV)
    for bad in (dict(K=K.float(), V=K.float()), dict(K=K, V=K[:, :, :2].contiguous()), dict(K=K[:, :1].contiguous(), V=K), dict(K=K.cpu(), V=K),
                dict(K=K, V=K, first=torch.zeros(2, device=DEV)), dict(K=K, V=K, first=torch.zeros(3, dtype=torch.int32, device=DEV)),
                dict(K=K, V=K, count=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            ctx.cache_write(cache, **bad)
    with pytest.raises(TypeError):
        ctx.cache_write((cache.k, cache.v), K, K)
    with pytest.raises(sp.SpotlightError) as e:
        ctx.cache_write(cache, K, K, 98)
    assert e.value.rc == sp.ERR_INVALID_ARG
    with pytest.raises(sp.SpotlightError):
        ctx.cache_read(cache, 101)
    with pytest.raises(ValueError):
        ctx.new_cache(torch.float8_e5m2)
    with pytest.raises(ValueError):
        ctx.new_cache(torch.int8, 48)
    other = _ctx(2, 2, 101)
    with pytest.raises(ValueError):
        other.cache_write(cache, K, K)
    ctx.close()
    other.close()


def test_another_stream_and_a_graph():
    """Positions in device memory: a captured append is replayed at other positions, with eager work between."""
    b, hkv, n, block = 2, 2, 200, 32
    ctx, host = _ctx(b, hkv, n), cc.HostCache(b, hkv, n, block, "i8")
    cache = ctx.new_cache(torch.int8, block)
    K = torch.zeros(b, hkv, 1, cc.D, dtype=torch.bfloat16, device=DEV)
    V = torch.zeros_like(K)
    pos = torch.zeros(b, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ctx.cache_write(cache, K, V, 0, pos)
    side.synchronize()
    host.write(K.cpu(), V.cpu(), 0, [0, 0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.cache_write(cache, K, V, 0, pos)
        out = ctx.cache_read(cache, 1, 0, pos)
    for t in range(40):
        k, v = (_rows(100 * t + j, b, hkv, 1).to(torch.bfloat16) for j in (1, 2))
        at = [t, 150 - t if t < 20 else t + 100]
        K.copy_(k); V.copy_(v); pos.copy_(torch.tensor(at, dtype=torch.int32))
        graph.replay()
        host.write(k, v, 0, at)
        if t % 3 == 0:
            torch.cuda.synchronize()
            _same(host, cache)
            for x, y in zip("kv", out):
                vals = host.values(x)
                assert all(torch.equal(y[i, :, 0].cpu().double(), vals[i, :, at[i]]) for i in range(b))
    torch.cuda.synchronize()
    _same(host, cache)
    ctx.close()


@pytest.mark.parametrize("code,kv,n", [("e4m3", "f32", 66001), ("i8", "bf16", 132003)])
def test_more_than_the_last_level_cache(code, kv, n):
    """Calls of over 256 MB of rows take other kernels: every code, scale and value.  (Whole blocks are new, so that the definition
    needs no loop.)"""
    b, hkv, block = 2, 2, 128
    ctx = _ctx(b, hkv, n + 1 + block, kv)
    cache = ctx.new_cache(cc.CODES[code], block)
    g = torch.Generator(device=DEV).manual_seed(3)
    rows = [(torch.randn(b, hkv, n, cc.D, generator=g, device=DEV) * torch.exp(torch.randn(b, hkv, n, 1, generator=g, device=DEV))).to(cc.KV[kv]) for _ in "kv"]
    ctx.cache_write(cache, *rows, block)
    got = ctx.cache_read(cache, n, block)
    for x, y, back in zip("kv", rows, got):
        y = torch.cat([y.double(), torch.zeros(b, hkv, -n % block, cc.D, dtype=torch.float64, device=DEV)], 2).view(b, hkv, -1, block, cc.D)
        a = y.abs().amax((3, 4))
        s = torch.tensor([cc.least_scale(v, code) for v in a.flatten().tolist()], dtype=torch.float64, device=DEV).view(a.shape)
        assert torch.equal(getattr(cache, x + "_scale")[:, :, 1:].double(), s)
        want = cc.nearest((y / s[..., None, None]).cpu(), code).to(DEV)      # (torch.ldexp is exact on the host)
        assert torch.equal(getattr(cache, x).view(torch.uint8)[:, :, block:block + n].view(cc.CODES[code]).double(), want.view(b, hkv, -1, cc.D)[:, :, :n])
        assert torch.equal(back.double(), (want * s[..., None, None]).view(b, hkv, -1, cc.D)[:, :, :n])
        assert int(getattr(cache, x).view(torch.uint8)[:, :, :block].max()) == 0 and int(getattr(cache, x).view(torch.uint8)[:, :, block + n:].max()) == 0
        del y, want
    ctx.close()


def test_no_rows():
    """Writing and reading nothing is no work, and no error."""
    ctx = _ctx(2, 2, 100)
    cache = ctx.new_cache(torch.int8, 32)
    K = torch.ones(2, 2, 40, 128, dtype=torch.bfloat16, device=DEV)
    ctx.cache_write(cache, K, K)
    before = cache.k.clone(), cache.k_scale.clone()
    ctx.cache_write(cache, K[:, :, :0], K[:, :, :0], 40)
    assert torch.equal(cache.k, before[0]) and torch.equal(cache.k_scale, before[1])
    k, v = ctx.cache_read(cache, 0, 40)
    assert k.shape == v.shape == (2, 2, 0, 128)
    ctx.close()
