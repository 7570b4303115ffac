"""Attention over the whole 8-bit cache where values are of very different sizes: a query loses nothing to keys that it does
not see, weighs 0 or weighs little, whatever their values are."""
import math

import pytest
import torch

import cache_common as cc
import paper_2508_19740_amd as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SCALE = 1.0 / math.sqrt(128)
U = 2.0 ** -24


def _ctx(hq, hkv, n, kv="bf16"):
    return sp.Spotlight(1, hq, hkv, 128, 256, n, 1, kv_dtype=cc.KV[kv], device=DEV)


def _q(seed, kv, *shape, size=1.0):
    return (torch.randn(*shape, cc.D, generator=torch.Generator().manual_seed(seed)) * size).to(cc.KV[kv])


def _want(q, host, h, n, nq, scale=SCALE):
    """The 64-bit result of a head's queries and how far a result may be off.  A score is off by the roundings of its
    products' sum, 136 units of sum |q k|, which moves a weight by as much; the exponential by 2 units; a weight that is split in
    two parts by 2^-22 (each rounded to 11 bits); sums by a rounding for every step of 32 keys and every part.  Of a weight
    that is small beside the largest it is split with, 2^-31 of that largest is lost at most (scaled to above 2^6, and the second
    part's smallest step is 2^-24): beside the largest of the 16 keys that share a product, or of the run where its values
    lie within 2^12 of each other.  Both at most: 2^-31 (sum of the block's |v|) times the block's largest weight, and 2^-31 times the
    sum of those |v| that are at most 2^12 times the least block's."""
    k, v = (host.values(x)[0, h, :n] for x in "kv")
    k = torch.nan_to_num(k)
    t = torch.arange(n)
    seen = t[None] <= (n - nq + torch.arange(nq))[:, None]
    want, mag, size = cc.attention(q, k, torch.nan_to_num(v), seen, scale)
    s = torch.where(seen, (q.double() @ k.T) * scale, -math.inf)
    p = torch.softmax(s, -1)
    pad = -n % 16
    top = torch.cat([p, torch.zeros(nq, pad, dtype=p.dtype)], 1).view(nq, -1, 16).amax(-1).repeat_interleave(16, 1)[:, :n]
    w = torch.nan_to_num(v).abs()
    least = host.scale["v"][0, h]
    least = float(least[torch.isfinite(least) & (least > 2.0 ** -126)].min())
    near = torch.where(w <= 128 * 2.0 ** 12 * least * 4, w, 0.0)
    lost = 2.0 ** -31 * (top @ w + torch.where(seen, 1.0, 0.0).double() @ near)
    tol = mag * (2.0 * torch.expm1(136 * U * size) + 2 * (2.0 ** -22 + (4 + 2 * (n // 32 + 16)) * U)) + lost + 1e-37
    return want, tol


def _check(got, want, tol, what):
    got = got.cpu().double()
    bad = ~((got - want).abs() <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} off, worst {float((got - want).abs().nan_to_num(9e9).max())}, wanted {want[bad][:3].tolist()}, got {got[bad][:3].tolist()}"


def _put_value(host, h, at, exponent, g):
    """A row of values of about 2^exponent at token `at`; other rows of its block are rounded to 0, as a write does."""
    top = 8 if host.code == "e4m3" else 6
    blk = at // host.block
    host.codes["v"][0, h, blk * host.block:(blk + 1) * host.block] = 0.0
    host.codes["v"][0, h, at] = cc.nearest(torch.rand(cc.D, generator=g, dtype=torch.float64) * cc.MOST[host.code], host.code)
    host.scale["v"][0, h, blk] = 2.0 ** (exponent - top)


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("nq,n,block", [(3, 70, 16), (20, 400, 64), (70, 2500, 16), (9, 9000, 128)])
def test_values_of_later_tokens(nq, n, block, code, kv):
    """A chunk of queries, and a value 2^31 to 2^127 times the others' size at one of its tokens: the queries before it."""
    hq, hkv = 4, 2
    at = n - (nq + 1) // 2
    for exponent in (13, 21, 31, 60, 126):
        host = cc.random_cache(1, hkv, n, block, code, 3)
        g = torch.Generator().manual_seed(1)
        _put_value(host, 0, at, exponent, g)
        ctx = _ctx(hq, hkv, n, kv)
        q = _q(2, kv, 1, hq, nq, size=2.0)
        out = ctx.dense_decode_cache(q.to(DEV), host.device(), n)
        before = at - (n - nq)
        for h in range(hq):
            rows = before if h // 2 == 0 else nq
            want, tol = _want(q[0, h], host, h // 2, n, nq)
            _check(out[0, h, :rows], want[:rows], tol[:rows], (exponent, h))
        ctx.close()


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("n,block", [(40, 16), (600, 32), (5000, 64)])
def test_values_that_weigh_little(n, block, code, kv):
    """One query, and a key of a huge value whose weight is 0, or so small that weight and value together are about 1, among
    keys of all other weights."""
    at = n // 2
    for exponent, nats in ((31, 31 * math.log(2)), (60, 60 * math.log(2)), (90, 90 * math.log(2)), (40, 400.0), (100, 400.0)):
        host = cc.random_cache(1, 1, n, block, code, 5)
        g = torch.Generator().manual_seed(2)
        _put_value(host, 0, at, exponent, g)
        q = _q(4, kv, 1, 2, 1)
        # the block's keys are opposite to the queries
        blk = at // block
        q[0, 1, 0] = q[0, 0, 0]
        size = float((q[0, 0, 0].double().abs().sum() * SCALE))
        c = nats / size                                       # k = -c sign(q): the score is -nats
        host.scale["k"][0, 0, blk] = cc.least_scale(c, code)
        host.codes["k"][0, 0, blk * block:(blk + 1) * block] = cc.nearest(-torch.sign(q[0, 0, 0].double()) * c / host.scale["k"][0, 0, blk], code)
        ctx = _ctx(2, 1, n, kv)
        out = ctx.dense_decode_cache(q.to(DEV), host.device(), n)
        for h in range(2):
            want, tol = _want(q[0, h], host, 0, n, 1)
            _check(out[0, h], want, tol, (exponent, nats, h))
        ctx.close()


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("nq,n", [(1, 33), (1, 3000), (17, 1000), (50, 700)])
def test_scales_far_apart_everywhere(nq, n, code, kv):
    """Every other block of 16 is 2^13, 2^40 or 2^70 larger, in half of the columns (the other half is the small blocks' own), or
    all zeros with the least scale there is."""
    hq, hkv, block = 2, 1, 16
    for apart in (13, 40, 70, None):
        host = cc.random_cache(1, hkv, n, block, code, 6)
        if apart is None:
            host.codes["v"].view(1, hkv, n, cc.D)[0, 0, torch.arange(n) // block % 2 == 1] = 0.0
            host.scale["v"][0, 0, 1::2] = 2.0 ** -126
        else:
            host.scale["v"][0, 0, 1::2] *= 2.0 ** -apart
            host.codes["v"][0, 0, torch.arange(n) // block % 2 == 0, 64:] = 0.0
        ctx = _ctx(hq, hkv, n, kv)
        q = _q(8, kv, 1, hq, nq, size=2.0)
        out = ctx.dense_decode_cache(q.to(DEV), host.device(), n)
        for h in range(hq):
            want, tol = _want(q[0, h], host, 0, n, nq)
            _check(out[0, h], want, tol, (apart, h))
        ctx.close()


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("nq,n,block", [(5, 80, 16), (20, 400, 32), (70, 400, 16)])
def test_nan_scales(nq, n, block, code, kv):
    """A block whose scale is NaN, of K, of V or of both: the queries that see a row of it get NaN, the others the result
    without it; with and without codes of NaN (E4M3) beside it."""
    hq, hkv = 4, 2
    blk = (n - nq // 2) // block
    for which, beside in (("k", False), ("v", False), ("kv", False), ("v", True)):
        host = cc.random_cache(1, hkv, n, block, code, 6)
        for x in which:
            host.scale[x][0, 0, blk] = math.nan
        first = blk * block
        if beside and code == "e4m3":
            first = max(first - 2, 0)
            host.codes["v"][0, 0, first, 7] = math.nan
        ctx = _ctx(hq, hkv, n, kv)
        q = _q(8, kv, 1, hq, nq)
        out = ctx.dense_decode_cache(q.to(DEV), host.device(), n).cpu()
        for h in range(hq):
            want, tol = _want(q[0, h], host, h // 2, n, nq)
            last = n - nq + torch.arange(nq)
            hit = (last >= blk * block) if h // 2 == 0 else torch.zeros(nq, dtype=torch.bool)
            assert bool(torch.isnan(out[0, h, hit]).all()), (which, h)
            clean = ~hit
            if beside and code == "e4m3" and h // 2 == 0:
                one = (last >= first) & clean
                assert bool(torch.isnan(out[0, h, one][:, 7]).all()) and int(torch.isnan(out[0, h, one]).sum()) == int(one.sum())
                clean &= ~one
            _check(out[0, h, clean], want[clean], tol[clean], (which, beside, h))
        ctx.close()


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("nq,n,block", [(1, 1, 16), (1, 2, 16), (1, 70, 32), (1, 4000, 64), (1, 8192, 128), (3, 3, 16), (20, 700, 16), (70, 300, 64)])
def test_values_near_the_largest_and_the_smallest(nq, n, block, code, kv):
    """Values up to the largest float's size, and down to 2^-110: weighted means of them are of their size, whatever sums are
    formed on the way.  (Scores are small: no key takes all the weight.)"""
    for size in (120, 127, -110):
        host = cc.random_cache(1, 1, n, block, code, 7, spread=0.0)
        top = 8 if code == "e4m3" else 6
        host.scale["v"][:] = 2.0 ** (size - top)
        host.codes["v"] = cc.nearest(torch.rand(1, 1, n, cc.D, generator=torch.Generator().manual_seed(n), dtype=torch.float64) * 1.75 * 2 ** top, code)
        ctx = _ctx(2, 1, n, kv)
        q = _q(4, kv, 1, 2, nq, size=0.5)
        out = ctx.dense_decode_cache(q.to(DEV), host.device(), n)
        for h in range(2):
            want, tol = _want(q[0, h], host, 0, n, nq)
            _check(out[0, h], want, tol - 1e-37 + 2.0 ** -135, (size, h))
        ctx.close()


@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("n,block", [(600, 32), (5000, 64)])
def test_the_largest_values_with_no_weight(n, block, code):
    """Keys of the largest values there are, a whole block of them, that weigh nothing."""
    host = cc.random_cache(1, 1, n, block, code, 5)
    blk = n // 2 // block
    rows = slice(blk * block, (blk + 1) * block)
    host.codes["v"][0, 0, rows] = cc.MOST[code]
    host.scale["v"][0, 0, blk] = 2.0 ** (119 if code == "e4m3" else 121)
    q = _q(4, "bf16", 1, 1, 1)
    c = 400.0 / float(q.double().abs().sum() * SCALE)
    host.scale["k"][0, 0, blk] = cc.least_scale(c, code)
    host.codes["k"][0, 0, rows] = cc.nearest(-torch.sign(q[0, 0, 0].double()) * c / host.scale["k"][0, 0, blk], code)
    ctx = _ctx(1, 1, n)
    out = ctx.dense_decode_cache(q.to(DEV), host.device(), n)
    want, tol = _want(q[0, 0], host, 0, n, 1)
    _check(out[0, 0], want, tol, n)
    ctx.close()
