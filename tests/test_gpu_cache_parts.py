"""How exact attention over the whole 8-bit cache is: queries and weights in several parts, none of which can be left out
(tests/test_cache_parts.py shows that each would be seen)."""
import pytest
import torch

import cache_common as cc
import cache_parts_common as pc
import paper_2508_19740_amd as sp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _check(host, q, scale, case, kv):
    hq, hkv, n, nq = case[:4]
    ctx = sp.Spotlight(1, hq, hkv, 128, 256, n, 1, kv_dtype=cc.KV[kv], device=DEV)
    out = ctx.dense_decode_cache(q.to(DEV), host.device(), n, scale=scale).cpu().double()
    for h in range(hq):
        k, v = (host.values(x)[0, h // (hq // hkv)] for x in "kv")
        want, tol = pc.want_and_tolerance(q[0, h], k, v, pc.seen_by(n, nq), scale, kv)
        worst = float(((out[0, h] - want).abs() / tol).max())
        assert worst <= 1.0, f"head {h}: {worst} of what is allowed"
    ctx.close()


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("case", pc.CASES, ids=str)
def test_parts(case, code, kv):
    for seed in range(3):
        host, q, scale = pc.make(case, code, kv, seed)
        _check(host, q, scale, case, kv)


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_sums_that_cancel(code):
    for seed in range(5):
        host, q, scale = pc.make_cancelling(code, seed)
        _check(host, q, scale, (1, 1, host.shape[2], 1), "f32")
