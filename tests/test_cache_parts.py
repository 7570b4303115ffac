"""The bounds that the GPU tests of parts hold results to, on the CPU: parts as the definition has them pass, and every part
that is left out fails."""
import pytest

import cache_parts_common as pc


def _worst(host, q, scale, case, kv, drop):
    hq, hkv, n, nq = case[:4]
    worst = 0.0
    for h in range(hq):
        k, v = (host.values(x)[0, h // (hq // hkv)] for x in "kv")
        seen = pc.seen_by(n, nq)
        want, tol = pc.want_and_tolerance(q[0, h], k, v, seen, scale, kv)
        got = pc.emulate(q[0, h], k, v, seen, scale, kv, drop)
        worst = max(worst, float(((got - want).abs() / tol).max()))
    return worst


@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("code", ["e4m3", "i8"])
@pytest.mark.parametrize("case", pc.CASES, ids=str)
def test_all_parts_are_needed(case, code, kv):
    host, q, scale = pc.make(case, code, kv, 1)
    assert _worst(host, q, scale, case, kv, None) < 0.5
    # of many keys the losses cancel, and what the third part holds is less than integers' scores are rounded by
    for drop in ("p2", "q2", "q3") if kv == "f32" else ("p2",):
        worst = _worst(host, q, scale, case, kv, drop)
        assert worst > 2.0 or (drop == "q3" and (case[2] < 16 or case[2] > 60)), (drop, worst)


@pytest.mark.parametrize("code", ["e4m3", "i8"])
def test_sums_that_cancel_need_a_common_grid(code):
    """Parts of 11 bits of each element, summed in 24 bits, lose in the large sums what the small ones need."""
    for seed in range(5):
        host, q, scale = pc.make_cancelling(code, seed)
        case = (1, 1, host.shape[2], 1)
        assert _worst(host, q, scale, case, "f32", None) < 0.5
        for drop in ("p2", "q2", "q11"):
            assert _worst(host, q, scale, case, "f32", drop) > 2.0, (seed, drop)
