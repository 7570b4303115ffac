"""Inputs and bounds of the tests of how exact attention over the whole 8-bit cache is.  Keys are whole numbers of few bits (E4M3: -15 to
15), and bfloat16 queries whole numbers up to 255, so that sums of products of the queries' first parts are exact (below
2^24 of their unit): what is left are the roundings of single numbers, which have narrow bounds."""
import math

import torch

import cache_common as cc

U = 2.0 ** -24
CASES = [  # hq, hkv, n, n_q, block, scores' spread
    (1, 1, 2, 1, 16, 3.0),
    (2, 1, 9, 1, 16, 3.0),
    (4, 1, 16, 5, 32, 4.0),
    (8, 2, 40, 1, 64, 4.0),
    (2, 2, 31, 20, 16, 3.0),
    (4, 2, 60, 40, 128, 4.0),
    (1, 1, 300, 1, 64, 5.0),
    (4, 1, 4000, 1, 64, 5.0),
]


def make(case, code, kv, seed):
    hq, hkv, n, nq, block, spread = case
    g = torch.Generator().manual_seed(seed)
    most = 15 if code == "e4m3" else 127
    host = cc.HostCache(1, hkv, n, block, code)
    host.codes["k"] = torch.randint(-most, most + 1, (1, hkv, n, cc.D), generator=g).double()
    host.codes["v"] = cc.nearest((torch.rand(1, hkv, n, cc.D, generator=g, dtype=torch.float64) * 2 - 1) * cc.MOST[code], code)
    if kv == "bf16":
        q = torch.randint(-255, 256, (1, hq, nq, cc.D), generator=g).to(torch.bfloat16)
    else:
        q = (torch.rand(1, hq, nq, cc.D, generator=g) * 2 - 1) * 255
    return host, q, spread / (255 / math.sqrt(3) * most / math.sqrt(3) * math.sqrt(cc.D))


def make_cancelling(code, seed):
    """Binary32 queries of pairs of large elements, whose products cancel, and of elements 2^-7 as large with finer bits, which
    make the scores: sums of a few units on the way to which there are sums thousands of times as large (a matrix product
    takes columns 8c .. 8c+7 of each 32, c = 0 .. 3 one after the other: the pairs are first and last)."""
    g = torch.Generator().manual_seed(seed)
    n, most = 24, 15 if code == "e4m3" else 127
    host = cc.HostCache(1, 1, n, 16, code)
    k = torch.randint(-most, most + 1, (n, cc.D), generator=g).double()
    first, last = (torch.arange(cc.D) % 32 // 8 == c for c in (0, 3))
    k[:, first] = torch.randint(most // 2, most + 1, (n, 32), generator=g).double()
    k[:, last] = -k[:, first]
    host.codes["k"][0, 0] = k
    host.codes["v"] = cc.nearest((torch.rand(1, 1, n, cc.D, generator=g, dtype=torch.float64) * 2 - 1) * cc.MOST[code], code)
    q = torch.randint(1, 3, (cc.D,), generator=g) * 64.0 + torch.randint(-8, 8, (cc.D,), generator=g) / 4.0
    q[first] = torch.randint(128, 255, (32,), generator=g) * 64.0
    q[last] = q[first]
    q = q.view(1, 1, 1, cc.D)
    return host, q, 3.0 / float((q[0, 0, 0].double() @ k.T).std())


def first_part(q):
    """The multiples of 2^-7 to 2^-8 of each row's largest that are nearest to its elements."""
    unit = torch.exp2(torch.floor(torch.log2(q.abs().amax(-1, keepdim=True))) - 7)
    return torch.round(q / unit) * unit


def want_and_tolerance(q, k, v, seen, scale, kv):
    """Rows of one head in 64 bits, and how far each element of a result may be off.  S: scores in units of log2.  Each is off by
    the roundings of scale log2(e) (three, of S less the row's largest: what all scores share cancels), of S itself and of S less
    the maximum (four, of at most |S - top| + |S| + 16), and, binary32, by 136 roundings of the sum over the queries' second and third
    parts.  The exponential is off by 2^-23.  In the numerator a weight's two
    parts are off by 2^-22 of it or 2^-32 of the largest.  Sums: a matrix instruction by 2^-22 of its terms, two a step of 32 keys,
    and 16 roundings for the parts that are joined."""
    q = q.double()
    scale = float(torch.tensor(scale, dtype=torch.float32))
    s = torch.where(seen, (q @ k.T) * scale / math.log(2), -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.softmax(s * math.log(2), -1)
    want = p @ v
    gap = torch.where(seen, (s - top).abs(), 0.0)
    size = torch.where(seen, s.abs(), 0.0)
    x = 3 * U * gap + 4 * U * (gap + size + 16)
    if kv == "f32":
        rest = (q - first_part(q)).abs() @ k.abs().T
        x = x + 136 * U * rest * scale / math.log(2)
    eta = math.log(2) * x + 2.0 ** -23
    steps = (seen.sum(-1, keepdim=True) + 31) // 32 + 1
    off = torch.stack([(p[r] * eta[r]) @ (v - want[r]).abs() for r in range(q.shape[0])])
    mag = p @ v.abs()
    lost = 2.0 ** -32 * (torch.where(seen, 1.0, 0.0).double() @ v.abs())
    return want, off + mag * (2.0 ** -22 + steps * 2 * 2.0 ** -22 + 16 * U) + lost


def emulate(q, k, v, seen, scale, kv, drop=None):
    """The result of queries and weights in parts, one of them dropped (drop: "q2", "q3", "p2"; or "q11": queries in two parts of 11
    bits whose sums round to 24 bits), all else in 64 bits."""
    q = q.double()
    if kv == "f32":
        most = q.abs().amax(-1, keepdim=True)
        unit = torch.exp2(torch.floor(torch.log2(most)) - 13)
        y = q / unit
        a = torch.round(y / 64) * 64
        b = torch.round((y - a) * 4) / 4
        c = (y - a - b).half().double()
        if drop == "q11":
            a = y.half().double()                                 # 11 bits of each element, and 11 more
            b, c = (y - a).half().double(), torch.zeros_like(y)
            s = torch.zeros(q.shape[0], k.shape[0], dtype=torch.float32)
            for j in [32 * i + 8 * c for c in range(4) for i in range(4)]:      # groups of eight products are summed exactly, then rounded
                s = (s.double() + a[:, j:j + 8] @ k[:, j:j + 8].T).float()
            s = s.double() + b @ k.T
        else:
            s = (a + (0 if drop == "q2" else b) + (0 if drop == "q3" else c)) @ k.T
        s = s * unit
    else:
        s = q @ k.T
    s = torch.where(seen, s * float(torch.tensor(scale, dtype=torch.float32)) / math.log(2), -math.inf)
    w = torch.exp2(s - torch.ceil(s.amax(-1, keepdim=True)) + 8)
    hi = w.half().double()
    lo = (w - hi).half().double()
    return ((hi + (0 if drop == "p2" else lo)) @ v) / w.sum(-1, keepdim=True)


def seen_by(n, nq):
    return torch.arange(n)[None] <= (n - nq + torch.arange(nq))[:, None]
