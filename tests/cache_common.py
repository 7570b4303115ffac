"""The 8-bit key-value cache step by step in 64 bits, for the tests: codes, scales, attention."""
import math

import torch

CODES = {"e4m3": torch.float8_e4m3fn, "i8": torch.int8}
KV = {"bf16": torch.bfloat16, "f32": torch.float32}
MOST = {"e4m3": 448.0, "i8": 127.0}
D = 128


def nearest(y, code):
    """y (float64) rounded to the code type's values, ties to even; NaN stays."""
    if code == "i8":
        return torch.round(y)
    _, e = torch.frexp(y)                                  # |y| = m 2^e, m in [1/2, 1)
    step = torch.ldexp(torch.ones_like(y), (e - 1).clamp(min=-6) - 3)
    return torch.round(y / step) * step


def least_scale(a, code):
    """The smallest 2^e, e >= -126, with a <= MOST 2^e (a a Python float)."""
    e = -126
    if a > 0:
        e = max(-126, math.frexp(a / MOST[code])[1] - 1)
        while a > MOST[code] * 2.0 ** e:
            e += 1
        while e > -126 and a <= MOST[code] * 2.0 ** (e - 1):
            e -= 1
    return 2.0 ** e


class HostCache:
    """Values (as codes in float64) and scales of one cache, written one block after the other."""

    def __init__(self, b, hkv, n, block, code):
        self.shape, self.block, self.code = (b, hkv, n), block, code
        self.codes = {x: torch.zeros(b, hkv, n, D, dtype=torch.float64) for x in "kv"}
        self.scale = {x: torch.ones(b, hkv, -(-n // block), dtype=torch.float64) for x in "kv"}

    def write(self, K, V, t0=0, first=None, count=None):
        b, hkv, n = self.shape
        for x, new in (("k", K), ("v", V)):
            for i in range(b):
                start = t0 + (first[i] if first is not None else 0)
                rows = min(max(count[i], 0), new.shape[2]) if count is not None else new.shape[2]
                lo, hi = max(start, 0), min(start + rows, n)
                for h in range(hkv):
                    for blk in range(lo // self.block, -(-hi // self.block) if hi > lo else 0):
                        self._block(x, i, h, blk, max(lo, blk * self.block), min(hi, (blk + 1) * self.block),
                                    new[i, h].double(), start, lo)

    def _block(self, x, i, h, blk, lo, hi, new, start, first_row):
        y = new[lo - start:hi - start]
        fine = torch.isfinite(y)
        s = least_scale(float(torch.where(fine, y, 0.0).abs().max()), self.code)
        old = float(self.scale[x][i, h, blk])
        poisoned = self.code == "i8" and not bool(fine.all())
        at = blk * self.block
        if at < first_row:                                 # rows from before
            poisoned |= old != old
            if not poisoned and s > old:
                c = self.codes[x][i, h, at:first_row]
                self.codes[x][i, h, at:first_row] = nearest(c * (old / s), self.code)
            if old == old:
                s = max(s, old)
        c = nearest(torch.where(fine, y / s, math.nan if self.code == "e4m3" else 0.0), self.code)
        self.codes[x][i, h, lo:hi] = c
        self.scale[x][i, h, blk] = math.nan if poisoned else s

    def values(self, x):
        return self.codes[x] * self.scale[x].repeat_interleave(self.block, 2)[:, :, :self.shape[2], None]

    def device(self, dev="cuda:0"):
        """The same cache as the library's."""
        import paper_2508_19740_amd as sp
        t = {x: self.codes[x].float().to(CODES[self.code]).to(dev) for x in "kv"}
        s = {x: self.scale[x].float().to(dev) for x in "kv"}
        return sp.Cache(t["k"], t["v"], s["k"], s["v"], self.block)


def random_cache(b, hkv, n, block, code, seed, spread=1.0):
    """A cache written in one go from rows whose sizes differ from token to token."""
    g = torch.Generator().manual_seed(seed)
    c = HostCache(b, hkv, n, block, code)
    for x in "kv":
        rows = torch.randn(b, hkv, n, D, generator=g, dtype=torch.float64)
        rows *= torch.exp(spread * torch.randn(b, hkv, n, 1, generator=g, dtype=torch.float64))
        pad = -n % block
        y = torch.cat([rows, torch.zeros(b, hkv, pad, D, dtype=torch.float64)], 2).view(b, hkv, -1, block, D)
        a = y.abs().amax((3, 4))
        s = torch.tensor([least_scale(v, code) for v in a.view(-1).tolist()], dtype=torch.float64).view(a.shape)
        c.scale[x] = s
        c.codes[x] = nearest(y / s[..., None, None], code).view(b, hkv, -1, D)[:, :, :n].contiguous()
    return c


def attention(q, k, v, seen, scale):
    """(softmax(scale q k^T) v, softmax(..) |v|, largest scale sum |q k| of each row) over the keys `seen` [rows, n]
    keeps, in 64 bits; a row that sees nothing is 0."""
    q = q.double()
    s = (q @ k.T) * scale
    size = abs(scale) * (q.abs() @ torch.nan_to_num(k).abs().T)
    out, mag = torch.zeros(q.shape[0], D, dtype=torch.float64), torch.zeros(q.shape[0], D, dtype=torch.float64)
    for r in range(q.shape[0]):
        t = seen[r].nonzero()[:, 0]
        if t.numel():
            p = torch.softmax(s[r, t], -1)
            out[r], mag[r] = p @ v[t], p @ v[t].abs()
    return out, mag, torch.where(seen, size, torch.zeros_like(size)).amax(-1, keepdim=True)


def tolerance(mag, size, chain, q_parts=1, p_err=0.0):
    """How far a result may be off: every score by (128 + 8) roundings of its products' sum (and, where binary32 rows of q
    are split in binary16 parts, 2^-20 of them: two parts, each rounded to 11 bits, lose no more, three of 8 bits less), which moves each weight by as much; the exponential by 2 units; p by
    p_err; sums by `chain` roundings.  Both the numerator and the denominator take the error."""
    u = 2.0 ** -24
    score = (136 * u + (2.0 ** -20 if q_parts == 2 else 0.0)) * size
    return mag * (2.0 * torch.expm1(score) + 2 * (p_err + (4 + 2 * chain) * u)) + 1e-30


def split_floor(v):
    """What the binary16 parts of the weights lose however small a weight is: a weight is scaled by 2^7, and of its second part
    binary16 drops at most half its smallest step, 2^-25.  So each key's weight (relative to the largest) is off by at most
    2^-32, and a column's sum by at most 2^-32 sum |v|; the denominator is at least 1.  v: the head's values [n, d]."""
    return 2.0 ** -32 * torch.nan_to_num(v).abs().sum(0)
