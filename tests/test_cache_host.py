"""What the 8-bit cache refuses and how its attention is shared out, without a GPU: the argument checks of the entry points
on a context made on the host, the rule that splits keys over workgroups, the binding's checks."""
import os
import subprocess
import types

import pytest
import torch

import cache_common as cc
import paper_2508_19740_amd as sp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2508_19740_amd", "csrc")

HEAD = r"""
#include <stdio.h>
#include <string.h>
#include <algorithm>
#include "cache.h"
using namespace spotlight;
static spotlight_config config(int B, int Hq, int Hkv, long n, int k)
{
    spotlight_config c;
    memset(&c, 0, sizeof(c));
    c.batch = B; c.n_q_heads = Hq; c.n_kv_heads = Hkv; c.head_dim = 128; c.code_bits = 128; c.hidden = 256;
    c.max_tokens = n; c.max_topk = k; c.kv_dtype = SPOTLIGHT_BF16; c.weight_dtype = SPOTLIGHT_BF16;
    return c;
}
"""

REFUSALS = HEAD + r"""
// pointers that are never followed: every call here is refused before the first HIP call, or does nothing
alignas(64) static char mem[256];
static int failed = 0;
#define WANT(rc, call) do { const int got = (call); if (got != (rc)) { printf("%d, not %d: %s\n", got, rc, #call); failed = 1; } } while (0)
int main()
{
    const spotlight_config cfg = config(2, 4, 2, 1000, 50);
    spotlight_ctx ctx;
    memset(&ctx, 0, sizeof(ctx));
    if (make_plan(&cfg, &ctx.plan) != SPOTLIGHT_OK) return 2;
    spotlight_hash_weights w = {mem, mem, mem};
    float* f = reinterpret_cast<float*>(mem);
    int32_t* i = reinterpret_cast<int32_t*>(mem);
    uint32_t* u = reinterpret_cast<uint32_t*>(mem);
    const spotlight_cache good = {mem, mem, f, f, SPOTLIGHT_E4M3, 64};
    const int bad = SPOTLIGHT_ERR_INVALID_ARG;
    for (int kind = 0; kind < 9; ++kind) {
        spotlight_cache c = good;
        if (kind == 0) c.k = nullptr;
        if (kind == 1) c.v = nullptr;
        if (kind == 2) c.k_scale = nullptr;
        if (kind == 3) c.v_scale = nullptr;
        if (kind == 4) c.code_type = SPOTLIGHT_BF16;
        if (kind == 5) c.block_tokens = 48;
        if (kind == 6) c.block_tokens = 256;
        if (kind == 7) c.k = mem + 8;
        if (kind == 8) c.block_tokens = 0;
        WANT(bad, spotlight_cache_write(&ctx, &c, mem, mem, 0, 1, nullptr, nullptr));
        WANT(bad, spotlight_cache_read(&ctx, &c, 0, 1, nullptr, mem, mem));
        WANT(bad, spotlight_sparse_decode_cache(&ctx, mem, &c, i, 5, 0.1f, f));
        WANT(bad, spotlight_dense_decode_cache(&ctx, mem, &c, 10, 1, nullptr, 0.1f, f));
        WANT(bad, spotlight_decode_step_cache(&ctx, mem, mem, mem, &c, &w, u, 10, 5, 0, 0, 0.1f, i, f));
    }
    WANT(bad, spotlight_cache_write(&ctx, nullptr, mem, mem, 0, 1, nullptr, nullptr));
    WANT(bad, spotlight_cache_write(&ctx, &good, nullptr, mem, 0, 1, nullptr, nullptr));
    WANT(bad, spotlight_cache_write(&ctx, &good, mem, nullptr, 0, 1, nullptr, nullptr));
    WANT(bad, spotlight_cache_write(&ctx, &good, mem + 2, mem, 0, 1, nullptr, nullptr));
    for (const int32_t* first : {static_cast<const int32_t*>(nullptr), static_cast<const int32_t*>(i)}) {
        WANT(bad, spotlight_cache_write(&ctx, &good, mem, mem, -1, 1, first, nullptr));
        WANT(bad, spotlight_cache_write(&ctx, &good, mem, mem, 0, -1, first, nullptr));
        WANT(bad, spotlight_cache_write(&ctx, &good, mem, mem, 0, 1001, first, nullptr));
        WANT(bad, spotlight_cache_write(&ctx, &good, mem, mem, 1001, 0, first, nullptr));
        WANT(bad, spotlight_cache_read(&ctx, &good, -1, 1, first, mem, mem));
        WANT(bad, spotlight_cache_read(&ctx, &good, 0, 1001, first, mem, mem));
        WANT(SPOTLIGHT_OK, spotlight_cache_write(&ctx, &good, mem, mem, 1000, 0, first, nullptr));
        WANT(SPOTLIGHT_OK, spotlight_cache_read(&ctx, &good, 1000, 0, first, mem, mem));
    }
    // an empty tensor has no address
    WANT(SPOTLIGHT_OK, spotlight_cache_write(&ctx, &good, nullptr, nullptr, 5, 0, nullptr, nullptr));
    WANT(SPOTLIGHT_OK, spotlight_cache_read(&ctx, &good, 5, 0, nullptr, nullptr, nullptr));
    WANT(SPOTLIGHT_OK, spotlight_hash_rows(&ctx, nullptr, &w, 5, 0, u));
    WANT(bad, spotlight_cache_write(&ctx, &good, nullptr, nullptr, 1001, 0, nullptr, nullptr));
    WANT(bad, spotlight_cache_write(&ctx, &good, mem, mem, 999, 2, nullptr, nullptr));
    WANT(bad, spotlight_cache_read(&ctx, &good, 999, 2, nullptr, mem, mem));
    WANT(bad, spotlight_cache_read(&ctx, &good, 0, 1, nullptr, nullptr, nullptr));
    WANT(bad, spotlight_cache_read(&ctx, &good, 0, 1, nullptr, mem + 4, nullptr));
    WANT(bad, spotlight_sparse_decode_cache(&ctx, mem, &good, i, 0, 0.1f, f));
    WANT(bad, spotlight_sparse_decode_cache(&ctx, mem, &good, i, 51, 0.1f, f));
    WANT(bad, spotlight_sparse_decode_cache(&ctx, mem, &good, nullptr, 5, 0.1f, f));
    WANT(bad, spotlight_sparse_decode_cache(&ctx, mem + 2, &good, i, 5, 0.1f, f));
    WANT(bad, spotlight_dense_decode_cache(&ctx, mem, &good, 0, 1, nullptr, 0.1f, f));
    WANT(bad, spotlight_dense_decode_cache(&ctx, mem, &good, 1001, 1, nullptr, 0.1f, f));
    WANT(bad, spotlight_dense_decode_cache(&ctx, mem, &good, 10, 0, nullptr, 0.1f, f));
    WANT(bad, spotlight_dense_decode_cache(&ctx, mem, &good, 10, 1001, nullptr, 0.1f, f));
    WANT(bad, spotlight_dense_decode_cache(&ctx, mem, &good, 10, 1, nullptr, 0.1f, nullptr));
    WANT(bad, spotlight_hash_rows(&ctx, nullptr, &w, 0, 1, u));
    WANT(bad, spotlight_hash_rows(&ctx, mem, nullptr, 0, 1, u));
    WANT(bad, spotlight_hash_rows(&ctx, mem, &w, 0, 1, nullptr));
    WANT(bad, spotlight_hash_rows(&ctx, mem, &w, 1000, 1, u));
    WANT(bad, spotlight_hash_rows(&ctx, mem, &w, -1, 1, u));
    WANT(SPOTLIGHT_OK, spotlight_hash_rows(&ctx, mem, &w, 0, 0, u));
    WANT(bad, spotlight_decode_step_cache(&ctx, mem, mem, mem, &good, &w, u, 1001, 5, 0, 0, 0.1f, i, f));
    WANT(bad, spotlight_decode_step_cache(&ctx, mem, mem, mem, &good, &w, u, 10, 11, 0, 0, 0.1f, i, f));
    WANT(bad, spotlight_decode_step_cache(&ctx, mem, mem, mem, &good, &w, u, 10, 5, 4, 4, 0.1f, i, f));
    WANT(bad, spotlight_decode_step_cache(&ctx, mem, nullptr, mem, &good, &w, u, 10, 5, 0, 0, 0.1f, i, f));
    WANT(bad, spotlight_decode_step_cache(&ctx, mem, mem, mem, nullptr, &w, u, 10, 5, 0, 0, 0.1f, i, f));
    // a long cache whose many rows leave no room for the splits it needs
    const spotlight_config lc = config(1, 1, 1, 1L << 27, 50);
    if (make_plan(&lc, &ctx.plan) != SPOTLIGHT_OK) return 2;
    cache::DensePlan d;
    WANT(SPOTLIGHT_ERR_UNSUPPORTED, cache::plan_dense(ctx.plan, 256, 1L << 27, 16384, nullptr, &d));
    WANT(SPOTLIGHT_ERR_UNSUPPORTED, cache::plan_dense(ctx.plan, 256, 1L << 27, 16384, i, &d));
    WANT(SPOTLIGHT_ERR_UNSUPPORTED, cache::plan_dense(ctx.plan, 256, 100, (1 << 24) + 1, nullptr, &d));
    WANT(SPOTLIGHT_OK, cache::plan_dense(ctx.plan, 256, 1L << 27, 1, nullptr, &d));
    WANT(SPOTLIGHT_OK, cache::plan_dense(ctx.plan, 256, 1L << 27, 1, i, &d));
    // a launch's threads are counted in 32 bits
    const spotlight_config wide = config(8, 64, 64, 1L << 20, 50);
    if (make_plan(&wide, &ctx.plan) != SPOTLIGHT_OK) return 2;
    WANT(SPOTLIGHT_ERR_UNSUPPORTED, cache::plan_dense(ctx.plan, 256, 100, 1 << 20, nullptr, &d));
    WANT(SPOTLIGHT_OK, cache::plan_dense(ctx.plan, 256, 100, (1 << 20) - 32, nullptr, &d));
    return failed;
}
"""

SPLITS = HEAD + r"""
int main()
{
    for (int B : {1, 2, 7, 16, 100})
        for (int Hkv : {1, 4, 8, 32})
            for (int G : {1, 2, 7, 8})
                for (long cap : {1L, 31L, 129L, 4096L, 100003L, 1L << 25, (1L << 25) + 1, (1L << 31) - 1}) {
                    if (B * Hkv * G > 65535) continue;
                    const spotlight_config cfg = config(B, Hkv * G, Hkv, cap, 1);
                    Plan p;
                    if (make_plan(&cfg, &p) != SPOTLIGHT_OK) return 2;
                    for (long n : {1L, cap / 3 + 1, cap})
                        for (long nq : {1L, 2L, 5L, 17L, 128L, 1000L, cap}) {
                            if (nq > cap || nq > 2147483647L) continue;
                            for (int ragged : {0, 1}) {
                                cache::DensePlan d;
                                int32_t one;
                                const int rc = cache::plan_dense(p, 256, n, static_cast<int>(nq), ragged ? &one : nullptr, &d);
                                const cache::DenseShares& s = d.shares;
                                const long rows = static_cast<long>(G) * nq, units = (n + 127) / 128;
                                if (rc == SPOTLIGHT_ERR_UNSUPPORTED && (n > 1 << 24 || rows > 1 << 24 || B * Hkv * rows / 32 > 1 << 23)) continue;
                                bool ok = rc == SPOTLIGHT_OK && (d.row_tiles == 1 || d.row_tiles == 2) && s.tile_rows * s.tiles >= rows &&
                                    s.tile_rows <= 16 * d.row_tiles && s.chunk * 128L <= (1L << 25) + 128 && d.grid <= 1 << 24;
                                long runs = 0;
                                if (!ragged) {
                                    runs = static_cast<long>(B) * s.nsplit;
                                    ok = ok && s.nsplit >= 1 && static_cast<long>(s.chunk) * s.nsplit >= units && static_cast<long>(s.chunk) * (s.nsplit - 1) < units;
                                } else {
                                    // lengths all alike, all short but one, none at all: the runs they make fit the grid and the workspace
                                    for (int kind = 0; kind < 3; ++kind) {
                                        long total = 0, made = 0;
                                        for (int b = 0; b < B; ++b) total += kind == 0 ? units : kind == 1 && b == B / 2 ? units : 0;
                                        long chunk = units;                  // as the kernel chooses it
                                        if (s.most_runs) {
                                            const long safe = (total + s.most_runs - B - 1) / (s.most_runs - B);
                                            chunk = std::max((total + s.most_runs - 1) / s.most_runs, 1L);
                                            for (int tries = 0; chunk < safe; ++tries) {
                                                long m = 0;
                                                for (int b = 0; b < B; ++b)
                                                    m += std::max(((kind == 0 ? units : kind == 1 && b == B / 2 ? units : 0) + chunk - 1) / chunk, 1L);
                                                if (m <= s.most_runs) break;
                                                chunk = tries < 3 ? std::max(chunk + 1, chunk * m / s.most_runs) : safe;
                                            }
                                            chunk = std::min(std::max(chunk, 1L), units);
                                        }
                                        ok = ok && chunk * 128 <= (1L << 25) + 128;
                                        for (int b = 0; b < B; ++b) {
                                            const long u = kind == 0 ? units : kind == 1 && b == B / 2 ? units : 0, r = std::max((u + chunk - 1) / chunk, 1L);
                                            ok = ok && r <= s.nsplit;
                                            made += r;
                                        }
                                        runs = std::max(runs, made);
                                    }
                                }
                                ok = ok && (s.tiles == 1 ? runs * Hkv <= d.grid : (runs * Hkv + 7) / 8 * 8 * s.tiles <= d.grid);
                                ok = ok && d.splits == (s.nsplit > 1) && (!d.splits || runs * Hkv * s.tiles * s.tile_rows <= p.dense_rows);
                                const size_t from = p.off_dense_ml, to = p.off_dense_acc + p.dense_rows * 512;
                                ok = ok && to <= p.total_bytes && p.off_dense_acc >= from + p.dense_rows * 8 && from % 256 == 0 && p.off_dense_acc % 256 == 0;
                                ok = ok && ((from >= p.off_gcum && to <= p.off_wnorm) || from >= p.off_open_counts) && to <= std::max(p.off_runs, p.off_wnorm);
                                ok = ok && (!d.joins || runs * Hkv * s.tiles <= kJoinGroups);
                                for (const cache::FastDiv& f : {s.by_nsplit, s.by_heads, s.by_tiles8, s.by_most, s.by_spare})
                                    for (uint32_t x : {0u, 1u, f.d - 1, f.d, f.d + 1, 5 * f.d - 1, 5 * f.d, 99999u, (1u << 24) + 1, (1u << 31) - 1})
                                        if (x < 1u << 31) ok = ok && x / f.d == static_cast<uint32_t>((static_cast<uint64_t>(x) * f.mul >> 32) + x) >> f.shift;
                                if (!ok) {
                                    printf("B %d Hkv %d G %d cap %ld n %ld nq %ld ragged %d: rc %d tiles %u nsplit %u chunk %u most %u runs %ld\n", B, Hkv, G, cap, n, nq,
                                           ragged, rc, s.tiles, s.nsplit, s.chunk, s.most_runs, runs);
                                    return 1;
                                }
                            }
                        }
                }
    return 0;
}
"""


@pytest.mark.parametrize("source", [REFUSALS, SPLITS], ids=["refusals", "splits"])
def test_host_rules(tmp_path, source):
    src, exe = tmp_path / "host.cpp", tmp_path / "host"
    src.write_text(source)
    lib = sp.lib._name
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-w", "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
                    "-I", CSRC, str(src), "-o", str(exe), lib, f"-Wl,-rpath,{os.path.dirname(lib)}", "-L/opt/rocm/lib",
                    "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"], check=True)
    run = subprocess.run([str(exe)], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout + run.stderr


def _tensors(n=100, block=32, code=torch.int8):
    k = torch.zeros(2, 3, n, 128, dtype=torch.uint8).view(code)
    s = torch.ones(2, 3, -(-n // block))
    return [k, k.clone(), s, s.clone()]


def test_cache_takes_matching_tensors():
    for code in (torch.int8, torch.float8_e4m3fn):
        assert sp.Cache(*_tensors(code=code), 32).block_tokens == 32


@pytest.mark.parametrize("change", [
    lambda t: (*t, 48), lambda t: (*t, 64), lambda t: (t[0].float(), *t[1:], 32), lambda t: (t[0], t[1][:, :, :99], *t[2:], 32),
    lambda t: (t[0], t[1].view(torch.float8_e4m3fn), *t[2:], 32), lambda t: (t[0], t[1], t[2].double(), t[3], 32),
    lambda t: (t[0], t[1], t[2], t[3][:, :, :3], 32), lambda t: (t[0].transpose(0, 1).contiguous().transpose(0, 1), *t[1:], 32),
    lambda t: (t[0][0], *t[1:], 32)])
def test_cache_refuses_other_tensors(change):
    with pytest.raises(ValueError):
        sp.Cache(*change(_tensors()))


def test_a_cache_keeps_its_tensors():
    """The calls take the addresses that a Cache was made with: other tensors, or other storage, are refused."""
    cache = sp.Cache(*_tensors(), 32)
    for name in ("k", "v", "k_scale", "v_scale", "block_tokens"):
        with pytest.raises(AttributeError):
            setattr(cache, name, getattr(cache, name))
    ctx = types.SimpleNamespace(_kv_shape=tuple(cache.k.shape), device=cache.k.device)
    assert sp.Spotlight._cache(ctx, cache) is not None
    cache.v_scale.fill_(2.0)
    assert sp.Spotlight._cache(ctx, cache) is not None
    for name in ("k", "v", "k_scale", "v_scale"):
        other = sp.Cache(*_tensors(), 32)
        t = getattr(other, name)
        t.data = t.data.clone()
        with pytest.raises(ValueError):
            sp.Spotlight._cache(ctx, other)


def test_the_reference_quantises_to_the_nearest_code():
    """The tests' own rounding against all codes of each type, and its scale against the definition."""
    g = torch.Generator().manual_seed(3)
    for code in ("e4m3", "i8"):
        if code == "i8":
            values = torch.arange(-127, 128, dtype=torch.float64)
        else:
            values = torch.arange(256, dtype=torch.int64).to(torch.uint8).view(torch.float8_e4m3fn).double()
            values = values[torch.isfinite(values)].unique()
        y = torch.cat([torch.randn(500, generator=g, dtype=torch.float64) * cc.MOST[code] / 5, torch.randn(200, generator=g, dtype=torch.float64) * 0.01])
        y = y.clamp(-cc.MOST[code], cc.MOST[code])
        got = cc.nearest(y, code)
        assert torch.equal((got - y).abs(), (values[None] - y[:, None]).abs().amin(1))
        between = (values[1:] + values[:-1]) / 2                   # ties: the even code of the two
        got = cc.nearest(between, code)
        assert bool(((got == values[1:]) | (got == values[:-1])).all())
        if code == "i8":
            assert bool((got % 2 == 0).all())
        else:
            assert bool((got.float().to(torch.float8_e4m3fn).view(torch.uint8) % 2 == 0).all())
        for a in (0.0, 1e-300, 2.0 ** -120, 0.9, cc.MOST[code], cc.MOST[code] * 1.0001, 3e38, cc.MOST[code] * 2.0 ** 17):
            s = cc.least_scale(a, code)
            assert a <= cc.MOST[code] * s and (s == 2.0 ** -126 or a > cc.MOST[code] * s / 2)
