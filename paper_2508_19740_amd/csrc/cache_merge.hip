// Merge of the partial results of attention over an 8-bit cache whose keys are split over many workgroups (cache.h).
#include "cache.h"

namespace spotlight {
using namespace cache;
namespace {

// 32 threads, with four columns each, fold the splits part, part + PARTS, ... of a row with a running maximum, up to eight loads ahead of the
// arithmetic; the row's PARTS groups of them are then combined in order.  A split without rows has sum 0 and is left
// out: its accumulator may hold anything.
template <int PARTS>
__global__ __launch_bounds__(kThreads) void cache_merge_kernel(const float2* __restrict__ part_ml, const float4* __restrict__ part_acc,
                                                               float4* __restrict__ out, MergeRows r)
{
    constexpr int NB = 8, QUADS = kHeadDim / 4, RPW = kThreads / QUADS / PARTS;   // rows of a workgroup
    __shared__ float s_m[PARTS][kThreads / PARTS], s_l[PARTS][kThreads / PARTS];
    __shared__ float4 s_a[PARTS][kThreads / PARTS];
    const int tid = threadIdx.x;
    const int c = tid % QUADS, part = tid / QUADS % PARTS, slot = tid / (QUADS * PARTS);
    const int64_t row = static_cast<int64_t>(blockIdx.x) * RPW + slot;
    const int64_t have = min(row, r.rows - 1);            // threads behind the last row repeat it
    int64_t at = have * r.nsplit, step = 1;
    int nsplit = r.nsplit;
    if (r.runs) {
        const uint32_t head = r.by_rows.over(static_cast<uint32_t>(have)), in_head = static_cast<uint32_t>(have) - head * r.by_rows.d;
        const uint32_t entry = r.by_heads.over(head), tile = r.by_tile.over(in_head);
        const RowParts p = parts_of(r, r.runs[entry], head - entry * r.by_heads.d, tile, in_head - tile * r.by_tile.d);
        at = p.at;
        step = p.step;
        nsplit = p.nsplit;
    }
    float m = -INFINITY, l = 0.0f;
    float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s0 = part; s0 < nsplit; s0 += PARTS * NB) {
        float2 v[NB];
        float4 av[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int sp = s0 + PARTS * i;
            const int64_t spc = at + (sp < nsplit ? sp : s0) * step;      // in-bounds stand-in, left out below
            v[i] = part_ml[spc];
            av[i] = part_acc[spc * QUADS + c];
            if (sp >= nsplit) v[i].y = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            if (v[i].y != 0.0f) {
                const float mn = fmaxf(m, v[i].x);
                const float fo = l != 0.0f ? __builtin_amdgcn_exp2f(m - mn) : 0.0f, fn = __builtin_amdgcn_exp2f(v[i].x - mn);
                a.x = __builtin_fmaf(a.x, fo, fn * av[i].x);
                a.y = __builtin_fmaf(a.y, fo, fn * av[i].y);
                a.z = __builtin_fmaf(a.z, fo, fn * av[i].z);
                a.w = __builtin_fmaf(a.w, fo, fn * av[i].w);
                l = __builtin_fmaf(l, fo, fn * v[i].y);
                m = mn;
            }
        }
    }
    if constexpr (PARTS > 1) {
        const int e = slot * QUADS + c;
        s_m[part][e] = m; s_l[part][e] = l; s_a[part][e] = a;
        __syncthreads();
        if (part != 0) return;
        m = -INFINITY;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) m = fmaxf(m, s_m[p][e]);
        l = 0.0f;
        a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            if (s_l[p][e] != 0.0f) {
                const float f = __builtin_amdgcn_exp2f(s_m[p][e] - m);
                const float4 o = s_a[p][e];
                a.x = __builtin_fmaf(f, o.x, a.x);
                a.y = __builtin_fmaf(f, o.y, a.y);
                a.z = __builtin_fmaf(f, o.z, a.z);
                a.w = __builtin_fmaf(f, o.w, a.w);
                l = __builtin_fmaf(f, s_l[p][e], l);
            }
        }
    }
    if (row >= r.rows || (r.runs && nsplit == 1)) return;      // a sequence of one run has its result already
    out[row * QUADS + c] = l != 0.0f ? make_float4(a.x / l, a.y / l, a.z / l, a.w / l) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
}

}  // namespace

int launch_cache_merge(spotlight_ctx* ctx, const void* part_ml, const void* part_acc, const MergeRows& r, int64_t about, float* out)
{
    StageTimer timer(ctx, SPOTLIGHT_STAGE_MERGE);
    // few splits: a row's are folded by the same threads, and a workgroup has eight rows
    const bool few = about <= 8;
    const int64_t per = few ? kThreads / (kHeadDim / 4) : 1;
    timer.launch(few ? cache_merge_kernel<1> : cache_merge_kernel<8>, dim3(static_cast<unsigned>((r.rows + per - 1) / per)), dim3(kThreads), 0,
                 static_cast<const float2*>(part_ml), static_cast<const float4*>(part_acc), reinterpret_cast<float4*>(out), r);
    return hip_rc(hipGetLastError());
}

}  // namespace spotlight
