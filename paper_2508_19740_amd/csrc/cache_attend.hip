// Attention over gathered rows of the 8-bit cache, and the merge of partial results that it shares with
// attention over the whole cache.
//
// As in attend.hip, the k rows of a query head are split over workgroups, a wavefront issues the loads of
// all its rows before it uses any (random rows: bound by the latency and bandwidth of memory), and
// forms scores, a softmax in binary32 and the weighted sum of its rows.  A row is 128 bytes here: eight
// lanes read it, 16 bytes a lane, so one load instruction fetches eight rows.  The scale of a row's block
// multiplies its score, or its weight.
#include "cache.h"

namespace spotlight {
using namespace cache;
namespace {

constexpr int kLanes = 8;               // lanes of a row
constexpr int kElems = 16;              // elements of a lane
constexpr int kRowsPerLoad = 64 / kLanes;
constexpr float kLog2e = 1.4426950408889634f;

// 16 bytes of a row that is used once: the rows of a step do not fit into a cache
__device__ __forceinline__ uint4 load16(const uint8_t* p)
{
    const uint4* s = reinterpret_cast<const uint4*>(p);
    uint4 r;
    r.x = __builtin_nontemporal_load(&s->x);
    r.y = __builtin_nontemporal_load(&s->y);
    r.z = __builtin_nontemporal_load(&s->z);
    r.w = __builtin_nontemporal_load(&s->w);
    return r;
}

template <typename CT>
__device__ __forceinline__ void decode16(const uint4& u, float (&o)[kElems])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float f[4];
        CT::decode(w[i], f);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[4 * i + e] = f[e];
    }
}

// Sum over the eight adjacent lanes of a row, the same bits in every lane.
__device__ __forceinline__ float add_across_row(float x)
{
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xb1, 0xf, 0xf, true));    // quad_perm 1,0,3,2
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4e, 0xf, 0xf, true));    // quad_perm 2,3,0,1
    x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x141, 0xf, 0xf, true));   // row_half_mirror
    return x;
}

__device__ __forceinline__ void load_q(const bf16_raw* q, float (&o)[kElems])
{
    const uint4* s = reinterpret_cast<const uint4*>(q);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint4 u = s[i];
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            o[8 * i + 2 * j] = __uint_as_float(w[j] << 16);
            o[8 * i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
    }
}
__device__ __forceinline__ void load_q(const float* q, float (&o)[kElems])
{
    const float4* s = reinterpret_cast<const float4*>(q);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 u = s[i];
        o[4 * i] = u.x; o[4 * i + 1] = u.y; o[4 * i + 2] = u.z; o[4 * i + 3] = u.w;
    }
}

struct AttendArgs {
    const void* q;
    const uint8_t* k;
    const uint8_t* v;
    const float* k_scale;
    const float* v_scale;
    const int32_t* idx;
    float2* part_ml;
    float* part_acc;
    float* out;
    int64_t Nmax, blocks;
    int topk, Hq, Hkv, nsplit, shift;
    float scale2;                       // scale * log2(e)
};

// RB rows per workgroup of NT threads, shared out evenly over its wavefronts.
template <typename CT, typename QT, int RB, int NT>
__global__ __launch_bounds__(NT) void cache_attend_kernel(AttendArgs a)
{
    constexpr int NW = NT / 64;
    constexpr int RPW = RB / NW;
    constexpr int ITERS = RPW / kRowsPerLoad;
    static_assert(ITERS >= 1 && RPW % kRowsPerLoad == 0, "row tiling");

    __shared__ float s_m[NW], s_l[NW];
    __shared__ float s_acc[NW][kHeadDim];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int split = blockIdx.x;
    const int64_t bh = blockIdx.y;
    const int64_t b = bh / a.Hq;
    const int hk = static_cast<int>(bh % a.Hq) / (a.Hq / a.Hkv);
    const int64_t head = b * a.Hkv + hk;
    const int sub = lane % kLanes, grp = lane / kLanes;

    const uint8_t* Kh = a.k + head * a.Nmax * kHeadDim + sub * kElems;
    const uint8_t* Vh = a.v + head * a.Nmax * kHeadDim + sub * kElems;
    const float* ks = a.k_scale + head * a.blocks;
    const float* vs = a.v_scale + head * a.blocks;

    // A missing row (past k, or an index outside the cache) loads row 0 and is masked below, so that
    // every load is unconditional and all of them are in flight together.
    const int row0 = split * RB + wave * RPW;
    int ridx[ITERS];
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int j = row0 + it * kRowsPerLoad + grp;
        ridx[it] = a.idx[bh * a.topk + (j < a.topk ? j : 0)];
        if (j >= a.topk || static_cast<int64_t>(ridx[it]) >= a.Nmax) ridx[it] = -1;
    }
    uint4 kr[ITERS], vr[ITERS];
    float kf[ITERS], vf[ITERS];
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int r = ridx[it] >= 0 ? ridx[it] : 0;
        kr[it] = load16(Kh + static_cast<int64_t>(r) * kHeadDim);
        kf[it] = ks[r >> a.shift];
    }
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int r = ridx[it] >= 0 ? ridx[it] : 0;
        vr[it] = load16(Vh + static_cast<int64_t>(r) * kHeadDim);
        vf[it] = vs[r >> a.shift];
    }
    float qf[kElems];
    load_q(static_cast<const QT*>(a.q) + bh * kHeadDim + sub * kElems, qf);

    // scores in units of log2
    float s[ITERS];
    float m = -INFINITY;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        float f[kElems];
        decode16<CT>(kr[it], f);
        float dot = 0.0f;
#pragma unroll
        for (int e = 0; e < kElems; ++e) dot = __builtin_fmaf(qf[e], f[e], dot);
        dot = add_across_row(dot);
        s[it] = ridx[it] >= 0 ? dot * kf[it] * a.scale2 : -INFINITY;
        m = fmaxf(m, s[it]);
    }
#pragma unroll
    for (int off = kLanes; off < 64; off <<= 1) m = fmaxf(m, __shfl_xor(m, off));

    // softmax numerators and the weighted sum of the rows; a row of NaN makes them NaN
    float l = 0.0f;
    float acc[kElems];
#pragma unroll
    for (int e = 0; e < kElems; ++e) acc[e] = 0.0f;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const bool have = ridx[it] >= 0;
        const float p = have ? __builtin_amdgcn_exp2f(s[it] - m) : 0.0f;
        const float pv = have ? p * vf[it] : 0.0f;
        l += p;
        if (!have) vr[it] = make_uint4(0u, 0u, 0u, 0u);   // the stand-in may hold NaN
        float f[kElems];
        decode16<CT>(vr[it], f);
#pragma unroll
        for (int e = 0; e < kElems; ++e) acc[e] = __builtin_fmaf(pv, f[e], acc[e]);
    }
#pragma unroll
    for (int off = kLanes; off < 64; off <<= 1) {
        l += __shfl_xor(l, off);
#pragma unroll
        for (int e = 0; e < kElems; ++e) acc[e] += __shfl_xor(acc[e], off);
    }
    if (grp == 0) {
#pragma unroll
        for (int e = 0; e < kElems; ++e) s_acc[wave][sub * kElems + e] = acc[e];
    }
    if (lane == 0) { s_m[wave] = m; s_l[wave] = l; }
    __syncthreads();

    // merge the waves; thread c < 128 owns output column c.  A wave without rows has l = 0.
    if (tid < kHeadDim) {
        float M = s_m[0];
#pragma unroll
        for (int w = 1; w < NW; ++w) M = fmaxf(M, s_m[w]);
        float o = 0.0f, lsum = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (s_l[w] != 0.0f) {
                const float f = __builtin_amdgcn_exp2f(s_m[w] - M);
                o = __builtin_fmaf(f, s_acc[w][tid], o);
                lsum = __builtin_fmaf(f, s_l[w], lsum);
            }
        }
        if (a.nsplit == 1) {   // the whole head is here
            a.out[bh * kHeadDim + tid] = lsum != 0.0f ? o / lsum : 0.0f;
            return;
        }
        const int64_t pi = bh * a.nsplit + split;
        a.part_acc[pi * kHeadDim + tid] = o;
        if (tid == 0) a.part_ml[pi] = make_float2(M, lsum);
    }
}

// Merge of a row's partial results {maximum in units of log2, sum} and accumulators.  32 threads, with four columns
// each, fold the splits part, part + PARTS, ... of a row with a running maximum, up to eight loads ahead of the
// arithmetic; the row's PARTS groups of them are then combined in order.  A split without rows has sum 0 and is left
// out: its accumulator may hold anything.
template <int PARTS>
__global__ __launch_bounds__(kThreads) void cache_merge_kernel(const float2* __restrict__ part_ml, const float4* __restrict__ part_acc,
                                                               float4* __restrict__ out, int64_t rows, int nsplit)
{
    constexpr int NB = 8, QUADS = kHeadDim / 4, RPW = kThreads / QUADS / PARTS;   // rows of a workgroup
    __shared__ float s_m[PARTS][kThreads / PARTS], s_l[PARTS][kThreads / PARTS];
    __shared__ float4 s_a[PARTS][kThreads / PARTS];
    const int tid = threadIdx.x;
    const int c = tid % QUADS, part = tid / QUADS % PARTS, slot = tid / (QUADS * PARTS);
    const int64_t row = static_cast<int64_t>(blockIdx.x) * RPW + slot;
    const int64_t at = min(row, rows - 1) * nsplit;       // threads behind the last row repeat it
    float m = -INFINITY, l = 0.0f;
    float4 a = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int s0 = part; s0 < nsplit; s0 += PARTS * NB) {
        float2 v[NB];
        float4 av[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int sp = s0 + PARTS * i;
            const int64_t spc = at + (sp < nsplit ? sp : s0);      // in-bounds stand-in, left out below
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
    if (row >= rows) return;
    out[row * QUADS + c] = l != 0.0f ? make_float4(a.x / l, a.y / l, a.z / l, a.w / l) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
}

template <typename CT, typename QT, int RB, int NT = kThreads>
void launch_rb(spotlight_ctx* ctx, StageTimer& timer, AttendArgs& a)
{
    const Plan& p = ctx->plan;
    a.nsplit = (a.topk + RB - 1) / RB;
    timer.launch(cache_attend_kernel<CT, QT, RB, NT>, dim3(static_cast<unsigned>(a.nsplit), static_cast<unsigned>(p.B * p.Hq)), dim3(NT), 0, a);
}

template <typename CT, typename QT>
int launch_t(spotlight_ctx* ctx, AttendArgs& a)
{
    const Plan& p = ctx->plan;
    const int64_t heads = static_cast<int64_t>(p.B) * p.Hq;
    {
        StageTimer timer(ctx, SPOTLIGHT_STAGE_ATTEND);
        if (a.topk <= 256) {
            if (timer.rec) timer.rec->whole = true;
            if (a.topk <= 128) launch_rb<CT, QT, 128, 1024>(ctx, timer, a);
            else launch_rb<CT, QT, 256, 1024>(ctx, timer, a);
            return hip_rc(hipGetLastError());
        }
        if (heads * ((a.topk + 127) / 128) >= 1024) launch_rb<CT, QT, 128>(ctx, timer, a);
        else if (heads * ((a.topk + 63) / 64) >= 1024) launch_rb<CT, QT, 64>(ctx, timer, a);
        else launch_rb<CT, QT, 32>(ctx, timer, a);
        if (hipGetLastError() != hipSuccess) return SPOTLIGHT_ERR_HIP;
    }
    return launch_cache_merge(ctx, a.part_ml, a.part_acc, heads, a.nsplit, a.out);
}

}  // namespace

int launch_cache_merge(spotlight_ctx* ctx, const void* part_ml, const float* part_acc, int64_t rows, int nsplit, float* out)
{
    StageTimer timer(ctx, SPOTLIGHT_STAGE_MERGE);
    // few splits: a row's are folded by the same threads, and a workgroup has eight rows
    const bool few = nsplit <= 8;
    const int64_t per = few ? kThreads / (kHeadDim / 4) : 1;
    timer.launch(few ? cache_merge_kernel<1> : cache_merge_kernel<8>, dim3(static_cast<unsigned>((rows + per - 1) / per)), dim3(kThreads), 0,
                 static_cast<const float2*>(part_ml), reinterpret_cast<const float4*>(part_acc), reinterpret_cast<float4*>(out), rows, nsplit);
    return hip_rc(hipGetLastError());
}

int launch_cache_attend(spotlight_ctx* ctx, const void* q, const spotlight_cache& c, const int32_t* idx, int k, float scale, float* out)
{
    const Plan& p = ctx->plan;
    AttendArgs a;
    a.q = q;
    a.k = static_cast<const uint8_t*>(c.k);
    a.v = static_cast<const uint8_t*>(c.v);
    a.k_scale = c.k_scale;
    a.v_scale = c.v_scale;
    a.idx = idx;
    a.part_ml = reinterpret_cast<float2*>(ctx->workspace + p.off_part_ml);
    a.part_acc = reinterpret_cast<float*>(ctx->workspace + p.off_part_acc);
    a.out = out;
    a.Nmax = p.Nmax;
    a.blocks = (p.Nmax + c.block_tokens - 1) / c.block_tokens;
    a.topk = k;
    a.Hq = p.Hq;
    a.Hkv = p.Hkv;
    a.nsplit = 1;
    a.shift = __builtin_ctz(static_cast<unsigned>(c.block_tokens));
    a.scale2 = scale * kLog2e;
    if (p.kv_dtype == SPOTLIGHT_BF16)
        return c.code_type == SPOTLIGHT_E4M3 ? launch_t<E4M3, bf16_raw>(ctx, a) : launch_t<I8, bf16_raw>(ctx, a);
    return c.code_type == SPOTLIGHT_E4M3 ? launch_t<E4M3, float>(ctx, a) : launch_t<I8, float>(ctx, a);
}

}  // namespace spotlight
