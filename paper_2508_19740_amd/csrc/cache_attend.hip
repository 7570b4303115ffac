// Attention over gathered rows of the 8-bit cache.
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
constexpr int kWholeThreads = 1024;     // threads of a workgroup that takes a whole head
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

// Lanes below 32 get a summed over the two halves of the wavefront, the others b.
__device__ __forceinline__ float add_halves(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// The same over the two quarters of each half: lanes with bit 4 clear get a, the others b.
__device__ __forceinline__ float add_quarters(float a, float b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
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
    Partials part;
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
    constexpr bool JOINS = NT == kThreads && RB == kAttendMinRows;   // small calls: few heads and rows
    static_assert(ITERS >= 1 && RPW % kRowsPerLoad == 0, "row tiling");

    __shared__ float s_m[NW], s_l[NW];
    __shared__ float s_acc[JOINS ? 2 * NW : NW][kHeadDim];     // twice: the join's
    __shared__ uint32_t s_before;

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
    // Sums over the eight rows of a load.  Halves of the wavefront, then of each half, exchange half of what they hold, so
    // that each lane ends with a quarter of its elements, summed over four rows; then neighbours of eight lanes.
#pragma unroll
    for (int off = kLanes; off < 64; off <<= 1) l += __shfl_xor(l, off);
    float part[4];
    {
        float a8[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) a8[e] = add_halves(acc[e], acc[e + 8]);
#pragma unroll
        for (int e = 0; e < 4; ++e) part[e] = add_quarters(a8[e], a8[e + 4]);
#pragma unroll
        for (int e = 0; e < 4; ++e) part[e] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(part[e]), 0x128, 0xf, 0xf, true));   // row_ror:8
    }
    // lane 32h + 16q + s (s < 8) has elements 8h + 4q .. + 3 of lane s's sixteen
    if ((lane & 8) == 0)
        *reinterpret_cast<float4*>(&s_acc[wave][sub * kElems + (lane >> 5) * 8 + (lane >> 4 & 1) * 4]) = make_float4(part[0], part[1], part[2], part[3]);
    if (lane == 0) { s_m[wave] = m; s_l[wave] = l; }
    __syncthreads();

    // merge the waves; thread c < 64 owns output columns 2c and 2c + 1
    if (wave == 0) {
        Join j;
#pragma unroll
        for (int w = 0; w < NW; ++w) j.add(f32x2{s_m[w], s_l[w]}, reinterpret_cast<const f32x2*>(s_acc[w])[lane]);
        if (NT == kWholeThreads) {   // the whole head is here
            reinterpret_cast<f32x2*>(a.out + bh * kHeadDim)[lane] = j.l != 0.0f ? f32x2{j.a.x / j.l, j.a.y / j.l} : f32x2{0.0f, 0.0f};
        } else {
            put_part(a.part, bh * a.nsplit + split, lane, j.m, j.l, j.a);
        }
    }
    if constexpr (JOINS) {
        if (!a.part.arrived) return;
        if (arrives_last(a.part, static_cast<uint32_t>(bh), static_cast<uint32_t>(a.nsplit), &s_before))
            join_rows<NT, 16>(a.part, static_cast<uint32_t>(bh) * a.nsplit, 1, 1, static_cast<uint32_t>(a.nsplit), a.out + bh * kHeadDim, reinterpret_cast<f32x2*>(&s_acc[0][0]));
    }
}

template <typename CT, typename QT, int RB, int NT = kThreads>
void launch_rb(spotlight_ctx* ctx, StageTimer& timer, AttendArgs& a)
{
    const Plan& p = ctx->plan;
    a.nsplit = (a.topk + RB - 1) / RB;
    if (NT == kWholeThreads || RB != kAttendMinRows || !joins_in_place(static_cast<int64_t>(p.B) * p.Hq * a.nsplit, 1, a.nsplit)) a.part.arrived = nullptr;
    if (timer.rec) timer.rec->whole = NT == kWholeThreads || a.part.arrived;
    timer.launch(cache_attend_kernel<CT, QT, RB, NT>, dim3(static_cast<unsigned>(a.nsplit), static_cast<unsigned>(p.B * p.Hq)), dim3(NT), 0, a);
}

// Rows of a workgroup.  Up to 256 rows a head's are in one workgroup of 16 wavefronts, without a merge; then as many a workgroup as leave
// 1024 workgroups, four a compute unit.  Measured (us, E4M3, caches of which nothing is in a cache; heads x rows: one
// workgroup a head / 128 / 64 / 32 rows a workgroup, where small grids are joined in place):
//   1 x 256      7.1 / 10.4 / 10.0 /  7.1      512 x 128   8.9 /  8.1 / 11.8 / 12.7      512 x 256  11.5 / 13.6 / 13.3 / 17.0
//   1 x 2048       - / 10.1 / 10.1 /  7.1      128 x 512     - / 10.7 / 10.6 / 12.5      512 x 512     - / 18.6 / 18.1 / 27.1
//  32 x 512        - / 10.3 / 10.8 / 10.7      128 x 2048    - / 18.2 / 18.1 / 26.9      512 x 4096    - / 84.5 / 91.4 / 156
// At the borders the rule is behind the best choice by up to 18 % (128 x 384 11.7 against 10.2, 1 x 8192 11.3 against 9.7, 8 x 8192
// 11.9 against 10.9, 512 x 64 8.4 against 7.9).
template <typename CT, typename QT>
int launch_t(spotlight_ctx* ctx, AttendArgs& a)
{
    const Plan& p = ctx->plan;
    const int64_t heads = static_cast<int64_t>(p.B) * p.Hq;
    {
        StageTimer timer(ctx, SPOTLIGHT_STAGE_ATTEND);
        if (a.topk <= 128) launch_rb<CT, QT, 128, kWholeThreads>(ctx, timer, a);
        else if (a.topk <= 256) launch_rb<CT, QT, 256, kWholeThreads>(ctx, timer, a);
        else if (heads * ((a.topk + 127) / 128) >= 1024) launch_rb<CT, QT, 128>(ctx, timer, a);
        else if (heads * ((a.topk + 63) / 64) >= 1024) launch_rb<CT, QT, 64>(ctx, timer, a);
        else launch_rb<CT, QT, 32>(ctx, timer, a);
        if (hipGetLastError() != hipSuccess) return SPOTLIGHT_ERR_HIP;
    }
    if (a.nsplit == 1 || a.part.arrived) return SPOTLIGHT_OK;
    return launch_cache_merge(ctx, a.part.ml, a.part.acc, MergeRows{heads, a.nsplit, nullptr, {}, {}, {}, 0, 0, 0}, a.nsplit, a.out);
}

}  // namespace

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
    a.part.ml = reinterpret_cast<unsigned long long*>(ctx->workspace + p.off_part_ml);
    a.part.acc = reinterpret_cast<unsigned long long*>(ctx->workspace + p.off_part_acc);
    a.part.arrived = reinterpret_cast<uint32_t*>(ctx->workspace + p.off_arrived);
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
