// Attention of the last n_q tokens of each sequence over the whole 8-bit cache.
//
// The rows of a key-value head are its G query heads times n_q queries, contiguous in q.  A wavefront
// takes tiles of 16 rows and a run of keys, 32 keys a step, and needs no barrier until its keys are done:
//
//   S^T = K Q^T     v_mfma_f32_16x16x32_f16.  Lane (g, i) = (lane / 16, lane % 16) loads 32 adjacent
//                   bytes of key i; four products take 8 of them each, and q lies in registers in the
//                   same order.  The result leaves lane (g, i) with keys 4g .. 4g+3 of query row i.
//   softmax         weights are relative to a maximum that was taken once, rounded up to a whole number (of log2).  Lanes compare
//                   their own scores with it, and only where one is more than 7 (a factor of 2^7) above it is the maximum taken
//                   anew, over the lanes, and what has been summed rescaled.  (Taken at every larger score, some row
//                   of 16 had one at most steps; at 4 above, at one step in three.)
//   O^T += V^T P^T  The lane holds the weights just where the second operand wants them (the keys of a
//                   product may come in any order).  The first operand wants the same keys of one
//                   column: lane (g, i) loads 8 bytes, columns 8i .. 8i+7, of each of its eight keys, and
//                   swaps keys for columns with byte permutes.
//
// Both codes are exact in binary16, so the products' only rounding is that of their binary32 sums:
//   q   is scaled by a power of two for each row to a largest magnitude in [2^13, 2^14), where bfloat16
//       rows are exact down to 2^-28 of it; binary32 rows are split in three parts, multiples of 2^6, of 2^-2, and the rest,
//       which is off by 2^-28 of the row's largest at most.  A matrix instruction is off by up to 4 units of its largest
//       term; but sums of the first part by integer codes are below 2^24 of its units, and exact.  They are kept apart from the
//       others' (2^-8 of them), and meet them in the score less the maximum.  (Error of the result, median of 40 seeds each of 6
//       shapes: 1.7e-7 to 2.3e-7, with parts of eight significant bits of each element 2.0e-7 to 2.7e-7, of torch operations in
//       binary32 4.9e-7 to 9.0e-7; of a single row of 4096 keys 9e-7 at most, theirs 1.7e-6, but less in 12 of 80.)
//   p   is scaled to a largest of 2^7 to 2^15 (below) and split in two parts: 22 bits, or 2^-32 of the largest weight
//       where that is more.  Both are rounded to nearest: what many small weights lose must not add up.
//   v   carries the ratio of its block's scale to the largest of the run's, times 2^5, which is exact down to 2^-20.
//
// Where the scales of a run's values lie further apart than 2^12 (a key of huge values, or a block of zeros, whose scale
// is the least there is), or one is NaN, a row must not lose the small values that it attends to a large one that it does not
// see, or weighs 0.  There, the 16 keys of a block have products of their own (v_mfma_f32_16x16x16_f16), with weights
// relative to the row's largest among them, and meet the others in binary32 with that weight and the block's scale: 64 more
// multiply-adds a tile.  (All runs so: 268 MB, 32 / 8 heads, 48.1 -> 53.4 us, 128 queries over 67 MB 122 -> 195 us; other runs lose
// nothing.  2^12: what the second part of p drops, 2^-32 of the largest weight, is then 2^-20 of the least block's
// values at most.)
//
// A row reads 256 bytes a key and key-value head, whatever G and n_q: with few rows the kernel is bound by
// memory.  The keys are split over workgroups, and a merge joins them.
#include <algorithm>

#include "cache.h"

namespace spotlight {
using namespace cache;
namespace {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int kStep = kDenseStep;       // keys of a step
constexpr int kVUp = 5;                 // v is scaled by 2^5, p by 2^8 less the maximum rounded up
constexpr float kPUp = 8.0f;
constexpr int kFar = 12;                // scales of values further apart than 2^12 have products of their own
// Partial results are sums of weights and of weighted values, the largest weight 2^7 to 2^15, times 2^-20: of values of
// the largest float's size, 2^13 with all the same weight add up without an overflow; and values are whole down to 2^-113.
constexpr int kSumUp = -20;
constexpr float kSlack = 7.0f;          // by which scores may pass the last maximum (log2, rounded up) before it is taken anew
constexpr int kInf = 0x7f800000;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ h8 join(h2 a, h2 b, h2 c, h2 d)
{
    return h8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

// The elements of the first or the last 16 keys of a step.
__device__ __forceinline__ h4 half_of(h8 x, int kt)
{
    return kt ? __builtin_shufflevector(x, x, 4, 5, 6, 7) : __builtin_shufflevector(x, x, 0, 1, 2, 3);
}

// Binary16 operands from codes.
template <typename CT> struct Operand;
template <> struct Operand<E4M3> {
    // eight codes of a key
    static __device__ __forceinline__ h8 row(uint32_t lo, uint32_t hi)
    {
        return join(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true),
                    __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true));
    }
    // four columns of the keys a and b, times a power of two: o[c] = (a[c], b[c])
    typedef float Ratio;
    static __device__ __forceinline__ Ratio ratio(float r) { return r; }
    static __device__ __forceinline__ void columns(uint32_t a, uint32_t b, Ratio r, h2 (&o)[4])
    {
        const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x05010400u), hi = __builtin_amdgcn_perm(b, a, 0x07030602u);
        o[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, r, false);
        o[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, r, true);
        o[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, r, false);
        o[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, r, true);
    }
};
template <> struct Operand<I8> {
    // 0x6400 | u is 1024 + u in binary16; u is the code with its sign bit flipped, code + 128
    static __device__ __forceinline__ h2 pair(uint32_t biased) { return __builtin_bit_cast(h2, biased) - h2{1152.0f16, 1152.0f16}; }
    static __device__ __forceinline__ h8 row(uint32_t lo, uint32_t hi)
    {
        lo ^= 0x80808080u;
        hi ^= 0x80808080u;
        return join(pair(__builtin_amdgcn_perm(lo, 0x64646464u, 0x00050004u)), pair(__builtin_amdgcn_perm(lo, 0x64646464u, 0x00070006u)),
                    pair(__builtin_amdgcn_perm(hi, 0x64646464u, 0x00050004u)), pair(__builtin_amdgcn_perm(hi, 0x64646464u, 0x00070006u)));
    }
    struct Ratio { h2 r, bias; };
    static __device__ __forceinline__ Ratio ratio(float r)
    {
        const _Float16 h = static_cast<_Float16>(r);
        return Ratio{h2{h, h}, h2{-1152.0f16 * h, -1152.0f16 * h}};
    }
    static __device__ __forceinline__ void columns(uint32_t a, uint32_t b, const Ratio& r, h2 (&o)[4])
    {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t w = __builtin_amdgcn_perm(a, b, 0x0c000c04u + 0x00010001u * c) ^ 0x64806480u;
            o[c] = __builtin_elementwise_fma(__builtin_bit_cast(h2, w), r.r, r.bias);
        }
    }
};

// Two numbers rounded to binary16 (to nearest: what many small weights lose must not add up).
__device__ __forceinline__ h2 to_half(float x, float y) { return __builtin_convertvector((f32x2{x, y}), h2); }

// x less the low or the high half of h, in one instruction.
__device__ __forceinline__ float less_low(float x, h2 h)
{
    float d;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(d) : "v"(h), "v"(x));
    return d;
}
__device__ __forceinline__ float less_high(float x, h2 h)
{
    float d;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(d) : "v"(h), "v"(x));
    return d;
}

struct DenseArgs {
    const void* q;
    const uint8_t* k;
    const uint8_t* v;
    const float* k_scale;
    const float* v_scale;
    Partials part;
    uint2* runs;                        // [batch] {first, number} of each sequence's runs, for the merge
    float* out;
    int64_t Nmax, blocks, n_tokens;
    DenseShares shares;
    FastDiv by_queries;
    uint32_t rows, n_q;                 // rows of a key-value head: G * n_q
    int shift;
    float scale2;                       // |scale| * log2(e)
    bool negate;                        // the scale is negative: q is negated
};

template <bool B> struct Flag { static constexpr bool value = B; };

// The nearest multiple of a power of two (|x| below 2^22 of them).
__device__ __forceinline__ float multiple_of(float unit, float x)
{
    const float c = 0x1.8p23f * unit;
    return (x + c) - c;
}

// A lane's 8 NF elements of a row, which LANES lanes (64 / LANES apart) share, scaled by a power of two that brings the row's largest into [2^13, 2^14), negated if
// asked and split into QP binary16 parts (multiples of 2^6, of 2^-2, and the rest); returns the exponent that takes the scaling back.
template <typename QT, int QP, int NF, int LANES>
__device__ __forceinline__ int load_row(const QT* q, bool negate, h8 (&frag)[QP][NF])
{
    constexpr int NV = 8 * NF * sizeof(QT) / 16;
    uint4 u[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) u[i] = reinterpret_cast<const uint4*>(q)[i];
    uint32_t most = 0;                           // bits of the largest magnitude
    if constexpr (sizeof(QT) == 2) {
        typedef uint16_t us2 __attribute__((ext_vector_type(2)));
        us2 top = {0, 0};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t w[4] = {u[i].x, u[i].y, u[i].z, u[i].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) top = __builtin_elementwise_max(top, __builtin_bit_cast(us2, w[j] & 0x7fff7fffu));
        }
        most = static_cast<uint32_t>(max(top.x, top.y)) << 16;
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            most = max(max(max(most, u[i].x & 0x7fffffffu), u[i].y & 0x7fffffffu), max(u[i].z & 0x7fffffffu, u[i].w & 0x7fffffffu));
    }
#pragma unroll
    for (int off = 64 / LANES; off < 64; off <<= 1) most = max(most, static_cast<uint32_t>(__shfl_xor(static_cast<int>(most), off)));
    // rows below 2^-113 are scaled as those at it; an infinity or a NaN makes the row's results NaN, however it is scaled
    const int ex = min(max(static_cast<int>(most >> 23) - 127, -113), 127);
    const float up = __uint_as_float(static_cast<uint32_t>(13 - ex + 127) << 23 | (negate ? 0x80000000u : 0u));
#pragma unroll
    for (int c = 0; c < NF; ++c) {
        h2 part[QP][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float x, y;
            if constexpr (sizeof(QT) == 2) {
                const uint32_t w = j == 0 ? u[c].x : j == 1 ? u[c].y : j == 2 ? u[c].z : u[c].w;
                x = __uint_as_float(w << 16);
                y = __uint_as_float(w & 0xffff0000u);
            } else {
                const uint4 w = u[2 * c + j / 2];
                x = __uint_as_float(j % 2 ? w.z : w.x);
                y = __uint_as_float(j % 2 ? w.w : w.y);
            }
            x *= up;
            y *= up;
#pragma unroll
            for (int p = 0; p < QP; ++p) {
                const float unit = p == 0 ? 0x1p6f : 0x1p-2f, hx = p + 1 < QP ? multiple_of(unit, x) : x, hy = p + 1 < QP ? multiple_of(unit, y) : y;
                part[p][j] = to_half(hx, hy);
                x -= hx;
                y -= hy;
            }
        }
#pragma unroll
        for (int p = 0; p < QP; ++p) frag[p][c] = join(part[p][0], part[p][1], part[p][2], part[p][3]);
    }
    return ex - 13;
}

constexpr int kWaves = kDenseWaves;
static_assert(kWaves == kThreads / 64, "wavefronts of a workgroup");

// Largest of 64 numbers that are not negative, by data-parallel-primitive moves.
__device__ __forceinline__ int wave_max(int x)
{
#define SPOTLIGHT_DPP_MAX(ctrl, rows) x = max(x, __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xf, true))
    SPOTLIGHT_DPP_MAX(0x111, 0xf);   // row_shr:1
    SPOTLIGHT_DPP_MAX(0x112, 0xf);   // row_shr:2
    SPOTLIGHT_DPP_MAX(0x114, 0xf);   // row_shr:4
    SPOTLIGHT_DPP_MAX(0x118, 0xf);   // row_shr:8
    SPOTLIGHT_DPP_MAX(0x142, 0xa);   // lane 15 of rows 0 and 2 to rows 1 and 3
    SPOTLIGHT_DPP_MAX(0x143, 0xc);   // lane 31 to rows 2 and 3
#undef SPOTLIGHT_DPP_MAX
    return __builtin_amdgcn_readlane(x, 63);
}

__device__ __forceinline__ float across_groups_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float across_groups_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// MT tiles of 16 rows a workgroup; its four wavefronts share out the keys of a run.  ONCE: no other workgroup reads them.
template <typename CT, typename QT, int MT, bool ONCE>
__global__ __launch_bounds__(kThreads, MT == 1 && sizeof(QT) == 2 ? 3 : 2) void cache_dense_kernel(DenseArgs a)
{
    constexpr int QP = sizeof(QT) == 2 ? 1 : 3, SP = QP == 1 ? 1 : 2;    // parts of q, sums of its products
    constexpr int kAux = ONCE ? 2 : 0;           // non-temporal
    constexpr bool TURN = MT == 1;               // keys pass through LDS (below)
    typedef Operand<CT> Op;
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    __shared__ alignas(16) float s_acc[kWaves][16][kHeadDim + 4];
    __shared__ uint32_t s_before;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int g = lane >> 4, i = lane & 15;
    // Workgroups go to the eight dies in turn: the tiles of one run and head, which read the same keys, to one die.
    uint32_t group = blockIdx.x, tile = 0;
    if (a.shares.tiles > 1) {
        const uint32_t eighth = a.shares.by_tiles8.over(blockIdx.x), in = blockIdx.x - eighth * a.shares.by_tiles8.d;
        group = eighth * 8 + in % 8;
        tile = in / 8;
    }
    const uint32_t number = a.shares.by_heads.over(group), heads = a.shares.by_heads.d, kv = group - number * heads;
    DenseRun run = find_run(a.shares, number, a.n_tokens);
    run.to_scalars();
    if (run.entry >= a.shares.batch) return;
    const uint32_t r0 = tile * (16 * MT), nsplit = run.nsplit;
    const int64_t head = static_cast<int64_t>(run.entry) * heads + kv, len = run.len;

    // The queries of the tile's rows: first of them, last of them, and those of the lane's rows.  Rows behind the
    // last repeat it.
    uint32_t q_least = 0, q_most = 0, query[MT], row[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) { row[t] = min(r0 + 16 * t + i, a.rows - 1); query[t] = 0; }
    if (a.n_q > 1) {
        const uint32_t last = min(r0 + 16 * MT, a.rows) - 1;
        q_least = r0 - a.by_queries.over(r0) * a.n_q;
        q_most = last - a.by_queries.over(last) * a.n_q;
        if (last - r0 >= a.n_q || q_least > q_most) { q_least = 0; q_most = a.n_q - 1; }
#pragma unroll
        for (int t = 0; t < MT; ++t) query[t] = row[t] - a.by_queries.over(row[t]) * a.n_q;
    }
    const int64_t before = len - a.n_q + 1;      // query x sees the keys before this + x

    // this wavefront's keys
    const int64_t c0 = static_cast<int64_t>(run.split) * run.chunk * kDenseUnit;
    const int64_t c1 = min(c0 + static_cast<int64_t>(run.chunk) * kDenseUnit, before + q_most);
    const int64_t share = (max(c1 - c0, static_cast<int64_t>(0)) + kDenseUnit - 1) / kDenseUnit * kStep, k0 = c0 + wave * share;
    const int n = static_cast<int>(min(max(c1 - k0, static_cast<int64_t>(0)), share));
    const int steps = (n + kStep - 1) / kStep;
    // the first steps, whose keys every row sees
    const int plain_steps = static_cast<int>(min(max(before + q_least - k0, static_cast<int64_t>(0)), static_cast<int64_t>(n))) / kStep;
    int sees[MT];                                // keys of the run that the lane's row sees
#pragma unroll
    for (int t = 0; t < MT; ++t) sees[t] = static_cast<int>(min(max(before + query[t] - k0, static_cast<int64_t>(0)), static_cast<int64_t>(n)));

    // Rows behind the run read as zeros: the buffer ends with it.  Offsets within it stay below 2^31 (the host
    // bounds a split), and all of them are in the instruction's checked part.
    const int64_t start = (head * a.Nmax + k0) * kHeadDim;
    const __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.k + start), 0, n * kHeadDim, 0x00020000);
    const __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.v + start), 0, n * kHeadDim, 0x00020000);
    u4 kreg[2][2];                               // lane (g, i): 32 bytes of the keys i and 16 + i
    u2 vreg[2][4];
    int koff = TURN ? lane * 16 : i * kHeadDim + g * 32, voff = g * (4 * kHeadDim) + i * 8;      // of the next step
    // Loaded like that, neighbouring lanes read different rows: 64 accesses of the vector cache an instruction.  With TURN an
    // instruction reads eight whole rows, a step further ahead, and the lanes exchange them through 4 KB of LDS that the
    // wavefront has to itself (its place for results): 16 bytes of row r at place (chunk ^ r % 8), without bank conflicts either
    // way.  Half as many cache accesses: 268 MB, 32 / 8 heads 50.6 -> 49.4 us, lengths of their own, 28 / 4 heads 57.6 -> 56.2 us.
    // With two tiles of rows vector and matrix instructions are the bound (112.4 -> 111.8 us).
    u4 kraw[TURN ? 4 : 1];
    uint8_t* const stage = reinterpret_cast<uint8_t*>(&s_acc[wave][0][0]);
    uint8_t* const put = stage + (lane >> 3) * kHeadDim + ((lane ^ lane >> 3) & 7) * 16;
    const int get = i * kHeadDim + ((2 * g ^ i) & 7) * 16;
    auto load_k = [&]() {
        if constexpr (TURN) {
#pragma unroll
            for (int t = 0; t < 4; ++t) kraw[t] = __builtin_amdgcn_raw_buffer_load_b128(kr, koff + t * (8 * kHeadDim), 0, kAux);
        } else {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    kreg[t][j] = __builtin_amdgcn_raw_buffer_load_b128(kr, koff + (t * (16 * kHeadDim) + j * 16), 0, kAux);
        }
        koff += kStep * kHeadDim;
    };
    // The keys of the next step, and loads of those behind them.  (LDS serves a wavefront in order: it needs no wait.)
    auto next_k = [&]() {
        if constexpr (TURN) {
#pragma unroll
            for (int t = 0; t < 4; ++t) *reinterpret_cast<u4*>(put + t * (8 * kHeadDim)) = kraw[t];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j) kreg[t][j] = *reinterpret_cast<const u4*>(stage + (get ^ 16 * j) + t * (16 * kHeadDim));
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
        load_k();
    };
    auto load_v = [&]() {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                vreg[t][r] = __builtin_amdgcn_raw_buffer_load_b64(vr, voff + (t * (16 * kHeadDim) + r * kHeadDim), 0, kAux);
        voff += kStep * kHeadDim;
    };
    // on their way while the queries and scales are read
    load_k();
    load_v();

    const float* ks = a.k_scale + head * a.blocks;
    const float* vs = a.v_scale + head * a.blocks;
    const uint32_t last_block = static_cast<uint32_t>(k0 + (n > 0 ? n - 1 : 0)) >> a.shift;   // tokens are below 2^31

    // the largest scale of the run's values, as bits (NaN is more than infinity), and how far the least lies below infinity
    int unit_bits = 0, low_bits = 0;
    if (n > 0)
        for (uint32_t j = (static_cast<uint32_t>(k0) >> a.shift) + lane; j <= last_block; j += 64) {
            const int v = reinterpret_cast<const int*>(vs)[j];
            unit_bits = max(unit_bits, v);
            low_bits = max(low_bits, kInf - v);
        }
    h8 qf[MT][QP][4];
    float factor[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int ex = load_row<QT, QP, 4, 4>(static_cast<const QT*>(a.q) + (head * a.rows + row[t]) * kHeadDim + g * 32, a.negate, qf[t]);
        factor[t] = ldexpf(a.scale2, ex);
    }
    unit_bits = wave_max(unit_bits);
    low_bits = wave_max(low_bits);
    const bool apart = unit_bits > kInf || unit_bits - (kInf - low_bits) > kFar << 23;       // the same for the wavefront
    if (unit_bits == 0) unit_bits = 127 << 23;
    const int to_sum = apart ? 0 : (unit_bits >> 23) - 127 - kVUp + kSumUp;                  // from the products' unit, log2
    unit_bits -= (127 + kVUp) << 23;

    f4 acc[MT][8];
    // kPUp less the maximum (infinite: none yet), and the lane's sum of weights.  Maxima are rounded up to whole numbers:
    // differences of them, in rescaling and in joining partial results, are then exact powers of two.
    float base[MT], l[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        base[t] = INFINITY;
        l[t] = 0.0f;
#pragma unroll
        for (int d = 0; d < 8; ++d) acc[t][d] = f4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    float next_ks[2];
    int next_vs[2];                              // as bits
    auto load_scales = [&](int s) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const uint32_t blk = min((static_cast<uint32_t>(k0) + s * kStep + 16 * t) >> a.shift, last_block);
            next_ks[t] = ks[blk];
            next_vs[t] = reinterpret_cast<const int*>(vs)[blk];
        }
    };
    if (steps > 0) load_scales(0);
    if constexpr (TURN) next_k();

    // alone: the blocks' values have products of their own
    auto step = [&](int s, auto masked, auto alone) {
        constexpr bool ALONE = decltype(alone)::value;
        // the scales of this step; the next one's are on their way from here on
        float kscale[2], vscale[2];
        typename Op::Ratio ratio[2];
        bool nan_block[2] = {false, false};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            kscale[t] = next_ks[t];
            if constexpr (ALONE) {
                nan_block[t] = next_vs[t] > kInf;
                vscale[t] = nan_block[t] ? 0.0f : __int_as_float(next_vs[t]);
                ratio[t] = Op::ratio(1.0f);
            } else {
                ratio[t] = Op::ratio(__int_as_float(next_vs[t] - unit_bits));   // powers of two: a difference of exponents
            }
        }
        load_scales(s + 1);
        // scores
        f4 sc[MT][SP][2];                                       // of the first part of q, and of the others
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int p = 0; p < SP; ++p) sc[t][p][0] = sc[t][p][1] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const h8 kf = Op::row(kreg[kt][c / 2][2 * (c % 2)], kreg[kt][c / 2][2 * (c % 2) + 1]);
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int p = 0; p < QP; ++p) sc[t][p ? SP - 1 : 0][kt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf, qf[t][p][c], sc[t][p ? SP - 1 : 0][kt], 0, 0, 0);
            }
        next_k();
        // softmax
        h8 hi[MT], lo[MT];
        float back[MT][2];                                      // takes a block's products to the sum's unit
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            float f[2], x[8];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) f[kt] = factor[t] * kscale[kt];
            // the large part and the number first: where the weight is large they nearly cancel, and little is rounded off
            auto score = [&](int e, float add) {
                const float y = __builtin_fmaf(sc[t][0][e / 4][e % 4], f[e / 4], add);
                return SP == 2 ? __builtin_fmaf(sc[t][SP - 1][e / 4][e % 4], f[e / 4], y) : y;
            };
            float top = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = score(e, base[t]);
                if constexpr (decltype(masked)::value)
                    if (s * kStep + 16 * (e / 4) + 4 * g + e % 4 >= sees[t]) x[e] = -INFINITY;
                top = fmaxf(top, x[e]);
            }
            if (__any(!(top <= (ALONE ? kPUp : kPUp + kSlack)))) {   // also before the first maximum
                float high = -INFINITY;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[e] = score(e, -0.0f);
                    if constexpr (decltype(masked)::value)
                        if (s * kStep + 16 * (e / 4) + 4 * g + e % 4 >= sees[t]) x[e] = -INFINITY;
                    high = fmaxf(high, x[e]);
                }
                high = across_groups_max(high);
                if (high > -INFINITY) {
                    const float to = fminf(kPUp - ceilf(high), base[t]);
                    const float down = __builtin_amdgcn_exp2f(to - base[t]);      // 0 before the first maximum
                    l[t] *= down;
#pragma unroll
                    for (int d = 0; d < 8; ++d) acc[t][d] *= down;
                    base[t] = to;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] > -INFINITY ? x[e] + base[t] : x[e];
            }
            float up[2] = {0.0f, 0.0f};                     // what the weights in the products are scaled by, log2
            if constexpr (ALONE) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    float most = -400.0f;                       // less weighs 0 whatever its value
#pragma unroll
                    for (int e = 4 * kt; e < 4 * kt + 4; ++e) most = fmaxf(most, x[e]);
                    most = ceilf(across_groups_max(most));
                    up[kt] = kPUp - most;
                    back[t][kt] = ldexpf(vscale[kt], static_cast<int>(-up[kt]) + kSumUp);
                }
            }
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f(x[e]);
                x[e] = ALONE ? __builtin_amdgcn_exp2f(x[e] + up[e / 4]) : w[e];
            }
            l[t] += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
            h2 h[4], r[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                h[e] = to_half(x[2 * e], x[2 * e + 1]);
                r[e] = to_half(less_low(x[2 * e], h[e]), less_high(x[2 * e + 1], h[e]));
            }
            hi[t] = join(h[0], h[1], h[2], h[3]);
            lo[t] = join(r[0], r[1], r[2], r[3]);
        }
        // A row's weight 0 must not meet a NaN of a key that it does not see: the products are formed without NaN, and the
        // sums of the rows that see one become NaN.
        if constexpr (ALONE) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
                if ((nan_block[0] && s * kStep < sees[t]) || (nan_block[1] && s * kStep + 16 < sees[t]))
#pragma unroll
                    for (int d = 0; d < 8; ++d) acc[t][d] += __builtin_nanf("");
        }
        if constexpr (decltype(masked)::value && CT::kHasNaN) {
            auto nan_bytes = [](uint32_t v) { return ((v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; };      // 7f and ff
            uint32_t any = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) any |= nan_bytes(vreg[e / 4][e % 4].x) | nan_bytes(vreg[e / 4][e % 4].y);
            if (__any(any != 0)) {
                h8 sees_key[MT];
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sees_key[t][j] = s * kStep + 16 * (j / 4) + 4 * g + j % 4 < sees[t] ? 1.0f16 : 0.0f16;
#pragma unroll
                for (int d = 0; d < 8; ++d) {
                    h8 is_nan;
#pragma unroll
                    for (int j = 0; j < 8; ++j) is_nan[j] = (vreg[j / 4][j % 4][d / 4] >> (8 * (d % 4)) & 0x7fu) == 0x7fu ? 1.0f16 : 0.0f16;
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        const f4 hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(is_nan, sees_key[t], f4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (hit[r] != 0.0f) acc[t][d][r] = __builtin_nanf("");
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    u2& v = vreg[e / 4][e % 4];
                    v = u2{v.x & ~((nan_bytes(v.x) >> 7) * 0xffu), v.y & ~((nan_bytes(v.y) >> 7) * 0xffu)};
                }
            }
        }
        // weighted values: four columns of the lane at a time
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            h2 col[4][4];                       // [pair of keys][column]
#pragma unroll
            for (int pr = 0; pr < 4; ++pr) Op::columns(vreg[pr / 2][2 * (pr % 2)][w], vreg[pr / 2][2 * (pr % 2) + 1][w], ratio[pr / 2], col[pr]);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const h8 vf = join(col[0][c], col[1][c], col[2][c], col[3][c]);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    if constexpr (ALONE) {
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) {
                            f4 sum = __builtin_amdgcn_mfma_f32_16x16x16f16(half_of(vf, kt), half_of(hi[t], kt), f4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
                            sum = __builtin_amdgcn_mfma_f32_16x16x16f16(half_of(vf, kt), half_of(lo[t], kt), sum, 0, 0, 0);
#pragma unroll
                            for (int r = 0; r < 4; ++r) acc[t][4 * w + c][r] = __builtin_fmaf(sum[r], back[t][kt], acc[t][4 * w + c][r]);
                        }
                    } else {
                        acc[t][4 * w + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, hi[t], acc[t][4 * w + c], 0, 0, 0);
                        acc[t][4 * w + c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, lo[t], acc[t][4 * w + c], 0, 0, 0);
                    }
                }
                if constexpr (ALONE) __builtin_amdgcn_sched_barrier(0);      // a column at a time: no registers for more
            }
        }
        load_v();
    };
    int s = 0;
    if (apart)
        for (; s < steps; ++s) step(s, Flag<true>{}, Flag<true>{});
    for (; s < plain_steps; ++s) step(s, Flag<false>{}, Flag<false>{});
    for (; s < steps; ++s) step(s, Flag<true>{}, Flag<false>{});

    // the wavefronts' results, joined: lane (g, i) has columns 32g .. 32g+31 of row i
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const float sum = across_groups_sum(l[t]);
        if (t) __syncthreads();
        if (g == 0) { s_m[wave][i] = kPUp - base[t]; s_l[wave][i] = ldexpf(sum, kSumUp); }
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int d = 0; d < 8; d += 4)
                *reinterpret_cast<f4*>(&s_acc[wave][i][g * 32 + r * 8 + d]) =
                    f4{ldexpf(acc[t][d][r], to_sum), ldexpf(acc[t][d + 1][r], to_sum), ldexpf(acc[t][d + 2][r], to_sum), ldexpf(acc[t][d + 3][r], to_sum)};
        __syncthreads();
        const int left = static_cast<int>(a.rows - min(r0 + 16 * t, a.rows));
        for (int e = tid; e < 16 * 64 && e / 64 < left; e += kThreads) {
            const int row = e / 64, pair = e % 64;
            Join j;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) j.add(f32x2{s_m[w][row], s_l[w][row]}, reinterpret_cast<const f32x2*>(s_acc[w][row])[pair]);
            if (nsplit == 1)
                reinterpret_cast<f32x2*>(a.out + (head * a.rows + r0 + 16 * t + row) * kHeadDim)[pair] = j.l != 0.0f ? f32x2{j.a.x / j.l, j.a.y / j.l} : f32x2{0.0f, 0.0f};
            else
                put_part(a.part, static_cast<size_t>(group * a.shares.tiles + tile) * a.shares.tile_rows + 16 * t + row, pair, j.m, j.l, j.a);
        }
    }
    // (No store may come before the scales have been read: they would not be scalar loads.)
    if (kv == 0 && tile == 0 && run.split == 0 && tid == 0) a.runs[run.entry] = make_uint2(run.first, nsplit);
    if (nsplit == 1 || !a.part.arrived) return;
    const uint32_t first = (run.first * heads + kv) * a.shares.tiles + tile;          // the same tile in the sequence's first run
    // sequences with as many runs begin at least that many runs apart (both are small: the quotient is off by less than 1 / 128)
    const uint32_t like = static_cast<uint32_t>((static_cast<float>(run.first) + 0.5f) * __builtin_amdgcn_rcpf(static_cast<float>(nsplit)));
    if (arrives_last(a.part, (like * heads + kv) * a.shares.tiles + tile, nsplit, &s_before))
        join_rows<kThreads, 16>(a.part, first * a.shares.tile_rows, heads * a.shares.tiles * a.shares.tile_rows, min(16u * MT, a.rows - r0), nsplit,
                                a.out + (head * a.rows + r0) * kHeadDim, reinterpret_cast<f32x2*>(&s_acc[0][0][0]));
}

// Codes that no other workgroup reads and no cache would hold until the next call: 268 MB, 32 / 8 heads 50.4 -> 45.3 us, with
// lengths of their own, 28 / 4 heads 57.2 -> 52.3 us, 1074 MB 189 -> 162 us,
// with 32 rows 206 -> 183 us; but 134 MB, called again, 27.3 -> 29.4 us.
template <typename CT, typename QT>
void launch_mt(StageTimer& timer, const DenseArgs& a, const DensePlan& d)
{
    const int64_t bytes = 2 * a.n_tokens * kHeadDim * a.shares.batch * a.shares.by_heads.d;
    const bool once = a.shares.tiles == 1 && bytes >= kCacheBytes;
    auto kern = once ? cache_dense_kernel<CT, QT, 1, true> : cache_dense_kernel<CT, QT, 1, false>;
    if constexpr (sizeof(QT) == 2)
        if (d.row_tiles == 2) kern = once ? cache_dense_kernel<CT, QT, 2, true> : cache_dense_kernel<CT, QT, 2, false>;
    timer.launch(kern, dim3(d.grid), dim3(kThreads), 0, a);
}

}  // namespace

namespace cache {
int plan_dense(const Plan& p, int n_cus, int64_t n_tokens, int n_q, const int32_t* lens, DensePlan* d, int code_type)
{
    const int64_t rows = static_cast<int64_t>(p.G) * n_q;
    if (rows > 1 << 24) return SPOTLIGHT_ERR_UNSUPPORTED;
    DenseShares& s = d->shares;
    // Two tiles of rows a workgroup share the reads of codes and their conversion; one has the faster loads, and shorter work
    // before and behind the keys.  Up to 32 rows, two pay where the codes are read from memory once and pass the last-level cache by, and
    // for integers, whose conversion takes twice the instructions, up to 24 rows from 96 MB on; of more rows, whose codes several
    // workgroups read, where there is enough to do: rows times bytes.  With one / two, us, nothing in a cache, 8 key-value
    // heads, E4M3:
    //     MB    17 rows      32 rows      33 rows      64 rows      128 rows     256 rows     1024 rows
    //      4    13.4 / 14.9  13.4 / 17.4  15.1 / 19.7  15.3 / 19.8  16.6 / 22.1  16.6 / 22.1  21.9 / 23.1
    //     16    15.3 / 16.7  15.9 / 19.5  18.0 / 21.4  18.1 / 22.1  23.8 / 27.6  35.6 / 39.1  72.9 / 60.5
    //     32    19.1 / 20.5  19.9 / 21.5  21.4 / 23.2  23.4 / 23.9  30.4 / 29.5  45.7 / 40.9  140 / 117
    //     64    25.4 / 29.7  26.4 / 32.2  29.6 / 33.4  33.7 / 33.7  48.8 / 45.1  79.1 / 66.7
    //    128    38.2 / 40.9  38.5 / 42.6  45.8 / 49.3  53.4 / 49.7  84.5 / 73.4  154 / 124
    //    192    47.6 / 50.0  48.6 / 53.0  61.0 / 60.9  73.0 / 62.9  123 / 102    226 / 180
    //    256    61.0 / 56.3  61.4 / 60.5  78.9 / 77.7  94.1 / 78.4  162 / 132    297 / 232
    //    512    111 / 94     111 / 98     143 / 139    173 / 143    310 / 247    582 / 449
    // Integers, two against one, mean of 10 layouts: 17 rows 64 MB +5 %, 96 MB -1 %, 144 MB -3 %, 208 MB -4 %; 24 rows +8, +2, -1, -2 %; 32
    // rows +11, +5, +3, 0 %.  E4M3: 17 rows +9, +3, +1, +2 %; 32 rows +16, +10, +7, +5 %.
    // Over 1418 such cells (1 to 128 heads of sequences and keys, both codes, 1 to 512 MB, 17 to 2048 rows) the rule is 0.5 % behind the faster
    // kernel on average, in 57 cells by over 5 %, at worst by 18 % (64 MB in 128 heads, 64 rows).  Binary32 rows, three parts each,
    // leave no registers for two (512 rows 165 / 173 us, 17 rows 34.7 / 45.4).
    const int64_t bytes = 2 * n_tokens * kHeadDim * p.B * p.Hkv;
    const int64_t few = code_type == SPOTLIGHT_I8 && rows <= 24 ? kCacheBytes / 8 * 3 : kCacheBytes;
    const bool two = rows > 32 ? rows >= (12 * kCacheBytes + bytes - 1) / bytes : rows > 16 && bytes >= few;
    d->row_tiles = two && p.kv_dtype == SPOTLIGHT_BF16 ? 2 : 1;
    const int64_t most_rows = 16 * d->row_tiles, tiles = (rows + most_rows - 1) / most_rows, per = tiles * p.Hkv;   // workgroups of a run
    s.lens = lens;
    s.batch = static_cast<uint32_t>(p.B);
    s.tiles = static_cast<uint32_t>(tiles);
    s.tile_rows = static_cast<uint32_t>(rows < most_rows ? rows : most_rows);
    const int64_t units = (n_tokens + kDenseUnit - 1) / kDenseUnit, B = p.B;
    // Runs of all sequences: two workgroups a compute unit, which it holds at once (of the kernel with 16 rows it would hold
    // three; with those, lengths that differ: 38 MB of codes 17.1 -> 17.8 us, 258 MB 54.7 -> 52.4 us, 711 MB 123 -> 124 us), as
    // far as there is room for their partial results.
    const int64_t hold = static_cast<int64_t>(n_cus) * 2 / per, room = p.dense_rows / (s.tile_rows * per);
    int64_t runs, most, chunk;
    s.most_runs = 0;
    if (!lens) {
        most = std::min({hold / B, room / B, units});
        const int64_t need = (n_tokens + kDenseMostKeys - 1) / kDenseMostKeys;
        if (most < need) {
            most = need;
            if (need > 1 && need > room / B) return SPOTLIGHT_ERR_UNSUPPORTED;
        }
        chunk = (units + most - 1) / most;
        most = (units + chunk - 1) / chunk;
        runs = B * most;
    } else {
        runs = std::min({std::max(hold, 2 * B), room, B * units});
        if (units > 1 && runs > B) {
            s.most_runs = static_cast<uint32_t>(runs);
            chunk = std::min((B * units + runs - B - 1) / (runs - B), units);
            most = std::min(units, runs - B + 1);
        } else {
            runs = B;
            chunk = units;
            most = 1;
        }
    }
    if (chunk * kDenseUnit > kDenseMostKeys + kDenseUnit) return SPOTLIGHT_ERR_UNSUPPORTED;
    const int64_t grid = (runs * p.Hkv + 7) / 8 * 8 * tiles;
    if (grid >= 1 << 24) return SPOTLIGHT_ERR_UNSUPPORTED;      // a launch has less than 2^32 threads a dimension
    s.units = static_cast<uint32_t>(units);
    s.chunk = static_cast<uint32_t>(chunk);
    s.nsplit = static_cast<uint32_t>(most);
    s.by_nsplit = fast_div(s.nsplit);
    s.by_most = fast_div(s.most_runs ? s.most_runs : 1);
    s.by_spare = fast_div(s.most_runs ? s.most_runs - s.batch : 1);
    s.by_heads = fast_div(static_cast<uint32_t>(p.Hkv));
    s.by_tiles8 = fast_div(8 * s.tiles);
    d->grid = static_cast<uint32_t>(tiles == 1 ? runs * p.Hkv : grid);
    d->splits = most > 1;
    d->about = runs / B;
    d->joins = joins_in_place(runs * per, s.tile_rows, most);
    return SPOTLIGHT_OK;
}
}  // namespace cache

int launch_cache_dense(spotlight_ctx* ctx, const void* q, const spotlight_cache& c, int64_t n_tokens, int n_q, const int32_t* lens,
                       float scale, float* out)
{
    const Plan& p = ctx->plan;
    DenseArgs a;
    a.q = q;
    a.k = static_cast<const uint8_t*>(c.k);
    a.v = static_cast<const uint8_t*>(c.v);
    a.k_scale = c.k_scale;
    a.v_scale = c.v_scale;
    a.part.ml = reinterpret_cast<unsigned long long*>(ctx->workspace + p.off_dense_ml);
    a.part.acc = reinterpret_cast<unsigned long long*>(ctx->workspace + p.off_dense_acc);
    a.out = out;
    a.Nmax = p.Nmax;
    a.blocks = (p.Nmax + c.block_tokens - 1) / c.block_tokens;
    a.n_tokens = n_tokens;
    a.rows = static_cast<uint32_t>(p.G) * static_cast<uint32_t>(n_q);
    a.n_q = static_cast<uint32_t>(n_q);
    a.shift = __builtin_ctz(static_cast<unsigned>(c.block_tokens));
    a.scale2 = fabsf(scale) * kLog2e;
    a.negate = scale < 0.0f;

    DensePlan d;
    const int rc = plan_dense(p, ctx->n_cus, n_tokens, n_q, lens, &d, c.code_type);
    if (rc != SPOTLIGHT_OK) return rc;
    a.shares = d.shares;
    a.by_queries = fast_div(a.n_q);
    a.runs = reinterpret_cast<uint2*>(ctx->workspace + p.off_runs);
    a.part.arrived = d.joins ? reinterpret_cast<uint32_t*>(ctx->workspace + p.off_arrived) : nullptr;
    const bool done = !d.splits || d.joins;                   // nothing is left to merge
    {
        StageTimer timer(ctx, SPOTLIGHT_STAGE_ATTEND);
        if (timer.rec) timer.rec->whole = done;
        if (p.kv_dtype == SPOTLIGHT_BF16) {
            if (c.code_type == SPOTLIGHT_E4M3) launch_mt<E4M3, bf16_raw>(timer, a, d);
            else launch_mt<I8, bf16_raw>(timer, a, d);
        } else {
            if (c.code_type == SPOTLIGHT_E4M3) launch_mt<E4M3, float>(timer, a, d);
            else launch_mt<I8, float>(timer, a, d);
        }
        if (hipGetLastError() != hipSuccess) return SPOTLIGHT_ERR_HIP;
    }
    if (done) return SPOTLIGHT_OK;
    const MergeRows r{static_cast<int64_t>(p.B) * p.Hkv * a.rows, 0, a.runs, fast_div(a.rows), fast_div(static_cast<uint32_t>(p.Hkv)),
                      fast_div(16u * d.row_tiles), d.shares.tiles, d.shares.tile_rows, p.dense_rows};
    return launch_cache_merge(ctx, a.part.ml, a.part.acc, r, d.about, out);
}

}  // namespace spotlight
