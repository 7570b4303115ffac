// Writing rows into the 8-bit cache and reading them back.
//
// Both move each byte once and are bound by memory.  A workgroup of the write has one block of tokens of
// one head of K or of V: it holds the block's new rows in registers, takes their largest magnitude, and
// encodes them, so that a row is read once.  Only the block that the first new row falls into can hold
// earlier rows; they keep the larger of the two scales, and where that is not their own, their codes are
// decoded, scaled by the (negative) power of two between the scales and rounded again.
#include "cache.h"

namespace spotlight {
using namespace cache;
namespace {

template <typename XT> struct Vec;      // 16 bytes of a row
template <> struct Vec<bf16_raw> {
    static constexpr int kElems = 8;
    static __device__ __forceinline__ void unpack(const uint4& u, float (&o)[8])
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { o[2 * i] = __uint_as_float(w[i] << 16); o[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    // largest magnitude, as the bits of a float
    static __device__ __forceinline__ uint32_t largest(const uint4& u)
    {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) a = max(max(a, (w[i] << 16) & 0x7fffffffu), w[i] & 0x7fff0000u);
        return a;
    }
};
template <> struct Vec<float> {
    static constexpr int kElems = 4;
    static __device__ __forceinline__ void unpack(const uint4& u, float (&o)[4])
    {
        o[0] = __uint_as_float(u.x); o[1] = __uint_as_float(u.y); o[2] = __uint_as_float(u.z); o[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint32_t largest(const uint4& u)
    {
        return max(max(u.x & 0x7fffffffu, u.y & 0x7fffffffu), max(u.z & 0x7fffffffu, u.w & 0x7fffffffu));
    }
};

constexpr uint32_t kInfBits = 0x7f800000u;

// Of kCacheBytes of rows and more, bfloat16, 32 heads of 131072 rows 558 -> 508 us, 16 of 65536 140 -> 125 us, binary32, 8 of 32768
// 61 -> 54 us; of less, 8 of 32768 in bfloat16, 134 MB, 31.2 -> 32.3 us, and a smaller write that is read back at once
// 21.2 -> 24.6 us.
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_once(const uint4* p)
{
    const u4 v = __builtin_nontemporal_load(reinterpret_cast<const u4*>(p));
    return make_uint4(v.x, v.y, v.z, v.w);
}

__device__ __forceinline__ void store_once(uint32_t* p, uint32_t v) { __builtin_nontemporal_store(v, p); }
__device__ __forceinline__ void store_once(uint2* p, uint2 v)
{
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    __builtin_nontemporal_store(u2{v.x, v.y}, reinterpret_cast<u2*>(p));
}

// kElems codes: one word or two
template <int E> struct CodeWord;
template <> struct CodeWord<4> { typedef uint32_t type; };
template <> struct CodeWord<8> { typedef uint2 type; };

template <typename CT>
__device__ __forceinline__ uint32_t encode4(const float* x, float inv, bool odd)
{
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        y[i] = x[i] * inv;
        // where the block has an infinity or a NaN (rare, the same for the workgroup)
        if (odd && !(fabsf(x[i]) < INFINITY)) y[i] = CT::kHasNaN ? __uint_as_float(0x7fc00000u) : 0.0f;
    }
    return CT::encode(y);
}

// Maximum over the workgroup, in every thread.  `lds` is free again after the next barrier.
__device__ __forceinline__ uint32_t workgroup_max(uint32_t a, uint32_t* lds)
{
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) a = max(a, static_cast<uint32_t>(__shfl_xor(static_cast<int>(a), off)));
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = a;
    __syncthreads();
    a = lds[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) a = max(a, lds[w]);
    return a;
}

struct RowsArgs {
    const void* x[2];         // new rows of K and of V
    void* out[2];             // rows read back
    uint8_t* codes[2];
    float* scale[2];
    const int32_t* first;
    const int32_t* count;
    int64_t t0, n, Nmax, blocks;   // blocks: scales of a head
    int Hkv;
    int shift;                     // log2 of the tokens of a block
};

template <typename CT, typename XT, int TB, bool ONCE>
__global__ __launch_bounds__(kThreads) void write_kernel(RowsArgs a)
{
    constexpr int E = Vec<XT>::kElems;
    constexpr int VR = kHeadDim / E;                  // vectors of a row
    constexpr int IT = TB * VR / kThreads;            // vectors of a thread
    static_assert(IT >= 1 && TB * VR % kThreads == 0, "a block is shared out evenly");
    typedef typename CodeWord<E>::type Codes;
    __shared__ uint32_t s_max[2][kThreads / 64];

    const int tid = threadIdx.x, z = blockIdx.z;
    const int64_t head = blockIdx.y, b = head / a.Hkv;
    const int64_t start = a.t0 + (a.first ? a.first[b] : 0);
    const int64_t rows = a.count ? min(max(static_cast<int64_t>(a.count[b]), static_cast<int64_t>(0)), a.n) : a.n;
    const int64_t lo = max(start, static_cast<int64_t>(0)), hi = min(start + rows, a.Nmax);
    if (lo >= hi) return;
    const uint4* x = static_cast<const uint4*>(a.x[z]) + head * a.n * VR;
    Codes* codes = reinterpret_cast<Codes*>(a.codes[z]) + head * a.Nmax * VR;
    float* scale = a.scale[z] + head * a.blocks;

    for (int64_t blk = lo / TB + blockIdx.x; blk * TB < hi; blk += gridDim.x) {
        const int64_t r0 = blk * TB;
        const bool keeps = r0 < lo;                   // rows from before
        const float old = keeps ? scale[blk] : 0.0f;
        uint4 u[IT];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int v = i * kThreads + tid;
            const int64_t row = r0 + v / VR;
            u[i] = make_uint4(0u, 0u, 0u, 0u);
            if (row >= lo && row < hi) {
                const uint4* from = x + (row - start) * VR + v % VR;
                u[i] = ONCE ? load_once(from) : *from;
            }
        }
#pragma unroll
        for (int i = 0; i < IT; ++i) most = max(most, Vec<XT>::largest(u[i]));
        __syncthreads();                              // the last block's maxima have been read
        most = workgroup_max(most, s_max[0]);
        const bool odd = most >= kInfBits;
        if (odd) {
            // an infinity or a NaN: the scale is that of the finite values
            most = 0;
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                float f[E];
                Vec<XT>::unpack(u[i], f);
#pragma unroll
                for (int e = 0; e < E; ++e) most = max(most, fabsf(f[e]) < INFINITY ? __float_as_uint(f[e]) & 0x7fffffffu : 0u);
            }
            most = workgroup_max(most, s_max[1]);
        }
        int ex = least_exponent<CT>(most);
        const bool poisoned = !CT::kHasNaN && (odd || old != old);   // integers have no NaN: the block's scale holds it
        if (keeps) {
            const int was = static_cast<int>(__float_as_uint(old) >> 23) - 127;
            if (was >= ex || poisoned) {
                if (was > ex && was < 128) ex = was;
            } else {
                // the scale grows: the earlier rows' codes follow it
                const float down = ldexpf(1.0f, was - ex);
                for (int v = tid; v < static_cast<int>(lo - r0) * VR; v += kThreads) {
                    Codes c = codes[r0 * VR + v];
                    uint32_t* w = reinterpret_cast<uint32_t*>(&c);
#pragma unroll
                    for (int j = 0; j < E / 4; ++j) {
                        float f[4];
                        CT::decode(w[j], f);
#pragma unroll
                        for (int e = 0; e < 4; ++e) f[e] *= down;
                        w[j] = CT::encode(f);
                    }
                    codes[r0 * VR + v] = c;
                }
            }
        }
        const float inv = power_of_two(-ex);
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int v = i * kThreads + tid;
            const int64_t row = r0 + v / VR;
            if (row >= lo && row < hi) {
                float f[E];
                Vec<XT>::unpack(u[i], f);
                Codes c;
                uint32_t* w = reinterpret_cast<uint32_t*>(&c);
#pragma unroll
                for (int j = 0; j < E / 4; ++j) w[j] = encode4<CT>(f + 4 * j, inv, odd);
                if constexpr (ONCE) store_once(codes + r0 * VR + v, c);
                else codes[r0 * VR + v] = c;
            }
        }
        if (tid == 0) scale[blk] = poisoned ? __uint_as_float(0x7fc00000u) : power_of_two(ex);
    }
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)
{
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(lo), static_cast<__bf16>(hi)});
}

// U vectors of 16 bytes a thread, loads first.  Beyond the last-level cache two measured best (32 heads of 131072 rows, bfloat16, with
// 1 / 2 / 4 / 8: 525 / 540 / 560 / 564 us; 16 of 65536, binary32: 265 / 218 / 234 / 238 us), below it four (4 heads of 10007
// rows just written, binary32, with 2 / 4: 12.5 / 10.3 us).
template <typename CT, typename XT, int U>
__global__ __launch_bounds__(kThreads) void read_kernel(RowsArgs a)
{
    constexpr int E = Vec<XT>::kElems, VR = kHeadDim / E;
    typedef typename CodeWord<E>::type Codes;
    const int tid = threadIdx.x, z = blockIdx.z;
    if (!a.out[z]) return;
    const int64_t head = blockIdx.y, b = head / a.Hkv;
    const int64_t start = a.t0 + (a.first ? a.first[b] : 0);
    uint4* out = static_cast<uint4*>(a.out[z]) + head * a.n * VR;
    const Codes* codes = reinterpret_cast<const Codes*>(a.codes[z]) + head * a.Nmax * VR;
    const float* scale = a.scale[z] + head * a.blocks;
    const int64_t total = a.n * VR;
    for (int64_t v0 = static_cast<int64_t>(blockIdx.x) * (U * kThreads); v0 < total; v0 += static_cast<int64_t>(gridDim.x) * (U * kThreads)) {
        Codes c[U];
        float s[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t v = v0 + i * kThreads + tid, row = start + v / VR;
            c[i] = Codes{};
            s[i] = 0.0f;
            if (v < total && row >= 0 && row < a.Nmax) {
                c[i] = codes[row * VR + v % VR];
                s[i] = scale[row >> a.shift];
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int64_t v = v0 + i * kThreads + tid;
            if (v >= total) continue;
            const uint32_t* w = reinterpret_cast<const uint32_t*>(&c[i]);
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < E / 4; ++j) {
                float f[4];
                CT::decode(w[j], f);
                if constexpr (E == 4) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = __float_as_uint(f[e] * s[i]);
                } else {
                    // exact: a code has at most 7 significant bits (below binary32's normal range it rounds)
                    o[2 * j] = bf16_pair(f[0] * s[i], f[1] * s[i]);
                    o[2 * j + 1] = bf16_pair(f[2] * s[i], f[3] * s[i]);
                }
            }
            out[v] = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

template <typename CT, typename XT, bool ONCE>
void launch_write_block(spotlight_ctx* ctx, const RowsArgs& a, int block, const dim3& grid)
{
    auto kern = block == 16 ? write_kernel<CT, XT, 16, ONCE> : block == 32 ? write_kernel<CT, XT, 32, ONCE>
              : block == 64 ? write_kernel<CT, XT, 64, ONCE> : write_kernel<CT, XT, 128, ONCE>;
    hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, ctx->stream, a);
}

// Workgroups beyond this many take a second turn, so that a grid stays within the launch limits.
constexpr int64_t kMaxGridX = 1 << 20;

template <typename CT, typename XT>
void launch_write(spotlight_ctx* ctx, const RowsArgs& a, int block, const dim3& grid)
{
    const int64_t bytes = 2 * a.n * ctx->plan.B * ctx->plan.Hkv * kHeadDim * static_cast<int64_t>(sizeof(XT));
    if (bytes >= kCacheBytes) launch_write_block<CT, XT, true>(ctx, a, block, grid);
    else launch_write_block<CT, XT, false>(ctx, a, block, grid);
}

template <typename CT, typename XT, int U>
void launch_read_vectors(spotlight_ctx* ctx, const RowsArgs& a)
{
    const int64_t wgs = (a.n * (kHeadDim / Vec<XT>::kElems) + U * kThreads - 1) / (U * kThreads);
    const dim3 grid(static_cast<unsigned>(wgs < kMaxGridX ? wgs : kMaxGridX), static_cast<unsigned>(ctx->plan.B * ctx->plan.Hkv), 2);
    hipLaunchKernelGGL((read_kernel<CT, XT, U>), grid, dim3(kThreads), 0, ctx->stream, a);
}

template <typename CT, typename XT>
void launch_read(spotlight_ctx* ctx, const RowsArgs& a)
{
    const int64_t bytes = 2 * a.n * ctx->plan.B * ctx->plan.Hkv * kHeadDim * static_cast<int64_t>(sizeof(XT));
    if (bytes >= kCacheBytes) launch_read_vectors<CT, XT, 2>(ctx, a);
    else launch_read_vectors<CT, XT, 4>(ctx, a);
}

RowsArgs rows_args(const spotlight_ctx* ctx, const spotlight_cache& c, int64_t t0, int64_t n, const int32_t* first, const int32_t* count)
{
    RowsArgs a;
    a.x[0] = a.x[1] = nullptr;
    a.out[0] = a.out[1] = nullptr;
    a.codes[0] = static_cast<uint8_t*>(c.k);
    a.codes[1] = static_cast<uint8_t*>(c.v);
    a.scale[0] = c.k_scale;
    a.scale[1] = c.v_scale;
    a.first = first;
    a.count = count;
    a.t0 = t0;
    a.n = n;
    a.Nmax = ctx->plan.Nmax;
    a.blocks = (ctx->plan.Nmax + c.block_tokens - 1) / c.block_tokens;
    a.Hkv = ctx->plan.Hkv;
    a.shift = __builtin_ctz(static_cast<unsigned>(c.block_tokens));
    return a;
}

}  // namespace

int launch_cache_write(spotlight_ctx* ctx, const spotlight_cache& c, const void* K, const void* V, int64_t t0, int64_t n,
                       const int32_t* first, const int32_t* count)
{
    const Plan& p = ctx->plan;
    RowsArgs a = rows_args(ctx, c, t0, n, first, count);
    a.x[0] = K;
    a.x[1] = V;
    const int64_t T = c.block_tokens;
    // blocks that n rows touch, from t0 on or wherever they begin
    const int64_t nblk = first ? (n + T - 2) / T + 1 : (t0 % T + n + T - 1) / T;
    const dim3 grid(static_cast<unsigned>(nblk < kMaxGridX ? nblk : kMaxGridX), static_cast<unsigned>(p.B * p.Hkv), 2);
    if (p.kv_dtype == SPOTLIGHT_BF16) {
        if (c.code_type == SPOTLIGHT_E4M3) launch_write<E4M3, bf16_raw>(ctx, a, c.block_tokens, grid);
        else launch_write<I8, bf16_raw>(ctx, a, c.block_tokens, grid);
    } else {
        if (c.code_type == SPOTLIGHT_E4M3) launch_write<E4M3, float>(ctx, a, c.block_tokens, grid);
        else launch_write<I8, float>(ctx, a, c.block_tokens, grid);
    }
    return hip_rc(hipGetLastError());
}

int launch_cache_read(spotlight_ctx* ctx, const spotlight_cache& c, int64_t t0, int64_t n, const int32_t* first, void* K, void* V)
{
    const Plan& p = ctx->plan;
    RowsArgs a = rows_args(ctx, c, t0, n, first, nullptr);
    a.out[0] = K;
    a.out[1] = V;
    if (p.kv_dtype == SPOTLIGHT_BF16) {
        if (c.code_type == SPOTLIGHT_E4M3) launch_read<E4M3, bf16_raw>(ctx, a);
        else launch_read<I8, bf16_raw>(ctx, a);
    } else {
        if (c.code_type == SPOTLIGHT_E4M3) launch_read<E4M3, float>(ctx, a);
        else launch_read<I8, float>(ctx, a);
    }
    return hip_rc(hipGetLastError());
}

}  // namespace spotlight
