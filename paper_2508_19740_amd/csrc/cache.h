// The key-value cache held in 8 bits: its two code types, and what its kernels share.
//
// A block of block_tokens rows of a head has one scale, a power of two: value = code * scale.  Scaling
// by a power of two is exact in binary32, so the only rounding between a row and its codes is that to
// the code type, a block whose scale grows is rescaled without the original rows, and a code goes into
// a product in any type that holds the code itself.
#pragma once
#include "internal.h"

namespace spotlight {
namespace cache {

// How attention over the whole cache is shared out (host): tiles of 16 rows a workgroup, and the keys of a
// split.  Partial results of all rows and splits fit the workspace's dense_rows, and a split's keys are
// a multiple of its wavefronts' steps.
constexpr int kDenseStep = 32, kDenseWaves = 4;
constexpr int64_t kDenseMostKeys = 1 << 25;   // of a split: a wavefront's quarter of them stays below 2^31 bytes
struct DenseSplit {
    int tiles, nsplit;
    int64_t chunk;
};
inline int split_dense(const Plan& p, int n_cus, int64_t n_tokens, int n_q, DenseSplit* s)
{
    const int64_t rows = static_cast<int64_t>(p.G) * n_q, heads = static_cast<int64_t>(p.B) * p.Hkv;
    if (rows > 1 << 24) return SPOTLIGHT_ERR_UNSUPPORTED;   // a grid's first dimension, and 32 bits for a row
    s->tiles = rows <= 16 ? 1 : 2;
    const int64_t groups = heads * ((rows + 16 * s->tiles - 1) / (16 * s->tiles));
    constexpr int64_t unit = kDenseStep * kDenseWaves;
    const int64_t room = p.dense_rows / (heads * rows), most = (n_tokens + unit - 1) / unit;
    int64_t n = (static_cast<int64_t>(n_cus) * (s->tiles == 2 ? 2 : 4) + groups - 1) / groups;
    if (n > room) n = room;
    if (n > most) n = most;
    if (n < 1) n = 1;
    if (n_tokens > n * kDenseMostKeys) {
        n = (n_tokens + kDenseMostKeys - 1) / kDenseMostKeys;
        if (n > room) return SPOTLIGHT_ERR_UNSUPPORTED;
    }
    s->chunk = ((n_tokens + n - 1) / n + unit - 1) / unit * unit;
    s->nsplit = static_cast<int>((n_tokens + s->chunk - 1) / s->chunk);
    return SPOTLIGHT_OK;
}

#if defined(__HIPCC__)

struct bf16_raw { uint16_t v; };

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Binary32 values of the four codes of a word, and the codes nearest (ties to even) to four values that
// the code type's largest magnitude bounds.  kTop and kMant are the exponent and the fraction bits of
// that magnitude: 448 = 1.75 * 2^8, 127 = 1.984375 * 2^6.
struct E4M3 {
    static constexpr int kTop = 8;
    static constexpr uint32_t kMant = 0x600000u;
    static constexpr bool kHasNaN = true;
    static __device__ __forceinline__ void decode(uint32_t w, float (&o)[4])
    {
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), false);
        const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w), true);
        o[0] = a.x; o[1] = a.y; o[2] = b.x; o[3] = b.y;
    }
    static __device__ __forceinline__ uint32_t encode(const float (&x)[4])
    {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
        return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], lo, true));
    }
};

struct I8 {
    static constexpr int kTop = 6;
    static constexpr uint32_t kMant = 0x7e0000u;
    static constexpr bool kHasNaN = false;
    static __device__ __forceinline__ void decode(uint32_t w, float (&o)[4])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = static_cast<float>(static_cast<int8_t>(w >> (8 * i)));
    }
    static __device__ __forceinline__ uint32_t encode(const float (&x)[4])
    {
        uint32_t w = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) w |= (static_cast<uint32_t>(static_cast<int>(rintf(x[i]))) & 0xffu) << (8 * i);
        return w;
    }
};

// The smallest exponent e >= -126 for which a magnitude (bits of a finite, non-negative float) is at
// most the code type's largest times 2^e.
template <typename CT>
__device__ __forceinline__ int least_exponent(uint32_t bits)
{
    const int e = static_cast<int>(bits >> 23) - 127 - CT::kTop + ((bits & 0x7fffffu) > CT::kMant ? 1 : 0);
    return e > -126 ? e : -126;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

#endif   // __HIPCC__

}  // namespace cache
}  // namespace spotlight
