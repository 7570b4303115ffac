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

// The last-level cache.  Calls with as many bytes that nothing reads twice pass it by (non-temporal loads and stores).
constexpr int64_t kCacheBytes = 256 << 20;

// Division of numbers below 2^31 by one that the host knows.
struct FastDiv {
    uint32_t d, mul, shift;
#if defined(__HIPCC__)
    __device__ __forceinline__ uint32_t over(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
#endif
};
inline FastDiv fast_div(uint32_t d)
{
    FastDiv f{d, 0, 0};
    while (f.shift < 31 && (1u << f.shift) < d) ++f.shift;
    f.mul = static_cast<uint32_t>((((1ull << f.shift) - d) << 32) / d + 1);
    return f;
}

// How attention over the whole cache is shared out.  A workgroup has a tile of rows of a key-value head and a run of
// keys, counted in units of 128.  Sequences of one length are split alike.  Where each has a length of its own, which the
// host does not know, the kernel takes runs of one size for all, about the smallest with which all sequences make no
// more than `most_runs`, so that every workgroup has about as much to do.  (Runs of a fixed part of
// n_tokens leave compute units idle: 16 sequences of 2049 .. 32769 tokens, 28 / 4 heads, 69 -> 62 us.)
constexpr int kDenseStep = 32, kDenseWaves = 4, kDenseUnit = kDenseStep * kDenseWaves;
constexpr int64_t kDenseMostKeys = 1 << 25;   // of a workgroup: a wavefront's quarter of them stays below 2^31 bytes
struct DenseShares {
    const int32_t* lens;
    uint32_t batch, units;      // units of n_tokens
    uint32_t chunk;             // units of a run, and
    uint32_t nsplit;            // runs of a sequence, without lens
    uint32_t most_runs;         // with lens: runs of all sequences, more than there are sequences (twice as many where there is room); 0: a run is a sequence
    uint32_t tile_rows;         // rows of a workgroup's partial result
    uint32_t tiles;             // tiles of rows of a key-value head
    FastDiv by_nsplit, by_most, by_spare, by_heads, by_tiles8;    // by_spare: most_runs - batch
};
struct DensePlan {
    DenseShares shares;
    int row_tiles;              // of 16 rows, a workgroup
    uint32_t grid;              // workgroups, at most
    int64_t about;              // runs of a sequence, on average
    bool splits, joins;         // whether there are partial results, and whether the last workgroup joins them
};
int plan_dense(const Plan& p, int n_cus, int64_t n_tokens, int n_q, const int32_t* lens, DensePlan* d, int code_type = SPOTLIGHT_E4M3);

// Whether the last workgroup of each group of rows joins its partial results, instead of a launch of its own: small
// calls, where the join is one round of loads (about 2 us, since nothing of it is in a cache; a launch takes 3.5 us of the
// host).  Against the merge kernel, called back to back: 1 head, 600 / 4096 / 8192 tokens 10.6 / 11.5 / 11.5 -> 8.7 / 8.4 /
// 8.8 us, gathered 300 / 2000 of them 10.2 / 10.4 -> 7.8 / 7.7 us, and no slower in a graph; with two rounds, 16384
// tokens 11.3 -> 11.2 us (graph 10.2 -> 11.2), 1000 tokens of 4 groups of 8, 11.6 -> 10.5 us (graph 9.0 -> 10.4).
inline bool joins_in_place(int64_t workgroups, int64_t rows, int64_t nsplit)
{
    const int64_t rounds = rows >= 4 ? (rows + 3) / 4 * ((nsplit + 15) / 16) : rows * ((nsplit + 63) / 64);
    return nsplit > 1 && rounds <= 1 && workgroups <= kJoinGroups;
}

// The counter of the at-th group of rows among those of a call that have nsplit parts (2 .. kJoinSplits; at < kJoinGroups /
// nsplit).  A counter belongs to one nsplit for good and wraps there, so that it is 0 again after any number of calls, also
// where a program lets calls overlap, whose results are then undefined: the next call's are not.  (A counter that the last
// workgroup clears would lose or keep counts then, and no workgroup of later calls would be the last.)
constexpr
#if defined(__HIPCC__)
__host__ __device__
#endif
uint32_t arrival_counter(uint32_t at, uint32_t nsplit)
{
    const uint32_t k = 31 - __builtin_clz(nsplit);
    return (k - 1) * kJoinGroups + (nsplit - (1u << k)) * (kJoinGroups >> k) + at;
}
static_assert(arrival_counter(0, 2) == 0 && arrival_counter(kJoinGroups / kJoinSplits - 1, kJoinSplits) < kArrivedCounters, "counters");

// The rows that the merge kernel joins: nsplit partial results each, one after the other; or (runs set) those of attention
// over the whole cache, where the runs of a sequence lie apart.
struct MergeRows {
    int64_t rows;
    int nsplit;
    const uint2* runs;          // [batch] {first, number}
    FastDiv by_rows, by_heads, by_tile;
    uint32_t tiles, tile_rows;
    int64_t room;               // partial results that the workspace holds
};

// Where the partial results of a row lie: nsplit of them, `step` apart.  The table of runs is read from the workspace.  Where a
// program lets calls overlap, it may be another call's, with more runs than this call's tiles leave room for: those are left out.
struct RowParts { int64_t at, step; int nsplit; };
#if defined(__HIPCC__)
__host__ __device__
#endif
inline RowParts parts_of(const MergeRows& r, uint2 run, uint32_t kv, uint32_t tile, uint32_t row)
{
    RowParts p;
    p.step = static_cast<int64_t>(r.by_heads.d) * r.tiles * r.tile_rows;
    p.at = ((static_cast<int64_t>(run.x) * r.by_heads.d + kv) * r.tiles + tile) * r.tile_rows + row;
    p.nsplit = static_cast<int>(run.y);
    if (p.at + (p.nsplit - 1) * p.step >= r.room) p.nsplit = 0;
    return p;
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

// Partial results of attention whose keys are split over workgroups: for every row and split {maximum in units of log2,
// sum of weights} and 128 weighted sums of values.  A split without keys has sum 0, and its sums may hold
// anything.
//
// A kernel of its own joins them (cache_merge.hip), or, in small calls, the workgroup that arrives last: that saves a launch.
// Its reads have to see what workgroups on other dies wrote: there, partial results are written and read with
// device-wide (relaxed atomic) accesses, which no die's cache holds back, and every wavefront waits for its writes
// before its workgroup counts itself as arrived.  (A release fence would write back all of the die's cache instead, once
// a workgroup.)
struct Partials {
    unsigned long long* ml;             // [rows][nsplit] float2
    unsigned long long* acc;            // [rows][nsplit][64] float2
    uint32_t* arrived;                  // the counters, kArrivedStride apart; null: another kernel joins
};

__device__ __forceinline__ void put_pair(unsigned long long* p, float x, float y)
{
    __hip_atomic_store(p, static_cast<unsigned long long>(__float_as_uint(y)) << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ f32x2 get_pair(const unsigned long long* p)
{
    return __builtin_bit_cast(f32x2, __hip_atomic_load(const_cast<unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// One workgroup's part: a pair of columns of a row, and the row's maximum and sum.
__device__ __forceinline__ void put_part(const Partials& p, size_t at, uint32_t pair, float m, float l, f32x2 a)
{
    if (p.arrived) {
        put_pair(p.acc + at * 64 + pair, a.x, a.y);
        if (pair == 0) put_pair(p.ml + at, m, l);
    } else {
        reinterpret_cast<f32x2*>(p.acc)[at * 64 + pair] = a;
        if (pair == 0) reinterpret_cast<f32x2*>(p.ml)[at] = f32x2{m, l};
    }
}

// Counts the workgroup as arrived once its writes are done; true for the last of the group's (arrival_counter).
__device__ __forceinline__ bool arrives_last(const Partials& p, uint32_t at, uint32_t nsplit, uint32_t* lds)
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) *lds = atomicInc(p.arrived + arrival_counter(at, nsplit) * kArrivedStride, nsplit - 1);
    __syncthreads();
    asm volatile("" ::: "memory");
    return *lds == nsplit - 1;
}

// What a run of keys belongs to: its sequence, which run of it, how many there are, and the first one's number.
struct DenseRun {
    uint32_t entry, split, nsplit, first, chunk, len;
    // All of it is the same for the wavefront; loads that depend on it alone are scalar ones.
    __device__ __forceinline__ void to_scalars()
    {
        entry = __builtin_amdgcn_readfirstlane(entry);
        split = __builtin_amdgcn_readfirstlane(split);
        nsplit = __builtin_amdgcn_readfirstlane(nsplit);
        first = __builtin_amdgcn_readfirstlane(first);
        chunk = __builtin_amdgcn_readfirstlane(chunk);
        len = __builtin_amdgcn_readfirstlane(len);
    }
};
__device__ __forceinline__ uint32_t units_of(uint32_t len) { return (len + kDenseUnit - 1) / kDenseUnit; }
// Sequence lengths, 64 at a time; the first 64 stay in a register.
struct Lengths {
    const DenseShares& s;
    uint32_t most, lane, first;
    __device__ __forceinline__ Lengths(const DenseShares& shares, uint32_t n_tokens) : s(shares), most(n_tokens), lane(threadIdx.x & 63), first(load(0)) {}
    __device__ __forceinline__ uint32_t load(uint32_t o) const
    {
        return o + lane < s.batch ? static_cast<uint32_t>(min(max(s.lens[o + lane], 0), static_cast<int32_t>(most))) : 0;
    }
    __device__ __forceinline__ uint32_t at(uint32_t o) const { return o ? load(o) : first; }
    // Runs of `chunk` units (inv: about its inverse).  Units are below 2^24, so that a binary32 quotient is off by one at most.  An
    // empty sequence has a run too: it writes zeros.
    __device__ __forceinline__ uint32_t runs(uint32_t o, uint32_t len, uint32_t chunk, float inv) const
    {
        const uint32_t u = units_of(len) + chunk - 1;
        uint32_t n = static_cast<uint32_t>(static_cast<float>(u) * inv);
        const int32_t left = static_cast<int32_t>(u - n * chunk);
        n += left < 0 ? -1 : left >= static_cast<int32_t>(chunk) ? 1 : 0;
        return o + lane < s.batch ? max(n, 1u) : 0;
    }
};
// Uniform over the wavefront.  entry == batch: there is no such run.
__device__ __forceinline__ DenseRun find_run(const DenseShares& s, uint32_t number, int64_t n_tokens)
{
    DenseRun r;
    if (!s.lens) {
        r.entry = s.by_nsplit.over(number);
        r.nsplit = s.nsplit;
        r.first = r.entry * s.nsplit;
        r.split = number - r.first;
        r.chunk = s.chunk;
        r.len = static_cast<uint32_t>(n_tokens);
        return r;
    }
    const Lengths lens(s, static_cast<uint32_t>(n_tokens));
    r.chunk = s.units;
    if (s.most_runs) {
        uint32_t total = 0;
        for (uint32_t o = 0; o < s.batch; o += 64) total += units_of(lens.at(o));
        total = wave_sum(total);
        // Each sequence rounds up to whole runs, so that total / most_runs may be too small.  With total / (most_runs -
        // batch) there are never too many.
        const uint32_t safe = s.by_spare.over(total + s.by_spare.d - 1);
        uint32_t chunk = max(s.by_most.over(total + s.most_runs - 1), 1u);
        for (int tries = 0; chunk < safe; ++tries) {
            uint32_t made = 0;
            const float inv = __builtin_amdgcn_rcpf(static_cast<float>(chunk));
            for (uint32_t o = 0; o < s.batch; o += 64) made += lens.runs(o, lens.at(o), chunk, inv);
            made = wave_sum(made);
            if (made <= s.most_runs) break;
            chunk = tries < 3 ? max(chunk + 1, s.by_most.over(chunk * made)) : safe;
        }
        r.chunk = min(max(chunk, 1u), s.units);
    }
    r.entry = s.batch;
    r.nsplit = r.first = r.split = 0;
    r.len = 0;
    const float inv = __builtin_amdgcn_rcpf(static_cast<float>(r.chunk));
    for (uint32_t o = 0, before = 0; o < s.batch; o += 64) {
        const uint32_t len = lens.at(o), n = lens.runs(o, len, r.chunk, inv);
        const uint32_t upto = before + wave_inclusive_scan(n);
        const unsigned long long past = __ballot(upto > number);
        if (past) {
            const int at = __builtin_ctzll(past);
            r.entry = o + at;
            r.nsplit = __builtin_amdgcn_readlane(n, at);
            r.first = __builtin_amdgcn_readlane(upto, at) - r.nsplit;
            r.split = number - r.first;
            r.len = __builtin_amdgcn_readlane(len, at);
            break;
        }
        before = __builtin_amdgcn_readlane(upto, 63);
    }
    return r;
}

// A running softmax sum of partial results.
struct Join {
    float m = -INFINITY, l = 0.0f;
    f32x2 a = {0.0f, 0.0f};
    __device__ __forceinline__ void add(f32x2 ml, f32x2 v)
    {
        if (ml.y == 0.0f) return;
        const float mn = fmaxf(m, ml.x);
        const float fo = l != 0.0f ? __builtin_amdgcn_exp2f(m - mn) : 0.0f, fn = __builtin_amdgcn_exp2f(ml.x - mn);
        a.x = __builtin_fmaf(a.x, fo, fn * v.x);
        a.y = __builtin_fmaf(a.y, fo, fn * v.y);
        l = __builtin_fmaf(l, fo, fn * ml.y);
        m = mn;
    }
};

// Joins the partial results of `rows` rows into out, in the workgroup that arrived last: those of row r are the nsplit ones
// at + r, at + r + step, ...  A group of 64 threads has a row, two columns a thread, and NB splits on their way
// at once; where there are fewer rows than groups, the groups share out each row's splits and are joined in order.  `lds`: 128
// f32x2 for each group but the first.
template <int NT, uint32_t NB>
__device__ __forceinline__ void join_rows(const Partials& p, uint32_t at, uint32_t step, uint32_t rows, uint32_t nsplit, float* out, f32x2* lds)
{
    constexpr uint32_t GROUPS = NT / 64;
    const uint32_t c = threadIdx.x & 63, group = threadIdx.x >> 6;
    f32x2* o = reinterpret_cast<f32x2*>(out);
    const bool alone = rows >= GROUPS;                    // a group has its rows to itself
    const uint32_t stride = alone ? 1 : GROUPS;
    for (uint32_t r = alone ? group : 0; r < rows; r += alone ? GROUPS : 1) {
        Join j;
        for (uint32_t s = alone ? 0 : group; s < nsplit; s += stride * NB) {
            f32x2 ml[NB], v[NB];
#pragma unroll
            for (uint32_t y = 0; y < NB; ++y) {
                const size_t from = at + r + static_cast<size_t>(min(s + stride * y, nsplit - 1)) * step;
                ml[y] = get_pair(p.ml + from);
                v[y] = get_pair(p.acc + from * 64 + c);
            }
#pragma unroll
            for (uint32_t y = 0; y < NB; ++y)
                if (s + stride * y < nsplit) j.add(ml[y], v[y]);
        }
        if (!alone) {
            __syncthreads();
            if (group > 0) {
                f32x2* to = lds + (group - 1) * 128;
                to[c] = f32x2{j.m, j.l};
                to[64 + c] = j.a;
            }
            __syncthreads();
            if (group > 0) continue;
#pragma unroll
            for (uint32_t k = 0; k + 1 < GROUPS; ++k) j.add(lds[k * 128 + c], lds[k * 128 + 64 + c]);
        }
        o[static_cast<size_t>(r) * 64 + c] = j.l != 0.0f ? f32x2{j.a.x / j.l, j.a.y / j.l} : f32x2{0.0f, 0.0f};
    }
}

#endif   // __HIPCC__

}  // namespace cache

// Joins partial results; `about`: splits of a row, on average.
int launch_cache_merge(spotlight_ctx* ctx, const void* part_ml, const void* part_acc, const cache::MergeRows& r, int64_t about, float* out);

}  // namespace spotlight
