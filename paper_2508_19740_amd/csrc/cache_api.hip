// Entry points of the 8-bit key-value cache: argument checks (host only, before any HIP call) and launches.
#include "internal.h"

using namespace spotlight;

namespace {

// Makes the context's device the current one for the time of a call.
struct DeviceGuard {
    int before = -1;
    bool ok = true;
    explicit DeviceGuard(const spotlight_ctx* ctx)
    {
        int now = 0;
        ok = hipGetDevice(&now) == hipSuccess;
        if (ok && now != ctx->device) {
            ok = hipSetDevice(ctx->device) == hipSuccess;
            if (ok) before = now;
        }
    }
    ~DeviceGuard() { if (before >= 0) (void)hipSetDevice(before); }
    DeviceGuard(const DeviceGuard&) = delete;
    DeviceGuard& operator=(const DeviceGuard&) = delete;
};

int check_cache(const spotlight_cache* c)
{
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return SPOTLIGHT_ERR_INVALID_ARG;
    if (c->code_type != SPOTLIGHT_E4M3 && c->code_type != SPOTLIGHT_I8) return SPOTLIGHT_ERR_INVALID_ARG;
    const int32_t T = c->block_tokens;
    if (T != 16 && T != 32 && T != 64 && T != 128) return SPOTLIGHT_ERR_INVALID_ARG;
    if (misaligned(c->k) || misaligned(c->v)) return SPOTLIGHT_ERR_INVALID_ARG;
    return SPOTLIGHT_OK;
}

// Rows t0 .. t0 + n - 1 of every sequence; with `first` the kernels leave out those that are not in the cache.
int check_rows(const Plan& p, int64_t t0, int64_t n, const int32_t* first)
{
    if (t0 < 0 || n < 0 || t0 > p.Nmax || n > p.Nmax) return SPOTLIGHT_ERR_INVALID_ARG;
    if (!first && n > p.Nmax - t0) return SPOTLIGHT_ERR_INVALID_ARG;
    return SPOTLIGHT_OK;
}

}  // namespace

extern "C" {

int spotlight_cache_write(spotlight_ctx* ctx, const spotlight_cache* cache, const void* K, const void* V, int64_t t0,
                          int64_t n_new, const int32_t* first, const int32_t* count)
{
    if (!ctx || (n_new != 0 && (!K || !V))) return SPOTLIGHT_ERR_INVALID_ARG;
    int rc = check_cache(cache);
    if (rc != SPOTLIGHT_OK) return rc;
    rc = check_rows(ctx->plan, t0, n_new, first);
    if (rc != SPOTLIGHT_OK) return rc;
    if (misaligned(K) || misaligned(V)) return SPOTLIGHT_ERR_INVALID_ARG;
    if (n_new == 0) return SPOTLIGHT_OK;
    DeviceGuard on(ctx);
    if (!on.ok) return SPOTLIGHT_ERR_HIP;
    return launch_cache_write(ctx, *cache, K, V, t0, n_new, first, count);
}

int spotlight_cache_read(spotlight_ctx* ctx, const spotlight_cache* cache, int64_t t0, int64_t n, const int32_t* first,
                         void* K, void* V)
{
    if (!ctx || (n != 0 && !K && !V)) return SPOTLIGHT_ERR_INVALID_ARG;
    int rc = check_cache(cache);
    if (rc != SPOTLIGHT_OK) return rc;
    rc = check_rows(ctx->plan, t0, n, first);
    if (rc != SPOTLIGHT_OK) return rc;
    if (misaligned(K) || misaligned(V)) return SPOTLIGHT_ERR_INVALID_ARG;
    if (n == 0) return SPOTLIGHT_OK;
    DeviceGuard on(ctx);
    if (!on.ok) return SPOTLIGHT_ERR_HIP;
    return launch_cache_read(ctx, *cache, t0, n, first, K, V);
}

int spotlight_sparse_decode_cache(spotlight_ctx* ctx, const void* q, const spotlight_cache* cache, const int32_t* idx,
                                  int32_t k, float scale, float* out)
{
    if (!ctx || !q || !idx || !out) return SPOTLIGHT_ERR_INVALID_ARG;
    const int rc = check_cache(cache);
    if (rc != SPOTLIGHT_OK) return rc;
    if (k < 1 || k > ctx->plan.max_topk) return SPOTLIGHT_ERR_INVALID_ARG;
    if (misaligned(q)) return SPOTLIGHT_ERR_INVALID_ARG;
    DeviceGuard on(ctx);
    if (!on.ok) return SPOTLIGHT_ERR_HIP;
    return launch_cache_attend(ctx, q, *cache, idx, k, scale, out);
}

int spotlight_dense_decode_cache(spotlight_ctx* ctx, const void* q, const spotlight_cache* cache, int64_t n_tokens,
                                 int32_t n_q, const int32_t* lens, float scale, float* out)
{
    if (!ctx || !q || !out) return SPOTLIGHT_ERR_INVALID_ARG;
    const int rc = check_cache(cache);
    if (rc != SPOTLIGHT_OK) return rc;
    if (n_tokens < 1 || n_tokens > ctx->plan.Nmax || n_q < 1 || n_q > ctx->plan.Nmax) return SPOTLIGHT_ERR_INVALID_ARG;
    if (misaligned(q)) return SPOTLIGHT_ERR_INVALID_ARG;
    DeviceGuard on(ctx);
    if (!on.ok) return SPOTLIGHT_ERR_HIP;
    return launch_cache_dense(ctx, q, *cache, n_tokens, n_q, lens, scale, out);
}

int spotlight_hash_rows(spotlight_ctx* ctx, const void* K, const spotlight_hash_weights* w, int64_t t0, int64_t n_new,
                        uint32_t* codes)
{
    if (!ctx || (n_new != 0 && !K) || !codes) return SPOTLIGHT_ERR_INVALID_ARG;
    const Plan& p = ctx->plan;
    int rc = check_weights(ctx, w);
    if (rc != SPOTLIGHT_OK) return rc;
    rc = check_rows(p, t0, n_new, nullptr);
    if (rc != SPOTLIGHT_OK) return rc;
    if (misaligned(K) || misaligned(codes)) return SPOTLIGHT_ERR_INVALID_ARG;
    if (n_new == 0) return SPOTLIGHT_OK;
    DeviceGuard on(ctx);
    if (!on.ok) return SPOTLIGHT_ERR_HIP;
    HashLaunch job = key_job(ctx, K, w, t0, n_new, codes);
    job.x_head_stride = n_new * kHeadDim;
    job.x_row0 = 0;
    return launch_hash(ctx, job, SPOTLIGHT_STAGE_HASH_KEYS);
}

int spotlight_decode_step_cache(spotlight_ctx* ctx, const void* q, const void* K, const void* V, const spotlight_cache* cache,
                                const spotlight_hash_weights* w, uint32_t* codes, int64_t n_tokens, int32_t k,
                                int32_t n_sink, int32_t n_local, float scale, int32_t* out_idx, float* out)
{
    int rc = check_step_args(ctx, q, K, V, w, codes, n_tokens, k, n_sink, n_local, out_idx, out);
    if (rc != SPOTLIGHT_OK) return rc;
    rc = check_cache(cache);
    if (rc != SPOTLIGHT_OK) return rc;
    DeviceGuard on(ctx);
    if (!on.ok) return SPOTLIGHT_ERR_HIP;
    // queries first: their workgroups also clear the histograms
    HashLaunch key = key_job(ctx, K, w, n_tokens - 1, 1, codes);
    key.x_head_stride = kHeadDim;
    key.x_row0 = 0;
    rc = launch_hash_pair(ctx, query_job(ctx, q, w), key, SPOTLIGHT_STAGE_HASH_QUERY);
    if (rc != SPOTLIGHT_OK) return rc;
    rc = launch_cache_write(ctx, *cache, K, V, n_tokens - 1, 1, nullptr, nullptr);
    if (rc != SPOTLIGHT_OK) return rc;
    rc = launch_retrieve(ctx, codes, n_tokens, k, n_sink, n_local, out_idx, nullptr);
    if (rc != SPOTLIGHT_OK) return rc;
    return launch_cache_attend(ctx, q, *cache, out_idx, k, scale, out);
}

}  // extern "C"
