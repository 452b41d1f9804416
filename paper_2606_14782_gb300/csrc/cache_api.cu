// C ABI of the 8-bit paged cache: argument checks and the handle.
#include <cmath>
#include <cstdlib>
#include <cstring>
#include <new>

#include "bacon.h"
#include "cache.h"
#include "common.cuh"
#include "host.h"
#include "rotary.cuh"
#include "step_host.h"

using namespace bacon;

struct bacon_cache {
    int device = 0;
    int max_requests = 0;
    int fault_pending = 0;  // test-only fault injection (BACON_FAULT=missing_page[:tile])
    CacheGeom g{};
    SplitScratch sc{};
};

namespace {

bacon_status check_call(const bacon_cache* c, int requests)
{
    if (!c) return fail(BACON_EINVAL, "null cache");
    if (requests < 1 || requests > c->max_requests)
        return fail(BACON_EINVAL, "requests must be in [1, %d], got %d", c->max_requests, requests);
    return BACON_OK;
}

bacon_status check_rows(const void* p, long long token_stride, long long head_stride, const char* what)
{
    if (!p || !aligned16(p))
        return fail(BACON_EINVAL, "%s must be a 16-byte aligned device pointer", what);
    if (token_stride % 8 || head_stride % 8 || token_stride < 0 || head_stride < 0)
        return fail(BACON_EINVAL, "the strides of %s must be multiples of 8 elements", what);
    return BACON_OK;
}

}  // namespace

extern "C" {

bacon_status bacon_cache_create(bacon_cache** out, const bacon_cache_desc* desc)
{
    g_last_error.clear();
    if (!out || !desc) return fail(BACON_EINVAL, "null argument");
    *out = nullptr;
    const bacon_cache_desc& d = *desc;
    if (d.layers < 1 || d.kv_heads < 1 || d.q_heads < 1 || d.pages < 1 || d.max_requests < 1 ||
        d.max_blocks < 1)
        return fail(BACON_EINVAL, "sizes must be positive");
    if (d.q_heads % d.kv_heads)
        return fail(BACON_EINVAL, "q_heads %d is not a multiple of kv_heads %d", d.q_heads, d.kv_heads);
    if (d.head_dim != 64 && d.head_dim != 128)
        return fail(BACON_EINVAL, "head_dim must be 64 or 128, got %d", d.head_dim);
    if (d.page != 16 && d.page != 32 && d.page != 64 && d.page != 128)
        return fail(BACON_EINVAL, "page must be 16, 32, 64 or 128, got %d", d.page);
    if ((long long)d.pages * d.page >= 1ll << 31)
        return fail(BACON_EINVAL, "pages * page must be below 2^31");
    if ((long long)d.max_blocks * d.page >= (1ll << 31) - 1024)
        return fail(BACON_EINVAL, "max_blocks * page must be below 2^31 - 1024");
    if ((long long)d.max_requests * d.layers * d.kv_heads >= 1ll << 31)
        return fail(BACON_EINVAL, "max_requests * layers * kv_heads must be below 2^31");
    if (d.format != BACON_E4M3 && d.format != BACON_INT8)
        return fail(BACON_EINVAL, "unknown format %d", d.format);
    if (d.dtype != BACON_BF16 && d.dtype != BACON_FP16)
        return fail(BACON_EINVAL, "unknown dtype %d", d.dtype);
    if (!d.k || !d.v || !aligned16(d.k) || !aligned16(d.v) || !d.k_scale || !d.v_scale)
        return fail(BACON_EINVAL, "pools must be non-null, k and v 16-byte aligned");
    bacon_cache* c = new (std::nothrow) bacon_cache;
    if (!c) return fail(BACON_ENOMEM, "host allocation failed");
    CacheGeom& g = c->g;
    c->max_requests = d.max_requests;
    g.layers = d.layers;
    g.hkv = d.kv_heads;
    g.hq = d.q_heads;
    g.group = d.q_heads / d.kv_heads;
    g.d = d.head_dim;
    g.page = d.page;
    for (g.page_log2 = 0; 1 << g.page_log2 < d.page;) ++g.page_log2;
    g.pages = d.pages;
    g.max_blocks = d.max_blocks;
    g.format = d.format;
    g.dtype = d.dtype;
    g.k = static_cast<uint8_t*>(d.k);
    g.v = static_cast<uint8_t*>(d.v);
    g.k_scale = d.k_scale;
    g.v_scale = d.v_scale;
    cudaError_t e = cudaGetDevice(&c->device);
    SplitScratch& sc = c->sc;
    if (e == cudaSuccess)
        e = cudaDeviceGetAttribute(&sc.sms, cudaDevAttrMultiProcessorCount, c->device);
    // one allocation: partial outputs, their sums, arrival counts, error word
    const size_t blocks = (size_t)sc.sms * kBlocksPerSm;
    const size_t out_bytes = 2 * blocks * 32 * 128 * sizeof(float);
    const size_t sum_bytes = 2 * blocks * 32 * 2 * sizeof(float);
    const size_t many_out_bytes = (size_t)sc.sms * 4 * 128 * 128 * sizeof(float);
    const size_t many_sum_bytes = (size_t)sc.sms * 4 * 128 * sizeof(float2);
    const size_t word_bytes = (blocks + 2 * (size_t)sc.sms + 1) * sizeof(int);
    if (e == cudaSuccess)
        e = cudaMalloc(reinterpret_cast<void**>(&sc.out),
                       out_bytes + sum_bytes + many_out_bytes + many_sum_bytes + word_bytes);
    if (e == cudaSuccess) {
        sc.sums = sc.out + out_bytes / sizeof(float);
        sc.many_out = sc.sums + sum_bytes / sizeof(float);
        sc.many_sums = reinterpret_cast<float2*>(sc.many_out + many_out_bytes / sizeof(float));
        sc.arrived = reinterpret_cast<int*>(sc.many_sums + many_sum_bytes / sizeof(float2));
        sc.many_arrived = sc.arrived + blocks;
        g.err = sc.many_arrived + 2 * (size_t)sc.sms;
        e = clear_now(sc.arrived, word_bytes);
    }
    if (e != cudaSuccess) {
        bacon_cache_destroy(c);
        const bacon_status rc = cuda_fail(e, "cache creation");
        return e == cudaErrorMemoryAllocation ? fail(BACON_ENOMEM, "device allocation failed") : rc;
    }
    const long long rows = (long long)g.pages * g.page;
    if (!encode_pool_map(&sc.kmap, g.k, g.d, rows) || !encode_pool_map(&sc.vmap, g.v, g.d, rows)) {
        bacon_cache_destroy(c);
        return fail(BACON_ECUDA, "cuTensorMapEncodeTiled failed");
    }
    const char* const fault = std::getenv("BACON_FAULT");
    if (fault && std::strcmp(fault, "missing_page") == 0) c->fault_pending = 1;
    if (fault && std::strncmp(fault, "missing_page:", 13) == 0) {
        const int tile = std::atoi(fault + 13);
        if (tile >= 0 && tile < 1 << 30) c->fault_pending = tile + 1;
    }
    *out = c;
    return BACON_OK;
}

void bacon_cache_destroy(bacon_cache* cache)
{
    if (!cache) return;
    DeviceGuard dg(cache->device);
    if (cache->sc.out) cudaFree(cache->sc.out);
    delete cache;
}

bacon_status bacon_cache_plan(bacon_cache* cache, int requests, const int32_t* lengths,
                              const int32_t* added, int per_unit, int32_t* table,
                              const int32_t* ring, const int32_t* state, int rows,
                              int32_t* slots, int32_t* lengths_out, int32_t* state_out,
                              bacon_stream stream)
{
    g_last_error.clear();
    if (bacon_status rc = check_call(cache, requests)) return rc;
    if (!lengths || !table || !ring || !state || !lengths_out || !state_out)
        return fail(BACON_EINVAL, "null argument");
    if (per_unit && !added) return fail(BACON_EINVAL, "per_unit needs the units' numbers of tokens");
    if (rows < 0 || (rows && !slots)) return fail(BACON_EINVAL, "rows is negative or slots is null");
    if (lengths == lengths_out || state == state_out)
        return fail(BACON_EINVAL, "lengths_out and state_out must not be the inputs");
    const CacheGeom& g = cache->g;
    PlanArgs a{requests * g.layers * g.hkv, requests, lengths, added, per_unit != 0, table, ring,
               state, rows, slots, lengths_out, state_out};
    DeviceGuard dg(cache->device);
    BACON_CUDA(launch_cache_plan(g, a, static_cast<cudaStream_t>(stream)), "plan launch");
    return BACON_OK;
}

bacon_status bacon_cache_locate(bacon_cache* cache, int requests, const int32_t* first,
                                const int32_t* count, const int32_t* table, int rows,
                                int32_t* slots, bacon_stream stream)
{
    g_last_error.clear();
    if (bacon_status rc = check_call(cache, requests)) return rc;
    if (!count || !table) return fail(BACON_EINVAL, "null argument");
    if (rows < 0 || (rows && !slots)) return fail(BACON_EINVAL, "rows is negative or slots is null");
    const CacheGeom& g = cache->g;
    PlanArgs a{requests * g.layers * g.hkv, requests, first, count, 1,
               const_cast<int32_t*>(table), nullptr, nullptr, rows, slots, nullptr, nullptr};
    DeviceGuard dg(cache->device);
    BACON_CUDA(launch_cache_plan(g, a, static_cast<cudaStream_t>(stream)), "locate launch");
    return BACON_OK;
}

bacon_status bacon_cache_release(bacon_cache* cache, int requests, const int32_t* done,
                                 int32_t* lengths, int32_t* table, int32_t* ring,
                                 int32_t* state, bacon_stream stream)
{
    g_last_error.clear();
    if (bacon_status rc = check_call(cache, requests)) return rc;
    if (!done || !lengths || !table || !ring || !state) return fail(BACON_EINVAL, "null argument");
    const CacheGeom& g = cache->g;
    DeviceGuard dg(cache->device);
    BACON_CUDA(launch_cache_release(g, requests * g.layers * g.hkv, done, nullptr, lengths, table,
                                    ring, state, static_cast<cudaStream_t>(stream)),
               "release launch");
    return BACON_OK;
}

bacon_status bacon_cache_shorten(bacon_cache* cache, int requests, const int32_t* fewer,
                                 int32_t* lengths, int32_t* table, int32_t* ring,
                                 int32_t* state, bacon_stream stream)
{
    g_last_error.clear();
    if (bacon_status rc = check_call(cache, requests)) return rc;
    if (!fewer || !lengths || !table || !ring || !state) return fail(BACON_EINVAL, "null argument");
    const CacheGeom& g = cache->g;
    DeviceGuard dg(cache->device);
    BACON_CUDA(launch_cache_release(g, requests * g.layers * g.hkv, nullptr, fewer, lengths, table,
                                    ring, state, static_cast<cudaStream_t>(stream)),
               "shorten launch");
    return BACON_OK;
}

bacon_status bacon_cache_store(bacon_cache* cache, int tokens, int heads, const void* k,
                               long long k_token_stride, long long k_head_stride, const void* v,
                               long long v_token_stride, long long v_head_stride,
                               const int32_t* slots, bacon_stream stream)
{
    g_last_error.clear();
    if (!cache) return fail(BACON_EINVAL, "null cache");
    if (tokens < 0 || heads < 1 || heads > 65535)
        return fail(BACON_EINVAL, "tokens must not be negative, heads in [1, 65535]");
    if (tokens == 0) return BACON_OK;
    if (!slots) return fail(BACON_EINVAL, "null argument");
    if (bacon_status rc = check_rows(k, k_token_stride, k_head_stride, "k")) return rc;
    if (bacon_status rc = check_rows(v, v_token_stride, v_head_stride, "v")) return rc;
    StoreArgs a{tokens, heads,
                {static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v)},
                {k_token_stride, v_token_stride}, {k_head_stride, v_head_stride}, slots};
    DeviceGuard dg(cache->device);
    BACON_CUDA(launch_cache_store(cache->g, a, static_cast<cudaStream_t>(stream)), "store launch");
    return BACON_OK;
}

bacon_status bacon_cache_store_rotated(bacon_cache* cache, const bacon_rotary* rotary, int tokens,
                                       const bacon_rows* q, const bacon_rows* k, const void* v,
                                       long long v_token_stride, long long v_head_stride,
                                       int weight_dtype, float eps, float weight_offset,
                                       const int32_t* positions, const int32_t* slots,
                                       bacon_stream stream)
{
    g_last_error.clear();
    if (!cache) return fail(BACON_EINVAL, "null cache");
    if (!rotary || !k) return fail(BACON_EINVAL, "null argument");
    const CacheGeom& g = cache->g;
    if (tokens < 0 || k->heads < 1 || k->heads > 65535)
        return fail(BACON_EINVAL, "tokens must not be negative, heads in [1, 65535]");
    RotaryArgs r;
    if (bacon_status rc = rotary_args(rotary, 1, tokens, q, k, false, g.dtype, weight_dtype, eps,
                                      weight_offset, 0, positions, &r))
        return rc;
    if (r.table.head_dim != g.d)
        return fail(BACON_EINVAL, "the rotation is of %d values, rows have %d", r.table.head_dim, g.d);
    if (tokens == 0) return BACON_OK;
    if (!slots) return fail(BACON_EINVAL, "null argument");
    if (reinterpret_cast<uintptr_t>(slots) % 4)
        return fail(BACON_EINVAL, "slots must be aligned to their type");
    if (bacon_status rc = check_rows(k->in, k->in_token, k->in_head, "k")) return rc;
    if (bacon_status rc = check_rows(v, v_token_stride, v_head_stride, "v")) return rc;
    StoreArgs a{tokens, k->heads,
                {static_cast<const uint16_t*>(k->in), static_cast<const uint16_t*>(v)},
                {k->in_token, v_token_stride}, {k->in_head, v_head_stride}, slots};
    DeviceGuard dg(cache->device);
    BACON_CUDA(launch_cache_store_rotated(g, a, r, static_cast<cudaStream_t>(stream)), "store launch");
    return BACON_OK;
}

bacon_status bacon_cache_load(bacon_cache* cache, int rows, const int32_t* slots, void* k_out,
                              void* v_out, bacon_stream stream)
{
    g_last_error.clear();
    if (!cache) return fail(BACON_EINVAL, "null cache");
    if (rows < 0) return fail(BACON_EINVAL, "rows must not be negative");
    if (rows == 0) return BACON_OK;
    if (!slots || !k_out || !v_out || !aligned16(k_out) || !aligned16(v_out))
        return fail(BACON_EINVAL, "slots is null or an output is not 16-byte aligned");
    DeviceGuard dg(cache->device);
    BACON_CUDA(launch_cache_load(cache->g, rows, slots, k_out, v_out,
                                 static_cast<cudaStream_t>(stream)),
               "load launch");
    return BACON_OK;
}

bacon_status bacon_cache_attend(bacon_cache* cache, int requests, int layer, int tokens,
                                const void* q, long long q_token_stride, long long q_head_stride,
                                const int32_t* starts, const int32_t* lengths,
                                const int32_t* table, int causal, float scale, void* out,
                                float* lse, bacon_stream stream)
{
    g_last_error.clear();
    if (bacon_status rc = check_call(cache, requests)) return rc;
    const CacheGeom& g = cache->g;
    if (layer < 0 || layer >= g.layers)
        return fail(BACON_EINVAL, "layer must be in [0, %d), got %d", g.layers, layer);
    if (tokens < 0) return fail(BACON_EINVAL, "tokens must not be negative");
    if (tokens == 0) return BACON_OK;
    if (!starts && tokens % requests)
        return fail(BACON_EINVAL, "%d tokens are not the same number for %d requests: starts is needed",
                    tokens, requests);
    if (bacon_status rc = check_rows(q, q_token_stride, q_head_stride, "q")) return rc;
    if (!lengths || !table) return fail(BACON_EINVAL, "null argument");
    if (!out || !aligned16(out)) return fail(BACON_EINVAL, "out must be a 16-byte aligned device pointer");
    if (!std::isfinite(scale) || scale < 0.0f)
        return fail(BACON_EINVAL, "scale must be finite and not negative");
    if (scale == 0.0f) scale = 1.0f / std::sqrt((float)g.d);
    AttendArgs a{requests, layer, tokens, causal != 0, static_cast<const uint16_t*>(q),
                 q_token_stride, q_head_stride, starts, lengths, table, scale,
                 static_cast<uint16_t*>(out), lse, cache->fault_pending, 0, 0};
    cache->fault_pending = 0;
    DeviceGuard dg(cache->device);
    BACON_CUDA(launch_cache_attend(g, a, cache->sc, static_cast<cudaStream_t>(stream)), "attend launch");
    return BACON_OK;
}

bacon_status bacon_cache_sync(bacon_cache* cache, bacon_stream stream)
{
    g_last_error.clear();
    if (!cache) return fail(BACON_EINVAL, "null cache");
    DeviceGuard dg(cache->device);
    // all of it on the caller's stream, which the next call on it follows
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    int flag = 0;
    BACON_CUDA(cudaMemcpyAsync(&flag, cache->g.err, sizeof(int), cudaMemcpyDeviceToHost, st),
               "error flag read");
    BACON_CUDA(cudaStreamSynchronize(st), "stream synchronisation");
    if (!flag) return BACON_OK;
    // cleared before it is reported, so that the next call starts clean on
    // whichever stream; a block that gave up may have left counts of parts behind
    BACON_CUDA(cudaMemsetAsync(cache->sc.arrived, 0,
                               (const char*)(cache->g.err + 1) - (const char*)cache->sc.arrived, st),
               "error flag reset");
    BACON_CUDA(cudaStreamSynchronize(st), "stream synchronisation");
    if (flag == kCacheBadIndex)
        return fail(BACON_EINVAL, "a length, slot, page or query range was outside its array");
    if (flag == kCacheNoPages) return fail(BACON_ENOMEM, "the ring holds too few pages");
    if (flag == kCacheTimeout)
        return fail(BACON_ETIMEOUT, "an attention kernel timed out waiting on its pipeline");
    return fail(BACON_ECUDA, "unknown device error code %d", flag);
}

}  // extern "C"
