// Kernel interfaces of the 8-bit paged cache.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace bacon {

// Codes of the cache's error word (bacon_cache_sync names them).
constexpr int kCacheBadIndex = 1;   // a slot, page, length or query range outside its array
constexpr int kCacheNoPages = 2;    // the ring holds too few pages
constexpr int kCacheTimeout = 3;    // a bounded pipeline wait ran out

// Geometry and pools of a cache.
struct CacheGeom {
    int layers, hkv, hq, group, d;
    int page, page_log2, pages, max_blocks;
    int format, dtype;  // bacon_cache_format, bacon_dtype
    uint8_t* k;
    uint8_t* v;
    float* k_scale;
    float* v_scale;
    int* err;
};

struct PlanArgs {
    int units, requests;
    const int32_t* lengths;  // null: 0 (locate only)
    const int32_t* added;    // null: 1 (per request only)
    int per_unit;
    int32_t* table;
    const int32_t* ring;     // null: pages are there already (locate)
    const int32_t* state;
    int rows;
    int32_t* slots;
    int32_t* lengths_out;
    int32_t* state_out;
};
cudaError_t launch_cache_plan(const CacheGeom& g, const PlanArgs& a, cudaStream_t st);
// Pages back to the ring: of requests that are done, or (fewer) of the last
// tokens of every request's units.
cudaError_t launch_cache_release(const CacheGeom& g, int units, const int32_t* done,
                                 const int32_t* fewer, int32_t* lengths, int32_t* table,
                                 int32_t* ring, int32_t* state, cudaStream_t st);

struct StoreArgs {
    int tokens, heads;
    const uint16_t* rows[2];      // K, V
    long long token_stride[2];
    long long head_stride[2];
    const int32_t* slots;
};
cudaError_t launch_cache_store(const CacheGeom& g, const StoreArgs& a, cudaStream_t st);
struct RotaryArgs;  // rotary.cuh
cudaError_t launch_cache_store_rotated(const CacheGeom& g, const StoreArgs& a,
                                       const RotaryArgs& rotary, cudaStream_t st);
cudaError_t launch_cache_load(const CacheGeom& g, int rows, const int32_t* slots, void* k_out,
                              void* v_out, cudaStream_t st);

struct AttendArgs {
    int requests, layer, tokens, causal;
    const uint16_t* q;
    long long q_token_stride, q_head_stride;
    const int32_t* starts;
    const int32_t* lengths;
    const int32_t* table;
    float scale;
    uint16_t* out;
    float* lse;
    int fault;              // test only: > 0 withholds a load of block 0's tile fault - 1
    long long above, upto;  // requests with more than `above` and at most `upto` rows
                            // (queries x heads of a kv-head) are the kernel's
};
// What a cache keeps for its attention calls: descriptors of the pools (rows
// of d bytes) and room for the partial sums of items that lie in several
// blocks, two a block.
constexpr int kBlocksPerSm = 3;
struct SplitScratch {
    CUtensorMap kmap, vmap;
    int sms;
    float* out;    // [2 sms kBlocksPerSm][32 columns][128]
    float* sums;   // [2 sms kBlocksPerSm][32 columns][maximum, sum]
    int* arrived;  // [sms kBlocksPerSm] parts that are there, 0 between calls
    float* many_out;    // [2 sms][2 row tiles][32 quads of dims][128 rows][4]
    float2* many_sums;  // [2 sms][2][128] maximum, sum
    int* many_arrived;  // [sms][2]
};
// Requests of up to a.upto rows by one kernel (`typical`: rows of most of them),
// of more than a.above by the other; launch_cache_attend chooses.
cudaError_t launch_cache_few(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc,
                             int typical, cudaStream_t st);
cudaError_t launch_cache_many(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc,
                              cudaStream_t st);
cudaError_t launch_cache_attend(const CacheGeom& g, const AttendArgs& a, const SplitScratch& sc,
                                cudaStream_t st);
// One descriptor over a pool of `rows` rows of d bytes, 16 of them a load.
bool encode_pool_map(CUtensorMap* out, const void* base, int d, long long rows);

}  // namespace bacon
