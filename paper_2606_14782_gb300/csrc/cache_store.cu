// Rows into the pages of the 8-bit cache and back: bound by their bytes, three
// of every element of a row one way or the other.  459k rows of K and V of 128
// are stored in 62 us and loaded in 54 (84 and 96 % of the measured copy
// bandwidth); a row of 256 units in 3.0 and 2.1.
//
// A run is the rows of one call that lie in one page one after the other.  A
// block takes a run of K and V: its rows are read once, into registers (2 x 4 x
// 16 bytes a thread at most), their largest finite magnitude gives the page's
// scale, and the codes leave as 8 bytes a thread.  A page that is appended to
// (the run starts above row 0) keeps its scale unless the new rows need a
// larger one; then its older rows are quantised again.  Blocks find their runs
// themselves: a run belongs to the block whose window of tokens it starts in,
// and one pass over the window's slots and a page's beyond marks where runs
// break.  The magnitudes are compared as 16-bit integers, two at a time; only
// when the largest is an infinity or NaN are they gone through again without
// such values.
#include "cache_store.cuh"

namespace bacon {
namespace {

// Eight codes as values.
template <int DTYPE, int FORMAT>
__device__ __forceinline__ uint4 values_of(uint2 c, float s)
{
    const float4 x = codes_float<FORMAT>(c.x), y = codes_float<FORMAT>(c.y);
    return make_uint4(pack16<DTYPE>(x.x * s, x.y * s), pack16<DTYPE>(x.z * s, x.w * s),
                      pack16<DTYPE>(y.x * s, y.y * s), pack16<DTYPE>(y.z * s, y.w * s));
}

// A thread takes 8 values of K and the same of V (one slot's latency for both)
// of two rows, so that a warp's stores are whole lines.
template <int DTYPE, int FORMAT, int D>
__global__ void __launch_bounds__(256)
load_kernel(CacheGeom g, int rows, const int32_t* slots, uint16_t* k_out, uint16_t* v_out)
{
    constexpr int kLanes = D / 8, kRows = 256 / kLanes;
    const int q = threadIdx.x % kLanes;
    const long long i0 = (long long)blockIdx.x * (2 * kRows) + threadIdx.x / kLanes;
    int slot[2];
    uint2 k[2], v[2];
    float ks[2], vs[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) slot[z] = i0 + z * kRows < rows ? slots[i0 + z * kRows] : -1;
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        k[z] = v[z] = make_uint2(0, 0);
        ks[z] = vs[z] = 0.0f;
        if (slot[z] >= 0 && slot[z] < (long long)g.pages << g.page_log2) {
            k[z] = *reinterpret_cast<const uint2*>(g.k + (size_t)slot[z] * D + q * 8);
            v[z] = *reinterpret_cast<const uint2*>(g.v + (size_t)slot[z] * D + q * 8);
            ks[z] = g.k_scale[slot[z] >> g.page_log2];
            vs[z] = g.v_scale[slot[z] >> g.page_log2];
        } else if (slot[z] != -1) {
            atomicCAS(g.err, 0, kCacheBadIndex);
        }
    }
#pragma unroll
    for (int z = 0; z < 2; ++z) {
        const long long i = i0 + z * kRows;
        if (i >= rows) break;
        *reinterpret_cast<uint4*>(k_out + i * D + q * 8) = values_of<DTYPE, FORMAT>(k[z], ks[z]);
        *reinterpret_cast<uint4*>(v_out + i * D + q * 8) = values_of<DTYPE, FORMAT>(v[z], vs[z]);
    }
}

template <int DTYPE, int FORMAT, int D>
struct Store {
    static cudaError_t go(const CacheGeom& g, const StoreArgs& a, dim3 grid, int window,
                          cudaStream_t st)
    {
        return launch_first(store_kernel<DTYPE, FORMAT, D, kNoPair, NoRotary>, grid,
                            g.page * D / 8 / kChunks, 0, st, g, a, window, NoRotary{});
    }
};
template <int DTYPE, int FORMAT, int D>
struct Load {
    static cudaError_t go(const CacheGeom& g, int rows, const int32_t* slots, void* k_out,
                          void* v_out, cudaStream_t st)
    {
        const int own = 2 * 256 / (D / 8);  // rows of a block
        return launch_first(load_kernel<DTYPE, FORMAT, D>, (unsigned)((rows + own - 1LL) / own),
                            256, 0, st, g, rows, slots, static_cast<uint16_t*>(k_out),
                            static_cast<uint16_t*>(v_out));
    }
};

}  // namespace

cudaError_t launch_cache_store(const CacheGeom& g, const StoreArgs& a, cudaStream_t st)
{
    const int window = store_window(g, a, 8);
    const dim3 grid((unsigned)((a.tokens + window - 1) / window), a.heads);
    return by_type<Store>(g, a, grid, window, st);
}

cudaError_t launch_cache_load(const CacheGeom& g, int rows, const int32_t* slots, void* k_out,
                              void* v_out, cudaStream_t st)
{
    return by_type<Load>(g, rows, slots, k_out, v_out, st);
}

}  // namespace bacon
