// Rows of K and V into the pages of the cache with the positions put into K on the
// way, and into Q by further blocks of the same launch.  K's rows are turned in the
// registers that the store keeps them in: what is saved against the two calls is a
// launch, and writing K and reading it again.
#include "cache_store.cuh"

namespace bacon {
namespace {

template <int DTYPE, int FORMAT, int D>
struct StoreTurned {
    template <int PAIR>
    static cudaError_t pair(const CacheGeom& g, const StoreArgs& a, const StoreRotary& rotary, dim3 grid,
                            int window, cudaStream_t st)
    {
        return launch_first(store_kernel<DTYPE, FORMAT, D, PAIR, StoreRotary>, grid,
                            g.page * D / 8 / kChunks, 0, st, g, a, window, rotary);
    }
    static cudaError_t go(const CacheGeom& g, const StoreArgs& a, const StoreRotary& rotary, dim3 grid,
                          int window, cudaStream_t st)
    {
        return rotary.args.pair == kPairLane  ? pair<kPairLane>(g, a, rotary, grid, window, st)
               : rotary.args.pair == kPairOwn ? pair<kPairOwn>(g, a, rotary, grid, window, st)
                                              : pair<kPairMemory>(g, a, rotary, grid, window, st);
    }
};

}  // namespace

cudaError_t launch_cache_store_rotated(const CacheGeom& g, const StoreArgs& a, const RotaryArgs& rotary,
                                       cudaStream_t st)
{
    StoreRotary r{rotary, {g.d == 128 ? 4 : 3, 1, {0, 0}}};
    r.args.rows[1].heads = 0;  // these are the store's
    const int window = store_window(g, a);
    dim3 grid((unsigned)((a.tokens + window - 1) / window), a.heads);
    const int heads = rotary.rows[0].heads;
    if (heads) {
        // a block's threads are the store's; its groups take as many heads each as
        // leave a few blocks per SM
        const long long rows = (long long)a.tokens * heads;
        const long long groups = (152LL * 2048) >> r.deal.log_lanes;
        while (r.deal.per < 32 && r.deal.per < heads && rows / r.deal.per > groups) r.deal.per *= 2;
        r.deal.chunks[0] = chunks_of(heads, r.deal.per);
        const long long items = (long long)a.tokens * r.deal.chunks[0], own = g.page / 4;
        const long long blocks = (items + own - 1) / own;
        const long long more = (blocks + grid.x - 1) / grid.x;
        if (grid.y + more > 65535) return cudaErrorInvalidConfiguration;
        grid.y += (unsigned)more;
    }
    return by_type<StoreTurned>(g, a, r, grid, window, st);
}

}  // namespace bacon
