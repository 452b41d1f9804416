// Rows of K and V into the pages of the cache with the positions put into K on the
// way, and into Q by further blocks of the same launch.  A run's rows of K are turned
// by lanes with eight pairs, through shared memory into the registers that the store
// keeps them in: what is saved against the two calls is a launch, and writing K and
// reading it again.  us: a token of 32 requests (32 and 8 heads, norms) 5.0, the two
// calls 3.1 and 3.1; turns of 5 requests, 3500 tokens (28 and 4 heads) 17.1, the two
// calls 8.7 and 9.5.  Short of the bytes' time (1.1 and 7 us): chains of a run's slots,
// its rows, its scale and its codes, which few blocks have anything beside.  Rotations
// that are not a multiple of sixteen have their pairs read again and spill 264 to 380
// bytes a thread: the same turns with 104 of 128 values turned 49 us with the pages loaded
// again, 24 with all.
#include "cache_store.cuh"

namespace bacon {
namespace {

template <int DTYPE, int FORMAT, int D>
struct StoreTurned {
    template <int PAIR>
    static cudaError_t pair(const CacheGeom& g, const StoreArgs& a, const StoreRotary& rotary, dim3 grid,
                            int window, cudaStream_t st)
    {
        const size_t stage = PAIR == kPairMemory ? 0 : (size_t)g.page * D * 2;
        return launch_first(store_kernel<DTYPE, FORMAT, D, PAIR, StoreRotary>, grid,
                            g.page * D / 8 / kChunks, stage, st, g, a, window, rotary);
    }
    static cudaError_t go(const CacheGeom& g, const StoreArgs& a, const StoreRotary& rotary, dim3 grid,
                          int window, cudaStream_t st)
    {
        return rotary.args.q_pair == kPairHalves    ? pair<kPairHalves>(g, a, rotary, grid, window, st)
               : rotary.args.q_pair == kPairSixteen ? pair<kPairSixteen>(g, a, rotary, grid, window, st)
                                                    : pair<kPairMemory>(g, a, rotary, grid, window, st);
    }
};

}  // namespace

cudaError_t launch_cache_store_rotated(const CacheGeom& g, const StoreArgs& a, const RotaryArgs& rotary,
                                       cudaStream_t st)
{
    StoreRotary r{rotary, {}};
    r.args.rows[1].heads = 0;  // these are the store's
    const int window = store_window(g, a, 2);
    dim3 grid((unsigned)((a.tokens + window - 1) / window), a.heads);
    if (r.args.rows[0].heads) {
        // blocks of the store's size, which begin when most of its own are through: more
        // and shorter pieces than rotary.cu has (3500 tokens of 28 heads: 17.1 us a call, 18.5
        // with its 512)
        const long long pieces = deal_rows(r.args, values_of_lane(r.args.q_pair), 2048, &r.deal);
        const int groups = (g.page * g.d / 8 / kChunks) >> r.deal.log_lanes;
        const long long blocks = (pieces + groups - 1) / groups;
        const long long more = (blocks + grid.x - 1) / grid.x;
        if (grid.y + more <= 65535) {
            grid.y += (unsigned)more;
        } else {  // so many heads that a grid has no room beside K's: Q by itself
            const cudaError_t e = launch_rotary(r.args, st);
            if (e != cudaSuccess) return e;
            r.args.rows[0].heads = 0;
        }
    }
    return by_type<StoreTurned>(g, a, r, grid, window, st);
}

}  // namespace bacon
