// Rotary positions of Q and K.  Bound by bytes: every value is read and written
// once.  A lane has eight neighbouring values of a row (16 bytes of 16-bit types),
// the lanes of a row form a group of a power of two, and a group turns several
// heads of one token with the same cosines and sines: per row what is left is
// two products a value.
#include "rotary.cuh"

namespace bacon {
namespace {

constexpr int kThreads = 256;

template <int DTYPE, int PAIR, bool NORM>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const __grid_constant__ RotaryArgs a, RotaryDeal deal)
{
    const unsigned groups = kThreads >> deal.log_lanes;
    rotate_piece<DTYPE, PAIR, NORM>(a, deal, blockIdx.x * groups + (threadIdx.x >> deal.log_lanes));
}

template <int DTYPE, int PAIR>
cudaError_t go(const RotaryArgs& a, cudaStream_t st)
{
    RotaryDeal deal{0, 1, {0, 0}};
    while (8 << deal.log_lanes < a.table.head_dim) ++deal.log_lanes;
    const int most = a.rows[0].heads > a.rows[1].heads ? a.rows[0].heads : a.rows[1].heads;
    // heads of a token that share a group and its angles: as few as fill the machine
    const long long rows = a.table.tokens * (a.rows[0].heads + a.rows[1].heads);
    const long long groups = 152LL * 2048 >> deal.log_lanes;
    while (deal.per < 32 && deal.per < most && rows / deal.per > groups) deal.per *= 2;
    for (int i = 0; i < 2; ++i) deal.chunks[i] = chunks_of(a.rows[i].heads, deal.per);
    const long long threads = a.table.tokens * (deal.chunks[0] + deal.chunks[1]) << deal.log_lanes;
    const unsigned blocks = (unsigned)((threads + kThreads - 1) / kThreads);
    if (a.rows[0].weight || a.rows[1].weight)
        return launch_first(rotary_kernel<DTYPE, PAIR, true>, blocks, kThreads, 0, st, a, deal);
    return launch_first(rotary_kernel<DTYPE, PAIR, false>, blocks, kThreads, 0, st, a, deal);
}

template <int DTYPE>
cudaError_t by_pair(const RotaryArgs& a, cudaStream_t st)
{
    return a.pair == kPairLane  ? go<DTYPE, kPairLane>(a, st)
           : a.pair == kPairOwn ? go<DTYPE, kPairOwn>(a, st)
                                : go<DTYPE, kPairMemory>(a, st);
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t st)
{
    return a.dtype == BACON_BF16   ? by_pair<BACON_BF16>(a, st)
           : a.dtype == BACON_FP16 ? by_pair<BACON_FP16>(a, st)
                                   : by_pair<BACON_FP32>(a, st);
}

}  // namespace bacon
