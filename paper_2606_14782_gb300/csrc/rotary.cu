// Rotary positions of Q and K.  Bound by bytes: every value is read and written
// once.  A lane has eight pairs of a row, as two groups of 16 bytes of 16-bit types,
// the lanes of a row form a group of a power of two, and a group turns several
// heads of one token with the same cosines and sines: per row what is left is two
// products a value.  Rows that do not allow it have eight values a lane.
#include "rotary.cuh"

namespace bacon {
namespace {

constexpr int kThreads = 256;

// Three blocks an SM where 80 registers do (four prompts of 16384 tokens: 163 us, 166
// with two), two with norms where lanes have whole pairs and where pairs are read again,
// which would spill far more.  Spilled all the same, bytes a thread: with eight values a
// lane and the others by shuffles 4, of fp32 20; fp32 interleaved without norms 16; fp32
// read again, with norms, 24.  Two prompts of 16384 tokens of 28 and 4 heads in bf16, 80 us of bytes:
// interleaved 82, with 104 of 128 values turned, whose pairs are read again, 206.  With
// norms, 95000 tokens of 6 and 2 heads of 128: 103 us for 58 of bytes; fp32, 2800 tokens
// of 48 and 16 heads: 42 for 27.
template <int DTYPE, int PAIR, bool NORM>
__global__ void __launch_bounds__(kThreads, PAIR == kPairMemory ? 2 : NORM && PAIR >= kPairHalves ? 2 : 3)
rotary_kernel(const __grid_constant__ RotaryArgs a, RotaryDeal deal)
{
    const unsigned groups = kThreads >> deal.log_lanes;
    rotate_piece<DTYPE, PAIR, NORM>(a, deal, blockIdx.x * groups + (threadIdx.x >> deal.log_lanes));
}

template <int DTYPE, int PAIR, bool NORM>
cudaError_t go(const RotaryArgs& a, cudaStream_t st)
{
    RotaryDeal deal;
    // (5003 tokens of 14 heads of 64, with norms: 6.2 us, and 10.0 with 2048)
    const long long threads = deal_rows(a, values_of_lane(PAIR), 512, &deal) << deal.log_lanes;
    const unsigned blocks = (unsigned)((threads + kThreads - 1) / kThreads);
    return launch_first(rotary_kernel<DTYPE, PAIR, NORM>, blocks, kThreads, 0, st, a, deal);
}

template <int DTYPE>
cudaError_t by_pair(const RotaryArgs& a, cudaStream_t st)
{
    const bool norm = a.rows[0].weight || a.rows[1].weight;
    switch (a.q_pair) {
        case kPairHalves: return norm ? go<DTYPE, kPairHalves, true>(a, st) : go<DTYPE, kPairHalves, false>(a, st);
        case kPairSixteen: return norm ? go<DTYPE, kPairSixteen, true>(a, st) : go<DTYPE, kPairSixteen, false>(a, st);
        case kPairLane: return go<DTYPE, kPairLane, true>(a, st);
        case kPairOwn: return go<DTYPE, kPairOwn, true>(a, st);
        default: return norm ? go<DTYPE, kPairMemory, true>(a, st) : go<DTYPE, kPairMemory, false>(a, st);
    }
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t st)
{
    return a.dtype == BACON_BF16   ? by_pair<BACON_BF16>(a, st)
           : a.dtype == BACON_FP16 ? by_pair<BACON_FP16>(a, st)
                                   : by_pair<BACON_FP32>(a, st);
}

}  // namespace bacon
