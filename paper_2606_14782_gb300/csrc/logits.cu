// Rules on logits: penalties, biases, masks, temperature, the best token and its
// log-probability in one pass.  Bound by bytes: a row's logits are read once and,
// if wanted, written once.
//
// A row belongs to a cluster of blocks, each with a part of the vocabulary.  The
// blocks read the row's history once between them and count every token in the
// block whose part it lies in, by atomics on distributed shared memory: a word a
// token, with the number of times in the answer, whether the history has it, and
// the last place of the row's bias list that names it.  Whole numbers only, so
// that no order changes a result.  The pass over the logits then looks at these
// words, and the maxima and sums of the parts meet in the first block.
#include "logits.h"

#include "common.cuh"
#include "values.cuh"

namespace bacon {
namespace {

constexpr int kThreads = 512;
constexpr float kLeast = 1e-30f;         // repetition and temperature
constexpr uint32_t kCount = 0xFFFFFu;    // of a token's word: times in the answer
constexpr uint32_t kSeen = 1u << 20;     // in the prompt
constexpr int kBiasShift = 21;           // place in the bias list, from 1
static_assert(kCount >= BACON_MAX_HISTORY && BACON_MAX_BIASES < 1 << (32 - kBiasShift), "a word's fields");

__device__ __forceinline__ void cluster_arrive()
{
    asm volatile("barrier.cluster.arrive;\n" ::: "memory");
}
__device__ __forceinline__ void cluster_wait()
{
    asm volatile("barrier.cluster.wait;\n" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_address(uint32_t local, int rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(a) : "r"(local), "r"(rank));
    return a;
}
__device__ __forceinline__ void cluster_add(uint32_t address, uint32_t v)
{
    asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;\n" ::"r"(address), "r"(v)
                 : "memory");
}
__device__ __forceinline__ void cluster_or(uint32_t address, uint32_t v)
{
    asm volatile("red.relaxed.cluster.shared::cluster.or.b32 [%0], %1;\n" ::"r"(address), "r"(v)
                 : "memory");
}

// A part's largest value, the sum of exp over it relative to that, and the key
// of its best token: the value's order, then the lowest number.
struct Part {
    float sum, top;
    unsigned long long best;
};

// Two parts as one; `rate` is log2(e) / temperature.
__device__ __forceinline__ Part join(const Part& a, const Part& b, float rate)
{
    Part p;
    p.best = a.best > b.best ? a.best : b.best;
    p.top = fmaxf(a.top, b.top);
    // an empty part (top -inf) has a sum of 0
    const float x = a.top == p.top ? a.sum : a.sum * fast_exp2((a.top - p.top) * rate);
    const float y = b.top == p.top ? b.sum : b.sum * fast_exp2((b.top - p.top) * rate);
    p.sum = x + y;
    return p;
}
__device__ __forceinline__ Part join_warp(Part p, float rate)
{
#pragma unroll
    for (int off = 16; off; off >>= 1) {
        Part o;
        o.sum = __shfl_xor_sync(0xFFFFFFFFu, p.sum, off);
        o.top = __shfl_xor_sync(0xFFFFFFFFu, p.top, off);
        o.best = __shfl_xor_sync(0xFFFFFFFFu, p.best, off);
        p = join(p, o, rate);
    }
    return p;
}

struct Rules {
    float repetition, frequency, presence, rate;  // rate: 1 / temperature
    const int32_t* bias_tokens;
    const float* bias_values;
};

// A logit under the rules before mask and temperature.
__device__ __forceinline__ float ruled(float x, uint32_t word, const Rules& r)
{
    if (word & (kCount | kSeen)) {
        x = x > 0.0f ? __fdiv_rn(x, r.repetition) : __fmul_rn(x, r.repetition);
        const uint32_t count = word & kCount;
        if (count) x = __fsub_rn(x, __fadd_rn(__fmul_rn(r.frequency, (float)count), r.presence));
    }
    if (word >> kBiasShift) x = __fadd_rn(x, r.bias_values[(word >> kBiasShift) - 1]);
    return x;
}

__device__ __forceinline__ float checked(const float* p, int row, float otherwise, bool positive, int* err)
{
    if (!p) return otherwise;
    const float v = p[row];
    if (isfinite(v) && (!positive || v >= kLeast)) return v;
    if (threadIdx.x == 0) atomicCAS(err, 0, kLogitsBadValue);
    return otherwise;
}

// kStep: values a thread takes at a time: 8 where rows start at 16 bytes, else 1.
template <int DTYPE, int OUT, int kStep>
__global__ void __launch_bounds__(kThreads)
logits_kernel(const __grid_constant__ bacon_logits_rows a, int vocab, int part, int blocks, int words,
              int* err)
{
    extern __shared__ uint32_t s_word[];  // [part], where there is a history or a list
    __shared__ Part s_part[16];
    __shared__ Part s_joined[16];
    const int row = blockIdx.x / blocks, rank = blockIdx.x % blocks;
    const int tid = threadIdx.x, lane = tid & 31;
    const int begin = min(vocab, rank * part), end = min(vocab, begin + part);
    const int length_in = a.lengths ? a.lengths[row] : 0;
    if (a.lengths && length_in == -1) return;  // all blocks of the row

    Rules rules;
    rules.repetition = checked(a.repetition, row, 1.0f, true, err);
    rules.frequency = checked(a.frequency, row, 0.0f, false, err);
    rules.presence = checked(a.presence, row, 0.0f, false, err);
    rules.rate = 1.0f / checked(a.temperature, row, 1.0f, true, err);
    rules.bias_tokens = a.bias_tokens ? a.bias_tokens + (long long)row * a.biases : nullptr;
    rules.bias_values = a.bias_tokens ? a.bias_values + (long long)row * a.biases : nullptr;

    const bool greedy = a.best || a.logprob || a.lse;
    // the row's blocks have all begun before one writes into another
    if (!words && greedy) cluster_arrive();
    if (words) {
        for (int i = tid; i < part; i += kThreads) s_word[i] = 0;
        cluster_arrive();
        cluster_wait();
        int length = a.tokens && a.lengths ? length_in : 0;
        const int prompt = a.prompt && length ? a.prompt[row] : 0;
        const int line = a.request ? a.request[row] : row;
        if (length && (length < 0 || length > a.capacity || prompt < 0 || prompt > length || line < 0 ||
                       line >= a.requests)) {
            if (tid == 0) atomicCAS(err, 0, kLogitsBadHistory);
            length = 0;
        }
        const int32_t* const history = a.tokens + (length ? line * a.token_stride : 0);
        const uint32_t base = smem_u32(s_word);
        for (int i = rank * kThreads + tid; i < length; i += blocks * kThreads) {
            const int token = history[i];
            if (token < 0 || token >= vocab) continue;
            const int owner = token / part;
            const uint32_t at = cluster_address(base + 4 * (token - owner * part), owner);
            if (i < prompt)
                cluster_or(at, kSeen);
            else
                cluster_add(at, 1);
        }
        cluster_arrive();
        cluster_wait();
        // the other fields of a word are settled: the largest word has the last place
        if (rules.bias_tokens) {
            for (int i = tid; i < a.biases; i += kThreads) {
                const int token = rules.bias_tokens[i];
                if (token >= begin && token < end) {
                    uint32_t* const w = &s_word[token - begin];
                    const uint32_t fields = *(volatile uint32_t*)w & (kCount | kSeen);
                    atomicMax(w, (uint32_t)(i + 1) << kBiasShift | fields);
                } else if ((token < -1 || token >= vocab) && rank == 0) {
                    atomicCAS(err, 0, kLogitsBadBias);
                }
            }
            __syncthreads();
        }
    }

    const float rate = rules.rate * 1.4426950408889634f;
    Part p{0.0f, -INFINITY, 0};
    const char* const in =
        static_cast<const char*>(a.logits) + row * a.row_stride * Eight<DTYPE>::kBytes;
    char* const out = a.out ? static_cast<char*>(a.out) + row * a.out_stride * Eight<OUT>::kBytes : nullptr;
    const uint32_t* const mask = a.mask ? a.mask + row * a.mask_stride : nullptr;
    // eight values at a time: neighbours, or every kThreads-th one
    constexpr int kGap = kStep == 8 ? 1 : kThreads;
    for (int v0 = begin + (kStep == 8 ? 8 * tid : tid); v0 < end; v0 += 8 * kThreads) {
        float x[8];
        if (kStep == 8 && v0 + 8 <= end) {
            Eight<DTYPE> raw;
            load_eight(raw, in + (long long)v0 * Eight<DTYPE>::kBytes);
            unpack_eight(raw, x);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int v = v0 + j * kGap;
                x[j] = v < end ? load_one<DTYPE>(in, v) : -INFINITY;
            }
        }
        if (words) {
            uint32_t w[8], any = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int v = v0 + j * kGap;
                w[j] = v < end ? s_word[v - begin] : 0;
                any |= w[j];
            }
            if (any)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (w[j]) x[j] = ruled(x[j], w[j], rules);
        }
        if (mask) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int v = v0 + j * kGap;
                if (v < end && !(mask[v >> 5] >> (v & 31) & 1)) x[j] = -INFINITY;
            }
        }
        if (out) {
            if (kStep == 8 && v0 + 8 <= end) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = x[j] * rules.rate;
                Eight<OUT> raw;
                pack_eight(raw, y);
                store_eight(out + (long long)v0 * Eight<OUT>::kBytes, raw);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int v = v0 + j * kGap;
                    if (v < end) store_one<OUT>(out, v, x[j] * rules.rate);
                }
            }
        }
        if (!greedy) continue;
        // numbers rise along j and along the loop: the first of equals stays
        float top = p.top;
        int at = -1;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (x[j] > top) {
                top = x[j];
                at = v0 + j * kGap;
            }
        if (at >= 0) {
            p.sum *= fast_exp2((p.top - top) * rate);  // 0 from -inf
            p.top = top;
            p.best = (unsigned long long)float_key(top + 0.0f) << 32 | (0xFFFFFFFFu - (uint32_t)at);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            // what is -inf adds nothing; NaN makes the sum NaN
            if (x[j] != -INFINITY) p.sum += fast_exp2((x[j] - p.top) * rate);
    }
    if (!greedy) return;

    if (!words) cluster_wait();
    p = join_warp(p, rate);
    if (lane == 0) s_part[tid >> 5] = p;
    __syncthreads();
    if (tid < 32) {
        p = tid < kThreads / 32 ? s_part[tid] : Part{0.0f, -INFINITY, 0};
        p = join_warp(p, rate);
        if (tid == 0) {
            const uint32_t to = cluster_address(smem_u32(&s_joined[rank]), 0);
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};\n" ::"r"(to), "f"(p.sum), "f"(p.top)
                         : "memory");
            asm volatile("st.shared::cluster.u64 [%0], %1;\n" ::"r"(to + 8), "l"(p.best) : "memory");
        }
    }
    cluster_arrive();
    cluster_wait();
    if (rank || tid >= 32) return;
    p = tid < blocks ? s_joined[tid] : Part{0.0f, -INFINITY, 0};
    p = join_warp(p, rate);
    if (tid == 0) {
        const bool none = p.best == 0 && !isnan(p.sum);
        const float more = logf(p.sum);
        if (a.best) a.best[row] = p.best ? (int)(0xFFFFFFFFu - (uint32_t)p.best) : -1;
        if (a.logprob) a.logprob[row] = none ? -INFINITY : p.best ? -more : NAN;
        if (a.lse)
            a.lse[row] = none ? -INFINITY : p.top == INFINITY ? INFINITY : p.top * rules.rate + more;
    }
}

template <int DTYPE, int OUT, int kStep>
cudaError_t go(const bacon_logits_rows& r, int vocab, int* err, cudaStream_t st)
{
    const bool words = (r.tokens && r.lengths) || (r.bias_tokens && r.biases);
    const int blocks = 8;
    const int part = ((vocab + blocks - 1) / blocks + 31) / 32 * 32;
    const size_t smem = words ? (size_t)part * 4 : 0;
    auto* const kernel = logits_kernel<DTYPE, OUT, kStep>;
    if (smem > 32 * 1024) {
        const cudaError_t e =
            cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = blocks;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)r.rows * blocks);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, r, vocab, part, blocks, (int)words, err);
}

template <int DTYPE, int OUT>
cudaError_t by_step(const bacon_logits_rows& r, int vocab, int* err, cudaStream_t st)
{
    const bool in = (reinterpret_cast<uintptr_t>(r.logits) & 15) == 0 &&
                    (r.rows == 1 || r.row_stride * Eight<DTYPE>::kBytes % 16 == 0);
    const bool out = !r.out || ((reinterpret_cast<uintptr_t>(r.out) & 15) == 0 &&
                                (r.rows == 1 || r.out_stride * Eight<OUT>::kBytes % 16 == 0));
    return in && out ? go<DTYPE, OUT, 8>(r, vocab, err, st) : go<DTYPE, OUT, 1>(r, vocab, err, st);
}

}  // namespace

cudaError_t launch_logits(const bacon_logits_rows& r, int vocab, int* err, cudaStream_t st)
{
    if (r.dtype == BACON_FP32) return by_step<BACON_FP32, BACON_FP32>(r, vocab, err, st);
    const bool wide = r.out_dtype == BACON_FP32;
    if (r.dtype == BACON_BF16)
        return wide ? by_step<BACON_BF16, BACON_FP32>(r, vocab, err, st)
                    : by_step<BACON_BF16, BACON_BF16>(r, vocab, err, st);
    return wide ? by_step<BACON_FP16, BACON_FP32>(r, vocab, err, st)
                : by_step<BACON_FP16, BACON_FP16>(r, vocab, err, st);
}

}  // namespace bacon
