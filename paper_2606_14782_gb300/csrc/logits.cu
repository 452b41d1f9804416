// Rules on logits: penalties, biases, masks, temperature, the best token and its
// log-probability in one pass.  Bound by bytes: a row's logits are read once and,
// if wanted, written once.
//
// A row belongs to a cluster of blocks, which have groups of 256 neighbouring tokens
// in turn, so that the many uses of a few low numbers are spread.  A block goes
// through the row's whole history and counts its own tokens by atomics on a word a
// token in its shared memory: the number of times in the answer, whether the prompt
// has it, and the last place of the row's bias list that names it.  Whole numbers
// only, so that no order changes a result.  (Each entry read by one block and counted
// in the block that has its token, by atomics on distributed shared memory, took
// about eight cycles an entry.)  Of long prompts, where one bit a token is enough,
// the blocks read a part each and exchange the bits: 4 rows with histories of 100000
// tokens 17 us, 31 without.  The pass over the logits then looks at these words, and
// the maxima and sums of the parts meet in the first block.  256 rows of 131072 fp32
// logits with all rules 92 us, 45 % of the measured copy bandwidth; without history
// and mask 53 us: counting and the rules take as many instructions as the pass, and
// a block's steps wait for one another.  One row of 32000: 5.7 us, a chain of its
// parameters, its history, its logits and the cluster's meeting.
#include "logits.h"

#include "common.cuh"
#include "values.cuh"

namespace bacon {
namespace {

// (24 warps of an SM in place of 48, by 256 threads a block: the largest case 115 us for 92)
constexpr int kThreads = 512;
constexpr int kGroup = 256;              // tokens that a warp takes together
constexpr int kSplit = 16384;           // tokens of a prompt that a row's blocks share
constexpr int kMostOfThree = 70;         // groups of a block of which three fit an SM's shared memory
constexpr int kMostOfTwo = 112;          // ... at most: of the largest vocabulary, by sixteen blocks
constexpr float kLeast = 1e-30f;         // repetition and temperature
constexpr uint32_t kCount = 0xFFFFFu;    // of a token's word: times in the answer
constexpr uint32_t kSeen = 1u << 20;     // in the prompt
constexpr int kBiasShift = 21;           // place in the bias list, from 1
static_assert(kMostOfTwo * kGroup * 16 >= BACON_MAX_VOCAB && kMostOfTwo >= kMostOfThree, "room for every vocabulary");
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
// Several parts' largest value, where it is first, and the sum of exp relative to it.
struct alignas(16) Part {
    float sum, top;
    uint32_t at;  // 0xFFFFFFFF: no value above -inf
};

// A warp's parts as one; `rate` is log2(e) / temperature.
__device__ __forceinline__ Part join_warp(const Part& p, float rate)
{
    Part all;
    const uint32_t key = float_key(p.top + 0.0f), most = __reduce_max_sync(0xFFFFFFFFu, key);  // (0 for -0)
    all.top = key_float(most);
    all.at = __reduce_min_sync(0xFFFFFFFFu, key == most ? p.at : 0xFFFFFFFFu);
    // an empty part (top -inf) has a sum of 0
    all.sum = key == most ? p.sum : p.sum * fast_exp2((p.top - all.top) * rate);
#pragma unroll
    for (int off = 16; off; off >>= 1) all.sum += __shfl_xor_sync(0xFFFFFFFFu, all.sum, off);
    return all;
}

// Whose a token is and where its word lies: the groups of kGroup tokens go to the
// blocks in turn.
struct Owner {
    uint32_t vocab, rank, others, words;  // others: blocks - 1; words: the shared address
    int log_blocks;
    __device__ __forceinline__ uint32_t apart(uint32_t t) const { return (t ^ rank * kGroup) & others * kGroup; }
    __device__ __forceinline__ bool has(uint32_t t) const { return t < vocab && apart(t) == 0; }
    __device__ __forceinline__ uint32_t place(uint32_t t) const
    {
        return (t >> log_blocks & ~(kGroup - 1u)) | (t & (kGroup - 1u));
    }
    // without a branch: in nearly every entry some lane has a token of the block
    __device__ __forceinline__ void said(uint32_t t) const
    {
        asm volatile(
            "{\n.reg .pred p;\nsetp.lt.u32 p, %1, %2;\nsetp.eq.and.u32 p, %3, 0, p;\n"
            "@p red.shared.add.u32 [%0], 1;\n}\n" ::"r"(words + 4 * place(t)),
            "r"(t), "r"(vocab), "r"(apart(t))
            : "memory");
    }
    // (a prompt may have one token many times on end)
    __device__ __forceinline__ void asked(uint32_t t, uint32_t before) const
    {
        asm volatile(
            "{\n.reg .pred p;\nsetp.lt.u32 p, %1, %2;\nsetp.eq.and.u32 p, %3, 0, p;\n"
            "setp.ne.and.u32 p, %1, %4, p;\n@p red.shared.or.b32 [%0], %5;\n}\n" ::"r"(words + 4 * place(t)),
            "r"(t), "r"(vocab), "r"(apart(t)), "r"(before), "r"(kSeen)
            : "memory");
    }
};
// A bit of a map of the whole vocabulary.
__device__ __forceinline__ void mark(uint32_t map, uint32_t t, uint32_t before, uint32_t vocab)
{
    asm volatile(
        "{\n.reg .pred p;\nsetp.lt.u32 p, %1, %2;\nsetp.ne.and.u32 p, %1, %3, p;\n"
        "@p red.shared.or.b32 [%0], %4;\n}\n" ::"r"(map + t / 32 * 4),
        "r"(t), "r"(vocab), "r"(before), "r"(1u << (t & 31))
        : "memory");
}

__device__ __forceinline__ uint32_t cluster_load(uint32_t address)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];\n" : "=r"(v) : "r"(address) : "memory");
    return v;
}

struct Rules {
    float repetition, frequency, presence, rate;  // rate: 1 / temperature
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

// A row's parameter, or what stands for it if it is out of its range.
__device__ __forceinline__ float checked(float v, float otherwise, bool positive, int* err)
{
    if (isfinite(v) && (!positive || v >= kLeast)) return v;
    if (threadIdx.x == 0) atomicCAS(err, 0, kLogitsBadValue);
    return otherwise;
}

// kStep: values a thread takes at a time: 8 where rows start at 16 bytes, else 1.
// kResident: blocks of an SM: 3 where there are as many (the largest case: 94 us for
// 107 with 2), else 2 and more registers (one row: 5.5 us for 5.8).
template <int DTYPE, int OUT, int kStep, int kResident>
__global__ void __launch_bounds__(kThreads, kResident)
logits_kernel(const __grid_constant__ bacon_logits_rows a, int vocab, int log_blocks, int words, int* err)
{
    extern __shared__ __align__(16) uint32_t s_word[];  // of the block's groups, if there is a history or list
    __shared__ Part s_part[16];
    __shared__ Part s_joined[16];
    const int blocks = 1 << log_blocks, row = blockIdx.x >> log_blocks, rank = blockIdx.x & (blocks - 1);
    const int tid = threadIdx.x, lane = tid & 31;
    // the block's k-th group is the row's number k blocks + rank
    const int groups = ((vocab + kGroup - 1) / kGroup - rank + blocks - 1) >> log_blocks;
    const Owner owner{(uint32_t)vocab, (uint32_t)rank, blocks - 1u, smem_u32(s_word), log_blocks};
    // all that the row's parameters say, on its way together
    const int length_in = a.lengths ? a.lengths[row] : 0;
    const int prompt_in = a.prompt ? a.prompt[row] : 0, line = a.request ? a.request[row] : row;
    const float repetition = a.repetition ? a.repetition[row] : 1.0f;
    const float frequency = a.frequency ? a.frequency[row] : 0.0f;
    const float presence = a.presence ? a.presence[row] : 0.0f;
    const float temperature = a.temperature ? a.temperature[row] : 1.0f;
    const int32_t* const bias_tokens = a.bias_tokens ? a.bias_tokens + (long long)row * a.biases : nullptr;
    const int first_bias = bias_tokens && tid < a.biases ? bias_tokens[tid] : -1;
    if (a.lengths && length_in == -1) return;  // all blocks of the row
    Rules rules;
    rules.repetition = checked(repetition, 1.0f, true, err);
    rules.frequency = checked(frequency, 0.0f, false, err);
    rules.presence = checked(presence, 0.0f, false, err);
    rules.rate = 1.0f / checked(temperature, 1.0f, true, err);
    rules.bias_values = a.bias_tokens ? a.bias_values + (long long)row * a.biases : nullptr;

    const char* const in =
        static_cast<const char*>(a.logits) + row * a.row_stride * Eight<DTYPE>::kBytes;
    const bool greedy = a.best || a.logprob || a.lse;
    // the row's blocks have all begun before one writes into another
    if (greedy) cluster_arrive();
    uint32_t* const s_seen = s_word + (((vocab + kGroup - 1) / kGroup + blocks - 1) >> log_blocks) * kGroup;
    bool split = false;  // what the prompt has is in s_seen, a bit a token
    if (words) {
        int length = a.tokens && a.lengths ? length_in : 0;
        if (length && (length < 0 || length > a.capacity || prompt_in < 0 || prompt_in > length || line < 0 ||
                       line >= a.requests)) {
            if (tid == 0) atomicCAS(err, 0, kLogitsBadHistory);
            length = 0;
        }
        const int prompt = length ? prompt_in : 0;
        const int32_t* const history = a.tokens + (length ? line * a.token_stride : 0);
        constexpr int kFlight = 4;  // loads of a thread that are on their way together
        int4 token[kFlight];
        // entries from .. to of the history: four a load, from the last multiple of 16
        // bytes before them; use(the first one's number, the four)
        const auto entries = [&](int from, int to, const auto& meanwhile, const auto& use) {
            const int lead = (int)(reinterpret_cast<uintptr_t>(history + from) >> 2) & 3;
            const int loads = (to - from + lead + 3) / 4;
            const auto fetch = [&](int g0) {
#pragma unroll
                for (int k = 0; k < kFlight; ++k) {
                    const int g = g0 + k * kThreads, i = from + 4 * g - lead;
                    token[k] = make_int4(-1, -1, -1, -1);
                    if (g >= loads) continue;
                    if (i >= from && i + 4 <= to) {
                        token[k] = *reinterpret_cast<const int4*>(history + i);
                    } else {
                        if (i >= from) token[k].x = history[i];
                        if (i + 1 >= from && i + 1 < to) token[k].y = history[i + 1];
                        if (i + 2 >= from && i + 2 < to) token[k].z = history[i + 2];
                        if (i + 3 < to) token[k].w = history[i + 3];
                    }
                }
            };
            if (tid < loads) fetch(tid);
            meanwhile();
            for (int g0 = tid; g0 < loads; g0 += kFlight * kThreads) {
                if (g0 != tid) fetch(g0);
#pragma unroll
                for (int k = 0; k < kFlight; ++k) {
                    use(from + 4 * (g0 + k * kThreads) - lead, token[k]);
                }
            }
        };
        const auto clear = [&](int count) {
            for (int i = tid; i < (count + 3) / 4; i += kThreads)
                reinterpret_cast<uint4*>(s_word)[i] = make_uint4(0, 0, 0, 0);
            __syncthreads();
        };
        split = prompt >= kSplit && blocks > 1;
        if (split) {
            // whether the prompt has a token is one bit: each block goes through a part
            // of a long prompt into a map of the whole vocabulary, and then takes its own
            // tokens' words from everybody's
            const int part = (prompt + blocks - 1) >> log_blocks, from = min(prompt, rank * part);
            entries(from, min(prompt, from + part), [&] { clear((vocab + kGroup - 1) / kGroup * (kGroup / 32)); },
                    [&](int, const int4& t) {
                        mark(owner.words, t.x, ~t.x, vocab);
                        mark(owner.words, t.y, t.x, vocab);
                        mark(owner.words, t.z, t.y, vocab);
                        mark(owner.words, t.w, t.z, vocab);
                    });
            if (greedy) cluster_wait();
            cluster_arrive();
            cluster_wait();
            for (int i = tid; i < groups * (kGroup / 32); i += kThreads) {
                const uint32_t at = owner.words + (((i >> 3) << log_blocks) + rank) * kGroup / 8 + (i & 7) * 4;
                uint32_t bits = 0;
                for (int r = 0; r < blocks; ++r) bits |= cluster_load(cluster_address(at, r));
                s_seen[i] = bits;
            }
            cluster_arrive();
            cluster_wait();
        }
        entries(split ? prompt : 0, length, [&] { clear(groups * kGroup); },
                [&](int i, const int4& t) {
                    if (i >= prompt) {
                        owner.said(t.x);
                        owner.said(t.y);
                        owner.said(t.z);
                        owner.said(t.w);
                    } else if (i + 4 <= prompt) {
                        owner.asked(t.x, ~t.x);
                        owner.asked(t.y, t.x);
                        owner.asked(t.z, t.y);
                        owner.asked(t.w, t.z);
                    } else {
                        owner.asked(t.x, ~t.x);
                        i + 1 < prompt ? owner.asked(t.y, ~t.y) : owner.said(t.y);
                        i + 2 < prompt ? owner.asked(t.z, ~t.z) : owner.said(t.z);
                        owner.said(t.w);
                    }
                });
        __syncthreads();
        // the other fields of a word are settled: the largest word has the last place
        if (bias_tokens) {
            for (int i = tid; i < a.biases; i += kThreads) {
                const int token = i == tid ? first_bias : bias_tokens[i];
                if (owner.has(token)) {
                    const uint32_t at = owner.place(token);
                    uint32_t* const w = &s_word[at];
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
    Part p{0.0f, -INFINITY, 0xFFFFFFFFu};
    char* const out = a.out ? static_cast<char*>(a.out) + row * a.out_stride * Eight<OUT>::kBytes : nullptr;
    const uint32_t* const mask = a.mask ? a.mask + row * a.mask_stride : nullptr;
    // a lane has eight neighbours of a group, or every 32nd token from its own
    constexpr int kGap = kStep == 8 ? 1 : 32;
    const Pair by_rate = pair_of(rules.rate, rules.rate), by_log = pair_of(rate, rate);
    for (int k = tid >> 5; k < groups; k += kThreads / 32) {
        const int v0 = ((k << log_blocks) + rank) * kGroup + (kStep == 8 ? 8 : 1) * lane;
        const bool whole = kStep == 8 && v0 + 8 <= vocab;
        Piece piece;
        if (whole) {
            Eight<DTYPE> raw;
            load_eight(raw, in + (long long)v0 * Eight<DTYPE>::kBytes);
            open_piece(raw, piece);
        } else {  // -inf behind the row's end
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int v = v0 + j * kGap;
                x[j] = v < vocab ? load_one<DTYPE>(in, v) : -INFINITY;
            }
            set_floats(piece, x);
        }
        if (words) {
            uint32_t* const words_here = s_word + k * kGroup + (kStep == 8 ? 8 : 1) * lane;
            uint32_t w[8], some = 0;
            const auto read = [&] {
                if (kStep == 8) {
                    const uint4* const q = reinterpret_cast<const uint4*>(words_here);
                    const uint4 lo = q[0], hi = q[1];
                    w[0] = lo.x, w[1] = lo.y, w[2] = lo.z, w[3] = lo.w;
                    w[4] = hi.x, w[5] = hi.y, w[6] = hi.z, w[7] = hi.w;
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) w[j] = words_here[32 * j];
                }
            };
            read();
#pragma unroll
            for (int j = 0; j < 8; ++j) some |= (w[j] != 0) << j;
            uint32_t seen = 0;
            if (split) {
                if (kStep == 8)
                    seen = reinterpret_cast<const uint8_t*>(s_seen)[k * (kGroup / 8) + lane];
                else
#pragma unroll
                    for (int j = 0; j < 8; ++j) seen |= (s_seen[k * 8 + j] >> lane & 1) << j;
                some |= seen;
            }
            if (some) {
                // few of the eight, so each in its turn: its word becomes the logit that
                // the rules make of it (eight at once: 103 us for 94 of the largest case)
                float x[8];
                get_floats(piece, x);
                for (uint32_t left = some; left; left &= left - 1) {
                    const int j = __ffs(left) - 1;
                    const float raw = load_one<DTYPE>(in, v0 + j * kGap);
                    words_here[j * kGap] = __float_as_uint(ruled(raw, words_here[j * kGap] | (seen >> j & 1 ? kSeen : 0), rules));
                }
                read();
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (some >> j & 1) x[j] = __uint_as_float(w[j]);
                set_floats(piece, x);
            }
        }
        if (mask) {
            uint32_t allowed = 0;
            if (kStep == 8) {
                if (v0 < vocab) allowed = reinterpret_cast<const uint8_t*>(mask)[v0 >> 3];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int v = v0 + j * kGap;
                    if (v < vocab) allowed |= (mask[v >> 5] >> (v & 31) & 1) << j;
                }
            }
            if (allowed != 0xFF) {
                float x[8];
                get_floats(piece, x);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (!(allowed >> j & 1)) x[j] = -INFINITY;
                set_floats(piece, x);
            }
        }
        if (out) {
            Piece y;
#pragma unroll
            for (int j = 0; j < 4; ++j) y.p[j] = mul2(piece.p[j], by_rate);
            if (whole) {
                Eight<OUT> raw;
                close_piece(raw, y);
                store_eight(out + (long long)v0 * Eight<OUT>::kBytes, raw);
            } else {
                float f[8];
                get_floats(y, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int v = v0 + j * kGap;
                    if (v < vocab) store_one<OUT>(out, v, f[j]);
                }
            }
        }
        if (!greedy) continue;
        float x[8];
        get_floats(piece, x);
        const float top = max3f(max3f(x[0], x[1], x[2]), max3f(x[3], x[4], x[5]), fmaxf(x[6], x[7]));
        if (top > p.top) {
            // numbers rise along j and along the loop: the first of equals stays
            int at = 0;
#pragma unroll
            for (int j = 7; j >= 0; --j)
                if (x[j] == top) at = j;
            p.sum *= fast_exp2((p.top - top) * rate);  // 0 from -inf
            p.top = top;
            p.at = v0 + at * kGap;
        }
        // what is -inf adds nothing, while there is nothing else too; an infinity makes the
        // sum one, and NaN makes it NaN
        const float less = fabsf(p.top) == INFINITY ? 0.0f : -p.top;
        const Pair off = pair_of(less, less);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = floats_of(mul2(add2(piece.p[j], off), by_log));
            p.sum += fast_exp2(f.x) + fast_exp2(f.y);
        }
    }
    if (!greedy) return;

    if (!split) cluster_wait();
    p = join_warp(p, rate);
    if (lane == 0) s_part[tid >> 5] = p;
    __syncthreads();
    if (tid < 32) {
        p = tid < kThreads / 32 ? s_part[tid] : Part{0.0f, -INFINITY, 0xFFFFFFFFu};
        p = join_warp(p, rate);
        if (tid == 0) {
            const uint32_t to = cluster_address(smem_u32(&s_joined[rank]), 0);
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};\n" ::"r"(to), "f"(p.sum), "f"(p.top)
                         : "memory");
            asm volatile("st.shared::cluster.u32 [%0], %1;\n" ::"r"(to + 8), "r"(p.at) : "memory");
        }
    }
    cluster_arrive();
    cluster_wait();
    if (rank || tid >= 32) return;
    p = tid < blocks ? s_joined[tid] : Part{0.0f, -INFINITY, 0xFFFFFFFFu};
    p = join_warp(p, rate);
    if (tid == 0) {
        const bool found = p.at != 0xFFFFFFFFu, none = !found && !isnan(p.sum);
        const float more = logf(p.sum);
        if (a.best) a.best[row] = found ? (int)p.at : -1;
        if (a.logprob) a.logprob[row] = none ? -INFINITY : found && p.top < INFINITY ? -more : NAN;
        if (a.lse) a.lse[row] = none ? -INFINITY : p.top * rules.rate + more;
    }
}

template <int DTYPE, int OUT, int kStep, int kResident>
cudaError_t start(const bacon_logits_rows& r, int vocab, int blocks, int* err, cudaStream_t st)
{
    const bool words = (r.tokens && r.lengths) || (r.bias_tokens && r.biases);
    int log_blocks = 0;
    while (1 << log_blocks < blocks) ++log_blocks;
    const int groups = ((vocab + kGroup - 1) / kGroup + blocks - 1) / blocks;  // of a block, at most
    const auto bytes = [](int groups) { return (size_t)groups * (kGroup + kGroup / 32) * 4; };
    const size_t smem = words ? bytes(groups) : 0;
    auto* const kernel = logits_kernel<DTYPE, OUT, kStep, kResident>;
    if (smem > 32 * 1024) {
        // what any call may need: the limit is the kernel's, and a smaller one could come
        // between another thread's limit and its launch
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)bytes(kResident == 3 ? kMostOfThree : kMostOfTwo));
        if (e != cudaSuccess) return e;
    }
    if (blocks > 8) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
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
    return cudaLaunchKernelEx(&cfg, kernel, r, vocab, log_blocks, (int)words, err);
}

template <int DTYPE, int OUT, int kStep>
cudaError_t go(const bacon_logits_rows& r, int vocab, int* err, cudaStream_t st)
{
    // blocks of a row: eight, or sixteen when rows are few; no more than have
    // something to do, be it logits or tokens of a long history
    int blocks = r.rows <= 152 / 8 ? 16 : 8;
    while (blocks > 1 && vocab <= blocks / 2 * kThreads * 8 && vocab <= BACON_MAX_VOCAB / 16 &&
           r.capacity <= blocks * kThreads)
        blocks /= 2;
    // so many words that three blocks would not fit an SM (34 rows of 255141 logits:
    // 47 us with eight, 30 with sixteen)
    if (vocab > kGroup * kMostOfThree * blocks) blocks = 16;
    const bool three = (long long)r.rows * blocks > 152 * 2 && vocab <= kGroup * kMostOfThree * blocks;
    return three ? start<DTYPE, OUT, kStep, 3>(r, vocab, blocks, err, st)
                 : start<DTYPE, OUT, kStep, 2>(r, vocab, blocks, err, st);
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
