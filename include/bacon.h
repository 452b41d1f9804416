/*
 * bacon.h -- C ABI of the GB300 (sm_103a) BACON KV-cache compression library.
 *
 * BACON (Boundary Attention CalibratiON) scores every cached prompt token of
 * every (layer, kv-head) at the end of prefill and keeps the best ones:
 *
 *   window score   B_i = mean over the window queries of their causal
 *                        attention to key i                       (Sec. 4.1, Eq. 1)
 *   last query     Q_i = attention of the last prompt query to i  (Sec. 4.2, Eq. 2)
 *   residual       E_i = max(Q_i - B_i, 0)                        (Sec. 4.2, Eq. 4)
 *   coherence      L   = radius-r box mean of E, truncated at the ends
 *                                                                 (Sec. 4.3, Eqs. 5-7)
 *   persistence    T   = mean of E over the preceding min(m, l) layers
 *                                                                 (Sec. 4.3, Eqs. 8-9)
 *   evidence       V   = E + L + T                                (Sec. 4.3, Eqs. 10-11)
 *   scale          lambda = gamma Std_M(B~) / (Std_M(V) + eps), M = the
 *                        top-min(rho K, |I|) candidates by B~     (Sec. 4.4, Eqs. 12-15)
 *   score          S_i = B~_i + lambda V_i                        (Sec. 4.4, Eq. 16)
 *   selection      the K best candidates by S                     (Sec. 4.4, Eq. 17)
 *   compaction     their K/V rows gathered into a dense cache     (Sec. 4.4, after Eq. 17)
 *
 * where B~ is B max-pooled (odd width `pool`, stride 1, out-of-range
 * positions ignored) over the candidates.  Readings where the paper is
 * silent: the G = q_heads / kv_heads query heads of a kv-head are averaged
 * into one B and one Q; the candidates are positions [0, N - W) and the W
 * window tokens are always kept, so K = budget - W; gamma = 1, eps = 1e-8;
 * Std is the population standard deviation; ties go to the lower position.
 *
 * Layouts (all row-major, contiguous, element type bf16 unless stated):
 *   q_win  [Hq][W][d]      the last W prompt queries of one layer, post-RoPE;
 *                          query w sits at position N - W + w
 *   k, v   [Hkv][N][d]     one layer's prefill cache
 *   idx    [Hkv][budget]   int32 kept positions, ascending per head
 *   k_out, v_out [Hkv][budget][d]
 * Only head_dim 64 and 128 are supported.  Every device pointer must be
 * 16-byte aligned.
 *
 * Ownership: the caller owns every tensor passed in or out.  The library
 * owns the context, its device scratch and the per-request state.  All calls
 * are asynchronous on the caller's CUDA stream (`bacon_stream` is a
 * cudaStream_t; NULL means the legacy default stream): a call's work starts
 * after all earlier work of the stream, and later work starts after it,
 * however the caller's own kernels are launched.  A call returns the
 * launch-time status; no exception crosses the ABI.  On error the message of
 * the failing call is available from bacon_last_error() on the same thread.
 *
 * Errors: BACON_EINVAL for a bad argument (null or misaligned pointer, a
 * size out of range, budget < W, q_heads not a multiple of kv_heads,
 * unsupported head_dim, seq_len above max_seq_len, requests above
 * max_requests); BACON_ENOMEM when device or host allocation fails;
 * BACON_ECUDA for a CUDA launch or copy failure; BACON_ESTATE when layers
 * of a request are scored out of order or select runs before any layer was
 * scored; BACON_EUNSUPPORTED for sizes beyond the allocation-free entry
 * point's static scratch.  Errors found on the device are latched in the
 * context and returned by the next bacon_sync (the first one wins):
 * BACON_ETIMEOUT when a kernel's bounded pipeline wait (about a second) ran
 * out, after which the kernel drained its own work and returned, so the
 * context stays usable; BACON_EINVAL when bacon_compact was given an index
 * outside [0, seq_len); BACON_ECUDA when an internal consistency check of a
 * selection kernel failed (it emitted a different number of positions than
 * its budget; never expected, its message says so).  A context must not be
 * used from two threads at once.
 */
#ifndef BACON_H
#define BACON_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    BACON_OK = 0,
    BACON_EINVAL = 1,
    BACON_ENOMEM = 2,
    BACON_ECUDA = 3,
    BACON_ESTATE = 4,
    BACON_ETIMEOUT = 5,
    BACON_EUNSUPPORTED = 6
} bacon_status;

typedef void* bacon_stream; /* a cudaStream_t */

typedef struct bacon_ctx bacon_ctx;
typedef struct bacon_state bacon_state;

/* Hyper-parameters (Secs. 4.3-4.4) and capacity limits. */
typedef struct {
    int r;            /* coherence radius, default 5 (Sec. 4.3)            */
    int m;            /* persistence depth, default 4 (Sec. 4.3)           */
    int rho;          /* scale-matching expansion, default 2 (Sec. 4.4)    */
    float gamma;      /* calibration strength, default 1 (Eq. 14)          */
    float eps;        /* stabiliser, default 1e-8 (Eq. 15)                 */
    int use_E;        /* terms of Eq. 10, default 1, 1, 1 (0 = ablated)    */
    int use_L;
    int use_T;
    int keep_window;  /* 1 (default): window kept, candidates [0, N - W)   */
    int max_seq_len;  /* largest N any call may pass (default 16384)       */
    int max_requests; /* largest request count of one call (default 4)     */
    int keep_scores;  /* 1: keep V, pooled B and S of the last whole-step
                         call for bacon_get_scores (default 0)            */
} bacon_params;

/* Fill *p with the defaults listed above. */
void bacon_default_params(bacon_params* p);

/* Create a context for one model shape.  `layers` transformer layers with
 * `q_heads` query heads sharing `kv_heads` kv heads of dimension head_dim;
 * window W; odd max-pool width `pool` (1 = no pooling); default budget.
 * p may be NULL for the defaults.  Allocates the device scratch for
 * max_requests x layers x kv_heads x max_seq_len scores on the current
 * device.  For tests of failure detection only: when the environment
 * variable BACON_FAULT is "missing_arrival" at this call, the context's
 * next two-pass window step withholds one K-tile load, its bounded pipeline
 * waits run out and bacon_sync reports BACON_ETIMEOUT (nothing faults). */
bacon_status bacon_init(bacon_ctx** out, int layers, int kv_heads, int q_heads,
                        int head_dim, int window, int pool, int budget,
                        const bacon_params* p);
void bacon_destroy(bacon_ctx* ctx);

/* Message of the last failing call on this thread ("" if none). */
const char* bacon_last_error(void);

/* Per-request state for layer-by-layer scoring: the residuals E of the
 * preceding m layers (persistence, Eqs. 8-9), the scores of the last scored
 * layer and the index of the next layer expected. */
bacon_status bacon_state_create(bacon_ctx* ctx, bacon_state** out);
bacon_status bacon_state_reset(bacon_state* st);
void bacon_state_destroy(bacon_state* st);

/* Score one layer of one request (Eqs. 1-16 for every kv-head).  Layers
 * must arrive as 0, 1, 2, ... per state, else BACON_ESTATE.  q_win and k
 * are device pointers in the layouts above.  scores_out, if not NULL,
 * receives S as fp32 [Hkv][seq_len] (0 at non-candidates). */
bacon_status bacon_score_layer(bacon_ctx* ctx, bacon_state* st, int layer,
                               const void* q_win, const void* k, int seq_len,
                               float* scores_out, bacon_stream stream);

/* Select (Eq. 17) on the last layer scored with `st`: idx_out receives
 * int32 [Hkv][min(budget, N)] kept positions, ascending per head. */
bacon_status bacon_select(bacon_ctx* ctx, bacon_state* st, int budget,
                          int32_t* idx_out, bacon_stream stream);

/* Gather the kept rows of one layer: k_out[h][j] = k[h][idx[h][j]] and the
 * same for v (bitwise copies).  `count` indices per head. */
bacon_status bacon_compact(bacon_ctx* ctx, const void* k, const void* v,
                           const int32_t* idx, int seq_len, int count,
                           void* k_out, void* v_out, bacon_stream stream);

/* The whole step for `requests` independent prompts of seq_len tokens:
 * every layer and kv-head is scored, selected and compacted.  The pointer
 * arrays are HOST arrays of DEVICE pointers, indexed [request * layers +
 * layer], each pointing at one layer's tensor in the layouts above.
 * idx_out is one device array int32 [requests][layers][Hkv][kept] with
 * kept = min(budget, seq_len).  The host pointer arrays may be reused as
 * soon as the call returns. */
bacon_status bacon_compress_all_layers(bacon_ctx* ctx, int requests,
                                       const void* const* q_win,
                                       const void* const* k,
                                       const void* const* v, int seq_len,
                                       int budget, void* const* k_out,
                                       void* const* v_out, int32_t* idx_out,
                                       bacon_stream stream);

/* The whole step with one budget per layer (window included), e.g. the
 * pyramid schedule of bacon_pyramid_budgets (PyramidKV-style allocation,
 * Sec. 5 / App. B: BACON replaces only the within-head score, the base
 * compressor's layer budgets are kept).  layer_budgets is a HOST array of
 * `layers` ints; K_{l,h} of Eq. 12 is the layer's own budget minus W.
 * idx_out is a HOST array of DEVICE pointers [request * layers + layer], each
 * int32 [Hkv][kept_l] with kept_l = min(layer_budgets[l], seq_len); k_out and
 * v_out point at [Hkv][kept_l][d] per pair.  Other arguments and errors as
 * bacon_compress_all_layers. */
bacon_status bacon_compress_layer_budgets(bacon_ctx* ctx, int requests,
                                          const void* const* q_win, const void* const* k,
                                          const void* const* v, int seq_len,
                                          const int* layer_budgets, void* const* k_out,
                                          void* const* v_out, int32_t* const* idx_out,
                                          bacon_stream stream);

/* The whole step when the caller's prefill attention already produced the
 * softmax normalisers of the window rows (a fused attention kernel keeps
 * the log-sum-exp of every query row; Eq. 1's rows need nothing else to be
 * normalised), so the first pass over K is skipped.  lse is a HOST array of
 * DEVICE pointers [request * layers + layer], each fp32 [Hq][W]: for window
 * query w of query head g, ln sum_{i <= N-W+w} exp(q . k_i / sqrt(d)).
 * Everything else, including outputs and errors, as bacon_compress_all_layers.
 * Results equal that call's up to the rounding of the supplied values. */
bacon_status bacon_compress_with_lse(bacon_ctx* ctx, int requests, const void* const* q_win,
                                     const void* const* k, const void* const* v,
                                     const float* const* lse, int seq_len, int budget,
                                     void* const* k_out, void* const* v_out, int32_t* idx_out,
                                     bacon_stream stream);

/* The whole step with AdaKV-style adaptive head budgets (Sec. 5 / App. B:
 * the base compressor spreads a layer's budget over its kv-heads; BACON
 * supplies the score, Eq. 16, with K of Eq. 12 the average per-head budget).
 * Per (request, layer), with K = min(budget, N) - W per head on average:
 * every head first keeps its own top floor(alpha K) candidates; the other
 * Hkv K - Hkv floor(alpha K) slots go to the best remaining candidates of
 * all heads together (larger score first, ties to the lower head, then the
 * lower position).  Outputs are flat per (request, layer) pair, heads in
 * order: idx_out[pair] -> int32 [Hkv * kept] (each head's kept positions
 * ascending, then its window), k_out/v_out[pair] -> [Hkv * kept][d], with
 * kept = min(budget, N); counts_out is a DEVICE int32 [requests][layers][Hkv]
 * array receiving each head's kept count (window included).  alpha in
 * [0, 1]; BACON_EUNSUPPORTED when kv_heads x candidates exceeds 204800.
 * Other arguments and errors as bacon_compress_all_layers. */
bacon_status bacon_compress_adaptive(bacon_ctx* ctx, int requests, const void* const* q_win,
                                     const void* const* k, const void* const* v, int seq_len,
                                     int budget, float alpha, void* const* k_out,
                                     void* const* v_out, int32_t* const* idx_out,
                                     int32_t* counts_out, bacon_stream stream);

/* Ablation / sensitivity sweep (Sec. 5's component ablation of E, L and T
 * and its sensitivity study over m and r): every unit is scored under
 * several hyper-parameter sets while the window passes (Eqs. 1-4, the
 * dominant cost) run once.  Each variant overrides these fields of the
 * context's parameters; eps, keep_window and the pool width stay the
 * context's. */
#define BACON_MAX_VARIANTS 32
typedef struct {
    int r;           /* coherence radius (Eqs. 5-7), >= 0              */
    int m;           /* persistence depth (Eqs. 8-9), >= 0; 0 = no T  */
    int rho;         /* scale-matching expansion (Eq. 12), >= 0        */
    float gamma;     /* calibration strength (Eq. 14), finite, >= 0    */
    int use_E;       /* terms of Eq. 10 (0 = ablated)                  */
    int use_L;
    int use_T;
} bacon_variant;

/* Selection (Eq. 17) of every (request, layer, kv-head) under each of
 * n_variants variants (1 <= n_variants <= BACON_MAX_VARIANTS, HOST array),
 * from one set of window passes.  q_win and k as in
 * bacon_compress_all_layers; no K/V is gathered.  idx_out is one device
 * array int32 [n_variants][requests][layers][Hkv][kept], kept =
 * min(budget, seq_len), each variant's block laid out as that call's;
 * lambda_out, if not NULL, a device array fp32
 * [n_variants][requests][layers][Hkv] receiving Eq. 15's lambda.  Variant j
 * gives the indices bacon_compress_all_layers gives with its fields in the
 * context's parameters.  Afterwards bacon_get_scores reports BACON_ESTATE
 * until the next whole-step call.  EINVAL for a variant field out of range;
 * other errors as bacon_compress_all_layers. */
bacon_status bacon_sweep(bacon_ctx* ctx, int requests, const void* const* q_win,
                         const void* const* k, int seq_len, int budget, int n_variants,
                         const bacon_variant* variants, int32_t* idx_out, float* lambda_out,
                         bacon_stream stream);

/* Pyramid budget schedule over `layers` layers averaging `budget` (window
 * included): with K = budget - window, K_min = floor(K / beta) and
 * K_max = 2 K - K_min, layer l keeps W + K_min +
 * floor((layers - 1 - l) (K_max - K_min) / (layers - 1)) tokens, so the first
 * layer keeps the most, the last the fewest, and the layers together keep
 * at most layers x budget.  Host-only; writes out[0 .. layers). */
void bacon_pyramid_budgets(int layers, int window, int budget, int beta, int* out);

/* The same step on HOST buffers: inputs are copied to library-owned device
 * buffers, compressed, and the outputs copied back, all on `stream`; the
 * call returns once the outputs are on the host.  Contiguous host layouts:
 *   q_win [requests][layers][Hq][W][d], k, v [requests][layers][Hkv][N][d],
 *   k_out, v_out [requests][layers][Hkv][kept][d],
 *   idx_out [requests][layers][Hkv][kept].
 * Page-locked host memory gives the full copy bandwidth.  When `v` is
 * page-locked memory the device can address (allocated or registered
 * through CUDA, 16-byte aligned), it is not uploaded: the gather reads only
 * the kept rows from it in place. */
bacon_status bacon_compress_host(bacon_ctx* ctx, int requests,
                                 const void* q_win, const void* k,
                                 const void* v, int seq_len, int budget,
                                 void* k_out, void* v_out, int32_t* idx_out,
                                 bacon_stream stream);

/* Intermediate per-token arrays of the last bacon_compress_all_layers /
 * bacon_compress_host call, for inspection: fp32 [requests][layers][Hkv][N]
 * (lambda: [requests][layers][Hkv]).  `out` is a device pointer of at least
 * `count` floats.  V, the pooled B and S are kept only when the context was
 * created with keep_scores = 1 (else BACON_ESTATE). */
typedef enum {
    BACON_SCORE_B = 0,      /* window score, Eq. 1               */
    BACON_SCORE_Q = 1,      /* last-query score, Eq. 2           */
    BACON_SCORE_E = 2,      /* residual, Eq. 4                   */
    BACON_SCORE_V = 3,      /* calibrated evidence, Eq. 10       */
    BACON_SCORE_BPOOL = 4,  /* pooled window score (0 off-candidates) */
    BACON_SCORE_S = 5,      /* final score, Eq. 16 (0 off-candidates) */
    BACON_SCORE_LAMBDA = 6  /* lambda, Eq. 15                    */
} bacon_score_kind;

bacon_status bacon_get_scores(bacon_ctx* ctx, bacon_score_kind kind,
                              float* out, size_t count, bacon_stream stream);

/* Per-kernel device timing of the whole-step path: when enabled, CUDA events
 * are recorded on the caller's stream around each launch of
 * bacon_compress_all_layers / bacon_compress_host. */
bacon_status bacon_profile_enable(bacon_ctx* ctx, int enable);

/* Kernel stages reported by bacon_profile_read, in this order. */
#define BACON_PROFILE_STAGES 5 /* window_stats, window_combine, window_scores,
                                  calibrate_select, gather */

/* Waits for the recorded work, then writes per stage the summed device time
 * in ms and the launch count since the previous read (arrays of at least
 * `n` entries; n <= BACON_PROFILE_STAGES), and clears the record.  A stage
 * that launched nothing in a call is not counted: when every unit's logits
 * fit in tensor memory (at most 32 window rows and 1024 tokens) the window
 * score is one kernel, reported as window_scores, with no window_stats or
 * window_combine launch. */
bacon_status bacon_profile_read(bacon_ctx* ctx, double* ms, int* launches, int n);

/* Window scores of one layer (B, Q and E of Eqs. 1, 2 and 4 for every
 * kv-head) WITHOUT ANY DEVICE ALLOCATION.  The paper has no counterpart:
 * this entry point exists for callers that cannot call cudaMalloc, such as
 * a serving engine that reserves all of HBM for its KV cache up front, or
 * code that must not pay the device-wide synchronisation of cudaMalloc /
 * cudaFree in the middle of prefill.  It needs no context: the kernels'
 * scratch (the softmax statistics) lives in one static __device__ array of
 * about 512 KiB, which every GPU that loads the library holds until the
 * process exits.
 *
 * Inputs as in the layouts above (q_win [Hq][W][d], k [Hkv][N][d] bf16);
 * outputs B_out, Q_out, E_out fp32 [Hkv][N], all caller-owned device
 * pointers, 16-byte aligned.  Limits: seq_len <= 16384,
 * q_heads * window <= 4096 and (q_heads / kv_heads) * window <= 512 (beyond
 * them: BACON_EUNSUPPORTED); malformed
 * arguments give BACON_EINVAL, a CUDA failure at launch BACON_ECUDA.  No
 * message is recorded for bacon_last_error.  The status is returned before
 * the kernels run, so an error found on the device (a bounded pipeline wait
 * of about a second that ran out) is reported in the outputs instead: B_out,
 * Q_out and E_out are then all NaN once the stream reaches the end of the
 * call.  A caller that must tell this case apart checks one output value
 * after synchronising.
 *
 * The first call on a device looks up the array's device address (with
 * that device current) and caches it.  Every call uses the same array:
 * calls whose work can overlap on the GPU (different streams, or several
 * host threads) race and must be serialised by the caller.  The array keeps
 * the last call's contents; its error word, the one entry that must start
 * at zero, is cleared again on the stream by the call that set it, and every
 * other entry a call reads it has written first. */
bacon_status bacon_window_scores_noalloc(int kv_heads, int q_heads, int head_dim, int window,
                                         const void* q_win, const void* k, int seq_len,
                                         float* B_out, float* Q_out, float* E_out,
                                         bacon_stream stream);

/* Wait for the stream and report any error latched by a kernel. */
bacon_status bacon_sync(bacon_ctx* ctx, bacon_stream stream);

/* ------------------------------------------------------------------------
 * Serving from the kept rows.  The paper ends at the compacted cache; these
 * calls hold it, and the tokens generated after it, in pages of 8-bit values
 * and attend to it.
 *
 * A unit is one (request, layer, kv-head); each has its own length, since
 * adaptive head budgets keep another number of rows per head.  A page holds
 * `page` tokens of one unit, with one fp32 scale for its K rows and one for
 * its V rows; a value is code * scale.  Arrays of the caller:
 *
 *   k, v           [pages][page][d]              8-bit codes
 *   k_scale,
 *   v_scale        [pages]                       fp32
 *   lengths        [requests][layers][Hkv]       int32 tokens of each unit
 *   table          [requests][layers][Hkv][max_blocks]
 *                                                int32 page of each block of
 *                                                `page` tokens
 *   ring, state    [pages], [2]                  int32 free pages:
 *                  ring[(state[0] + i) mod pages], 0 <= i < state[1]
 *   slots                                        int32 page * `page` + row of
 *                                                a token, -1 for none
 *
 * A decoding program plans the new tokens of a step once (bacon_cache_plan),
 * then per layer stores their K and V (bacon_cache_store) and attends
 * (bacon_cache_attend).  The calls are asynchronous on `stream` like those
 * above, allocate nothing and may be captured.  One cache must not be used
 * from two threads or on two streams at once.  What is found wrong on the
 * device is latched and returned by bacon_cache_sync. */
typedef struct bacon_cache bacon_cache;

typedef enum {
    BACON_E4M3 = 0, /* scale: the least power of two with amax <= 448 scale  */
    BACON_INT8 = 1  /* scale: amax / 127 rounded up to 8 significant bits    */
} bacon_cache_format; /* either scale is at least 2^-60 */

typedef enum { BACON_BF16 = 0, BACON_FP16 = 1 } bacon_dtype;

typedef struct {
    int layers, kv_heads, q_heads, head_dim; /* head_dim 64 or 128            */
    int page;         /* tokens per page: 16, 32, 64 or 128                  */
    int pages;        /* pages of the pool; pages * page < 2^31              */
    int max_requests; /* largest request count of one call                   */
    int max_blocks;   /* columns of a table; max_blocks * page < 2^31 - 1024  */
    int format;       /* bacon_cache_format                                  */
    int dtype;        /* bacon_dtype of rows, queries and outputs            */
    void* k;          /* device arrays as above, kept by the caller for the  */
    void* v;          /* life of the cache; k and v 16-byte aligned          */
    float* k_scale;
    float* v_scale;
} bacon_cache_desc;

/* Creates a cache over the caller's pools on the current device: holds the
 * split attention's scratch (about 55 MB) and the error word.  For tests of
 * failure detection only: when the environment variable BACON_FAULT is
 * "missing_page", or "missing_page:<tile>", at this call, the cache's next
 * attention withholds one load of 16 rows of its first block's first tile, or
 * of tile <tile> if it has that many, its bounded pipeline waits run out and
 * bacon_cache_sync reports BACON_ETIMEOUT (nothing faults; that call's outputs
 * are undefined, the cache stays usable). */
bacon_status bacon_cache_create(bacon_cache** out, const bacon_cache_desc* desc);
void bacon_cache_destroy(bacon_cache* cache);

/* Pages and slots for the tokens that the units are about to get.  Unit u
 * (in order r, l, h) with n tokens and a new ones takes
 * ceil((n + a) / page) - ceil(n / page) pages from the ring, the units one
 * after the other; they are entered in its row of the table.  lengths_out
 * receives n + a, state_out the ring's state afterwards; neither may overlap
 * its input.  With per_unit != 0, `added` is [requests][layers][Hkv] and
 * slots [rows] takes the units' tokens one after the other: the order of the
 * rows of bacon_compress_adaptive.  With per_unit == 0, `added` is
 * [requests], or NULL for one token each, and slots is [layers][rows][Hkv],
 * the requests' tokens one after the other.  Entries beyond the last token
 * are -1.  When the ring holds too few pages (BACON_ENOMEM), or a length is
 * negative or exceeds max_blocks * page, or the tokens exceed `rows`
 * (BACON_EINVAL, both at bacon_cache_sync), nothing is given: lengths_out
 * and state_out repeat the input and every slot is -1.  A plan of which nothing
 * is used is undone by going on with its inputs; where some of the tokens are
 * not kept (rejected drafts), bacon_cache_shorten takes them back.  A length
 * that is put back by hand leaves its pages in the table, where the next plan
 * writes others over them. */
bacon_status bacon_cache_plan(bacon_cache* cache, int requests, const int32_t* lengths,
                              const int32_t* added, int per_unit, int32_t* table,
                              const int32_t* ring, const int32_t* state, int rows,
                              int32_t* slots, int32_t* lengths_out, int32_t* state_out,
                              bacon_stream stream);

/* Slots of the positions [first, first + count) of each unit (first NULL: 0),
 * the units one after the other; -1 beyond.  Errors as bacon_cache_plan. */
bacon_status bacon_cache_locate(bacon_cache* cache, int requests, const int32_t* first,
                                const int32_t* count, const int32_t* table, int rows,
                                int32_t* slots, bacon_stream stream);

/* Returns the pages of every request with done[r] != 0 to the ring (units in
 * order, blocks in order); their lengths become 0, their table rows -1.
 * Nothing changes when an entry is no page or the ring would overflow
 * (BACON_EINVAL at bacon_cache_sync). */
bacon_status bacon_cache_release(bacon_cache* cache, int requests, const int32_t* done,
                                 int32_t* lengths, int32_t* table, int32_t* ring,
                                 int32_t* state, bacon_stream stream);

/* Takes the last fewer[r] tokens of every unit of request r back ([requests],
 * 0 for none): lengths become smaller, pages that held none of the tokens kept
 * go back to the ring (units in order, blocks in order) and leave the table.
 * What stays is untouched, a page's scale too.  Nothing changes when a unit has
 * fewer tokens than that, a number is negative, an entry is no page or the ring
 * would overflow (BACON_EINVAL at bacon_cache_sync). */
bacon_status bacon_cache_shorten(bacon_cache* cache, int requests, const int32_t* fewer,
                                 int32_t* lengths, int32_t* table, int32_t* ring,
                                 int32_t* state, bacon_stream stream);

/* Quantises rows into their slots.  Row (t, h) of k starts at element
 * t * k_token_stride + h * k_head_stride, the same for v (strides multiples
 * of 8 elements, rows 16-byte aligned); slots is [tokens][heads], so heads is
 * Hkv for token-major rows of one layer and 1 for rows one after the other.
 * The rows of one page must follow one another in tokens and positions: two
 * runs of a page in one call would both write its scale and codes.  Rows that
 * do not follow the row before them in their page are left out and reported
 * (BACON_EINVAL at bacon_cache_sync); runs of a page with others between them
 * (rows of several kv-heads in turn with heads = 1, say) are not noticed.  A
 * page that gets its first row has its scale from the new rows; one that is
 * appended to keeps its scale if that holds them, and its older rows are
 * quantised again with the larger scale if not.  Infinities saturate; NaN
 * stays NaN in e4m3 and becomes 0 in int8; neither counts for the scale. */
bacon_status bacon_cache_store(bacon_cache* cache, int tokens, int heads, const void* k,
                               long long k_token_stride, long long k_head_stride, const void* v,
                               long long v_token_stride, long long v_head_stride,
                               const int32_t* slots, bacon_stream stream);

/* The values of `rows` slots as [rows][d] each; zeros for -1. */
bacon_status bacon_cache_load(bacon_cache* cache, int rows, const int32_t* slots, void* k_out,
                              void* v_out, bacon_stream stream);

/* Attention of `tokens` new queries of one layer over their units' tokens
 * (lengths and table include the new ones): query head g of kv-head
 * h = g / (Hq / Hkv).  q row (t, g) starts at element t * q_token_stride +
 * g * q_head_stride (multiples of 8 elements).  Request r has the queries
 * starts[r] .. starts[r + 1], starts[0] = 0 and starts[requests] = tokens
 * (otherwise, or when one ends before it starts, nothing is attended:
 * BACON_EINVAL at bacon_cache_sync); starts NULL: tokens / requests each.  With
 * causal != 0, query j of a request with a sees the positions up to
 * n - a + j, else all n.  scale multiplies the logits; 0 means 1/sqrt(d).
 * out is [tokens][Hq][d], lse (may be NULL) fp32 [tokens][Hq] receives the
 * natural log-sum-exp.  A query that sees nothing gets zeros and -inf. */
bacon_status bacon_cache_attend(bacon_cache* cache, int requests, int layer, int tokens,
                                const void* q, long long q_token_stride, long long q_head_stride,
                                const int32_t* starts, const int32_t* lengths,
                                const int32_t* table, int causal, float scale, void* out,
                                float* lse, bacon_stream stream);

/* Wait for the stream and report any error latched by these kernels. */
bacon_status bacon_cache_sync(bacon_cache* cache, bacon_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* BACON_H */
