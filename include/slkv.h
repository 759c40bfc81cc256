/*
 * slkv.h -- C ABI of the SurfaceLogicKV prefill KV-cache compression library (CUDA, sm_100a).
 *
 * One call per step of the paper's method:
 *   slkv_behavior_scores Stage 1, SF_sc / LG_sc / INF_sc of attention rows               (Sec. 3.2, Algorithm 1)
 *   slkv_alloc_budgets   Stage 2, per-head KV budgets from the INF_sc table     (Sec. 3.3, Eq. 6, Algorithm 2)
 *   slkv_score           relevance of every history key to the query window     (Sec. 3.4, Eq. 7, Alg. 3 l.4-6)
 *   slkv_compress        score -> top-(C - window) history rows + window, gather (Sec. 3.4, Eq. 8, Algorithm 3)
 *   slkv_compress_host   the same, from/to host buffers (copies included)
 *   slkv_compress_overlapped / slkv_join   the same, successive layers overlapped on the GPU
 *   slkv_cp_*            the same for one sequence whose keys are split over ranks (context parallel)
 *   slkv_row_lse         the window rows' log-sum-exp over their softmax domain       (Eq. 3-4, Eq. 7)
 *   slkv_q4_*            the compressed cache in decoding: held in 4 bits, attended to, evicted from
 *   slkv_prompt_attend   the prompt's own attention, which leaves the window rows' log-sum-exp for the compression
 *   slkv_paged_*         the compressed cache in pages: planned, written, attended to by trees of drafted tokens
 *
 * Conventions
 *   - "dev" pointers are device memory of the current CUDA device, "host" pointers are host memory.
 *   - The caller owns every buffer.  The library allocates no device memory; scratch comes from the
 *     caller's `workspace` (size from slkv_workspace_bytes) and must stay untouched until the enqueued
 *     work has finished.  Nothing is freed or retained by the library.  One exception, for callers that
 *     have no workspace to give: slkv_score_noalloc works in a fixed array of SLKV_NOALLOC_SCRATCH_BYTES
 *     that is part of the library's device image (see there for when it comes into being and how long it
 *     lives).
 *   - All device work is enqueued on `stream` (a cudaStream_t passed as void*; NULL = default stream).
 *     No call synchronises the device except slkv_compress_host, which returns after its results are
 *     in the host buffers.
 *   - Every function returns SLKV_OK (0) or a negative slkv_status.  Argument errors are found on the
 *     host before anything is enqueued.  Errors only visible in device data (a negative INF_sc, an
 *     output capacity that turns out too small) are written to the optional device word `status`
 *     (untouched when nothing is wrong -- zero it first), never raised as a device fault.
 *
 * Tensor layouts (element = float for SLKV_F32, bfloat16 for SLKV_BF16; head_dim contiguous)
 *   K, V   packed varlen, token-major: element (t, h, p) at t*stride_tok + h*stride_head + p,
 *          t in [0, total_tokens), sequences delimited by cu_seqlens[n_seqs+1] (cu[0] = 0).
 *   Q_win  the queries of each sequence's last `window` tokens: element (s, i, h, p) at
 *          s*q_stride_seq + i*q_stride_row + h*q_stride_head + p; row i is token len_s - window + i.
 *          (Rows are unused for sequences not longer than the window.)
 *   GQA    query head h scores against KV head h / (n_q_heads / n_kv_heads).
 *   pooled ragged float array: sequence s, KV head h, history position j (j < n_hist_s = max(len_s -
 *          window, 0)) at  n_kv_heads * sum_{s'<s} n_hist_s'  +  h * n_hist_s  +  j.
 *   packed output: segment seg = s*n_kv_heads + h owns rows offsets[seg] .. offsets[seg+1]-1 of k_out /
 *          v_out / kept_idx; its rows are the selected history positions in ascending order followed by
 *          the window positions; a row is head_dim contiguous elements.  kept_idx holds positions
 *          within the sequence (0-based).
 */
#ifndef SLKV_H_
#define SLKV_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum slkv_status {
  SLKV_OK = 0,
  SLKV_ERR_NULL_PTR = -1,       /* a required pointer is NULL */
  SLKV_ERR_BAD_SHAPE = -2,      /* a size / count / stride is out of the supported range */
  SLKV_ERR_BAD_DTYPE = -3,      /* dtype / mode enum not recognised or not supported by the chosen path */
  SLKV_ERR_BAD_ALIGN = -4,      /* a pointer or stride breaks the 16-byte row alignment rule */
  SLKV_ERR_BUDGET_SUM = -5,     /* total < n_layers*n_heads*fixed, or fixed < 0 */
  SLKV_ERR_NEG_INF_SC = -6,     /* an INF_sc entry is negative or not finite (device status word) */
  SLKV_ERR_CAPACITY = -7,       /* out_capacity_rows smaller than the rows to write */
  SLKV_ERR_WORKSPACE = -8,      /* workspace NULL or smaller than slkv_workspace_bytes */
  SLKV_ERR_CUDA = -9,           /* a CUDA runtime call failed (see slkv_last_cuda_error) */
  SLKV_ERR_DEVICE_TIMEOUT = -10 /* a bounded device-side wait ran out (device status word) */
} slkv_status;

enum { SLKV_F32 = 0, SLKV_BF16 = 1 };                 /* slkv_params.dtype */
enum { SLKV_POOL_MAX = 0, SLKV_POOL_AVG = 1 };        /* slkv_params.pool_mode */
enum { SLKV_HISTORY = 0,                              /* slkv_params.softmax_domain: softmax over the history keys */
       SLKV_ALL_CAUSAL = 1 };                         /*   over every key a window query sees causally */
enum { SLKV_LSE_LN = 0, SLKV_LSE_LOG2 = 1 };          /* slkv_params.lse_units: natural log / base-2 log */
enum { SLKV_PATH_AUTO = 0,                            /* slkv_params.score_path */
       SLKV_PATH_SIMT = 1,                            /*   fp32 FMA kernels (any dtype, head_dim 64/128) */
       SLKV_PATH_TENSOR = 2 };                        /*   tcgen05 + TMA kernels (bf16, up to 256 score rows per KV head) */

/* Shapes and options shared by slkv_score / slkv_compress. Strides are in elements. */
typedef struct slkv_params {
  int32_t n_seqs;          /* >= 1 */
  int32_t n_q_heads;       /* multiple of n_kv_heads */
  int32_t n_kv_heads;
  int32_t head_dim;        /* 64 or 128 */
  int32_t window;          /* w >= 1: observation window (last w tokens), always kept */
  int32_t pool_kernel;     /* odd >= 1 (1 = no pooling) */
  int32_t dtype;           /* SLKV_F32 | SLKV_BF16: element type of Q_win, K, V and the packed outputs */
  int32_t pool_mode;       /* SLKV_POOL_MAX | SLKV_POOL_AVG */
  int32_t softmax_domain;  /* SLKV_HISTORY | SLKV_ALL_CAUSAL: the keys a window row's softmax runs over */
  int32_t score_path;      /* SLKV_PATH_AUTO picks TENSOR when the shape allows it, else SIMT */
  int32_t lse_units;       /* SLKV_LSE_LN | SLKV_LSE_LOG2: units of lse_opt / slkv_row_lse's output */
  int32_t history_only;    /* 0: the last `window` rows of every sequence in K / V are the window rows (never scored);
                              1: K holds history rows only -- a range of a longer sequence's keys whose window rows
                              live elsewhere (context-parallel sharding).  n_seqs must be 1; taken by slkv_score,
                              slkv_row_lse and slkv_score_noalloc, SLKV_ERR_BAD_SHAPE from the compress entry points;
                              the softmax then runs over the rows given, whatever softmax_domain says */
  int64_t k_stride_tok, k_stride_head;
  int64_t v_stride_tok, v_stride_head;
  int64_t q_stride_seq, q_stride_row, q_stride_head;
} slkv_params;

/* Human-readable name of a status code (static string, never NULL). */
const char* slkv_strerror(int status);

/* Last CUDA runtime error code seen by a call that returned SLKV_ERR_CUDA on this thread (0 = none). */
int slkv_last_cuda_error(void);

/*
 * Stage-1 attention behaviour analysis (Sec. 3.2, Algorithm 1), for a batch of attention rows (one row = the
 * attention weights of one head for one probe prompt's answering position, over the context).
 * For each row with needle positions N and top-k positions T (both as sets):
 *     WO = sum of W over N and T,  WD = sum over T without N,  TNW = sum over N,  WS = max(0, TNW - WO)
 *     SF_sc = WO / (WO + WD),  LG_sc = WO / (WO + WS),  INF_sc = 2 SF_sc LG_sc / (SF_sc + LG_sc)     (0/0 = 0)
 *   attn         dev, float: row r starts at attn + r*row_stride and has row_len weights (row_stride 0 shares one row)
 *   needle_idx   dev, int32: row r's needle positions at needle_idx + r*needle_stride, n_needle entries
 *                (needle_stride 0: one list for all rows); entries outside [0, row_len) are padding
 *   topk_idx     dev, int32: likewise the positions of the row's k largest weights (n_topk entries, topk_stride)
 *   sf_sc, lg_sc, inf_sc   dev, out, float[n_rows]
 * An index listed twice counts once.  Averaging the per-row scores into the per-(layer, head) INF_sc table that
 * slkv_alloc_budgets takes is left to the caller (the paper does not print how it aggregates over prompts).
 * Limits: n_needle, n_topk <= 4096.
 */
int slkv_behavior_scores(const float* attn, int64_t n_rows, int32_t row_len, int64_t row_stride,
                         const int32_t* needle_idx, int32_t n_needle, int64_t needle_stride, const int32_t* topk_idx,
                         int32_t n_topk, int64_t topk_stride, float* sf_sc, float* lg_sc, float* inf_sc, void* stream);

/*
 * Stage-2 budget allocation (Sec. 3.3, Eq. 6; Algorithm 2).
 *   inf_sc   dev, float[n_layers*n_heads], row-major (layer, head); INF_sc >= 0, finite
 *   fixed    fixed part every head receives (= b_c (1 - 1/beta) in the paper's notation)
 *   total    sum of all budgets (= b_c * n_layers * n_heads); dynamic pool D = total - N*fixed >= 0
 *   budgets  dev, out, int32[n_layers*n_heads]
 *   status   dev, optional: set to SLKV_ERR_NEG_INF_SC (budgets then left unwritten)
 * Head (i, j) receives fixed + its share of D in proportion to Algorithm 2's weight
 * (0.01 + L_i/L_s) * (inf_ij/L_s), L_i the layer's INF_sc sum, L_s the grand sum; shares are rounded by
 * largest remainder (ties: lower index first) so that the budgets sum to `total` exactly.  All-zero
 * INF_sc gives uniform shares.  fp64 arithmetic in a fixed order: results are reproducible bit for bit.
 * Limits: n_layers <= 1024, n_layers*n_heads <= 16384, total < 2^31 (else SLKV_ERR_BAD_SHAPE).
 */
int slkv_alloc_budgets(const float* inf_sc, int32_t n_layers, int32_t n_heads, int32_t fixed, int64_t total,
                       int32_t* budgets, int32_t* status, void* stream);

/*
 * The same allocation with the readings Sec. 3.3 leaves open (Eq. 6 and its prose; Algorithm 2's last line).
 *   head_normaliser  SLKV_NORM_GLOBAL: a head's share S_ij = inf_ij / L_s of the grand sum, as Algorithm 2 prints it;
 *                    SLKV_NORM_WITHIN_LAYER: inf_ij / L_i of its own layer's sum, as the prose under Eq. 6 describes
 *                    it (an all-zero layer shares evenly).  Under the second one a layer's total follows
 *                    (0.01 + L_i/L_s) / (1 + 0.01 n_layers): the 0.01 "minimum layer budget" really is a floor.
 *   rounding         SLKV_ROUND_SUM_EXACT: normalised weights, largest remainder, sum == total (as slkv_alloc_budgets);
 *                    SLKV_ROUND_PAPER: Algorithm 2's own C = floor(max(0, fixed + D * weight) + 0.5) per head with
 *                    D = total - N*fixed; the weights are not normalised, so the sum is whatever it comes to.
 *   cap              0: none.  > 0: no head gets more than `cap` (say, the sequence length: budget beyond it could
 *                    never be used).  With SLKV_ROUND_SUM_EXACT what a full head cannot take goes to the others in
 *                    proportion to their weights, again and again until nobody is above the cap, and the budgets
 *                    still sum to `total` (needs cap >= fixed and total <= N * cap, else SLKV_ERR_BUDGET_SUM); with
 *                    SLKV_ROUND_PAPER the budgets are just clipped.  The paper has no cap.
 * opt == NULL means {SLKV_NORM_GLOBAL, SLKV_ROUND_SUM_EXACT, 0}.  Other arguments, limits and errors as
 * slkv_alloc_budgets; an unknown enum value gives SLKV_ERR_BAD_DTYPE.  Bit-reproducible like slkv_alloc_budgets.
 */
enum { SLKV_NORM_GLOBAL = 0, SLKV_NORM_WITHIN_LAYER = 1 };     /* slkv_alloc_options.head_normaliser */
enum { SLKV_ROUND_SUM_EXACT = 0, SLKV_ROUND_PAPER = 1 };       /* slkv_alloc_options.rounding */
typedef struct slkv_alloc_options {
  int32_t head_normaliser;
  int32_t rounding;
  int64_t cap;
} slkv_alloc_options;
int slkv_alloc_budgets_ex(const float* inf_sc, int32_t n_layers, int32_t n_heads, int32_t fixed, int64_t total,
                          const slkv_alloc_options* opt, int32_t* budgets, int32_t* status, void* stream);

/* Bytes of workspace slkv_score / slkv_compress need for these shapes (0 on invalid arguments).
 * cu_seqlens_host: host, int32[n_seqs+1]. */
size_t slkv_workspace_bytes(const slkv_params* p, const int32_t* cu_seqlens_host);

/* Number of floats in the ragged `pooled` array: n_kv_heads * sum_s max(len_s - window, 0) (-1 on error). */
int64_t slkv_pooled_elems(const slkv_params* p, const int32_t* cu_seqlens_host);

/* Upper bound of packed rows for any budgets: n_kv_heads * total_tokens (-1 on error). */
int64_t slkv_packed_rows_upper_bound(const slkv_params* p, const int32_t* cu_seqlens_host);

/*
 * Relevance scores (Sec. 3.4, Eq. 7; Algorithm 3 lines 4-6; scale and softmax axis from Eq. 3-4).
 * For every sequence s, KV head g and history key j < n_hist_s:
 *     vote[j]   = (1/G) * sum_{query heads h of group g} sum_{window rows i} exp(q_i . k_j / sqrt(head_dim) - lse_i)
 *     pooled[j] = max (or zero-padded mean) of vote over [j - pool_kernel/2, j + pool_kernel/2] within the history
 * where lse_i is the log-sum-exp of row i's scaled scores over its softmax domain: the history keys
 * (SLKV_HISTORY: Eq. 7 and Algorithm 3 as printed) or the history keys plus the window keys up to the
 * row's own position (SLKV_ALL_CAUSAL: the prefill attention's own softmax, the reading of the prior work
 * Sec. 3.4 refers to; the window columns get no vote).  (The paper leaves the reduction over the window
 * rows, the GQA reduction and the pooling to prior work; this is the reading used here.)
 *   q_win, k         dev, layouts above
 *   cu_seqlens_dev   dev, int32[n_seqs+1];  cu_seqlens_host: the same values on the host (sizes the launch)
 *   lse_opt          dev, optional, float[n_seqs][n_q_heads][window] in p->lse_units: the rows' log-sum-exp
 *                    when the caller has it already (a prefill attention kernel that keeps its softmax
 *                    statistics has exactly the SLKV_ALL_CAUSAL one).  NULL: computed here, which costs a
 *                    second pass over K.  The values are used as given, whatever softmax_domain says.
 *   pooled           dev, out, float[slkv_pooled_elems]
 *   status           dev, optional: SLKV_ERR_DEVICE_TIMEOUT if a bounded wait inside a kernel ran out
 *                    (pooled is then incomplete)
 * Accuracy: fp32 accumulation; relative error of pooled <= 1e-3 of the exact value.
 */
int slkv_score(const slkv_params* p, const void* q_win, const void* k, const int32_t* cu_seqlens_dev,
               const int32_t* cu_seqlens_host, const float* lse_opt, float* pooled, int32_t* status,
               void* workspace, size_t workspace_bytes, void* stream);

/*
 * The row statistics alone (Eq. 3-4 with Eq. 7's key set): lse_out[s][h][i] = log sum_j exp(q_i . k_j /
 * sqrt(head_dim)) over the softmax domain of p->softmax_domain, in p->lse_units, for the window rows of
 * every sequence longer than the window (rows of shorter sequences are left untouched).  It is what
 * slkv_score computes first when lse_opt is NULL; fed back as lse_opt it reproduces that call with SLKV_LSE_LOG2
 * (the kernels' own unit), and to rounding with SLKV_LSE_LN.  Callers that shard the keys of one sequence over
 * several devices merge these per shard and pass the result as lse_opt.
 * "Reproduces", here and where the overlapped calls promise the results of single ones: a row's sum is added up from
 * the fp32 sums of its tiles (128 keys; 32 on the FMA path) by fp64 additions whose order varies from launch to launch.
 * Where the largest and the smallest of a row's n tile sums are no more than a factor 2^29 / n apart (2^19 at 131072
 * keys) these additions are exact, and everything is the same bit for bit.  Beyond that, sums agree to 2^-53 times
 * a few: the fp32 log-sum-exp of about one row in 10^8 differs in its last bit, its votes by 10^-6 of their value, and
 * which of two positions is kept whose scores are that close.  With scores beyond fp64's range (900 in log2 units)
 * the log-sum-exps agree to fp32 rounding.
 *   lse_out   dev, out, float[n_seqs][n_q_heads][window]
 * Other arguments and errors as slkv_score.
 */
int slkv_row_lse(const slkv_params* p, const void* q_win, const void* k, const int32_t* cu_seqlens_dev,
                 const int32_t* cu_seqlens_host, float* lse_out, int32_t* status, void* workspace,
                 size_t workspace_bytes, void* stream);

/*
 * KV entry selection and gather for one layer (Sec. 3.4, Eq. 8; Algorithm 3).
 * For each segment (s, h) with budget C = budgets[h]:  kept = min(len_s, max(C, window)) rows survive:
 * everything if len_s <= C (Alg. 3 l.1-3), else the window rows plus the kept - window history positions
 * with the largest pooled score (ties: lower position first), in ascending position order (l.7-10).
 *   budgets            dev, int32[n_kv_heads]: this layer's row of slkv_alloc_budgets' output
 *   lse_opt            dev, optional: as in slkv_score
 *   k_out, v_out       dev, out, [out_capacity_rows, head_dim] elements of p->dtype
 *   offsets            dev, out, int32[n_seqs*n_kv_heads + 1]
 *   kept_idx           dev, out, int32[out_capacity_rows]
 *   pooled_opt         dev, optional out, float[slkv_pooled_elems]: the scores the selection used
 *   status             dev, optional: SLKV_ERR_CAPACITY if offsets[last] > out_capacity_rows (rows beyond
 *                      the capacity are then not written; offsets are still complete)
 * Gathered rows are bit copies of the input rows.
 */
int slkv_compress(const slkv_params* p, const void* q_win, const void* k, const void* v,
                  const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host, const int32_t* budgets,
                  const float* lse_opt, void* k_out, void* v_out, int64_t out_capacity_rows, int32_t* offsets, int32_t* kept_idx,
                  float* pooled_opt, int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/*
 * slkv_compress with the calls of successive layers overlapped on the GPU (Algorithm 3, same results).
 *
 * The layers of a prefill are independent problems, and inside one layer the vote pass needs every key's row
 * statistics first (the softmax of Eq. 7 runs over all keys).  This entry point therefore works on several layers
 * at once: a call queues its layer, and a list of layers goes out as three launches on `stream` -- the score kernel, in
 * which the row-statistics pass of later layers runs between the vote passes of earlier ones, then the selections and the
 * gathers of all layers of the list -- when the queued layers come to some 0.4 ms of work, which is eight to thirty-two
 * layers (thirty-two of up to 16k tokens, sixteen of 32k, eight of 64k and more, at 8 KV heads and 128 score rows), or at
 * slkv_join.  Consequences:
 *   - Nothing of a call needs to have been enqueued when it returns: slkv_join(stream) enqueues whatever is still
 *     queued and makes `stream` wait for every overlapped call made so far on the current device (no host wait);
 *     consume outputs, or free / overwrite any input, output or workspace buffer -- q_win, k, v, cu_seqlens_dev
 *     and budgets included -- only behind it.  cu_seqlens_host is read during the call only.  Any other slkv_*
 *     call that uses a workspace joins by itself first, but for these.  slkv_prompt_attend and slkv_paged_attend leave what is queued
 *     where it is, so that a prefill's layers still come together into lists; where their workspace overlaps that of overlapped calls, or their
 *     lse_opt one that a queued layer takes, what is concerned goes out, and `stream` waits for it, first.  slkv_paged_plan and
 *     slkv_paged_write send out what is queued on their own stream.  Of the slkv_q4_* calls, slkv_q4_pack sends out what is queued on its
 *     own stream, so that it finds the rows of calls made there before it; the others do not look at queued layers, and no
 *     slkv_q4_* call waits for another stream: a cache that is filled on one and read on another needs an order from the caller.
 *   - Streams and host threads: the calls made on one stream form one sequence (queue, workspace);
 *     calls made on another stream -- by another host thread or the same one -- form another, and the two do not
 *     disturb each other as long as each has its own workspace (calls on two streams that share a workspace are
 *     serialised: the later one waits for what the other stream has in flight).  A join orders its stream behind
 *     the calls of every stream but settles only its own stream's: each stream that consumes results joins for
 *     itself.  The entry points may be called from several host threads at once (one lock inside); up to eight
 *     streams per device keep a sequence each, a ninth takes over the one used longest ago once that one's
 *     stream has been made to wait for what it had in flight.
 *   - workspace must hold slkv_workspace_bytes_overlapped: votes, source-row lists and row statistics for the
 *     layers of a list (one layer's worth for shapes that are not taken as lists).  Successive calls share one
 *     workspace; a call with another shape or workspace first sends out what is queued.  q_win, k, v, budgets and the
 *     outputs of calls that may be in flight together must not alias each other's outputs.
 *   - The call sequence is stream-ordered and allocates nothing on the device, so a step's calls plus the join can be
 *     captured in a CUDA graph.
 *   - Lists take bf16 and (n_q_heads / n_kv_heads) * window <= 256, at most 64 sequences, segments the one-launch
 *     selections take (up to 262116 history positions with pool_kernel <= 9, up to 131040 with pool_kernel <= 129).  Other shapes run as slkv_compress does, on `stream`, after a join.
 *   - Long lists with max pooling, without pooled_opt and lse_opt, take one product with every key instead of two where that is quicker, with
 *     the same results.  out_capacity_rows tells which: as many rows as the budgets make, or room for all, lets the line be drawn best.
 * Arguments, results and error codes otherwise as slkv_compress.
 */
int slkv_compress_overlapped(const slkv_params* p, const void* q_win, const void* k, const void* v,
                             const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host, const int32_t* budgets,
                             const float* lse_opt, void* k_out, void* v_out, int64_t out_capacity_rows, int32_t* offsets,
                             int32_t* kept_idx, float* pooled_opt, int32_t* status, void* workspace,
                             size_t workspace_bytes, void* stream);
size_t slkv_workspace_bytes_overlapped(const slkv_params* p, const int32_t* cu_seqlens_host);
/* Enqueues the layers still queued by slkv_compress_overlapped and orders `stream` after every overlapped call made
 * so far on the current device (see above). */
int slkv_join(void* stream);

/*
 * Context-parallel compression of ONE long sequence whose history keys are split over ranks (Sec. 3.4, Eq. 7-8;
 * Algorithm 3; same kept set as slkv_compress on the whole sequence, up to the score tolerance).
 *
 * Rank r of n_parts holds K / V rows of a contiguous range of history positions [b_r, e_r) plus up to pool_kernel/2
 * rows of each neighbour's range on either side (so that pooling needs nothing from the neighbours); the last rank
 * also holds the `window` rows behind the history.  Every rank holds q_win.  Per layer, on every rank:
 *   1. slkv_row_lse over the rows it OWNS (history_only = 1 on all ranks but the last, whose range is an ordinary
 *      sequence tail): the rows' log-sum-exp over this rank's keys.            all-gather over ranks
 *   2. slkv_cp_merge_lse: log-sum-exp over the ranks = the rows' log-sum-exp over all keys.
 *   3. slkv_score with lse_opt = that, over the owned rows plus the neighbours' margins: pooled scores.
 *   4. slkv_cp_select_init once, then for level = 0, 1, 2: slkv_cp_histogram over the owned positions,
 *      all-reduce (sum) of the histograms over ranks, slkv_cp_descend on the sum.  prefix[] then holds the bit
 *      pattern of every head's threshold score, need[] how many positions with exactly that score are kept.
 *   5. slkv_cp_local_ties (from the rank's OWN level-2 histogram): all-gather over ranks; slkv_cp_emit packs the
 *      rank's kept rows (the ties go to the lowest positions, i.e. in rank order) and its window rows.
 * The packed cache of head h is the concatenation over ranks of each rank's rows of head h; offsets[] are local.
 * The collectives (two all-gathers of a few hundred bytes and three all-reduces of n_kv_heads x 2048 int32 per layer)
 * are the caller's: the library launches no communication.  Everything is enqueued on `stream`; all pointers are
 * device pointers unless stated.
 *   lse_parts  [n_parts][n_q_heads][window] in p->lse_units (-inf for a rank without keys); lse_out [n_q_heads][window]
 *   prefix, need, ties  [n_kv_heads]; hist  [n_kv_heads][2048] int32 (zeroed by slkv_cp_histogram)
 *   pooled     [n_kv_heads][row_stride]: slkv_score's output for this rank's rows; the owned positions are
 *              own_begin .. own_begin + own_count - 1 of every row (the margins before and after them are not owned)
 *   pos0       position in the whole sequence of the first owned row
 *   rows       rows of k / v on this rank; row j of k / v is position j of pooled; window_rows = 0, or on the last rank
 *              the number of window rows, which are the last window_rows rows of k / v at positions window_pos0 ..
 *   ties_all   [n_parts][n_kv_heads]: every rank's slkv_cp_local_ties; part = this rank's index
 *   offsets    out, int32[n_kv_heads + 1]; kept_idx out, positions in the whole sequence; k_out, v_out as slkv_compress
 *   status     optional: SLKV_ERR_CAPACITY if offsets[n_kv_heads] > out_capacity_rows
 *
 * slkv_cp_step is steps 4 and 5 up to the packing with one launch between two collectives:
 *   level 0            what slkv_cp_select_init does, then the level-0 histogram
 *   level 1, 2         slkv_cp_descend of the level before on hist_sum, then this level's histogram
 *   level 3            slkv_cp_descend of level 2, then the owned positions above the threshold and those equal to it:
 *                      totals[0 .. n_kv_heads) above, totals[n_kv_heads .. 2 n_kv_heads) equal (= the ties to all-gather),
 *                      and counts by slice into the workspace for slkv_cp_emit_counted (workspace: level 3 only)
 *   state      int32 [4][2][n_kv_heads]: prefix and need after each level; state[3] goes to slkv_cp_emit_counted
 *   hist, totals  ADDED to: zeroed by the caller before the call; hist_sum: the histograms of the level before, summed
 *              over ranks
 *   clear      optional: clear_bytes (a multiple of 16, from a 16-byte boundary) are set to zero by the same launch --
 *              a share of k_out / v_out, where rows that nothing is packed into should be zero
 * slkv_cp_emit_counted is slkv_cp_emit on those totals and counts (same workspace contents); it also sets kept_idx to -1
 * behind the last packed row.  totals == NULL: exactly slkv_cp_emit.
 */
int slkv_cp_step(const int32_t* budgets, int32_t n_kv_heads, int32_t window, int64_t seq_len, int32_t level,
                 int32_t* state, const int32_t* hist_sum, const float* pooled, int64_t row_stride, int32_t own_begin,
                 int32_t own_count, int32_t* hist, int32_t* totals, void* clear, size_t clear_bytes, void* workspace,
                 size_t workspace_bytes, void* stream);
int slkv_cp_emit_counted(const slkv_params* p, const void* k, const void* v, int64_t rows, const float* pooled,
                         int64_t row_stride, int32_t own_begin, int32_t own_count, int64_t pos0,
                         const uint32_t* threshold, const int32_t* need, const int32_t* ties_all, int32_t n_parts,
                         int32_t part, int32_t window_rows, int64_t window_pos0, const int32_t* totals, void* k_out,
                         void* v_out, int64_t out_capacity_rows, int32_t* offsets, int32_t* kept_idx, int32_t* status,
                         void* workspace, size_t workspace_bytes, void* stream);
int slkv_cp_merge_lse(const slkv_params* p, const float* lse_parts, int32_t n_parts, float* lse_out, void* stream);
/* slkv_row_lse on a workspace that is zero throughout (step 1: a caller that clears several buffers at once spares the call its
 * own clearing, which stands between the kernels before and the statistics). */
int slkv_cp_row_lse(const slkv_params* p, const void* q_win, const void* k, const int32_t* cu_seqlens_dev,
                    const int32_t* cu_seqlens_host, float* lse_out, int32_t* status, void* zeroed_workspace,
                    size_t workspace_bytes, void* stream);
int slkv_cp_select_init(const int32_t* budgets, int32_t n_kv_heads, int32_t window, int64_t seq_len, uint32_t* prefix,
                        int32_t* need, void* stream);
int slkv_cp_histogram(const float* pooled, int32_t n_kv_heads, int64_t row_stride, int32_t own_begin, int32_t own_count,
                      int32_t level, const uint32_t* prefix, int32_t* hist, void* stream);
int slkv_cp_descend(const int32_t* hist, int32_t n_kv_heads, int32_t level, uint32_t* prefix, int32_t* need,
                    void* stream);
int slkv_cp_local_ties(const int32_t* hist_local, const uint32_t* prefix, int32_t n_kv_heads, int32_t* ties,
                       void* stream);
size_t slkv_cp_workspace_bytes(int32_t n_kv_heads, int32_t own_count, int64_t out_capacity_rows);
int slkv_cp_emit(const slkv_params* p, const void* k, const void* v, int64_t rows, const float* pooled,
                 int64_t row_stride, int32_t own_begin, int32_t own_count, int64_t pos0, const uint32_t* threshold,
                 const int32_t* need, const int32_t* ties_all, int32_t n_parts, int32_t part, int32_t window_rows,
                 int64_t window_pos0, void* k_out, void* v_out, int64_t out_capacity_rows, int32_t* offsets,
                 int32_t* kept_idx, int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/* Bytes of device arena slkv_compress_host needs (inputs, outputs and workspace; 0 on invalid arguments). */
size_t slkv_compress_host_arena_bytes(const slkv_params* p, const int32_t* cu_seqlens_host,
                                      int64_t out_capacity_rows);

/*
 * slkv_compress for callers whose tensors live in host memory (Algorithm 3, same semantics).
 * q_win, k, v, budgets are HOST inputs (dense layouts: the strides in `p` must describe contiguous
 * [n_seqs, window, n_q_heads, head_dim] and [total_tokens, n_kv_heads, head_dim] arrays); k_out, v_out,
 * offsets, kept_idx are HOST outputs.  `arena` is caller-owned DEVICE memory of at least
 * slkv_compress_host_arena_bytes, 256-byte aligned.  The call copies the inputs to the arena, runs the
 * kernels, copies offsets, kept_idx and the packed rows back and waits for `stream` before returning, so
 * the outputs are valid on return.  Page-locked host buffers make it fast (of V only the kept rows then cross
 * the link, and the outputs are written without a copy); pageable ones work.  Returns SLKV_ERR_CAPACITY if out_capacity_rows is too small (nothing is copied back then
 * except offsets).  *rows_out (optional) receives offsets[last].
 */
int slkv_compress_host(const slkv_params* p, const void* q_win, const void* k, const void* v,
                       const int32_t* cu_seqlens_host, const int32_t* budgets, void* k_out, void* v_out,
                       int64_t out_capacity_rows, int32_t* offsets, int32_t* kept_idx, int64_t* rows_out,
                       void* arena, size_t arena_bytes, void* stream);

/*
 * slkv_score without a workspace argument, for callers that cannot allocate device memory.  (The paper has
 * no counterpart: this is a property of the library, not of the method.)
 *
 * Who needs it: code that runs inside a host application which has already handed every free byte of the
 * GPU to its own pool (a serving engine that sizes its KV-cache blocks from "all memory that is left"), or a
 * plug-in that is given tensors but no handle to the host's allocator.  There cudaMalloc fails, or succeeds
 * only by synchronising the whole device and shrinking somebody else's pool, and torch's allocator is not
 * the caller's to use.  Such a caller still owns its inputs and outputs; what it lacks is scratch.
 *
 * The scratch is a fixed array of SLKV_NOALLOC_SCRATCH_BYTES (and 10 KB for what the CTAs of a launch tell one
 * another) inside the library's device image: every GPU that loads the library holds that much memory until the
 * process exits, used or not.  The call computes exactly what slkv_score computes, with the same kernels and the
 * same results.
 *   - Shapes whose slkv_workspace_bytes exceed the array are rejected with SLKV_ERR_WORKSPACE before anything
 *     is enqueued (32k tokens x 8 KV heads x 128 score rows needs about 5.3 MB).
 *   - The first call on each device looks up the array's device address (a CUDA runtime query, made with that
 *     device current) and keeps it.  With the CUDA runtime's lazy module loading the array comes into being at
 *     that query, not when the library is loaded: make the first call at start-up, while SLKV_NOALLOC_SCRATCH_BYTES
 *     of device memory are still free (otherwise it returns SLKV_ERR_CUDA), and outside any stream capture.
 *   - The library itself calls no cudaMalloc, cudaFree or other allocating routine, on the first call or later.
 *   - All calls on a device share the one array.  It keeps whatever the previous call left; nothing in it has
 *     to be zero, each call overwrites what it reads.  Two calls whose kernels may overlap on the GPU
 *     (different streams, no ordering between them) race on it: order them.
 * Arguments and return value as slkv_score, minus workspace / workspace_bytes.  If the address query fails
 * the call returns SLKV_ERR_CUDA and slkv_noalloc_last_cuda_error() gives the runtime's code.
 */
#define SLKV_NOALLOC_SCRATCH_BYTES (8u << 20)
int slkv_score_noalloc(const slkv_params* p, const void* q_win, const void* k, const int32_t* cu_seqlens_dev,
                       const int32_t* cu_seqlens_host, const float* lse_opt, float* pooled, int32_t* status,
                       void* stream);
size_t slkv_noalloc_scratch_bytes(void);      /* = SLKV_NOALLOC_SCRATCH_BYTES */
int slkv_noalloc_last_cuda_error(void);

/*
 * The compressed cache in decoding (no counterpart in the paper, which ends with the prefill): the rows that slkv_compress kept, held in
 * 4 bits, attended to by new tokens, and kept within their heads' budgets while tokens come in.
 *
 * A cache has n_seqs * n_kv_heads segments, seg = s * n_kv_heads + h as in the packed output.  Segment seg owns the slots
 * starts[seg] .. starts[seg+1]-1; the first lens[seg] of them are filled.  starts with no slack is slkv_compress' offsets; with slack,
 * tokens can be appended.  starts and lens are device arrays that the host never reads: lengths that do not fit their segments and
 * segments that do not fit the cache are cut to what fits.  Per slot:
 *   records  slkv_q4_record_bytes(head_dim) = head_dim * 5 / 4 bytes: the token's K and V row in groups of 32 channels.  A group has a
 *            scale and a zero in bf16, a channel a 4-bit code; it stands for zero + scale * code.
 *              zero = the minimum of the group rounded down to bf16, scale = (maximum - zero) / 15 rounded up to bf16,
 *              code = (x - zero) / scale in fp32, rounded to the nearest integer, ties to even: 0 .. 15
 *            so that |x - value| <= scale / 2 up to fp32 rounding.  A group with a NaN or an infinity, or with a range that fp32 does
 *            not hold or a zero that bf16 does not, stands for NaN throughout.
 *            Layout: head_dim/2 bytes K codes, head_dim/2 bytes V codes, then head_dim/32 bf16 each of K scales, K zeros, V scales and
 *            V zeros.  K codes: 32-bit word t * head_dim/32 + j has channels 32 j + 8 t + e in its nibbles e = 0 .. 7, lowest first; V
 *            codes: 16-bit unit g * head_dim/32 + j has channels 32 j + 4 g + e in its nibbles e = 0 .. 3.
 *   pos      the token's position in its sequence (kept_idx).  Slots need not be in the order of their positions.
 *   weight   the attention the row has received: 0 when it comes in, added to by slkv_q4_attend, read by slkv_q4_evict.  May be NULL
 *            for callers that never evict.
 * Everything is enqueued on `stream`, nothing is allocated, every call can be captured.  A cache and a workspace belong to one call at a
 * time: calls on several streams, and graphs that are replayed beside each other, need their own or an order between them.  Results are
 * the same bit for bit from call to call.  n_seqs * n_kv_heads <= 16384, 1 <= capacity_rows < 2^31; records, rows and workspaces 16-byte aligned.
 */
typedef struct slkv_q4_cache {
  int32_t n_seqs, n_kv_heads, head_dim;   /* head_dim 64 or 128 */
  int32_t reserved;
  int64_t capacity_rows;                  /* slots of the arrays below */
  void* records;                          /* dev */
  int32_t* pos;                           /* dev */
  float* weight;                          /* dev, optional */
  const int32_t* starts;                  /* dev, int32[n_seqs*n_kv_heads + 1], ascending */
  int32_t* lens;                          /* dev, int32[n_seqs*n_kv_heads] */
} slkv_q4_cache;

size_t slkv_q4_record_bytes(int32_t head_dim);   /* 0 for a head_dim that is not supported */

/*
 * A packed layer into the cache: rows offsets[seg] .. offsets[seg+1]-1 of k, v (the k_out, v_out, offsets and kept_idx of slkv_compress)
 * become the segment's first rows, lens[seg] their number, their positions kept_idx, their weights 0.
 *   k, v       dev, [n_rows, head_dim] elements of dtype (SLKV_F32 | SLKV_BF16), contiguous; n_rows: rows that may be read
 *   offsets    dev, int32[n_seqs*n_kv_heads + 1];  kept_idx dev, int32[n_rows]
 *   status     dev, optional: SLKV_ERR_CAPACITY if a segment has more rows than slots, or offsets run past n_rows (the rest is dropped)
 * Behind slkv_compress_overlapped calls on the same stream no slkv_join is needed (what is queued goes out, so pack behind the last
 * layer, not between the layers); behind those of another stream it is.
 */
int slkv_q4_pack(const slkv_q4_cache* c, int32_t dtype, const void* k, const void* v, int64_t n_rows, const int32_t* offsets,
                 const int32_t* kept_idx, int32_t* status, void* stream);

/*
 * New tokens' rows behind the filled slots of every segment.
 *   k, v       dev: element (s, i, h, p) at s*stride_seq + i*stride_tok + h*stride_head + p, i < n_tokens <= 65536
 *   pos        dev, int32[n_seqs][n_tokens]: the tokens' positions
 *   lens_out   dev, optional: takes the new lengths in place of c->lens, which then keeps the old ones (tokens that are drafted, and
 *              may have to go again)
 *   status     dev, optional: SLKV_ERR_CAPACITY if a segment has not enough slots left (it takes the tokens that fit)
 */
int slkv_q4_append(const slkv_q4_cache* c, int32_t dtype, const void* k, const void* v, int32_t n_tokens, int64_t k_stride_seq,
                   int64_t k_stride_tok, int64_t k_stride_head, int64_t v_stride_seq, int64_t v_stride_tok, int64_t v_stride_head,
                   const int32_t* pos, int32_t* lens_out, int32_t* status, void* stream);

/*
 * The values that records stand for, as rows of dtype (rounded to nearest for bf16).
 *   slots_opt    dev, optional, int32[n]: row i of k_out, v_out [n, head_dim] is slot slots_opt[i]'s, filled or not (tokens that were
 *                drafted lie behind the filled ones); entries outside the cache are padding, whose rows are left as they are.
 *                NULL: row i is slot i's, for the filled slots (n is capacity_rows whatever is passed); the other rows are left as they are.
 */
int slkv_q4_unpack(const slkv_q4_cache* c, int32_t dtype, const int32_t* slots_opt, int64_t n, void* k_out, void* v_out, void* stream);

/*
 * Attention of n_tokens new tokens per sequence over the cache (their own rows appended or not).  For query head qh of KV head h and
 * token i, over the filled slots r of segment (s, h):
 *     x[r] = scale * q . K[r];  softcap > 0: x = softcap * tanh(x / softcap);  slopes: x += slopes[qh] * (pos[r] - q_pos[s][i])
 *     visible: every filled slot; with q_pos those with pos[r] <= q_pos[s][i]
 *     out = sum p V, p = softmax of x over the visible slots;  lse = log sum exp x
 * A query that sees no slot gets zeros and -infinity.  A slot that is not visible to a query gives it nothing, whatever it holds.
 *   q, out     dev, elements of dtype: element (s, i, qh, p) at s*stride_seq + i*stride_tok + qh*stride_head + p
 *   q_pos_opt  dev, optional, int32[n_seqs][n_tokens];  slopes_opt dev, optional, float[n_q_heads] (needs q_pos_opt)
 *   lse_opt    dev, optional out, float[n_seqs][n_q_heads][n_tokens] in lse_units
 *   accumulate 1: weight[r] = weight_decay * weight[r] + (1/G) sum over the G query heads of h and over the tokens of p[r], for every
 *              filled slot (the reduction slkv_score uses over window rows and heads)
 *   status     dev, optional: SLKV_ERR_DEVICE_TIMEOUT if a wait inside the kernel ran out (a copy that takes a second).  out and lse of
 *              the query heads concerned are then NaN, and with accumulate the weights of their segments too; the rest is as ever
 * Limits: n_q_heads / n_kv_heads * n_tokens <= 256.  Positions are >= 0.  Queries are below 2^67 in magnitude (a head with a larger
 * one, or a NaN, gets NaN), sums of products q . K below 2^200, scores below 2^124, values below 2^119 over the number of a segment's
 * rows (outputs are summed before they are divided by the softmax's sum); beyond these a head may get NaN.  A score is off by up to
 * |scale| * |K| * 2^-58 beside its roundings, which shows only for queries far below 2^-40.
 * fp32 accumulation throughout; with bf16 rows, probabilities times scales are rounded to bf16 for the product with V: up to 2^-8 of
 * each term p * scale * |code - 8|.  With fp32 rows, over the same cache, they keep 24 bits.
 * The workspace is some 64 bytes per segment and block of 8 columns, 8 MB at most for outputs of pieces, and with accumulate a float
 * per slot of the cache (filled or not) and column (query head of a KV head, and token): 16 bytes a slot for 4 heads and one token.
 */
typedef struct slkv_q4_attend_params {
  int32_t n_q_heads;        /* multiple of the cache's n_kv_heads */
  int32_t n_tokens;         /* per sequence, >= 1 */
  int32_t dtype;            /* SLKV_F32 | SLKV_BF16: q and out */
  int32_t lse_units;        /* SLKV_LSE_LN | SLKV_LSE_LOG2 */
  float scale;              /* 1 / sqrt(head_dim), usually; at most 2^54 in magnitude */
  float softcap;            /* 0: none; else >= 1e-20 */
  float weight_decay;       /* 1: a plain sum */
  int32_t reserved;
  int64_t q_stride_seq, q_stride_tok, q_stride_head;
  int64_t o_stride_seq, o_stride_tok, o_stride_head;
} slkv_q4_attend_params;
size_t slkv_q4_attend_workspace_bytes(const slkv_q4_cache* c, const slkv_q4_attend_params* p, int32_t accumulate);   /* 0: bad arguments */
int slkv_q4_attend(const slkv_q4_cache* c, const slkv_q4_attend_params* p, const void* q, const int32_t* q_pos_opt,
                   const float* slopes_opt, void* out, float* lse_opt, int32_t accumulate, int32_t* status, void* workspace,
                   size_t workspace_bytes, void* stream);

/*
 * Eviction: segment (s, h) with len rows keeps kept = min(len, max(budgets[h], window)) of them -- the rows with
 * pos > newest[s] - window first, then those with the largest weights (NaN counts as less than any number; ties: lower slot first).
 * Slot i < kept of the result holds row i where that is kept; the slots of rows that go take the kept rows from slots kept, kept + 1, ..
 * in ascending order.  to->lens[seg] = kept.
 *   from, to   the same cache (in place: records, pos, weight, starts and capacity the same, lens the same array or another), or another
 *              one with the same numbers of sequences and heads that shares no memory with it and may lay out its segments otherwise.
 *              Slots behind the kept rows are left as they are.
 *   budgets    dev, int32[n_kv_heads];  newest dev, int32[n_seqs]: the position of the sequence's newest token;  window >= 1
 *   status     dev, optional: SLKV_ERR_CAPACITY if a segment of `to` has fewer slots than rows are kept (it takes the first ones)
 */
size_t slkv_q4_evict_workspace_bytes(const slkv_q4_cache* from);     /* 0: bad arguments */
int slkv_q4_evict(const slkv_q4_cache* from, const slkv_q4_cache* to, const int32_t* budgets, int32_t window, const int32_t* newest,
                  int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Attention of whole prompts, causal (Eq. 1-5; the attention whose keys slkv_compress then selects from).  Sequence s has nq = cu_q[s+1] -
 * cu_q[s] queries and nk = cu_k[s+1] - cu_k[s] keys, the queries being its last tokens (nk > nq: what lies before them was there
 * already, a prompt in chunks).  For token i < nq, query head qh of KV head h, over the keys j <= i + nk - nq:
 *     out = sum p V[j],  p = softmax of scale * q . K[j];   lse = log sum exp(scale * q . K[j])
 * A query that sees no key (nk < nq) gets zeros and -infinity.  A key that a query does not see gives it nothing, whatever K and V hold
 * there; sequences do not see one another.
 *   q, out        dev, elements of dtype: element (t, qh, p) at t*stride_tok + qh*stride_head + p, t in [0, cu_q[n_seqs])
 *   k, v          dev, likewise by KV head, t in [0, cu_k[n_seqs])
 *   cu_q_dev      dev, int32[n_seqs+1], cu_q[0] = 0;  cu_q_host: the same values on the host (they size the launch)
 *   cu_k_*_opt    both or neither; NULL: the keys are the queries' own tokens
 *   lse_opt       dev, optional out, float[n_seqs][n_q_heads][window] in lse_units: row i of a sequence is its token nq - window + i; rows
 *                 before its first query are left as they are.  With the window of slkv_params this is the lse_opt of slkv_score and
 *                 slkv_compress (SLKV_ALL_CAUSAL), which spares them their pass over K for it.
 *   status        dev, optional: SLKV_ERR_DEVICE_TIMEOUT if a wait inside a kernel ran out; rows concerned are then left as they were or NaN
 * Limits: n_q_heads / n_kv_heads <= 64, at most 2^31 - 512 tokens, n_seqs * n_kv_heads < 2^31.  Strides of axes longer than one: head_dim at
 * least, below 2^38, multiples of 16 bytes, as are addresses.  Scores below fp32's range in magnitude: where a query or a key that it sees is not
 * finite, its results may be NaN.  An infinite value that a query sees makes the output infinite, or NaN where its probability rounds to 0.
 * fp32 accumulation throughout; with bf16, probabilities are rounded to bf16 for the product with V (2^-8 of each term).  fp32 rows are
 * exact sums of three bf16 parts, whose products with less than 2^-24 of a term are left out.  Results are the same bit for bit from call
 * to call.  out is none of the inputs.  A workspace belongs to one call at a time.
 * Layers queued by slkv_compress_overlapped stay queued, but for those that take the log-sum-exps which lse_opt overwrites (see there); their other
 * inputs and outputs are not to be overwritten in front of slkv_join, by out neither.
 */
typedef struct slkv_prompt_params {
  int32_t n_seqs;
  int32_t n_q_heads;        /* multiple of n_kv_heads */
  int32_t n_kv_heads;
  int32_t head_dim;         /* 64 or 128 */
  int32_t window;           /* >= 1: rows of lse_opt */
  int32_t dtype;            /* SLKV_F32 | SLKV_BF16 */
  int32_t lse_units;        /* SLKV_LSE_LN | SLKV_LSE_LOG2 */
  float scale;              /* 1 / sqrt(head_dim), usually; 2^-54 .. 2^54 */
  int64_t q_stride_tok, q_stride_head, k_stride_tok, k_stride_head, v_stride_tok, v_stride_head, o_stride_tok, o_stride_head;
} slkv_prompt_params;
size_t slkv_prompt_attend_workspace_bytes(const slkv_prompt_params* p, const int32_t* cu_q_host, const int32_t* cu_k_host_opt);   /* 0: bad arguments */
int slkv_prompt_attend(const slkv_prompt_params* p, const void* q, const void* k, const void* v, const int32_t* cu_q_dev,
                       const int32_t* cu_q_host, const int32_t* cu_k_dev_opt, const int32_t* cu_k_host_opt, void* out, float* lse_opt,
                       int32_t* status, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The compressed cache in pages (no counterpart in the paper): rows as slkv_compress packs them, with room to grow.  Budgets differ per
 * head, so every segment has a length of its own: a page belongs to one segment of one layer, and all layers share the pool.
 *
 * Segment seg = (layer * n_seqs + s) * n_kv_heads + h has lens[seg] rows; row r is row r % page_rows of page tables[seg][r / page_rows].
 * A slot is page * page_rows + row.  free_pages[0 .. n_free) is a stack of the pages that no segment has.  Tables, lengths and stack are
 * device arrays that the host never reads: lengths beyond max_pages pages are cut to them, entries of tables outside the pool are read as
 * pages of zeros (status: SLKV_ERR_BAD_SHAPE).
 * Everything is enqueued on `stream`, nothing is allocated, every call can be captured.  A cache and a workspace belong to one call at a
 * time.  n_seqs * n_kv_heads <= 16384, n_layers times that <= 2^20, that times max_pages < 2^31; n_pages and max_pages times page_rows
 * <= 2^31 - 512; pages, rows and workspaces 16-byte aligned.
 */
typedef struct slkv_paged_cache {
  int32_t n_layers, n_seqs, n_kv_heads;
  int32_t head_dim;         /* 64 or 128 */
  int32_t dtype;            /* SLKV_F32 | SLKV_BF16 */
  int32_t page_rows;        /* 16, 32, 64 or 128 */
  int32_t n_pages;          /* of the pool */
  int32_t max_pages;        /* entries of a segment's table */
  void *k_pages, *v_pages;  /* dev, [n_pages][page_rows][head_dim] */
  int32_t* tables;          /* dev, [n_layers*n_seqs*n_kv_heads][max_pages] */
  int32_t* lens;            /* dev, [n_layers*n_seqs*n_kv_heads] */
  int32_t* free_pages;      /* dev, [n_pages] */
  int32_t* n_free;          /* dev, [1] */
} slkv_paged_cache;

/*
 * New lengths for all segments: pages that are no longer needed go back to the stack, pages that are come from it, and new rows get
 * their slots.  Wanted lengths, by mode:
 *   SLKV_PAGED_LENGTHS  want[n_segments]: the length itself (0: the sequence is done; less than it has: drafted rows go again)
 *   SLKV_PAGED_OFFSETS  want[n_layers][n_seqs*n_kv_heads + 1]: offsets as slkv_compress writes them, a segment's rows being its length
 *   SLKV_PAGED_ADD      want[n_seqs]: rows that every segment of the sequence gets in addition (below 0 counts as 0)
 * First all pages are returned, so that the first segment's first returned page ends up on top of the stack, the next ones below it; then
 * the segments take theirs from the top, in order.  Taking and returning are each other's inverse: going back to the old lengths leaves
 * stack and tables as they were.  Where the pages run out (or a table is full) a segment gets what there is, the ones behind it nothing,
 * and lengths are cut to the pages: status is SLKV_ERR_CAPACITY.
 *   slots_opt        dev, optional out, int32[n_slots]: the slots of the rows that come in (old length .. new length - 1).
 *                    slot_width = 0: one segment's behind the other's, from slot_offsets[seg] on (slot_offsets_opt: int32[n_segments+1],
 *                    required); -1 behind the last one.  A fresh cache's slots so lie in the order of slkv_compress' packed rows.
 *                    slot_width > 0: segment seg's from seg * slot_width on, -1 behind them.
 *                    Rows beyond n_slots or slot_width get none (status: SLKV_ERR_CAPACITY).
 *   lens_out, n_free_out   dev, optional, both or neither: take the new values in place of c->lens and c->n_free, which then keep the old
 *                    ones: c still describes the cache as it was (tokens that are drafted), until a plan from there takes the pages again.
 *                    lens_out is c->lens or does not overlap it.
 * OFFSETS behind slkv_compress_overlapped calls on the same stream needs no slkv_join: what is queued there goes out first.
 */
enum { SLKV_PAGED_LENGTHS = 0, SLKV_PAGED_OFFSETS = 1, SLKV_PAGED_ADD = 2 };
int slkv_paged_plan(const slkv_paged_cache* c, int32_t mode, const int32_t* want, int32_t* slots_opt, int64_t n_slots, int32_t slot_width,
                    int32_t* slot_offsets_opt, int32_t* lens_out, int32_t* n_free_out, int32_t* status, void* stream);

/*
 * Rows into slots: for every sequence s, head h and r < n_slots with a slot inside the pool, token t = take_opt[s][r] (NULL: r) of k and v,
 * bit for bit.  Slots outside the pool are padding, and so are tokens outside 0 .. n_tokens - 1.  A slot is to be named once.
 *   k, v       dev, elements of the cache's dtype: element (s, t, h, p) at s*stride_seq + t*stride_tok + h*stride_head + p
 *   slots      dev, int32[n_seqs][n_heads][n_slots]: a layer's part of what slkv_paged_plan wrote
 *   take_opt   dev, optional, int32[n_seqs][n_slots]: which tokens (of a tree, the accepted ones)
 * A packed layer (k_out, v_out of slkv_compress) is one sequence and one head of n_tokens = its rows.  Behind slkv_compress_overlapped
 * calls on the same stream no slkv_join is needed.
 */
int slkv_paged_write(const slkv_paged_cache* c, const void* k, const void* v, int32_t n_seqs, int32_t n_heads, int32_t n_tokens,
                     int64_t k_stride_seq, int64_t k_stride_tok, int64_t k_stride_head, int64_t v_stride_seq, int64_t v_stride_tok,
                     int64_t v_stride_head, const int32_t* slots, int32_t n_slots, const int32_t* take_opt, void* stream);

/*
 * Attention of n_tokens <= 64 tokens per sequence over one layer of the cache and over each other.  Token i of sequence s sees all rows of
 * the segment (s, h) and, with has_new, those tokens j whose bit is set in tree[s][i]; their K and V rows are k_new and v_new, which are
 * not in the cache (tokens that are refused leave no trace; the accepted ones go in by slkv_paged_plan and slkv_paged_write).
 * out and lse as slkv_prompt_attend; a token that sees nothing gets zeros and -infinity, what it does not see gives it nothing.
 *   q, out         dev: element (s, i, qh, p) at s*stride_seq + i*stride_tok + qh*stride_head + p
 *   k_new, v_new   dev, with has_new: element (s, i, h, p) likewise
 *   tree_opt       dev, optional, uint64[n_seqs][n_tokens]; NULL: token i sees the tokens 0 .. i
 *   n_new_opt      dev, optional, int32[n_seqs]: tokens of each sequence; the rows behind them are padding: not read by others, outputs left as they are
 *   lse_opt        dev, optional out, float[n_seqs][n_q_heads][n_tokens] in lse_units
 * Limits, precision, status and workspace as slkv_prompt_attend.  Tiles are counted in 32 bits, whatever lengths there are: n_seqs * n_kv_heads
 * times the blocks of 2 * (128 / G) tokens (fp32: of 128 / G; G = n_q_heads / n_kv_heads, quotients rounded down) that n_tokens make times
 * max_pages * page_rows / 128 + 4 (fp32: / 64) < 2^31, counts rounded up.
 */
typedef struct slkv_paged_attend_params {
  int32_t n_q_heads;        /* multiple of the cache's n_kv_heads */
  int32_t n_tokens;         /* per sequence, 1 .. 64 */
  int32_t layer;            /* of the cache */
  int32_t has_new;          /* 1: the tokens' own rows are in k_new, v_new; 0: only the cache is seen */
  int32_t lse_units;        /* SLKV_LSE_LN | SLKV_LSE_LOG2 */
  float scale;
  int64_t q_stride_seq, q_stride_tok, q_stride_head, o_stride_seq, o_stride_tok, o_stride_head;
  int64_t k_stride_seq, k_stride_tok, k_stride_head, v_stride_seq, v_stride_tok, v_stride_head;
} slkv_paged_attend_params;
size_t slkv_paged_attend_workspace_bytes(const slkv_paged_cache* c, const slkv_paged_attend_params* p);   /* 0: bad arguments */
int slkv_paged_attend(const slkv_paged_cache* c, const slkv_paged_attend_params* p, const void* q, const void* k_new, const void* v_new,
                      const uint64_t* tree_opt, const int32_t* n_new_opt, void* out, float* lse_opt, int32_t* status, void* workspace,
                      size_t workspace_bytes, void* stream);

/* Number of kernels the most recent slkv_score / slkv_compress / slkv_compress_host / slkv_q4_* / slkv_prompt_* / slkv_paged_* call on
 * this thread enqueued (launch accounting for benchmarks). */
int slkv_last_launch_count(void);

/*
 * Per-kernel timing for benchmarks (no counterpart in the paper).  While enabled on the calling thread,
 * every kernel the library enqueues is bracketed by a CUDA event pair on its stream (events are created
 * on demand and reused; this adds host work per launch, so headline timings are taken with it off).
 * on = 1: every kernel (each then waits for the one before it to end, so that the step is slower than untimed); on = 2:
 * the score kernels only -- their times in the regime of an untimed step; on = 0: off.
 * slkv_profile_collect waits for the recorded events, adds each kernel's elapsed milliseconds and launch
 * count into total_ms[id] / launches[id] (arrays of n_kernels entries, overwritten) and forgets the records.
 * Kernel ids run from 0 to slkv_kernel_count()-1; slkv_kernel_name gives their names.
 */
int slkv_profile_enable(int on);
int slkv_profile_collect(float* total_ms, int32_t* launches, int32_t n_kernels);
const char* slkv_kernel_name(int kernel_id);
int slkv_kernel_count(void);

/*
 * Timeline tracing of the tensor-core score kernels (diagnostics; no counterpart in the paper).
 * With a device buffer set on the calling thread, every CTA of the score kernel stores %globaltimer nanosecond stamps
 * into it, 64 uint64 slots per CTA: 0 CTA start, 1 past its wait for the launch before, 3 first log-sum-exps of a vote
 * phase there, 4 CTA end, 60 / 61 the SM cycle counter at CTA start / end.  The buffer that is set when a launch is
 * enqueued is the one it writes (the overlapped entry point enqueues a list when it is full, or at a join).  The buffer must
 * hold n_cta * 64 * 8 bytes (n_cta <= number of SMs); smaller buffers switch tracing off.  NULL switches it off.
 */
int slkv_trace_set_buffer(void* dev_buf, size_t bytes);

/*
 * Test hook for the bounded waits (no counterpart in the paper).  Where the CTAs of a launch wait for one another
 * (the counters between the two passes of the score kernel; row sums and votes between the CTAs of a segment where one launch does
 * a short layer), and where warps of slkv_q4_attend, slkv_prompt_attend or slkv_paged_attend wait for copies and products, every wait
 * gives up after one second, sets SLKV_ERR_DEVICE_TIMEOUT in the call's status word, releases what the CTA holds and returns.  With the
 * hook armed (on != 0) the next such launch made by the calling thread waits for one arrival more than there are -- on = 1: where the CTAs
 * of a score launch wait for the statistics, 2: for their clearing, 3: where those of a one-launch layer wait for the row sums, 4: for the
 * votes, 5: where the first CTA of slkv_q4_attend waits for rows, or those of slkv_prompt_attend or slkv_paged_attend for probabilities --
 * so that exactly this path runs: the call's results are then incomplete and its status word says so; the calls after it are unaffected.
 * While it is armed with 1 or 2, short layers go the way of the others; a list that goes with one product with every key
 * (slkv_debug_list_way) waits for statistics only where some head needs all its votes.  One-shot: the launch that takes it disarms it.
 */
int slkv_debug_expire_next_wait(int on);

/*
 * Test hook for lists of overlapped calls whose pooled scores nobody asks for (no counterpart in the paper).  Such a list goes with one
 * product with every key or with two, which keep the same positions, by a rule on its size and its layers' capacities.  way = 1: lists
 * that the calling thread sends out go with one product wherever the kernels take the shape, 2: with two, 0: by the rule.
 */
int slkv_debug_list_way(int way);

/* Library version, major*10000 + minor*100 + patch. */
int slkv_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SLKV_H_ */
