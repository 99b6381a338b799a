/*
 * qgemm.h - C ABI of the MI355X (gfx950) block-quantised prefill GEMM library.
 *
 * The library computes the prompt-processing (prefill) matrix multiplies the
 * paper routes onto matrix units (Section 3.1): dense projection GEMMs over
 * 4-bit / 8-bit block-quantised weights, and the MoE expert GEMM that
 * evaluates each active expert's projection over the tokens routed to it,
 * plus the SiLU-gated activation between the MoE projections (Section 3.1,
 * fused gate/up item) and the router-weighted combine of the experts' outputs.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - Pointers are DEVICE pointers (memory the HIP runtime of this process
 *   allocated on the current device) unless the comment says HOST.
 * - Arrays are dense and row-major; no strides, but for the row strides that the
 *   serving entry points take. Every device pointer must be 16-byte aligned,
 *   except fp16 scale arrays, which need 2-byte alignment, and the tables of
 *   the serving entry points and qgemm_rope's rows, which need that of their
 *   elements (QGEMM_EALIGN otherwise).
 * - Work is enqueued on `stream` (0 = the null stream) and the call returns
 *   without synchronising; device faults surface at the caller's next sync.
 *   The caller keeps every buffer alive until the stream has passed the call.
 * - Outputs are written, never accumulated into (but for qgemm_adapters' y), and must not alias inputs.
 * - Return value: QGEMM_OK (0) or a negative QGEMM_E* code. On an error return
 *   nothing has been enqueued and no output is written;
 *   qgemm_last_error() gives a message. No entry point throws.
 * - A zero-sized problem (M, T or rows == 0) returns QGEMM_OK and launches
 *   nothing.
 *
 * Storage formats (the paper names 4-bit and 8-bit block quantisation without a
 * byte layout; this is the layout the library reads):
 * - activations x: bf16 [rows][K].
 * - QGEMM_Q8 weights: int8 [N][K]; element (n, k) means q * s.
 * - QGEMM_Q4 weights: uint8 [N][K/2]; byte j of a row holds element 2j in
 *   bits 0-3 and element 2j+1 in bits 4-7; a nibble u means (u - 8) * s.
 * - scales: fp16 [N][K/32]; s = scales[n][k / 32] (one scale per 32
 *   consecutive K elements of a row).
 * - K must be a multiple of 32.
 * - results: fp32, y[m][n] = sum_k x[m][k] * s[n][k/32] * q[n][k]; the
 *   library rounds each dequantised weight to bf16 and accumulates in fp32.
 */
#ifndef QGEMM_H
#define QGEMM_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#ifndef __HIP_INCLUDE_HIP_HIP_RUNTIME_API_H__
typedef struct ihipStream_t* hipStream_t;
#endif

enum qgemm_fmt { QGEMM_Q8 = 0, QGEMM_Q4 = 1 };

enum qgemm_type { QGEMM_F32 = 0, QGEMM_BF16 = 1 };

enum qgemm_rope_scaling {
  QGEMM_ROPE_PLAIN = 0,
  QGEMM_ROPE_LINEAR = 1,
  QGEMM_ROPE_LLAMA3 = 2,
  QGEMM_ROPE_YARN = 3
};

enum qgemm_status {
  QGEMM_OK = 0,
  QGEMM_EINVAL = -1,       /* bad size, format, null pointer or routing table */
  QGEMM_EALIGN = -2,       /* a device pointer is not 16-byte aligned */
  QGEMM_EUNSUPPORTED = -3, /* a size beyond what the library handles */
  QGEMM_EHIP = -4          /* the HIP runtime reported an error */
};

/*
 * Dense block-quantised GEMM (Section 3.1, dense GEMM item):
 *   y[M][N] = x[M][K] . dequant(wq, scales)^T
 * x: bf16 [M][K]; wq: int8 [N][K] (Q8) or uint8 [N][K/2] (Q4);
 * scales: fp16 [N][K/32]; y: fp32 [M][N].
 * Sizes: M >= 0, 1 <= N, 32 <= K, K % 32 == 0, every element count < 2^31.
 * When few output tiles meet a long K, the call splits K over several
 * workgroups and sums their fp32 partials in split order (deterministic) in a
 * library-owned workspace (grown on first use, freed by qgemm_release);
 * concurrent calls on different streams must not share it.
 * M <= 16 (decode and speculative-draft verification, the memory-bound
 * regime of Section 2.3 and the batched verification of Section 5.2) takes a
 * separate bandwidth-oriented kernel: weights dequantised straight into
 * matrix-core registers, K split over waves (and over workgroups when N is
 * small, through the same workspace). The same kernel, in blocks of 16
 * activation rows, serves 16 < M <= 128 when ceil(N/128) times the number of
 * 16-row blocks (rounded up to 2, 4 or 8) is at most 512: short prompts whose
 * few 128x128 output tiles would leave most CUs idle. Its results are bitwise
 * reproducible but not bitwise equal to the tile kernels' (another summation
 * order).
 */
int qgemm_dense(const void* x, const void* wq, const void* scales, float* y,
                int M, int N, int K, int fmt, hipStream_t stream);

/*
 * MoE expert GEMM (Section 3.1, MoE expert GEMM item): every token slot
 * ("assignment") a = t*topk + j is multiplied by the weights of its expert:
 *   y[a][:] = dequant(wq[e], scales[e]) . x[a / topk][:],  e = token_expert_idx[a]
 * Only experts with at least one assignment read their weights.
 * x: bf16 [T][K].
 * token_expert_idx: int32 [T*topk], values in [0, E).
 * expert_offsets: int32 [E+1], exclusive prefix sum of the per-expert
 *   assignment counts (offsets[0] == 0, offsets[E] == T*topk).
 * wq, scales: HOST arrays of E device pointers, each laid out as for
 *   qgemm_dense with the same N and K.
 * y: fp32 [T*topk][N], in assignment (token-slot) order.
 * Sizes: 1 <= E <= 4096, 1 <= topk <= E, T*topk < 2^31, T*K < 2^31.
 * The call buckets the assignments by expert into a library-owned workspace
 * (grown on first use, then reused; freed by qgemm_release) and runs the
 * grouped GEMM. Routing tables that disagree with each other are a caller
 * error: every access stays in bounds, and the rows of y that depend on the
 * inconsistent expert are written as NaN. With the environment variable
 * QGEMM_VALIDATE=1 the call synchronises `stream` and returns QGEMM_EINVAL
 * in that case.
 * Calls that share the workspace are ordered only by their streams: do not
 * run two qgemm_moe calls concurrently on different streams.
 */
int qgemm_moe(const void* x, const int32_t* token_expert_idx,
              const int32_t* expert_offsets, const void* const* wq,
              const void* const* scales, float* y, int T, int E, int topk,
              int N, int K, int fmt, hipStream_t stream);

/*
 * qgemm_moe for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): the
 * same arguments, results bitwise equal to qgemm_moe, and no hipMalloc, hipFree
 * or other allocation on any call. The bucketing buffers (permutation,
 * per-block expert histograms, error flag) live in a static device array of
 * 2 MiB + 256 bytes that each device holds until the process ends; the first
 * call on a device looks up its address there. Limits: T*topk <= 262144 and
 * ceil-blocks(T*topk) * E <= 262144 (the bucketing uses blocks of 512 slots,
 * at most 1024 blocks); larger problems return QGEMM_EUNSUPPORTED before
 * anything is enqueued. Every call on a device shares that device's array and
 * leaves its contents behind: calls that can overlap on one device (other
 * streams, other host threads) race and must be ordered by the caller.
 * QGEMM_VALIDATE is not consulted (the call never synchronises); inconsistent
 * routing tables still give NaN rows as for qgemm_moe.
 */
int qgemm_moe_noalloc(const void* x, const int32_t* token_expert_idx,
                      const int32_t* expert_offsets, const void* const* wq,
                      const void* const* scales, float* y, int T, int E, int topk,
                      int N, int K, int fmt, hipStream_t stream);

/*
 * The two halves of qgemm_moe, for callers that keep their own bucketing
 * buffer (the MoE expert GEMM of Section 3.1 needs each expert's routed
 * token list).
 * qgemm_moe_bucket: perm: int32 [n_assign], caller-owned. Writes the
 *   assignments grouped by expert: perm[expert_offsets[e] + r] is the r-th
 *   assignment (in increasing order) routed to expert e. Stable and
 *   deterministic. Entries for an expert whose count disagrees with
 *   expert_offsets are written as -1.
 * qgemm_moe_grouped: same arguments as qgemm_moe with perm in place of
 *   token_expert_idx; perm entries outside [0, T*topk) are skipped.
 */
int qgemm_moe_bucket(const int32_t* token_expert_idx, const int32_t* expert_offsets,
                     int32_t* perm, int n_assign, int E, hipStream_t stream);
int qgemm_moe_grouped(const void* x, const int32_t* perm, const int32_t* expert_offsets,
                      const void* const* wq, const void* const* scales, float* y,
                      int T, int E, int topk, int N, int K, int fmt, hipStream_t stream);

/*
 * Fused MoE gate/up projection with the SiLU-gated activation in its epilogue
 * (Section 3.1, fused gate/up item): for every assignment a routed to expert e
 * (perm and expert_offsets as for qgemm_moe_grouped) and i < inter,
 *   g = (dequant(wq[e], scales[e]) . x[a / topk])[i]
 *   u = (dequant(wq[e], scales[e]) . x[a / topk])[inter + i]
 *   h[a][i] = bf16_rne(silu(g) * u)
 * with g and u the same fp32 values qgemm_moe_grouped writes to y[a][i] and
 * y[a][inter + i], and silu evaluated as in qgemm_swiglu, so h equals
 * qgemm_swiglu applied to qgemm_moe_grouped's output bit for bit; the fp32
 * [T*topk][2*inter] intermediate is never stored.
 * wq[e], scales[e]: the gate rows (0 .. inter-1) and then the up rows
 * (inter .. 2*inter-1) of one [2*inter][K] matrix per expert, laid out as for
 * qgemm_dense with N = 2*inter; each matrix spans less than 4 GiB.
 * h: bf16 [T*topk][inter] in assignment order; rows of assignments absent
 * from perm are not written.
 * Sizes as for qgemm_moe with N = 2*inter, inter >= 1.
 */
int qgemm_moe_gate_up_swiglu(const void* x, const int32_t* perm, const int32_t* expert_offsets,
                             const void* const* wq, const void* const* scales, void* h,
                             int T, int E, int topk, int inter, int K, int fmt,
                             hipStream_t stream);

/*
 * MoE down projection with the router-weighted combine fused into it (the
 * MoE expert GEMM of Section 3.1 over the SiLU-gated activations, followed by
 * the weighted sum of each token's selected experts):
 *   y2[a][:] = dequant(wq[e], scales[e]) . h[a][:]        (a routed to expert e)
 *   out[t][n] = sum_{j < topk} route_w[t*topk + j] * y2[t*topk + j][n]
 * h: bf16 [T*topk][K], one row per token slot (as qgemm_moe_gate_up_swiglu
 * writes it); perm, expert_offsets: as for qgemm_moe_grouped over the T*topk
 * slots; wq, scales: HOST arrays of E device pointers, each [N][K] as for
 * qgemm_dense; route_w: fp32 [T*topk]; y2: fp32 [T*topk][N], caller-owned,
 * written with exactly the values qgemm_moe_grouped(h, perm, ..., topk = 1)
 * writes; out: fp32 [T][N], bitwise equal to qgemm_moe_combine(y2, route_w)
 * (each sum runs in increasing j from zero with fp32 fused multiply-adds).
 * The tile that stores the last of a token's topk slot rows for a column tile
 * sums them there, so the separate combine pass over y2 disappears; results
 * do not depend on which tile that is. Arrival counters live in a
 * library-owned workspace (grown on first use, freed by qgemm_release) and
 * are cleared by a kernel at the start of every call; calls that share it are
 * ordered only by their streams.
 * Sizes: as for qgemm_moe_grouped with T*topk rows; N % 4 == 0; y2 spans less
 * than 4 GiB (T*topk*N*4 bytes, else QGEMM_EUNSUPPORTED). Tokens whose slots
 * are not all present in perm (inconsistent routing tables) are not written.
 */
int qgemm_moe_down_combine(const void* h, const int32_t* perm, const int32_t* expert_offsets,
                           const void* const* wq, const void* const* scales, const float* route_w,
                           float* y2, float* out, int T, int E, int topk, int N, int K, int fmt,
                           hipStream_t stream);

/*
 * SiLU-gated activation between the MoE projections (Section 3.1, fused
 * gate/up item): for r < rows, i < inter,
 *   h[r][i] = bf16_rne(silu(y1[r][i]) * y1[r][inter + i]),  silu(z) = z / (1 + e^-z)
 * evaluated in fp32 with the hardware exponential and reciprocal (about one
 * fp32 ulp each, below the bf16 rounding of h).
 * y1: fp32 [rows][2*inter]; h: bf16 [rows][inter]. inter % 8 == 0.
 */
int qgemm_swiglu(const float* y1, void* h, int rows, int inter, hipStream_t stream);

/*
 * Router-weighted combine of the selected experts' outputs:
 *   out[t][n] = sum_{j < topk} route_w[t*topk + j] * y2[t*topk + j][n]
 * summed in increasing j in fp32. y2: fp32 [T*topk][N]; route_w: fp32
 * [T*topk]; out: fp32 [T][N]. N % 4 == 0.
 */
int qgemm_moe_combine(const float* y2, const float* route_w, float* out,
                      int T, int topk, int N, hipStream_t stream);

/* Message of the last non-OK return on the calling thread ("" if none). */
const char* qgemm_last_error(void);

/*
 * Prefill attention (Section 3.1, prefill attention item): softmax attention of a prompt's
 * queries over its keys, with the score product and the output product on the matrix cores and
 * an exact online softmax (running row maximum) between them. For every batch entry b, query
 * head h and query position i:
 *   s_j = scale * (q[b][i][h] . k[b][j][g]),  g = h / (H / Hkv)   (grouped-query attention)
 *   o[b][i][h] = sum_j softmax(s)_j v[b][j][g]
 * over the keys j <= i (causal = 1: prefill from an empty cache) or all keys j < S (causal = 0).
 * q, o: bf16 [B][S][H][D]; k, v: bf16 [B][S][Hkv][D]; every tensor contiguous, token-major,
 * 16-byte aligned; caller-owned device memory. D is 64 or 128; H a multiple of Hkv;
 * S*H*D < 2^31. Accumulation is fp32; the softmax weights enter the output product as bf16
 * and o is rounded to bf16 (nearest even). scale > 0 (1/sqrt(D) for the usual models).
 * Returns QGEMM_EINVAL / QGEMM_EUNSUPPORTED / QGEMM_EALIGN before launching anything (o is
 * untouched) and QGEMM_EHIP if the launch fails; B == 0 or S == 0 is a no-op.
 */
int qgemm_attention_prefill(const void* q, const void* k, const void* v, void* o,
                            int B, int S, int H, int Hkv, int D,
                            float scale, int causal, hipStream_t stream);

/*
 * Serving: what stands between the QKV and the output projection of a step over
 * a ragged batch (decode, Section 2.3, and prompts of different lengths).
 *
 *   qgemm_kv_plan -> QKV projection -> qgemm_rope -> qgemm_kv4_store ->
 *   qgemm_attention_packed (prompts) / qgemm_attention_kv4 (over the cache)
 *
 * The step's T rows hold the new tokens of R requests end to end, request r in
 * rows cu_q[r] .. cu_q[r+1]-1. Row strides are in elements; the heads of a row
 * are contiguous, so query, key and value heads can be views of one projection
 * row. Rows at or past cu_q[R] belong to no request and are left as they are.
 * Tables live in device memory and the host does not read them: tables that
 * contradict each other or the sizes are a caller error, every access stays in
 * bounds, and each entry point says what it makes of them.
 *
 * The 4-bit cache: uint8 [pages][Hkv][page*(D + D/16)], page a power of two in
 * [16, 1024], D 64 or 128. The record of one page and head holds the key codes
 * [page][D/2], the value codes [page][D/2], the key scales [page][D/32] and the
 * value scales [page][D/32] (microscaled 4-bit floating point): a code is an
 * e2m1 number (bit 3 the sign; 0, 0.5, 1, 1.5, 2, 3, 4, 6), element 2j in the
 * low nibble of byte j; a scale byte E stands for 2^(E-127), 255 for NaN.
 * Token p of a request is at slot block_table[r][p / page] * page + p % page.
 */

/*
 * Block tables, slots and positions of a step, from the requests' lengths, in one
 * launch. For request r with kv_len[r] tokens in the cache and q_len[r] new
 * ones (negative lengths count as 0; sums below 2^31):
 *   have = ceil(kv_len / page), need = ceil((kv_len + q_len) / page)
 *   block_table[r][j] = free_pages[f + j - have] for have <= j < need,
 *     f the sum of (need - have) over the requests before r; entries below
 *     have are read, those from need on left as they are
 *   cu_q[r] = sum of q_len before r; total_len[r] = kv_len[r] + q_len[r]
 *   the row t = cu_q[r] + i of new token i: positions[t] = kv_len[r] + i,
 *     slots[t] = its slot
 *   used[0] = sum of (need - have); rows at or past cu_q[R]: position 0, slot -1
 * kv_len, q_len, total_len: int32 [R]; block_table: int32 [R][W]; free_pages:
 * int32 [F]; cu_q: int32 [R+1]; positions, slots: int32 [T]; used: int32 [1].
 * No array that is written (block_table too) may share memory with another: a total_len that is the next
 * step's kv_len needs a second one to be written there (QGEMM_EINVAL otherwise). Where the free list ends (used[0] > F)
 * table entries become -1; such a token, one past W pages, one of a negative
 * table entry and one whose slot is 2^31 or more have slot -1. Tokens past T are
 * not planned (nor the pages that begin with them). R <= 4096.
 */
int qgemm_kv_plan(const int32_t* kv_len, const int32_t* q_len, int32_t* block_table,
                  const int32_t* free_pages, int32_t* cu_q, int32_t* positions, int32_t* slots,
                  int32_t* total_len, int32_t* used, int R, int W, int F, int page, int T,
                  hipStream_t stream);

/*
 * Frequencies of qgemm_rope for rot dimensions (host only, no launch):
 *   f_i = base^(-2i / rot), 0 <= i < rot/2, then by `scaling`
 *   PLAIN: f_i.   LINEAR: f_i / factor.
 *   LLAMA3, YARN: w f_i + (1 - w) f_i / factor, clamped to 0 <= w <= 1, with
 *     LLAMA3: w = (length f_i / 2 pi - low) / (high - low): turns over the
 *       original context, from `low` (divided) to `high` (kept);
 *     YARN: w = 1 - (i - from) / (to - from), from = max(floor d(high), 0),
 *       to = min(ceil d(low), rot - 1), d(t) = rot ln(length / 2 pi t) / 2 ln base
 *       (to - from taken as 0.001 if not positive).
 * inv_freq: HOST double [rot/2]; gain: HOST, the factor of the sine and cosine,
 * 0.1 ln(factor) + 1 for YARN and 1 otherwise. rot even, at most 512; base > 1;
 * factor >= 1; LLAMA3 and YARN: 0 < low < high and length > 0 (what a scaling
 * does not use is ignored).
 */
int qgemm_rope_frequencies(double* inv_freq, float* gain, int rot, double base, int scaling,
                           double factor, double low, double high, double length);

/*
 * Rotary positions on rows of heads, and their conversion to bf16:
 *   for the first rot_heads heads and the pairs (a, b) of a head's first rot
 *   elements, pair i at (i, i + rot/2) or, interleaved = 1, at (2i, 2i + 1), with
 *   the angle positions[t] * inv_freq[i]:
 *     a' = gain (a cos - b sin),  b' = gain (a sin + b cos)
 *   every other element is only rounded.
 * So one call takes whole QKV rows, with rot_heads = query and key heads.
 * x: fp32 (as qgemm_dense writes it) or bf16 [T][heads][D] at x_stride elements
 * between rows, x_type QGEMM_F32 or QGEMM_BF16; y: bf16 at y_stride; bf16 x may
 * be y itself at the same stride, and may not overlap it otherwise. positions:
 * int32 [T]; inv_freq: double [rot/2] in device memory. The angle's turns are
 * taken in fp64 and its sine, cosine and the rotation in fp32; bf16 rounding to
 * nearest even. D and rot even, rot <= min(D, 512); any stride >= heads*D and
 * addresses aligned to the elements (16 elements are moved at once where D, rot,
 * strides and addresses are multiples of 16 elements or bytes, else two).
 */
int qgemm_rope(const void* x, int x_type, const int32_t* positions, const double* inv_freq, void* y,
               int T, int heads, int rot_heads, int D, int rot, int64_t x_stride, int64_t y_stride,
               int interleaved, float gain, hipStream_t stream);

/*
 * Keys and values of T tokens into the 4-bit cache. k, v: bf16 [T][Hkv][D] at
 * k_stride / v_stride elements between rows (multiples of 8); slots: int32 [T],
 * tokens whose slot is outside [0, pages*page) are skipped; two tokens of one
 * slot leave it unspecified. For each block of 32 elements of a head:
 *   E = floor(log2(largest magnitude, rounded to two significant bits, ties up)) - 2,
 *     between -126 and 125; codes = x / 2^E to the nearest level, ties to the even code
 * (so a block's largest magnitudes are at most half a level step off, 7 going to
 * 8 and not to 6; from 1.75 * 2^127 on all are held as 6 * 2^125). A block with an infinity or NaN is held as NaN.
 */
int qgemm_kv4_store(const void* k, const void* v, const int32_t* slots, void* cache, int T, int Hkv,
                    int D, int64_t k_stride, int64_t v_stride, int pages, int page,
                    hipStream_t stream);

/*
 * The cache's keys and values of T slots, as the bf16 numbers they stand for
 * (exact but below bf16's range): k, v: bf16 [T][Hkv][D], dense. Rows whose slot is outside
 * [0, pages*page) are left as they are.
 */
int qgemm_kv4_load(const void* cache, const int32_t* slots, void* k, void* v, int T, int Hkv, int D,
                   int pages, int page, hipStream_t stream);

/*
 * Prefill attention over prompts of different lengths packed end to end, each
 * causal in itself: as qgemm_attention_prefill for every prompt, row t of
 * prompt r (rows cu[r] .. cu[r+1]-1) over the keys cu[r] .. t.
 * q, o: bf16 [T][H][D]; k, v: bf16 [T][Hkv][D], at their strides (elements,
 * multiples of 8); cu: int32 [R+1], ascending, cu[0] == 0, cu[R] <= T; prompts
 * of no rows may stand among them. Rows at or past cu[R] are not written, and
 * what they hold changes nothing, but q is loaded for all T rows. A prompt's rows depend on no other prompt, whatever that holds
 * (infinities and NaN included), nor on later rows. D is 64 or 128; T*H*D < 2^31;
 * q, k and v each span less than 4 GiB. Precision as qgemm_attention_prefill.
 * A cu that does not ascend gives unspecified rows.
 */
int qgemm_attention_packed(const void* q, const void* k, const void* v, const int32_t* cu, void* o,
                           int T, int R, int H, int Hkv, int D, int64_t q_stride, int64_t k_stride,
                           int64_t v_stride, int64_t o_stride, float scale, hipStream_t stream);

/*
 * Attention of new tokens over the 4-bit cache (their own keys and values stored
 * there before): single tokens, drafted tokens, the chunk of a long prompt. With
 * n = cu_q[r+1] - cu_q[r] new tokens (1 for every request if cu_q is null; then
 * T == R) and kv_len[r] keys in all, new token i is at position
 * p = kv_len[r] - n + i and sees the keys 0 .. p:
 *   o[cu_q[r] + i][h] = sum_j softmax_j(scale q . k_j[g]) v_j[g],  g = h / (H / Hkv)
 * A row that sees no key (p < 0) gives 0, one whose scores are all -inf NaN.
 * q: bf16 [T][H][D] at q_stride elements between rows (a multiple of 8); o: bf16
 * [T][H][D], dense; cache, block_table as above, kv_len: int32 [R]; cu_q: int32
 * [R+1], ascending, or null. fp32 scores, sums and accumulation; the softmax
 * weights enter the output product as bf16 (and the sum that divides it with that
 * rounding, but without it in the tiles of 128 rows that chunks of prompts take). Keys of a page outside [0, pages) or
 * past the table's W entries make the rows that see them NaN, and a value block of scale
 * byte 253 or 254, which passes bf16's range, counts as one of NaN; nothing else that
 * the pages hold behind a row's position reaches it. How the work was split shows in the
 * order of the fp32 sums, and in the weights' rounding to bf16, which is relative to a maximum
 * of the keys that came before; results are the same on every call.
 * workspace: caller-owned device memory, 16-byte aligned, of the bytes that
 * qgemm_attention_kv4_workspace gives for the same sizes; it needs no
 * initialisation, and calls that can overlap need one each. W*page <= 2^30,
 * T*H*D < 2^31, R <= 2^20, (T*H/Hkv/16 + R) * Hkv * (W*page/128 + 2) < 2^31. R == 0 or T == 0 is a no-op.
 * A cu_q that does not ascend gives unspecified rows.
 */
int qgemm_attention_kv4(const void* q, const void* cache, const int32_t* block_table,
                        const int32_t* kv_len, const int32_t* cu_q, void* o, void* workspace,
                        int64_t workspace_bytes, int T, int R, int H, int Hkv, int D, int W, int pages,
                        int page, int64_t q_stride, float scale, hipStream_t stream);
int qgemm_attention_kv4_workspace(int T, int R, int H, int Hkv, int D, int W, int page, int64_t* bytes);

/*
 * Many continuations and many tenants: a step of beam search, or of a batch whose requests share a prompt or have
 * adapters of their own.
 *
 *   projections + qgemm_adapters -> ... -> qgemm_attention_kv4_shared -> ... -> logits -> qgemm_beam_select ->
 *   qgemm_kv_reorder -> qgemm_kv4_copy (each layer's cache) -> the next step's qgemm_kv_plan
 */

/*
 * qgemm_attention_kv4 for requests that share their first keys: the same result but for rounding, with the shared keys read
 * and unpacked once for all rows of a group (decode, Section 2.3, is bound by those bytes). As there the softmax weights
 * enter the output product as bf16, rounded relative to a maximum that the split of the work decides, so the two differ
 * by that too: by 0.2 to 0.3% of o's norm where the split differs, each 0.20 to 0.23% from the exact result (0.17 of it
 * the rounding of o), over random keys of some thousand.
 * Group g holds the requests groups[g] .. groups[g+1]-1, whose first prefix_len[g] keys are the same: the keys that are
 * taken as shared are read through the table of the group's first request that has new tokens, the others through each
 * request's own. Shared are min(prefix_len[g], the fewest keys that a request of the group has before its new tokens), down
 * to a multiple of 64; a prefix_len of 0 or less, or one past the table, asks for none, or for no more than the table
 * has. Requests before groups[0] or from groups[G] on share nothing.
 * groups: int32 [G+1], ascending; prefix_len: int32 [G]; the other arguments as qgemm_attention_kv4, o unaliased.
 * Rows behind the last request are left as they are. Keys of a page outside [0, pages) or past the table make the rows
 * that see them NaN, shared ones those of the whole group. groups or a cu_q that do not ascend leave o unspecified.
 * Where the tables agree, qgemm_attention_kv4 gives the same rows: it is faster for a few requests over short prefixes (4
 * beams over 1000 keys 10.9 us against 12.6; 64 requests behind 7919 keys 78.2 against 34.8).
 * Results are the same on every call. workspace as there, of qgemm_attention_kv4_shared_workspace's bytes.
 * R and G <= 2048; else the limits of qgemm_attention_kv4, with the larger of R and G in the last.
 */
int qgemm_attention_kv4_shared(const void* q, const void* cache, const int32_t* block_table,
                               const int32_t* kv_len, const int32_t* cu_q, const int32_t* groups,
                               const int32_t* prefix_len, void* o, void* workspace, int64_t workspace_bytes,
                               int T, int R, int G, int H, int Hkv, int D, int W, int pages, int page,
                               int64_t q_stride, float scale, hipStream_t stream);
int qgemm_attention_kv4_shared_workspace(int T, int R, int G, int H, int Hkv, int D, int W, int page,
                                         int64_t* bytes);

/*
 * The K best continuations of every request's B beams: of the candidates (beam b, token v), worth
 *   scores[r][b] + x[v] - log sum_u exp x[u],  x the row r*B + b of logits,
 * the K of largest value, in descending order:
 *   out_scores[r][k] its value, out_parents[r][k] = b, out_tokens[r][k] = v
 * Of a beam the larger logit comes first, of equal ones the lower token, also where a large score hides the difference from the
 * value; beams are compared by their candidates' values in fp64, equal ones the lower beam first.
 * A beam with finished[r][b] != 0 has one candidate, the token `end` at its own score; its logits do not matter. No
 * candidates are those worth -inf or NaN: all of a beam whose score is (a beam that is not there: before the first
 * selection all but one of a prompt's), tokens of logit -inf, and all of a row that holds NaN or +inf. Behind the last
 * candidate stand score -inf, parent -1 and token `end`. So finished is (out_tokens == end) for the next selection.
 * logits: fp32 (as qgemm_dense writes them) or bf16 [R*B][V] at `stride` elements between rows, aligned to their
 * elements; scores: fp32 [R][B]; finished: uint8 [R][B] or null; outputs [R][K], which share no memory with an input or each other. A row's
 * exponentials are taken in fp32 and added in fp64, values are fp64, rounded once: candidates of different beams may change
 * places where their values are closer than 1e-6 (sums of 1000 to 128000 logits are off by up to 2e-7 of themselves).
 * Results are the same on every call.
 * B <= 64, K <= 128 (of more than one beam K = B continues as many, K = 2B leaves a choice; the time of many beams with
 * many candidates goes with the square of B*K: 1.8 ms for 64 beams and K = 128), R*B <= 2^20, V <= 2^30. workspace: caller-owned, 16-byte aligned,
 * of the bytes that qgemm_beam_select_workspace gives, without initialisation; calls that can overlap need one each.
 */
int qgemm_beam_select(const void* logits, int type, const float* scores, const uint8_t* finished,
                      float* out_scores, int32_t* out_parents, int32_t* out_tokens, void* workspace,
                      int64_t workspace_bytes, int R, int B, int V, int K, int64_t stride, int end,
                      hipStream_t stream);
int qgemm_beam_select_workspace(int R, int B, int V, int K, int64_t* bytes);

/*
 * Block tables of the beams after a selection. Rows come in requests of B; row k of a request continues its old row
 * p = parents[r*B + k] in [0, B), and with any other parent nothing: it then has no tokens. With have = ceil(kv_len[p] / page):
 *   new_len = kv_len[p]; new_table[j] = block_table[p][j] for j < have, -1 from there on
 * A last page that is filled only in part is written by the next token, so one row alone may hold it: the first row (the lowest k)
 * of a parent has it, and the others a page each of free_pages, by request and k, with its number in dst and the
 * parent's in src (both -1 for all other rows): qgemm_kv4_copy brings the keys and values over. used[0]: pages taken; where
 * the free list ends (used[0] > F) entries become -1, with nothing to copy. (A parent whose own last entry is none, as
 * such a row's, has nothing to give: the other children's pages hold what they held.)
 * released: the pages that no new row of their request holds in the column that they had, each once, by request,
 * column and old row; -1 behind them. n_released[0] counts them; with more than Q those past Q are missing from the
 * list. Not listed: the first keep[r] columns (pages of a prompt that others hold too; keep may be null: none), and
 * negative entries.
 * block_table, new_table: int32 [R*B][W]; kv_len (negative counts as 0), parents, new_len, src, dst: int32 [R*B];
 * free_pages: int32 [F]; keep: int32 [R]; used, n_released: int32 [1]; released: int32 [Q]. Nothing that is written may share
 * memory with another array: a loop keeps two tables that take turns. B <= 64, R*B <= 65536, R*B*W < 2^31. R == 0 is a no-op.
 * workspace: caller-owned, 4-byte aligned, of qgemm_kv_reorder_workspace's bytes, without initialisation.
 */
int qgemm_kv_reorder(const int32_t* block_table, const int32_t* kv_len, const int32_t* parents,
                     const int32_t* free_pages, const int32_t* keep, int32_t* new_table, int32_t* new_len,
                     int32_t* src, int32_t* dst, int32_t* used, int32_t* released, int32_t* n_released,
                     void* workspace, int64_t workspace_bytes, int R, int B, int W, int F, int Q, int page,
                     hipStream_t stream);
int qgemm_kv_reorder_workspace(int R, int B, int W, int64_t* bytes);

/*
 * Whole pages within a 4-bit cache: page src[i] (all heads) to page dst[i] for i < n. Pairs with a page outside
 * [0, pages) are skipped. No page may be a dst twice, nor a dst of one pair and the src of another (what such pages hold
 * afterwards is unspecified). src, dst: int32 [n].
 */
int qgemm_kv4_copy(void* cache, const int32_t* src, const int32_t* dst, int n, int Hkv, int D, int pages,
                   int page, hipStream_t stream);

/*
 * Low-rank adapters of many requests on top of a shared projection's output (qgemm_dense of the same x):
 *   y[m][c] += gain[i] sum_{j < r} b[i][c][j] (sum_k a[i][j][k] x[m][k]),  i = ids[request of row m]
 * The rows cu_q[q] .. cu_q[q+1]-1 are request q's (cu_q ascending; null: M == R, row q is request q's). Rows of no
 * request, and of one whose id is outside [0, n), are neither read into a result nor written.
 * x: bf16 [M][K] at x_stride elements between rows (a multiple of 8); a: bf16 [n][r][K]; b: bf16 [n][N][r]; ids: int32 [R];
 * gain: fp32 [n] or null (1); y: fp32 [M][N] at y_stride elements, so that the columns of one projection within a wider
 * row can be given. y is read and written (the one output here that is added to), and shares no memory with an input.
 * K and r multiples of 8 (an adapter of lower rank has zeros behind it), r <= 128, M <= 2^25, N, K and R <= 2^28. fp32
 * accumulation; the inner sums, times gain, enter the second product as three bf16 numbers each, which hold them whole (of
 * those below 2^-110 in size what is below 2^-133 is lost). An infinite weight or sum gives the formula's infinity or NaN
 * (an infinite b with an inner sum that is not 0 but below 2^-90 in size may give NaN too). What one adapter or request
 * holds (infinities and NaN included) reaches no other's rows. Results are the same on every call.
 * Rows of an adapter that stand next to each other share the reading of its weights.
 * workspace: caller-owned, 16-byte aligned, of qgemm_adapters_workspace's bytes, without initialisation; calls that can
 * overlap need one each.
 */
int qgemm_adapters(const void* x, const void* a, const void* b, const int32_t* ids, const int32_t* cu_q,
                   const float* gain, float* y, void* workspace, int64_t workspace_bytes, int M, int N, int K,
                   int r, int n, int R, int64_t x_stride, int64_t y_stride, hipStream_t stream);
int qgemm_adapters_workspace(int M, int N, int K, int r, int64_t* bytes);

/*
 * Measurement utility, not part of the GEMM path: runs `iters` rounds of four
 * independent bf16 MFMAs (the GEMM's v_mfma_f32_32x32x16_bf16) in eight waves on
 * every CU at once, synchronises `stream`, and returns through HOST pointers
 * the median shader clock the CUs held (MHz; cycle counter over the device's
 * constant-rate real-time counter) and the bf16 dense matrix throughput the
 * launch reached (TFLOP/s, from HIP events on `stream`): the practical matrix-core
 * ceiling at the sustained clock, beside the nominal 2.4 GHz peak. Allocates and
 * frees its own small buffers. QGEMM_EINVAL for iters < 1 or null outputs.
 */
int qgemm_probe_mfma_clock(int iters, double* sclk_mhz, double* mfma_tflops, hipStream_t stream);

/* Frees the library-owned workspaces (MoE bucketing, split-K partials); the
 * next call that needs one grows it again. The caller must have synchronised
 * every stream that used them. */
int qgemm_release(void);

/* Library ABI version, (major << 16) | minor. */
int qgemm_version(void);

#ifdef __cplusplus
}
#endif

#endif /* QGEMM_H */
