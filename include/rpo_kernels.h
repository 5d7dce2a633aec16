/*
 * rpo_kernels.h -- building-block entry points of librpo, exported so that the
 * dense contraction can be checked on its own and so that tests can run the whole
 * path through the generic (vector-ALU) kernels as a cross-check of the MFMA ones.
 * Same conventions as rpo.h (caller-owned device buffers, stream as void*, int
 * error codes, rpo_last_error()).
 */
#ifndef RPO_KERNELS_H
#define RPO_KERNELS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* C[M,N] (op)= A[M,K] * W[N,K]^T with fp32 accumulation: the projection y = x W^T
 * used by every linear layer of the decoder (QKV, O, gate/up, down, LM head).
 *   a_dev  device, [M, K] row-major, row stride lda (elements), dtype RPO_F32 / RPO_BF16
 *   w_dev  device, [N, K] row-major, row stride ldw, same dtype
 *   c_dev  device, [M, N] row-major, row stride ldc
 *   epilogue 0: C = result in `dtype`; 1: C = result as fp32; 2: C (fp32) += result;
 *            3: SwiGLU: W rows are [gate (F rows); up (F rows)], N = 2F, and
 *               C[M, F] = silu(A Wgate^T) * (A Wup^T) in `dtype` (ldc >= F)
 *   ws_dev   device scratch for K-split partial sums, ws_bytes long, or NULL / 0: skinny
 *            problems are then not split along K (same result, fewer busy CUs)
 * bf16 operands with K, lda, ldw multiples of 8 and 16-byte aligned bases run on the
 * matrix cores (SwiGLU also needs F a multiple of 32); anything else on the generic
 * kernel.  Errors: RPO_EINVAL, RPO_EHIP. */
int rpo_gemm_nt(const void *a_dev, int64_t lda, const void *w_dev, int64_t ldw, void *c_dev, int64_t ldc,
                int32_t M, int32_t N, int32_t K, int32_t dtype, int32_t epilogue, void *ws_dev,
                size_t ws_bytes, void *stream);

/* What rpo_gemm_nt would launch for dense, aligned operands of these sizes and ws_bytes of scratch (0: none), or a model
 * whose projections and LM head are turn_bytes long (0: a call by itself), so that tests can check the choice; runs on
 * the host alone.  plan_out, 6 values: the kernel id (as rpo_profile_start's), the K ranges whose sums go through the
 * scratch (1: K is not split), the rows of the first of two launches (0: one launch), 1 where the generic kernel deals K
 * to the lanes of a wave (0: it works in tiles), 1 where the weights count as coming from HBM, 1 where an RMSNorm between
 * an accumulating (epilogue 2) and a SwiGLU (3) projection would be taken apart as far as this one is concerned.
 * Errors: RPO_EINVAL. */
int rpo_gemm_plan(int32_t M, int32_t N, int32_t K, int32_t dtype, int32_t epilogue, size_t ws_bytes, size_t turn_bytes,
                  int32_t *plan_out);

/* The shared-prefix decode attention of ONE layer on its own (the kernel rpo_decode_step runs
 * between the QKV and the output projection), so that it can be checked against a plain
 * softmax(q K^T / sqrt(dh)) V and profiled alone.  For rollout rows [0, n_rows) of a forked batch:
 * one query row per rollout attends to [the group's shared prefix pages || the rollout's private
 * pages], i.e. to positions [0, prefix_len(group) + n_suffix) of whatever keys / values the batch's
 * pages hold for `layer` (the prefix after rpo_prefill_prefix + rpo_kv_fork; private positions
 * that no decode step or log-prob pass has written hold zeros).
 *   q_dev      device, [n_rows, n_q_heads * head_dim], model dtype, already rotated
 *   n_suffix   private tokens each rollout sees, 0..max_suffix
 *   active_dev device uint8 [n_rows] or NULL; rows with 0 are skipped (their output row is untouched)
 *   out_dev    device, [n_rows, n_q_heads * head_dim], model dtype
 * Uses the batch's workspace (attention partials): not concurrently with other calls on the batch.
 * Errors: RPO_ESTATE unless forked; RPO_EINVAL. */
struct rpo_batch;
int rpo_attn_decode(struct rpo_batch *b, int32_t layer, const void *q_dev, int32_t n_rows, int32_t n_suffix,
                    const uint8_t *active_dev, void *out_dev, void *stream);

/* ---- a paged cache outside a batch ---------------------------------------------------------------
 * Keys and values of n_seqs sequences in pages of one layer: what a batch keeps, as building blocks for caches whose size is
 * bounded (a sliding window with sinks, or eviction by accumulated attention weight).
 * Page p of the pool starts p * page_stride elements in and holds, for every KV head, a key block [page_tokens][head_dim],
 * then for every KV head a value block [page_tokens / 8][head_dim][8] (eight tokens of a channel side by side).  The slots
 * [k * page_tokens, (k + 1) * page_tokens) of sequence s lie in page table_dev[s * table_stride + k]; slots are numbered from 0
 * without a gap, whatever positions the tokens had, and keys lie in the cache as they are multiplied (already rotated).
 *   pool_dev      device, 16-byte aligned; page_stride >= 2 * n_kv_heads * page_tokens * head_dim, a multiple of 8
 *   table_dev     device int32 [n_seqs, table_stride]; table_stride * page_tokens at most 2^30
 *   len_dev       device int32 [n_seqs]: slots in use.  What lies in other slots does not matter, NaN included
 *   n_seqs at most 65535; page_tokens a power of two, >= 16; head_dim even, <= 256; dtype RPO_F32 or RPO_BF16
 * What lies on the device cannot be checked on the host.  Every index from there is bounded by the kernels: a table entry
 * outside [0, n_pages) means that its tokens are not there (not visible, neither read nor written), a length beyond
 * table_stride * page_tokens is taken for that (by rpo_kv_append: as it is, the slots behind the table's end do not exist),
 * row ranges end with the row arrays.  Several sequences may share pages that are only read. */
typedef struct {
    void *pool_dev;
    const int32_t *table_dev;
    const int32_t *len_dev;
    int64_t page_stride;
    int32_t n_pages, n_seqs, table_stride, page_tokens, n_kv_heads, head_dim, dtype;
} rpo_paged_kv;

/* One layer of a forked batch as such a cache: its pool and the page tables of its n_groups * G rollouts, where position =
 * slot.  len_dev is left NULL for the caller to fill in (prefix_len + tokens appended per rollout).  The rollouts of a group
 * share their prefix pages: do not append below prefix_len.  Host only.  Errors: RPO_ESTATE unless forked; RPO_EINVAL. */
int rpo_batch_kv(const struct rpo_batch *b, int32_t layer, rpo_paged_kv *out);

/* The rows of a call (below): sequence s has rows cu_rows_dev[s] .. cu_rows_dev[s + 1] - 1 of the row arrays, any number from
 * 0 up to max_new (the longest, below 2^26; a host bound that sizes the launch: rows of a sequence beyond it are not looked
 * at).  They are the last tokens of its cache: with n rows, row i sits at slot len - n + i.  cu_rows_dev: device int32
 * [n_seqs + 1], not decreasing.  Rows of the arrays that belong to no sequence are left as they were.
 *
 * rpo_kv_append: write the rows' keys and values into their slots (len_dev counts them already).
 *   k_dev, v_dev  device, n_rows rows of n_kv_heads * head_dim values, k_stride / v_stride elements apart
 * Rows that would lie below slot 0 or beyond the table are dropped: a full cache stays as it is.  Errors: RPO_EINVAL, RPO_EHIP. */
int rpo_kv_append(const rpo_paged_kv *kv, const void *k_dev, int64_t k_stride, const void *v_dev, int64_t v_stride,
                  const int32_t *cu_rows_dev, int32_t n_rows, int32_t max_new, void *stream);

/* Attention of the rows over their sequences' caches, single tokens and whole chunks alike: query head h of a row at slot t
 * reads KV head h / (n_q_heads / n_kv_heads) and sees the slots j <= t, with a window only those of them with j < n_sinks or
 * j > t - window.  out = softmax(scale q k^T) v over what it sees; zeros where it sees nothing.
 *   q_dev       device, n_rows rows of n_q_heads * head_dim values (head h at column h * head_dim), q_stride elements apart
 *   max_len     no cache is longer (host; chooses how the work is split)
 *   window      0: all earlier slots; n_sinks counts only with a window
 *   out_dev     device, like q_dev with out_stride; must not overlap q_dev
 *   lse_out_dev device fp32 [n_rows, n_q_heads] or NULL: ln sum exp(scale q k^T), -infinity where nothing is seen
 *   ws_dev      device, 16-byte aligned, at least rpo_attn_paged_ws_bytes for the same arguments, or NULL / 0: the tokens of
 *               a sequence are then not split (few rows over long caches are slower).  Nothing in it needs clearing; calls
 *               that may run at the same time (captured graphs among them) need one each.
 * bf16 and fp32 with head_dim 32, 64 or 128 and rows that start at multiples of 16 bytes run on the matrix cores, anything
 * else on a generic kernel.  Sums and statistics are fp32; with bf16 the weights p are rounded to bf16 before they multiply
 * the values, as in the batch's attention, and those of a chunk are divided by their sum as rounded, so that equal values come
 * out as they are.  A NaN or infinity in a slot reaches the rows that see it (in a value: its channel of
 * theirs) and no others; rows that are computed together with such rows are computed once more, which takes longer.
 * On the matrix cores n_seqs * n_kv_heads times the pieces of 64 or 128 of max_new * n_q_heads / n_kv_heads columns must stay
 * below 2^24.  Errors: RPO_EINVAL, RPO_ENOMEM (ws_bytes), RPO_EHIP. */
size_t rpo_attn_paged_ws_bytes(const rpo_paged_kv *kv, int32_t n_rows, int32_t max_new, int32_t max_len, int32_t n_q_heads,
                               int32_t window, int32_t n_sinks);
int rpo_attn_paged(const rpo_paged_kv *kv, const void *q_dev, int64_t q_stride, const int32_t *cu_rows_dev, int32_t n_rows,
                   int32_t max_new, int32_t max_len, int32_t n_q_heads, float scale, int32_t window, int32_t n_sinks,
                   void *out_dev, int64_t out_stride, float *lse_out_dev, void *ws_dev, size_t ws_bytes, void *stream);

/* Attention weight that the cached tokens receive from the rows: for every slot j < len of every KV head
 *   score_out = score_in + sum over rows and the head's query heads that see j of exp(scale q k_j - lse)
 * lse_dev device fp32 [n_rows, n_q_heads]: what rpo_attn_paged left for the same rows (a row with -infinity gives nothing,
 * whatever its query holds).
 *   score_in_dev  device fp32 [n_seqs, n_kv_heads, score_stride] or NULL: zeros; score_out_dev the same layout, may be the
 *                 same array.  score_stride >= the longest cache (slots beyond it get no score); slots from len on are left
 *                 as they were.  The sums run in a fixed order: equal inputs give equal bits.
 *   ws_dev        as for rpo_attn_paged, rpo_kv_score_ws_bytes long
 * The other arguments as for rpo_attn_paged; slots from max_len on get no score.  n_seqs * n_kv_heads * max_len / 256 (fp32: 128)
 * must stay below 2^24.  Errors: RPO_EINVAL, RPO_ENOMEM, RPO_EHIP. */
size_t rpo_kv_score_ws_bytes(const rpo_paged_kv *kv, int32_t n_rows, int32_t max_new, int32_t max_len, int32_t n_q_heads,
                             int32_t window, int32_t n_sinks);
int rpo_kv_score(const rpo_paged_kv *kv, const void *q_dev, int64_t q_stride, const int32_t *cu_rows_dev, int32_t n_rows,
                 int32_t max_new, int32_t max_len, int32_t n_q_heads, float scale, int32_t window, int32_t n_sinks,
                 const float *lse_dev, const float *score_in_dev, float *score_out_dev, int64_t score_stride, void *ws_dev,
                 size_t ws_bytes, void *stream);

/* Evict what was attended to least: every sequence that holds more than `budget` tokens keeps, per KV head, its first
 * n_sinks and its last n_recent slots and of the others the budget - n_sinks - n_recent with the highest scores (ties: the
 * lower slot; NaN below every number).  What is kept goes, in order, to slots 0 .. of `dst`: other pages, so that pages
 * which other sequences share stay as they are.  A shorter sequence goes over whole.
 *   score_dev     device fp32 [n_seqs, n_kv_heads, score_stride], score_stride >= the longest cache (tokens beyond it are
 *                 not looked at)
 *   budget        >= 1, >= n_sinks + n_recent, at most what a row of dst's table holds and 2^30 - 64
 *   dst           same n_seqs, n_kv_heads, head_dim and dtype as src; its len_dev is not read and may be NULL; no page that
 *                 its tables name may be one that src's name.  Slots beyond the kept ones are left as they were
 *   len_out_dev   device int32 [n_seqs]: min(len, budget); may be src's or dst's len_dev
 *   score_out_dev device fp32 [n_seqs, n_kv_heads, score_out_stride] or NULL, score_out_stride >= budget, not score_dev: the
 *                 kept tokens' scores, 0 in the rest of the row
 *   kept_out_dev  device int32 [n_seqs, n_kv_heads, budget]: the old slot of every new one, -1 beyond the length
 * A kept token whose page is not there leaves its new slot as it was.  Errors: RPO_EINVAL, RPO_EHIP. */
int rpo_kv_evict(const rpo_paged_kv *src, const float *score_dev, int64_t score_stride, int32_t budget, int32_t n_sinks,
                 int32_t n_recent, const rpo_paged_kv *dst, int32_t *len_out_dev, float *score_out_dev,
                 int64_t score_out_stride, int32_t *kept_out_dev, void *stream);

/* rpo_gemm_nt for callers that cannot allocate or pass a workspace (code under HIP graph capture,
 * tight serving loops, harnesses that forbid hipMalloc): the same contraction, kernels and
 * results, with the K-split partial sums in a fixed 16 MiB device array that belongs to the
 * library (one copy per GPU, held until the process ends).  Allocates nothing, on the host or the
 * device; the first call on a GPU has the runtime load the kernels' code there, if no other call has
 * (a few MB), so that no later one does.  Arguments as rpo_gemm_nt.  A problem whose K split needs more than 16 MiB of partial
 * sums (splits * M * N * 4 bytes; only skinny problems with a deep K are split) is rejected with
 * RPO_ENOMEM and nothing is enqueued, unless it is a gate/up problem of more than 256 rows that the tiles
 * which never split hold in a few rounds, or a problem of more than 512 rows (epilogues 0 and 2) that 128x128 tiles hold
 * in one: those take it (rpo_gemm_nt with 16 MiB of workspace does the same).  All calls on one GPU share the array: calls that may run
 * concurrently on one GPU (different streams, different threads) race on it; calls on one
 * stream are safe.  Nothing in the array needs clearing between calls (every partial sum is
 * written before it is read).  Errors: RPO_EINVAL, RPO_ENOMEM, RPO_EHIP. */
int rpo_gemm_nt_noalloc(const void *a_dev, int64_t lda, const void *w_dev, int64_t ldw, void *c_dev, int64_t ldc,
                        int32_t M, int32_t N, int32_t K, int32_t dtype, int32_t epilogue, void *stream);

/* Practical ceilings of the GPU the library runs on, for roofline reports: the rate of a plain
 * device-to-device copy of `bytes` bytes (read + write counted, GB/s, best of three launches) and
 * of a back-to-back bf16 32x32x16 MFMA issue loop with changing operands (TFLOP/s, two workgroups
 * of four waves per CU, about 0.1 s, best of two).
 *   src_dev, dst_dev  device, `bytes` long each (a multiple of 16, at least 1 MiB), not overlapping
 *   scratch_dev       device, 512 * 256 floats, overwritten
 *   copy_gbps, mfma_tflops  host, results
 * Synchronises the stream.  Errors: RPO_EINVAL, RPO_EHIP. */
int rpo_probe_peaks(const void *src_dev, void *dst_dev, size_t bytes, float *scratch_dev, double *copy_gbps,
                    double *mfma_tflops, void *stream);

/* TEST AND TUNING SWITCH, process-wide: 0 = fastest available kernel for the shape (default, and
 * the only value a product run uses),
 * 1 = generic vector-ALU kernels for GEMM and attention regardless of shape (the tests run whole
 *     rollouts through them as a cross-check of the MFMA kernels),
 * 2 = MFMA GEMM with register-staged LDS fills instead of direct-to-LDS loads (the fallback
 *     used when K is not a multiple of 64; selectable so that the tests reach it at any K),
 * 16 + k (k = 1, 3..6, 11, 13, 14) = MFMA GEMM with the fixed tile shape of kernel id k, so that the tests
 *     can force every tile shape onto one problem (attention as in 0).
 * Unsynchronised: set it from the thread that issues the compute calls, between calls.
 * Errors: RPO_EINVAL. */
int rpo_set_kernel_path(int path);

/* Per-kernel timing for roofline reports.  rpo_profile_start(kernel_id, every) makes every
 * `every`-th later launch of that kernel (the 1st, the every+1-th, ...; process-wide, any stream)
 * bracketed by a pair of HIP events recorded on the launch stream; several kernel ids may be
 * timed at once.  rpo_profile_stop(kernel_id, ...) waits for that kernel's last event and returns
 * the number of bracketed launches, their summed event time in milliseconds, and their summed
 * ALGORITHMIC flops and bytes as the library counts them (GEMM: 2MNK flops, operands + result
 * bytes; decode attention: K/V bytes with a group's shared prefix counted once per group;
 * sampler: the logits rows read once).  Kernel ids:
 * (MFMA GEMM tile shapes <BM, BN, waves along M, waves along N>)
 *   1  <256,256,2,4> (prefill-sized problems, LM heads), every epilogue but SwiGLU; also the <128,256,2,4>
 *      tile of an LM head of 33 to 128 rows with its row maxima
 *   12 <256,256,2,4> with the fused SwiGLU epilogue: the gate/up projection of prefill and
 *      log-prob chunks, one instantiation, the heaviest kernel of a rollout step
 *   3  <128,128,2,2> (decode-sized problems with a deep K, gate/up of 65 to 128 rows, chunks of up to a few
 *      thousand rows)
 *   4  <64,128,1,2> (up to 64 rows, where kernel 15 does not take them)
 *   5  <32,128,1,4> / <64,128,1,4> / <128,128,2,2> (QKV projection of a decode step of more rows than kernel 15 takes,
 *      and of small chunks: rotary embedding and KV page write in the epilogue, the rows of a tile such that
 *      one round of workgroups holds them)
 *   6  <64,64,2,2> (decode-sized problems and small chunks with a shallow K, no K split)
 *      (all epilogues of a tile shape together; a K-split launch includes its reduction)
 *   11 <256,192,4,2> (large M with a narrow N: fewer idle CUs in the last round of workgroups)
 *   13 <256,160,4,1> (gate/up projection of a decode step, where one round holds its tiles, and of a small
 *      chunk, where it fills its rounds better)
 *   14 <128,160,4,1> (gate/up projection of a decode step, where one round holds its tiles)
 *   15 gemm_skinny_kernel (up to 64 rows, and narrow projections of up to 512 in groups of 64; every
 *      epilogue; a K-split launch includes its reduction)
 *   7  gemm_generic_wave_kernel / gemm_generic_kernel      8  attn_decode_mfma_kernel (+ merge)   9  attn_chunk_mfma_kernel
 *   10 sample_kernel
 * The timing state and rpo_set_kernel_path's switch are process-wide and unsynchronised: use them
 * from the one thread that issues the compute calls, and not while another thread is inside one.
 * Host-side only (event create / record / synchronise).
 * Errors: RPO_EINVAL (unknown id, every < 1, NULL), RPO_EHIP. */
int rpo_profile_start(int kernel_id, int every);
int rpo_profile_stop(int kernel_id, int64_t *n_launches, double *total_ms, double *total_flops,
                     double *total_bytes);

#ifdef __cplusplus
}
#endif
#endif /* RPO_KERNELS_H */
