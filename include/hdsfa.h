/*
 * hdsfa.h -- C ABI of libhdsfa.so: GB300 (sm_103a) kernels for Hidden Decoding's
 * multi-stream token expansion and Stream-Factorized Attention (SFA).
 *
 * Notation (0-indexed): a batch holds B sequences of L tokens; each token is
 * expanded into n streams, giving nL positions.  Token t, stream s sits at
 * position p = t*n + s (the paper's 1-indexed t = (i-1)n + k, Eq. 1).
 *
 * Conventions shared by every entry point
 *   - Ownership: the caller allocates and owns every buffer (device memory).
 *     The library never allocates, frees or synchronises; all work is enqueued
 *     asynchronously on `stream` (0 = legacy default stream).
 *   - Layout: dense row-major, no padding.  bf16 is IEEE bfloat16 (uint16 bits).
 *       tables  [n][V][D]        ids [B][L] int32      expanded [B][nL][D]
 *       q, o, dout, dq  [B][nL][Hq][Dh]      k, v, dk, dv  [B][nL][Hkv][Dh]
 *       lse [B][Hq][nL] float32, natural-log log-sum-exp of each softmax row.
 *   - Grouped K/V: query head h reads K/V head h / (Hq / Hkv).
 *   - Host-side argument errors return before anything is enqueued.
 *   - dev_status (nullable): a device int32 the kernels OR error bits into
 *     (HD_DEVBIT_*); the caller zeroes it, synchronises, then reads it.
 *     Kernels never trap.
 *   - Pointers must be 16-byte aligned; D and Dh must make rows a multiple of
 *     16 bytes.
 */
#ifndef HDSFA_H
#define HDSFA_H

#include <stddef.h>
#include <stdint.h>
#include <cuda_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  HD_OK = 0,
  HD_ERR_INVALID_ARG = 1, /* null / misaligned pointer, non-positive size, Hq % Hkv != 0 */
  HD_ERR_UNSUPPORTED = 2, /* valid but not implemented (e.g. Dh not in {64, 128, 256}) */
  HD_ERR_CUDA = 3,        /* a CUDA runtime/driver call or kernel launch failed */
  HD_ERR_WORKSPACE = 4,   /* workspace null or smaller than sfa_bwd_workspace_bytes() */
  HD_ERR_TIMEOUT = 5,     /* reserved: a bounded device wait expired (see HD_DEVBIT_TIMEOUT) */
  HD_ERR_INDEX = 6,       /* reserved: an index was out of range (see HD_DEVBIT_INDEX) */
  HD_ERR_SCRATCH_LIMIT = 7 /* sfa_bwd_noalloc: sizes need more than SFA_BWD_NOALLOC_MAX_BYTES */
} hd_status_t;

/* Bits the kernels OR into *dev_status. */
#define HD_DEVBIT_INDEX 1   /* a token id outside [0, V): hd_expand_embed zeroed its n output
                               rows; hd_expand_embed_bwd left it out of the sums.  A sequence
                               length outside its range in sfa_decode / sfa_kv_append; a length,
                               page, offset or sequence index outside its range in the paged
                               and packed calls below */
#define HD_DEVBIT_TIMEOUT 2 /* a bounded pipeline wait expired; outputs are invalid */
#define HD_DEVBIT_PAGES 4   /* no page was free for a sequence of hd_pages_grow or a fork of
                               hd_pages_fork: it was left as it was */

/* Attention mask of one SFA layer (Sec. 2.2, Eq. 4 and Fig. 2). */
typedef enum {
  SFA_WITHIN = 0, /* intra-stream: p' <= p and p' = p (mod n)                 (Eq. 4, Fig. 2c) */
  SFA_CROSS = 1,  /* full cross-stream: standard causal mask over nL, p' <= p (Fig. 2a)        */
  SFA_LOCAL = 2,  /* local cross-stream: causal window, p - window < p' <= p  (Fig. 2b)        */
  SFA_WITHIN_NAIVE = 3 /* measurement mode: the SFA_WITHIN result (same mask, same outputs)
                          computed over the full causal tile schedule of nL positions, with
                          the stream condition applied per pair instead of skipping the
                          other streams' tiles: n times the work, what the skipping saves.
                          sfa_fwd / sfa_bwd (and their parts) at Dh = 128 only.          */
} sfa_mode_t;

/*
 * hd_expand_embed -- multi-stream token expansion (Eq. 1, Sec. 2.1):
 *   out[b][t*n + s][:] = tables[s][ids[b][t]][:]   for t < L, s < n.
 * tables: bf16 [n][V][D] (read-only); ids: int32 [B][L]; out: bf16 [B][n*L][D].
 * An id outside [0, V) writes zero rows and sets HD_DEVBIT_INDEX.
 * Requires D % 8 == 0 (16-byte rows) and 16-byte aligned tables/out.
 * Bit-exact copy; HBM-bound.
 */
hd_status_t hd_expand_embed(const void* tables, const int32_t* ids, void* out, int B, int L, int n,
                            int V, int D, int32_t* dev_status, cudaStream_t stream);

/*
 * hd_expand_embed_bwd -- backward of the expansion (adjoint of Eq. 1, Sec. 2.1):
 *   dtables[s][v][:] += sum over (b, t) with ids[b][t] = v of dout[b][t*n + s][:]
 * for every s < n and every v in [0, V) that occurs in ids.
 *   dout: bf16 [B][n*L][D] (read-only); ids: int32 [B][L]; dtables: float32 [n][V][D],
 *   accumulated in place (rows of ids that do not occur are not touched; zero the
 *   tables first for a plain gradient).
 *   Deterministic: every element of dtables is read and written once, by one thread,
 *   which sums the occurrences of its id in fp32 in an order fixed by their number
 *   (ascending token order b*L + t; for ids with more than 32 occurrences, eight
 *   consecutive token blocks, each in ascending order, whose sums are added in
 *   block order) and adds the sum to dtables: repeated calls on the same inputs give
 *   identical bits.
 *   An id outside [0, V) contributes nothing and sets HD_DEVBIT_INDEX.
 *   workspace: device memory of at least hd_expand_embed_bwd_workspace_bytes(B, L)
 *   bytes, 16-byte aligned, overwritten (no contents need to survive between calls;
 *   the size is independent of n, V and D).
 *   Requires D % 8 == 0, B*L < 2^31, n*D < 2^31, 16-byte aligned dout/dtables;
 *   HBM-bound.
 */
size_t hd_expand_embed_bwd_workspace_bytes(int B, int L); /* 0 for invalid sizes */
hd_status_t hd_expand_embed_bwd(const void* dout, const int32_t* ids, float* dtables, int B, int L,
                                int n, int V, int D, void* workspace, size_t workspace_bytes,
                                int32_t* dev_status, cudaStream_t stream);
/*
 * The same in two parts.  hd_expand_embed_bwd_plan reads only ids: it sorts the
 * tokens by id and lists each id's run of tokens in the workspace (the "plan"), so a
 * caller can build it as soon as the ids are known (e.g. on a side stream during the
 * forward pass) and keep it for several applies.  hd_expand_embed_bwd_apply adds the
 * gradient rows into dtables following a plan of the same ids, B, L and V; the
 * workspace must hold that plan, unmodified, when the apply runs (order a plan on
 * another stream before the apply with an event).  plan + apply == hd_expand_embed_bwd.
 * An apply on a workspace that does not hold such a plan gives meaningless sums but
 * never reads or writes outside dout, dtables and the workspace: records and token
 * indexes outside the plan's ranges are skipped.
 */
hd_status_t hd_expand_embed_bwd_plan(const int32_t* ids, int B, int L, int V, void* workspace,
                                     size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream);
hd_status_t hd_expand_embed_bwd_apply(const void* dout, float* dtables, int B, int L, int n, int V,
                                      int D, const void* workspace, size_t workspace_bytes,
                                      cudaStream_t stream);

/*
 * hd_select_final_stream -- the positions the loss reads (Eq. 2, Sec. 2.1): the loss
 * is taken only on each token's final stream, 0-indexed position t*n + n-1.
 *   y[b][t][:] = x[b][t*n + n-1][:]   x: bf16 [B][n*L][D], y: bf16 [B][L][D].
 * hd_select_final_stream_bwd -- its adjoint:
 *   dx[b][t*n + n-1][:] = dy[b][t][:], every other row of dx is set to zero.
 * Bit-exact copies; D % 8 == 0, 16-byte aligned pointers; HBM-bound.
 */
hd_status_t hd_select_final_stream(const void* x, void* y, int B, int L, int n, int D,
                                   cudaStream_t stream);
hd_status_t hd_select_final_stream_bwd(const void* dy, void* dx, int B, int L, int n, int D,
                                       cudaStream_t stream);

/*
 * sfa_fwd -- SFA forward over the expanded sequence (Sec. 2.2; Eq. 3-4; Fig. 2):
 *   O[b][p][h] = sum_{p' visible from p} softmax_p'(scale * q_p . k_p') v_p',
 *   lse[b][h][p] = log sum_{p' visible} exp(scale * q_p . k_p').
 * q: bf16 [B][nL][Hq][Dh]; k, v: bf16 [B][nL][Hkv][Dh]; o: bf16 like q (written);
 * lse: float32 [B][Hq][nL] (written).  softmax_scale <= 0 selects 1/sqrt(Dh).
 * window is used only by SFA_LOCAL (must be >= 1 there).  Dh in {64, 128, 256}: the
 * forward and the backward run on tcgen05 kernels at every head dim (256 is the
 * paper's 80B configuration, Table 6).
 * Every position sees itself, so no softmax row is empty.
 */
hd_status_t sfa_fwd(const void* q, const void* k, const void* v, void* o, float* lse, int B, int L,
                    int n, int Hq, int Hkv, int Dh, float softmax_scale, sfa_mode_t mode,
                    int window, int32_t* dev_status, cudaStream_t stream);

/* Bytes of device workspace sfa_bwd needs for these sizes and mode (fp32 dQ
 * accumulator [B][nL][Hq][Dh] plus two fp32 row terms of about B*Hq*nL each; when the
 * backward's grid would leave SMs idle, also fp32 dK and dV partial sums [B][nL][Hkv][Dh]
 * for each of the query-head chunks it then splits the work into).
 * Returns 0 for invalid sizes. */
size_t sfa_bwd_workspace_bytes(int B, int L, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode);

/*
 * sfa_bwd -- gradient of sfa_fwd (the paper trains with SFA but does not write
 * the gradient; this is the derivative of the forward above):
 *   P = exp(scale q k^T - lse) on visible pairs, dP = dO v^T,
 *   dS = P * (dP - rowsum(dO * O)),
 *   dq = scale dS k,  dk = scale sum_{h in group} dS^T q,  dv = sum_{h in group} P^T dO.
 * Inputs q, k, v, o, dout (bf16) and lse (float32, as written by sfa_fwd).
 * Outputs dq [B][nL][Hq][Dh], dk, dv [B][nL][Hkv][Dh] (bf16, overwritten).  dq may lie in the
 * buffer of an input (dout's or q's; it is then rounded from the workspace after the last
 * read, two passes more); dk and dv may not.
 * workspace: device buffer of at least sfa_bwd_workspace_bytes(...) bytes, 256-byte
 * aligned; its contents on entry do not matter.
 */
hd_status_t sfa_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse,
                    const void* dout, void* dq, void* dk, void* dv, int B, int L, int n, int Hq,
                    int Hkv, int Dh, float softmax_scale, sfa_mode_t mode, int window,
                    void* workspace, size_t workspace_bytes, int32_t* dev_status,
                    cudaStream_t stream);

/*
 * The backward in three phases, in order on one stream, for a caller that overlaps or
 * times them separately or adds up dQ in fp32.  Same sizes, mode and workspace as sfa_bwd.
 *   sfa_bwd_prep     : delta = rowsum(dO * O) and lse * log2(e) into the workspace
 *                      (fp32, stream-major), and zero its fp32 dQ accumulator.
 *   sfa_bwd_main     : recompute P on visible pairs, add every dQ contribution into
 *                      the accumulator and write dk, dv (overwritten).
 *   sfa_bwd_finalize : dq = bf16(scale * accumulator).
 * (sfa_bwd itself runs the row terms and the main pass only: its dq is written as bf16
 * by the main pass, from the same fp32 sums, and needs no accumulator.)
 * A later phase reads what the earlier one left in the workspace.
 * sfa_bwd_prep is itself the two halves below, for a caller that overlaps them:
 *   sfa_bwd_row_terms: the delta and lse terms only (needs o, so after sfa_fwd);
 *   sfa_bwd_clear    : only the zeroing of the dQ accumulator.  It needs nothing from
 *                      the forward, so it may run on another stream beside sfa_fwd,
 *                      ordered after the previous sfa_bwd_finalize that read the same
 *                      workspace and before sfa_bwd_main.
 */
hd_status_t sfa_bwd_prep(const void* o, const void* dout, const float* lse, int B, int L, int n, int Hq,
                         int Hkv, int Dh, sfa_mode_t mode, void* workspace, size_t workspace_bytes,
                         cudaStream_t stream);
hd_status_t sfa_bwd_row_terms(const void* o, const void* dout, const float* lse, int B, int L, int n,
                              int Hq, int Hkv, int Dh, sfa_mode_t mode, void* workspace,
                              size_t workspace_bytes, cudaStream_t stream);
hd_status_t sfa_bwd_clear(int B, int L, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode, void* workspace,
                          size_t workspace_bytes, cudaStream_t stream);
hd_status_t sfa_bwd_main(const void* q, const void* k, const void* v, const void* dout, void* dk, void* dv,
                         int B, int L, int n, int Hq, int Hkv, int Dh, float softmax_scale,
                         sfa_mode_t mode, int window, void* workspace, size_t workspace_bytes,
                         int32_t* dev_status, cudaStream_t stream);
hd_status_t sfa_bwd_finalize(void* dq, int B, int L, int n, int Hq, int Hkv, int Dh,
                             float softmax_scale, sfa_mode_t mode, void* workspace,
                             size_t workspace_bytes, cudaStream_t stream);

/*
 * sfa_fwd_final / sfa_bwd_final -- attention of the final-stream queries only (the
 * positions t*n + n-1 the loss reads, Eq. 2) against the layer's keys over all nL
 * positions: the layers that run only the final stream while the other streams' K/V
 * stay as context (Sec. 3.1, KV-mirror layers).  The mask is the layer's own (Eq. 4,
 * Fig. 2): the query of token t at position p = t*n + n-1 sees key p' iff
 *   WITHIN  p' <= p and p' = n-1 (mod n)   (only stream n-1's keys)
 *   CROSS   p' <= p
 *   LOCAL   p - window < p' <= p
 * which equals rows t*n + n-1 of sfa_fwd over the full sequence.
 *   q, o, dout, dq : bf16 [B][L][Hq][Dh]  (dense: only the final-stream rows)
 *   k, v, dk, dv   : bf16 [B][n*L][Hkv][Dh]
 *   lse            : float32 [B][Hq][L], natural log (written by sfa_fwd_final)
 * dk, dv are fully overwritten (zero for keys no final-stream query sees); dq as in sfa_bwd.
 * workspace: >= sfa_bwd_final_workspace_bytes(...) bytes, 256-byte aligned.
 * Dh in {64, 128, 256}, on the same tcgen05 kernels as sfa_fwd / sfa_bwd.
 */
hd_status_t sfa_fwd_final(const void* q, const void* k, const void* v, void* o, float* lse, int B, int L,
                          int n, int Hq, int Hkv, int Dh, float softmax_scale, sfa_mode_t mode, int window,
                          int32_t* dev_status, cudaStream_t stream);
size_t sfa_bwd_final_workspace_bytes(int B, int L, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode);
hd_status_t sfa_bwd_final(const void* q, const void* k, const void* v, const void* o, const float* lse,
                          const void* dout, void* dq, void* dk, void* dv, int B, int L, int n, int Hq,
                          int Hkv, int Dh, float softmax_scale, sfa_mode_t mode, int window,
                          void* workspace, size_t workspace_bytes, int32_t* dev_status,
                          cudaStream_t stream);

/*
 * sfa_decode -- one decoding step over the expanded KV cache (Sec. 3.2 "Inference
 * Cost"; masks of Eq. 4 and Fig. 2).  Generation runs each new token's n streams
 * together: with T = lens[b] tokens in sequence b's cache (the new token included,
 * its K/V rows already appended, see sfa_kv_append), the new token's positions
 * p = (T-1)*n + s attend to the cached positions p' < T*n that the layer's mask lets
 * them see: WITHIN p' = s (mod n) and p' <= p (only stream s's rows are read for it),
 * CROSS p' <= p, LOCAL p - window < p' <= p.  The result equals rows (T-1)*n .. T*n-1
 * of sfa_fwd over the sequence.
 *   q, o     : bf16 [B][n][Hq][Dh], the new token's n positions.
 *   k_cache, v_cache : bf16 [B][Lcap*n][Hkv][Dh], position p at row p (the layout of
 *              sfa_fwd's k / v, so a prefilled forward's K/V is a cache); read-only.
 *   lens     : int32 device array [B], tokens in each sequence's cache (ragged batch).
 *   lse      : float32 [B][Hq][n] natural-log LSE of each row, or NULL.
 *   max_tokens: a bound on every lens[b] (<= Lcap); the work is split for it.
 *   workspace: device memory of >= sfa_decode_workspace_bytes(B, max_tokens, n, Hq,
 *              Hkv, Dh, mode, window) bytes, 16-byte aligned (partial results).
 * A sequence with lens outside [1, max_tokens] gets zero rows, LSE = -inf and
 * HD_DEVBIT_INDEX.  Dh in {64, 128, 256}; Lcap*n <= 2^30.  HBM-bound (reads the
 * visible cached rows once per step).
 */
size_t sfa_decode_workspace_bytes(int B, int max_tokens, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode,
                                  int window); /* 0 for invalid sizes */
hd_status_t sfa_decode(const void* q, const void* k_cache, const void* v_cache, const int32_t* lens, void* o,
                       float* lse, int B, int max_tokens, int Lcap, int n, int Hq, int Hkv, int Dh,
                       float softmax_scale, sfa_mode_t mode, int window, void* workspace,
                       size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream);

/*
 * sfa_kv_append -- the new token's n K and V rows into the cache (Sec. 3.2: each
 * decoded token adds n stream positions):
 *   k_cache[b][(T-1)*n + s] = k_new[b][s], likewise v, with T = lens[b] (the length
 *   including the new token), s < n.
 *   k_new, v_new: bf16 [B][n][Hkv][Dh]; caches as in sfa_decode.  Bit copy.
 * A length outside [1, Lcap] writes nothing for that sequence and sets HD_DEVBIT_INDEX.
 */
hd_status_t sfa_kv_append(const void* k_new, const void* v_new, void* k_cache, void* v_cache,
                          const int32_t* lens, int B, int Lcap, int n, int Hkv, int Dh,
                          int32_t* dev_status, cudaStream_t stream);

/*
 * sfa_fwd_packed -- sfa_fwd over B whole prompts of different lengths, packed one behind
 * another without padding: sequence b's tokens are offsets[b] .. offsets[b+1]-1 of N, its
 * positions count from its own first token, and no query sees another sequence's keys.
 *   q, o : bf16 [N*n][Hq][Dh]      k, v : bf16 [N*n][Hkv][Dh]      lse : float32 [Hq][N*n]
 *   offsets : int32 device array [B+1], 0 <= offsets[0] <= ... <= offsets[B] <= N.
 * Sequences of no tokens are allowed; rows of o and lse before offsets[0] and from offsets[B]
 * on are left as they were, and q, k, v there may hold anything.  Offsets that descend or leave
 * [0, N] write nothing and set HD_DEVBIT_INDEX.  What a mask hides has no effect, infinities and
 * NaN in it included.  Masks, limits and head dims are those of sfa_fwd with B = 1 and L = N
 * (no SFA_WITHIN_NAIVE); forward only.  A sequence's results do not depend on what is packed around
 * it, to the bit where it has more than 48 rows (n per token, or one in SFA_WITHIN); shorter ones share
 * tiles, where their place may change the rounding.
 * o and lse overlap no input (rows are read again where values are not finite).
 * workspace: >= sfa_fwd_packed_workspace_bytes(...) bytes, 16-byte aligned (the list of query
 * tiles, built by each call), not shared by calls that may run at the same time.
 */
size_t sfa_fwd_packed_workspace_bytes(int B, int N, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode); /* 0 for invalid sizes */
hd_status_t sfa_fwd_packed(const void* q, const void* k, const void* v, void* o, float* lse, const int32_t* offsets,
                           int B, int N, int n, int Hq, int Hkv, int Dh, float softmax_scale, sfa_mode_t mode, int window,
                           void* workspace, size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream);

/*
 * Paged cache.  K and V rows of many sequences share one pool each (one pair of pools a
 * layer), cut into pages of P = page_tokens tokens, all n streams of a token together:
 *   k_pages, v_pages : bf16 [num_pages][P*n][Hkv][Dh]
 *   page_table       : int32 [B][max_pages], a sequence's pages in order
 *   lens             : int32 [B], tokens of each sequence (0: an empty slot)
 * Token t, stream s of sequence b is row (t mod P)*n + s of page page_table[b][t / P].  Any
 * P >= 1 will do.  A contiguous cache [B][Lcap*n][Hkv][Dh] with P dividing Lcap is a pool
 * with page_table[b][i] = b*Lcap/P + i.  Entries of a table behind the pages in use are never
 * looked at, and neither are rows of a page behind its sequence's tokens.
 * Limits: max_pages*P*n <= 2^30, num_pages*P*n < 2^31, B*max_pages < 2^31.
 *
 * sfa_kv_append_paged -- new tokens' K and V rows into the pages: sfa_kv_append for a paged
 * cache, and for whole prompts.  lens counts the new tokens already.
 *   offsets NULL: one new token a sequence: N = B, k_new, v_new bf16 [B][n][Hkv][Dh], to
 *     token lens[b]-1.  A slot with lens[b] = 0 is left out.
 *   offsets int32 [B+1]: packed rows k_new, v_new bf16 [N*n][Hkv][Dh]; sequence b's new
 *     tokens are offsets[b] .. offsets[b+1]-1, its last ones: token i goes to token
 *     lens[b] - offsets[b+1] + i.  Rows before offsets[0] and from offsets[B] on are not
 *     read.  N = 0 is allowed.
 * Bit copy.  The pages must be held by the sequence alone.  Rows whose page is not in the
 * pool, and the rows of a sequence whose offsets descend, leave [0, N] or hold more tokens
 * than lens[b], are not written and set HD_DEVBIT_INDEX (so does a length outside
 * [0, max_pages*P]).  With offsets that descend anywhere, rows of other sequences may be left out as
 * well.
 *
 * sfa_kv_append_paged_served -- the same after a hd_pages_grow_served whose result nobody has looked at:
 *   served int32 [B], its output.  A sequence that got fewer tokens than it brings (one, or
 *   offsets[b+1] - offsets[b]) is left out, without a bit of its own.  (The plain call cannot tell: to it
 *   lens[b]-1 is the new token, and where a grow was refused that is the token before, in a page that
 *   others may share.)
 */
hd_status_t sfa_kv_append_paged(const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                                const int32_t* page_table, const int32_t* lens, const int32_t* offsets, int B, int N,
                                int num_pages, int page_tokens, int max_pages, int n, int Hkv, int Dh,
                                int32_t* dev_status, cudaStream_t stream);
hd_status_t sfa_kv_append_paged_served(const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                                       const int32_t* page_table, const int32_t* lens, const int32_t* offsets,
                                       const int32_t* served, int B, int N, int num_pages, int page_tokens, int max_pages,
                                       int n, int Hkv, int Dh, int32_t* dev_status, cudaStream_t stream);

/*
 * sfa_decode_paged -- sfa_decode over a paged cache: the same masks, outputs and limits (Dh,
 * n*Hq), with the rows found through page_table.  B <= 65535; max_tokens <= max_pages*P.
 *   An empty slot (lens[b] = 0) gets zero rows and LSE = -inf, and is no error.  A length
 *   outside [0, max_tokens], or a page that is needed and not in the pool, gives the
 *   sequence zero rows, LSE = -inf and HD_DEVBIT_INDEX; the others are not affected.
 *   SFA_LOCAL needs only the pages that the window of the new token's positions touches.
 *   What a mask hides has no effect, infinities and NaN in it included.
 *   workspace: >= sfa_decode_paged_workspace_bytes(...) bytes, 16-byte aligned, not shared by
 *   calls that may run at the same time.  With the other sizes the same, the bytes for some
 *   max_tokens and window are enough for every smaller max_tokens and window, any pages and any
 *   table width; another B asks anew (fewer sequences are split more).
 */
size_t sfa_decode_paged_workspace_bytes(int B, int max_tokens, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode,
                                        int window); /* 0 for invalid sizes */
hd_status_t sfa_decode_paged(const void* q, const void* k_pages, const void* v_pages, const int32_t* page_table,
                             const int32_t* lens, void* o, float* lse, int B, int max_tokens, int num_pages,
                             int page_tokens, int max_pages, int n, int Hq, int Hkv, int Dh, float softmax_scale,
                             sfa_mode_t mode, int window, void* workspace, size_t workspace_bytes,
                             int32_t* dev_status, cudaStream_t stream);

/*
 * Who holds which page.  The state is page_table and lens as above and
 *   refs : int32 [num_pages], the number of sequences that hold each page (0: free).
 * Start with refs and lens zero.  A sequence of T tokens holds the first ceil(T / P) entries
 * of its table; the calls keep it so.  Free pages are given out lowest id first, so results
 * depend on the state alone.  One table serves every layer; the copies that fork and compact
 * list are to be made in each layer's pools (hd_pages_copy) before the pages are written again.
 * The calls of one state are to be ordered on one stream; the workspace (>=
 * hd_pages_workspace_bytes(B, num_pages) bytes, 16-byte aligned) holds nothing between them.
 * Shared pages are always full, as long as lens only changes through these calls.
 *
 * hd_pages_grow : lens[b] += add[b], with the pages for it: sequence b, in ascending order,
 *   gets them if all that b and those before it ask for are free; else it and its length are
 *   left as they were (HD_DEVBIT_PAGES).  add[b] < 0, or a length that leaves
 *   [0, max_pages*P], is left out with HD_DEVBIT_INDEX.  Nothing is to be appended to a sequence that was
 *   left as it was: look at the status first, or use
 * hd_pages_grow_served : the same, and served [B] (a buffer of its own) is the tokens that each
 *   sequence got, add[b] or 0, for sfa_kv_append_paged_served (and the caller: o of a decoding step that
 *   follows is no token's for a sequence that got none).
 * hd_pages_fork : for i < F, the empty slot dst[i] gets the first tokens[i] tokens of src[i]
 *   (tokens NULL: all of them): floor(tokens/P) pages are shared, the rest of the prefix gets
 *   a page of its own and copies[i] = (page of src, page of dst), else (-1, -1).  src may name
 *   a slot many times.  A fork that finds no free page is left out (HD_DEVBIT_PAGES); with
 *   HD_DEVBIT_INDEX one whose slots are out of range or the same, whose dst is not empty or
 *   was named by an earlier fork, whose tokens exceed lens[src], or whose pages are not held.
 *   (A slot that the same call forks to counts as empty as a source.)  F <= B.
 * hd_pages_free : slots seqs[0 .. F-1] are emptied: lens 0, their table entries -1, one holder
 *   less for their pages.  An empty slot, or a slot named before, is no error; an index, a
 *   length or a table entry out of range, or a page that nobody holds, sets HD_DEVBIT_INDEX.
 * hd_pages_compact : the K pages in use get the ids 0 .. K-1: the j-th page in use with an id
 *   >= K goes to the j-th free id below K, moves[j] = (old, new); the other moves are
 *   (-1, -1).  new_refs and new_table (entries behind a sequence's pages -1) may be refs and
 *   page_table themselves.  moves: int32 [num_pages/2][2].
 * hd_pages_copy : for i < F, page copies[i][0] onto page copies[i][1] in both pools
 *   (page_bytes a page, a multiple of 16), as listed above; pairs of negative ids are left
 *   out, others outside the pool set HD_DEVBIT_INDEX.  No page may be written twice, or
 *   written and read.
 * F = 0 is allowed and does nothing.  refs is 16-byte, copies and moves 8-byte aligned.
 */
size_t hd_pages_workspace_bytes(int B, int num_pages); /* 0 for invalid sizes */
hd_status_t hd_pages_grow(int32_t* refs, int32_t* page_table, int32_t* lens, const int32_t* add, int B, int max_pages,
                          int num_pages, int page_tokens, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                          cudaStream_t stream);
hd_status_t hd_pages_grow_served(int32_t* refs, int32_t* page_table, int32_t* lens, const int32_t* add, int32_t* served,
                                 int B, int max_pages, int num_pages, int page_tokens, void* workspace,
                                 size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream);
hd_status_t hd_pages_fork(int32_t* refs, int32_t* page_table, int32_t* lens, const int32_t* src, const int32_t* dst,
                          const int32_t* tokens, int F, int32_t* copies, int B, int max_pages, int num_pages,
                          int page_tokens, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                          cudaStream_t stream);
hd_status_t hd_pages_free(int32_t* refs, int32_t* page_table, int32_t* lens, const int32_t* seqs, int F, int B,
                          int max_pages, int num_pages, int page_tokens, int32_t* dev_status, cudaStream_t stream);
hd_status_t hd_pages_compact(const int32_t* refs, const int32_t* page_table, const int32_t* lens, int32_t* new_refs,
                             int32_t* new_table, int32_t* moves, int B, int max_pages, int num_pages, int page_tokens,
                             void* workspace, size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream);
hd_status_t hd_pages_copy(void* k_pages, void* v_pages, const int32_t* copies, int F, int num_pages, size_t page_bytes,
                          int32_t* dev_status, cudaStream_t stream);

/*
 * Paged cache in 8 bits.  The same tables, lengths and page calls as above; the pools of a layer hold
 *   k_pages, v_pages   : e4m3 codes, 1 byte each, [num_pages][Hkv][P*n][Dh]: a page's rows of one head together
 *   k_scales, v_scales : uint8 [num_pages][Hkv][P/block_tokens], a scale for each block of block_tokens tokens (which
 *                        divides P; all n streams of a token together) and head: a power of two 2^e as the byte e + 127
 * A code c of a block stands for c * 2^e, which is exact in bf16.  e lies in [-64, 50] (bytes 63 ... 177; others
 * are read as the nearest of these): values below 2^-74 become 0, values above 448 * 2^50 saturate.
 * Pools and scales are 16-byte aligned.  Limits beside those above: Dh a multiple of 16, n*Hkv*Dh <= 2^24,
 * block_tokens*n*Dh <= 2^30, Hkv <= 32767, num_pages*P*n*Hkv < 2^32.
 *
 * sfa_kv_append_paged_q8 -- sfa_kv_append_paged into such a cache: the same arguments, rows and refusals; served
 *   (nullable) as in sfa_kv_append_paged_served.  Of a block, the call brings some last tokens.  If no token before
 *   them is in the block, its e is the smallest with 448 * 2^e no smaller than their largest finite magnitude
 *   (within [-64, 50]); else the larger of that and the e that it has, and where that is larger than it was the codes
 *   of the tokens before them are rounded again (exactly, but for values that become subnormal in e4m3).  Values are
 *   rounded to the nearest code, ties to even; infinities and NaN become NaN.  Rows of the block behind the
 *   sequence's tokens are left as they were.  So the same tokens in the same calls give the same bits, and in other
 *   calls differ by one rounding more at most for each growth.
 *
 * sfa_kv_read_paged_q8 -- the way back: packed rows k, v bf16 [N*n][Hkv][Dh] of the last tokens of each sequence,
 *   sequence b's to offsets[b] .. offsets[b+1]-1 (token lens[b] - offsets[b+1] + i to packed token i; lens may be less
 *   than the sequence holds).  Exact.  Rows before offsets[0] and from offsets[B] on are left as they were, and so
 *   are, with HD_DEVBIT_INDEX, the rows of what sfa_kv_append_paged would refuse.
 *
 * sfa_decode_paged_q8 -- sfa_decode_paged over such a cache: the same masks, outputs, errors and workspace rules (with
 *   its own workspace size).  The result is that of the values that the codes stand for.  Dh 64, 128 or 256.
 *   To what: o is rounded to bf16.  Sums are in 32 bits.  A position's weight is held to 2^-9 of itself, or, where the
 *   weight times its block's 2^e (of V) lies below 2^-19 of the row's largest such product, to 2^-28 of that: 2^-22 of the
 *   row's largest weight at most where its block's e lies no more than 6 below the largest, and else, for all such
 *   positions of a row together, 2^-7 of the sum of its weights.  A score is off by at most 2^-8 (in log2 units) for what
 *   is held of a query's values below 2^-13 of its row's largest.  Rows for which these bounds do not hold (blocks of V
 *   some 2^10 and more apart, or query values as far apart that meet K as much larger) are computed in 32 bits, position
 *   by position: as exact, but a step with many such rows takes 40 to 200 times as long.
 *
 * hd_pages_copy_q8 -- hd_pages_copy for codes (page_bytes = Hkv*P*n*Dh, a multiple of 16) and scales (page_scales =
 *   Hkv*P/block_tokens bytes a page).
 */
hd_status_t sfa_kv_append_paged_q8(const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                                   uint8_t* k_scales, uint8_t* v_scales, const int32_t* page_table, const int32_t* lens,
                                   const int32_t* offsets, const int32_t* served, int B, int N, int num_pages,
                                   int page_tokens, int max_pages, int n, int Hkv, int Dh, int block_tokens,
                                   int32_t* dev_status, cudaStream_t stream);
hd_status_t sfa_kv_read_paged_q8(const void* k_pages, const void* v_pages, const uint8_t* k_scales,
                                 const uint8_t* v_scales, const int32_t* page_table, const int32_t* lens,
                                 const int32_t* offsets, void* k, void* v, int B, int N, int num_pages, int page_tokens,
                                 int max_pages, int n, int Hkv, int Dh, int block_tokens, int32_t* dev_status,
                                 cudaStream_t stream);
size_t sfa_decode_paged_q8_workspace_bytes(int B, int max_tokens, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode,
                                           int window); /* 0 for invalid sizes */
hd_status_t sfa_decode_paged_q8(const void* q, const void* k_pages, const void* v_pages, const uint8_t* k_scales,
                                const uint8_t* v_scales, const int32_t* page_table, const int32_t* lens, void* o,
                                float* lse, int B, int max_tokens, int num_pages, int page_tokens, int max_pages, int n,
                                int Hq, int Hkv, int Dh, int block_tokens, float softmax_scale, sfa_mode_t mode,
                                int window, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                                cudaStream_t stream);
hd_status_t hd_pages_copy_q8(void* k_pages, void* v_pages, uint8_t* k_scales, uint8_t* v_scales, const int32_t* copies,
                             int F, int num_pages, size_t page_bytes, size_t page_scales, int32_t* dev_status,
                             cudaStream_t stream);

/*
 * sfa_bwd_noalloc -- sfa_bwd without a caller-supplied workspace.  The paper has no
 * counterpart: this is an interface for callers that cannot hand the library device
 * memory of their own (a runtime that commits its whole device-memory budget at
 * start-up and forbids allocation while serving, or C code with no device allocator).
 * Same arguments, outputs and status codes as sfa_bwd, minus the workspace.
 *
 * The workspace lives in a fixed device array of the library, SFA_BWD_NOALLOC_MAX_BYTES
 * long, present in every CUDA context that loads the library's module; the call
 * allocates and frees nothing.  Sizes whose sfa_bwd_workspace_bytes() exceeds that
 * limit return HD_ERR_SCRATCH_LIMIT before anything is enqueued (use sfa_bwd there).
 *   - Set-up: every call looks up the array's device address in the calling thread's
 *     current CUDA context (the address belongs to that context, so it is not cached);
 *     the first call in a context also loads the library's module there, so make that
 *     first call before any stream capture.  A failed look-up returns HD_ERR_CUDA.
 *   - Sharing: every call on a device uses the same array, which keeps the last call's
 *     contents; each call writes what it reads before reading it.  Calls that may run
 *     concurrently on one device (unordered streams, several host threads) race on
 *     the array: the caller must order them.
 */
#define SFA_BWD_NOALLOC_MAX_BYTES ((size_t)64 << 20)
hd_status_t sfa_bwd_noalloc(const void* q, const void* k, const void* v, const void* o,
                            const float* lse, const void* dout, void* dq, void* dk, void* dv, int B,
                            int L, int n, int Hq, int Hkv, int Dh, float softmax_scale,
                            sfa_mode_t mode, int window, int32_t* dev_status, cudaStream_t stream);

/* Human-readable name of a status code (static string). */
const char* hd_status_string(hd_status_t status);

/*
 * hd_selftest_bounded_wait -- diagnostic of the failure path shared by the tensor-core
 * kernels (no counterpart in the paper).  Launches one warp that waits, with the same
 * bounded mbarrier wait those kernels use, on a barrier nothing arrives on.  After the
 * bound (about a second) the wait gives up: HD_DEVBIT_TIMEOUT is ORed into *dev_status
 * and *dev_result is set to 0 (1 would mean the wait completed).  No fault, no trap: the
 * kernel returns and the context stays usable.
 *   dev_status, dev_result: device int32 words (dev_status may be NULL; dev_result not).
 */
hd_status_t hd_selftest_bounded_wait(int32_t* dev_status, int32_t* dev_result, cudaStream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* HDSFA_H */
