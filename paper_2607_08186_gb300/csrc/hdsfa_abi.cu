// C ABI of libhdsfa.so (declared in include/hdsfa.h): host-side validation,
// problem geometry and kernel dispatch.  No allocation, no synchronisation.
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include "common.cuh"
#include "decode_plan.cuh"
#include "nvtx_range.h"
#include "packed.cuh"

namespace hdsfa {
cudaError_t launch_expand_embed(const void* tables, const int32_t* ids, void* out, int B, int L,
                                int n, int V, int D, int32_t* status, cudaStream_t stream);
size_t expand_bwd_ws_bytes(long long N);
cudaError_t launch_expand_bwd_plan(const int32_t* ids, int B, int L, int V, void* ws, int32_t* status,
                                   cudaStream_t st);
cudaError_t launch_expand_bwd_apply(const void* dx, float* de, int B, int L, int n, int V, int D, const void* ws,
                                    cudaStream_t st);
cudaError_t launch_select_final(const void* x, void* y, int B, int L, int n, int D, cudaStream_t st);
cudaError_t launch_select_final_bwd(const void* dy, void* dx, int B, int L, int n, int D, cudaStream_t st);
cudaError_t launch_sfa_decode(const void* q, const void* kc, const void* vc, const int32_t* lens, void* o,
                              float* lse, int B, int maxT, int Lcap, int n, int Hq, int Hkv, int Dh, float scale,
                              int mode, int window, void* ws, int32_t* status, cudaStream_t st);
cudaError_t launch_bounded_wait_selftest(int32_t* status, int32_t* result, cudaStream_t st);
cudaError_t launch_kv_append(const void* kn, const void* vn, void* kc, void* vc, const int32_t* lens, int B,
                             int Lcap, int n, int Hkv, int Dh, int32_t* status, cudaStream_t st);
cudaError_t launch_sfa_decode_paged(const void* q, const void* kp, const void* vp, const int32_t* table,
                                    const int32_t* lens, void* o, float* lse, int B, int maxT, int num_pages, int P,
                                    int max_pages, int n, int Hq, int Hkv, int Dh, float scale, int mode, int window,
                                    void* ws, size_t ws_bytes, int32_t* status, cudaStream_t st);
cudaError_t launch_kv_append_paged(const void* kn, const void* vn, void* kp, void* vp, const int32_t* table,
                                   const int32_t* lens, const int32_t* offsets, const int32_t* served, int B, int N,
                                   int num_pages, int P, int max_pages, int n, int Hkv, int Dh, int32_t* status,
                                   cudaStream_t st);
cudaError_t launch_kv_append_paged_q8(const void* kn, const void* vn, void* kc, void* vc, uint8_t* ks, uint8_t* vs,
                                      const int32_t* table, const int32_t* lens, const int32_t* offsets,
                                      const int32_t* served, int B, int N, int num_pages, int P, int max_pages, int n,
                                      int Hkv, int Dh, int T, int32_t* status, cudaStream_t st);
cudaError_t launch_kv_read_paged_q8(const void* kc, const void* vc, const uint8_t* ks, const uint8_t* vs,
                                    const int32_t* table, const int32_t* lens, const int32_t* offsets, void* k, void* v,
                                    int B, int N, int num_pages, int P, int max_pages, int n, int Hkv, int Dh, int T,
                                    int32_t* status, cudaStream_t st);
size_t decode_paged_q8_ws_bytes(int B, int maxT, int n, int Hq, int Hkv, int Dh, int mode, int window);
cudaError_t launch_sfa_decode_paged_q8(const void* q, const void* kc, const void* vc, const uint8_t* ks, const uint8_t* vs,
                                       const int32_t* table, const int32_t* lens, void* o, float* lse, int B, int maxT,
                                       int num_pages, int P, int max_pages, int n, int Hq, int Hkv, int Dh, int T,
                                       float scale, int mode, int window, void* ws, size_t ws_bytes, int32_t* status,
                                       cudaStream_t st);
cudaError_t launch_pages_copy_q8(void* kc, void* vc, uint8_t* ks, uint8_t* vs, const int32_t* copies, int F,
                                 int num_pages, size_t page_bytes, int page_scales, int32_t* status, cudaStream_t st);
size_t pages_ws_bytes(int B, int num_pages);
cudaError_t launch_pages_grow(int32_t* refs, int32_t* table, int32_t* lens, const int32_t* add, int32_t* served, int B,
                              int max_pages, int num_pages, int P, void* ws, int32_t* status, cudaStream_t st);
cudaError_t launch_pages_fork(int32_t* refs, int32_t* table, int32_t* lens, const int32_t* src, const int32_t* dst,
                              const int32_t* tokens, int F, int32_t* copies, int B, int max_pages, int num_pages, int P,
                              void* ws, int32_t* status, cudaStream_t st);
cudaError_t launch_pages_free(int32_t* refs, int32_t* table, int32_t* lens, const int32_t* seqs, int F, int B,
                              int max_pages, int num_pages, int P, int32_t* status, cudaStream_t st);
cudaError_t launch_pages_compact(const int32_t* refs, const int32_t* table, const int32_t* lens, int32_t* new_refs,
                                 int32_t* new_table, int32_t* moves, int B, int max_pages, int num_pages, int P,
                                 void* ws, int32_t* status, cudaStream_t st);
cudaError_t launch_pages_copy(void* kp, void* vp, const int32_t* copies, int F, int num_pages, int page16,
                              int32_t* status, cudaStream_t st);
cudaError_t launch_sfa_fwd_tc(const void* q, const void* k, const void* v, void* o, float* lse,
                              const SfaGeom& g, int Dh, float scale, int32_t* status, cudaStream_t st);
cudaError_t launch_sfa_fwd_tc256(const void* q, const void* k, const void* v, void* o, float* lse,
                                 const SfaGeom& g, float scale, int32_t* status, cudaStream_t st);
cudaError_t launch_sfa_fwd_packed_tc(const void* q, const void* k, const void* v, void* o, float* lse, const SfaGeom& g,
                                     int Dh, float scale, const PackedList& list, const int32_t* offsets,
                                     bool shared, long long max_items, int32_t* status, cudaStream_t st);
cudaError_t launch_sfa_fwd_packed_tc256(const void* q, const void* k, const void* v, void* o, float* lse,
                                        const SfaGeom& g, float scale, const PackedList& list, const int32_t* offsets,
                                        long long max_items, int32_t* status, cudaStream_t st);
cudaError_t launch_sfa_bwd_prep(const void* o, const void* dout, const float* lse, float* lse2_ws,
                                float* delta_ws, float* dq_ws, const SfaGeom& g, int Dh,
                                cudaStream_t st, bool zero = true);
cudaError_t launch_sfa_bwd_clear(float* dq_ws, const SfaGeom& g, int Dh, cudaStream_t st);
cudaError_t launch_sfa_bwd_main_tc(const void* q, const void* k, const void* v, const void* dout, void* dq_out,
                                   void* dk, void* dv, const float* lse2_ws, const float* delta_ws, float* dq_ws,
                                   float* dkv_ws, const SfaGeom& g, int Dh, float scale, int32_t* status,
                                   cudaStream_t st);
cudaError_t launch_sfa_bwd_main_tc256(const void* q, const void* k, const void* v, const void* dout, void* dq_out,
                                      void* dk, void* dv, const float* lse2_ws, const float* delta_ws, float* dq_ws,
                                      float* dkv_ws, const SfaGeom& g, float scale, int32_t* status,
                                      cudaStream_t st);
cudaError_t launch_sfa_bwd_finalize(void* dq, const float* dq_ws, const SfaGeom& g, int Dh,
                                    float scale, cudaStream_t st);
}  // namespace hdsfa

namespace {

bool aligned16(const void* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned_to(const void* p, uintptr_t a) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
bool aligned_or_null(const void* p, uintptr_t a) { return p == nullptr || aligned_to(p, a); }

// Validates sizes shared by sfa_fwd / sfa_bwd and builds the virtual-problem geometry.

hd_status_t make_geom(int B, int L, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode, int window,
                      SfaGeom* g) {
  if (B <= 0 || L <= 0 || n <= 0 || Hq <= 0 || Hkv <= 0 || Dh <= 0) return HD_ERR_INVALID_ARG;
  if (Hq % Hkv != 0) return HD_ERR_INVALID_ARG;
  if (mode != SFA_WITHIN && mode != SFA_CROSS && mode != SFA_LOCAL && mode != SFA_WITHIN_NAIVE)
    return HD_ERR_INVALID_ARG;
  if (mode == SFA_LOCAL && window <= 0) return HD_ERR_INVALID_ARG;
  if (Dh != 64 && Dh != 128 && Dh != 256) return HD_ERR_UNSUPPORTED;
  // the naive schedule exists on the head-dim-128 kernels only
  if (mode == SFA_WITHIN_NAIVE && Dh != 128) return HD_ERR_UNSUPPORTED;
  const long long nL = (long long)n * L;
  // Every row index, head product and tile count must fit the kernels' int math.
  if (nL > (1LL << 30) || (long long)B * nL * Hq > (1LL << 31) / 2) return HD_ERR_UNSUPPORTED;
  g->B = B;
  g->nL = (int)nL;
  g->Hq = Hq;
  g->Hkv = Hkv;
  g->n = n;
  if (mode == SFA_WITHIN) {
    g->Lv = L;
    g->ns = n;
    g->rs = n;
    g->window = 0;
  } else {  // CROSS, LOCAL, and the naive WITHIN schedule
    g->Lv = (int)nL;
    g->ns = 1;
    g->rs = 1;
    // a window of nL positions already sees every earlier key; larger ones ("no limit",
    // up to INT_MAX) are cut to it, so that sums of a row and the window stay in 32 bits
    g->window = mode == SFA_LOCAL ? (window < nL ? window : (int)nL) : 0;
  }
  g->smod = mode == SFA_WITHIN_NAIVE ? n : 0;
  // queries are the key rows themselves
  g->Lq = g->Lv;
  g->qstep = 1;
  g->qoff = 0;
  g->q_nL = g->nL;
  g->q_ns = g->ns;
  g->q_rs = g->rs;
  g->kv_s0 = 0;
  return HD_OK;
}

// A final-stream problem: the L final-stream queries (positions t*n + n-1, the rows
// the loss reads, Eq. 2) in dense [B][L] tensors against the keys of the layer's mask.
hd_status_t make_final_geom(int B, int L, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode, int window,
                            SfaGeom* g) {
  if (mode == SFA_WITHIN_NAIVE) return HD_ERR_UNSUPPORTED;
  hd_status_t st = make_geom(B, L, n, Hq, Hkv, Dh, mode, window, g);
  if (st != HD_OK) return st;
  g->Lq = L;
  g->q_nL = L;
  g->q_ns = 1;
  g->q_rs = 1;
  if (mode == SFA_WITHIN) {  // the problem of stream n-1: query row t is its key row t
    g->qstep = 1;
    g->qoff = 0;
    g->kv_s0 = n - 1;
  } else {  // query row t at position t*n + n-1 of the nL key rows
    g->qstep = n;
    g->qoff = n - 1;
    g->kv_s0 = 0;
  }
  return HD_OK;
}

float resolve_scale(float s, int Dh) { return s > 0.f ? s : 1.0f / sqrtf((float)Dh); }

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// Workspace layout: fp32 dQ accumulator [B][nL][Hq][Dh], then -lse*log2(e) and
// -delta, each fp32 [B][Hq][ns][Lvp] (stream-major rows, Lvp = row_terms_pitch(Lv)),
// then on small grids the fp32 dV / dK partial sums of the head chunks, one slice per
// chunk (bwd_dkv_slice elements each).
struct BwdWs {
  float* dq;
  float* lse2;
  float* delta;
  float* dkv;
};

// Sizes follow the query side (query_geom): the accumulator and row terms are per query row.
size_t ws_bytes(const SfaGeom& gk, int Dh) {
  const SfaGeom g = query_geom(gk);
  const size_t rows = (size_t)g.B * g.nL * g.Hq;
  const size_t trows = (size_t)g.B * g.Hq * g.ns * (size_t)row_terms_pitch(g.Lv);
  const size_t dkv = (size_t)bwd_head_chunks(gk, Dh) * 2 * bwd_dkv_slice(gk, Dh) * sizeof(float);
  return align256(rows * Dh * sizeof(float)) + 2 * align256(trows * sizeof(float)) + align256(dkv);
}

hd_status_t split_ws(const SfaGeom& gk, int Dh, void* ws, size_t bytes, BwdWs* out) {
  if (ws == nullptr || bytes < ws_bytes(gk, Dh) || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0)
    return HD_ERR_WORKSPACE;
  const SfaGeom g = query_geom(gk);
  const size_t rows = (size_t)g.B * g.nL * g.Hq;
  const size_t trows = (size_t)g.B * g.Hq * g.ns * (size_t)row_terms_pitch(g.Lv);
  char* p = static_cast<char*>(ws);
  out->dq = reinterpret_cast<float*>(p);
  p += align256(rows * Dh * sizeof(float));
  out->lse2 = reinterpret_cast<float*>(p);
  p += align256(trows * sizeof(float));
  out->delta = reinterpret_cast<float*>(p);
  p += align256(trows * sizeof(float));
  out->dkv = bwd_dkv_slice(gk, Dh) > 0 ? reinterpret_cast<float*>(p) : nullptr;
  return HD_OK;
}

hd_status_t cuda_status(cudaError_t e) { return e == cudaSuccess ? HD_OK : HD_ERR_CUDA; }

// The main pass at any head dim; dq null: fp32 dQ added into the accumulator.
cudaError_t main_pass(const void* q, const void* k, const void* v, const void* dout, void* dq, void* dk, void* dv,
                      const BwdWs& ws, const SfaGeom& g, int Dh, float scale, int32_t* status, cudaStream_t st) {
  if (Dh == 256)
    return hdsfa::launch_sfa_bwd_main_tc256(q, k, v, dout, dq, dk, dv, ws.lse2, ws.delta, ws.dq, ws.dkv, g, scale, status,
                                            st);
  return hdsfa::launch_sfa_bwd_main_tc(q, k, v, dout, dq, dk, dv, ws.lse2, ws.delta, ws.dq, ws.dkv, g, Dh, scale, status,
                                       st);
}

bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + b_bytes && y < x + a_bytes;
}

// The backward after its argument checks.  dQ leaves the main pass as bf16 (no accumulator to
// clear or convert), unless dq is the buffer of an operand that the pass reads until its end
// (dout's, say): then the sums go through the accumulator.
cudaError_t backward(const void* q, const void* k, const void* v, const void* o, const float* lse, const void* dout,
                     void* dq, void* dk, void* dv, const BwdWs& ws, const SfaGeom& g, int Dh, float scale,
                     int32_t* status, cudaStream_t st) {
  const SfaGeom gq = query_geom(g);
  const size_t qb = (size_t)g.B * g.q_nL * g.Hq * Dh * 2, kb = (size_t)g.B * g.nL * g.Hkv * Dh * 2;
  const bool in_place =
      overlap(dq, qb, q, qb) || overlap(dq, qb, dout, qb) || overlap(dq, qb, k, kb) || overlap(dq, qb, v, kb);
  cudaError_t e = hdsfa::launch_sfa_bwd_prep(o, dout, lse, ws.lse2, ws.delta, ws.dq, gq, Dh, st, in_place);
  if (e == cudaSuccess && g.ns > g.q_ns) {
    // a WITHIN layer's final-stream queries see only stream n-1's keys: the other rows are zero
    e = cudaMemsetAsync(dk, 0, kb, st);
    if (e == cudaSuccess) e = cudaMemsetAsync(dv, 0, kb, st);
  }
  if (e == cudaSuccess) e = main_pass(q, k, v, dout, in_place ? nullptr : dq, dk, dv, ws, g, Dh, scale, status, st);
  if (e == cudaSuccess && in_place) e = hdsfa::launch_sfa_bwd_finalize(dq, ws.dq, gq, Dh, scale, st);
  return e;
}

}  // namespace

extern "C" {

hd_status_t hd_expand_embed(const void* tables, const int32_t* ids, void* out, int B, int L, int n,
                            int V, int D, int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("hd_expand_embed");
  if (!aligned16(tables) || !aligned16(out) || ids == nullptr) return HD_ERR_INVALID_ARG;
  if (B <= 0 || L <= 0 || n <= 0 || V <= 0 || D <= 0 || D % 8 != 0) return HD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(ids) & 3u) != 0) return HD_ERR_INVALID_ARG;
  return hdsfa::launch_expand_embed(tables, ids, out, B, L, n, V, D, dev_status, stream) == cudaSuccess
             ? HD_OK
             : HD_ERR_CUDA;
}

size_t hd_expand_embed_bwd_workspace_bytes(int B, int L) {
  if (B <= 0 || L <= 0 || (long long)B * L >= (1LL << 31)) return 0;
  return hdsfa::expand_bwd_ws_bytes((long long)B * L);
}

hd_status_t hd_expand_embed_bwd_plan(const int32_t* ids, int B, int L, int V, void* workspace,
                                     size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("hd_expand_embed_bwd_plan");
  if (ids == nullptr || (reinterpret_cast<uintptr_t>(ids) & 3u) != 0) return HD_ERR_INVALID_ARG;
  if (B <= 0 || L <= 0 || V <= 0) return HD_ERR_INVALID_ARG;
  const size_t need = hd_expand_embed_bwd_workspace_bytes(B, L);
  if (need == 0) return HD_ERR_UNSUPPORTED;
  if (!aligned16(workspace) || workspace_bytes < need) return HD_ERR_WORKSPACE;
  return cuda_status(hdsfa::launch_expand_bwd_plan(ids, B, L, V, workspace, dev_status, stream));
}

hd_status_t hd_expand_embed_bwd_apply(const void* dout, float* dtables, int B, int L, int n, int V, int D,
                                      const void* workspace, size_t workspace_bytes, cudaStream_t stream) {
  HD_NVTX_RANGE("hd_expand_embed_bwd_apply");
  if (!aligned16(dout) || !aligned16(dtables)) return HD_ERR_INVALID_ARG;
  if (B <= 0 || L <= 0 || n <= 0 || V <= 0 || D <= 0 || D % 8 != 0) return HD_ERR_INVALID_ARG;
  const size_t need = hd_expand_embed_bwd_workspace_bytes(B, L);
  if (need == 0 || (long long)n * D >= (1LL << 31)) return HD_ERR_UNSUPPORTED;
  if (!aligned16(workspace) || workspace_bytes < need) return HD_ERR_WORKSPACE;
  return cuda_status(hdsfa::launch_expand_bwd_apply(dout, dtables, B, L, n, V, D, workspace, stream));
}

hd_status_t hd_expand_embed_bwd(const void* dout, const int32_t* ids, float* dtables, int B, int L, int n,
                                int V, int D, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                                cudaStream_t stream) {
  HD_NVTX_RANGE("hd_expand_embed_bwd");
  // every argument is checked before the plan is enqueued
  if (!aligned16(dout) || !aligned16(dtables) || ids == nullptr) return HD_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(ids) & 3u) != 0) return HD_ERR_INVALID_ARG;
  if (B <= 0 || L <= 0 || n <= 0 || V <= 0 || D <= 0 || D % 8 != 0) return HD_ERR_INVALID_ARG;
  const size_t need = hd_expand_embed_bwd_workspace_bytes(B, L);
  if (need == 0 || (long long)n * D >= (1LL << 31)) return HD_ERR_UNSUPPORTED;
  if (!aligned16(workspace) || workspace_bytes < need) return HD_ERR_WORKSPACE;
  hd_status_t st = hd_expand_embed_bwd_plan(ids, B, L, V, workspace, workspace_bytes, dev_status, stream);
  if (st != HD_OK) return st;
  return hd_expand_embed_bwd_apply(dout, dtables, B, L, n, V, D, workspace, workspace_bytes, stream);
}

hd_status_t hd_select_final_stream(const void* x, void* y, int B, int L, int n, int D, cudaStream_t stream) {
  HD_NVTX_RANGE("hd_select_final_stream");
  if (!aligned16(x) || !aligned16(y)) return HD_ERR_INVALID_ARG;
  if (B <= 0 || L <= 0 || n <= 0 || D <= 0 || D % 8 != 0) return HD_ERR_INVALID_ARG;
  return cuda_status(hdsfa::launch_select_final(x, y, B, L, n, D, stream));
}

hd_status_t hd_select_final_stream_bwd(const void* dy, void* dx, int B, int L, int n, int D,
                                       cudaStream_t stream) {
  HD_NVTX_RANGE("hd_select_final_stream_bwd");
  if (!aligned16(dy) || !aligned16(dx)) return HD_ERR_INVALID_ARG;
  if (B <= 0 || L <= 0 || n <= 0 || D <= 0 || D % 8 != 0) return HD_ERR_INVALID_ARG;
  return cuda_status(hdsfa::launch_select_final_bwd(dy, dx, B, L, n, D, stream));
}

hd_status_t sfa_fwd(const void* q, const void* k, const void* v, void* o, float* lse, int B, int L,
                    int n, int Hq, int Hkv, int Dh, float softmax_scale, sfa_mode_t mode,
                    int window, int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_fwd");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(lse))
    return HD_ERR_INVALID_ARG;
  SfaGeom g;
  hd_status_t st = make_geom(B, L, n, Hq, Hkv, Dh, mode, window, &g);
  if (st != HD_OK) return st;
  const float scale = resolve_scale(softmax_scale, Dh);
  // head dim 256: one query tile per CTA (its O takes half of TMEM)
  if (Dh == 256) return cuda_status(hdsfa::launch_sfa_fwd_tc256(q, k, v, o, lse, g, scale, dev_status, stream));
  return cuda_status(hdsfa::launch_sfa_fwd_tc(q, k, v, o, lse, g, Dh, scale, dev_status, stream));
}

size_t sfa_bwd_workspace_bytes(int B, int L, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode) {
  SfaGeom g;
  if (make_geom(B, L, n, Hq, Hkv, Dh, mode, mode == SFA_LOCAL ? 1 : 0, &g) != HD_OK) return 0;
  return ws_bytes(g, Dh);
}

hd_status_t sfa_bwd_prep(const void* o, const void* dout, const float* lse, int B, int L, int n, int Hq,
                         int Hkv, int Dh, sfa_mode_t mode, void* workspace, size_t workspace_bytes,
                         cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_bwd_prep");
  if (!aligned16(o) || !aligned16(dout) || !aligned16(lse)) return HD_ERR_INVALID_ARG;
  SfaGeom g;
  hd_status_t st = make_geom(B, L, n, Hq, Hkv, Dh, mode, mode == SFA_LOCAL ? 1 : 0, &g);
  if (st != HD_OK) return st;
  BwdWs ws;
  if ((st = split_ws(g, Dh, workspace, workspace_bytes, &ws)) != HD_OK) return st;
  return cuda_status(hdsfa::launch_sfa_bwd_prep(o, dout, lse, ws.lse2, ws.delta, ws.dq, query_geom(g), Dh, stream));
}

hd_status_t sfa_bwd_row_terms(const void* o, const void* dout, const float* lse, int B, int L, int n, int Hq,
                              int Hkv, int Dh, sfa_mode_t mode, void* workspace, size_t workspace_bytes,
                              cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_bwd_row_terms");
  if (!aligned16(o) || !aligned16(dout) || !aligned16(lse)) return HD_ERR_INVALID_ARG;
  SfaGeom g;
  hd_status_t st = make_geom(B, L, n, Hq, Hkv, Dh, mode, mode == SFA_LOCAL ? 1 : 0, &g);
  if (st != HD_OK) return st;
  BwdWs ws;
  if ((st = split_ws(g, Dh, workspace, workspace_bytes, &ws)) != HD_OK) return st;
  return cuda_status(
      hdsfa::launch_sfa_bwd_prep(o, dout, lse, ws.lse2, ws.delta, ws.dq, query_geom(g), Dh, stream, false));
}

hd_status_t sfa_bwd_clear(int B, int L, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode, void* workspace,
                          size_t workspace_bytes, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_bwd_clear");
  SfaGeom g;
  hd_status_t st = make_geom(B, L, n, Hq, Hkv, Dh, mode, mode == SFA_LOCAL ? 1 : 0, &g);
  if (st != HD_OK) return st;
  BwdWs ws;
  if ((st = split_ws(g, Dh, workspace, workspace_bytes, &ws)) != HD_OK) return st;
  return cuda_status(hdsfa::launch_sfa_bwd_clear(ws.dq, query_geom(g), Dh, stream));
}

hd_status_t sfa_bwd_main(const void* q, const void* k, const void* v, const void* dout, void* dk, void* dv,
                         int B, int L, int n, int Hq, int Hkv, int Dh, float softmax_scale,
                         sfa_mode_t mode, int window, void* workspace, size_t workspace_bytes,
                         int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_bwd_main");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(dout) || !aligned16(dk) ||
      !aligned16(dv))
    return HD_ERR_INVALID_ARG;
  SfaGeom g;
  hd_status_t st = make_geom(B, L, n, Hq, Hkv, Dh, mode, window, &g);
  if (st != HD_OK) return st;
  BwdWs ws;
  if ((st = split_ws(g, Dh, workspace, workspace_bytes, &ws)) != HD_OK) return st;
  // the fp32 sums of dQ are added into the workspace's accumulator
  return cuda_status(main_pass(q, k, v, dout, nullptr, dk, dv, ws, g, Dh, resolve_scale(softmax_scale, Dh), dev_status,
                               stream));
}

hd_status_t sfa_bwd_finalize(void* dq, int B, int L, int n, int Hq, int Hkv, int Dh,
                             float softmax_scale, sfa_mode_t mode, void* workspace,
                             size_t workspace_bytes, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_bwd_finalize");
  if (!aligned16(dq)) return HD_ERR_INVALID_ARG;
  SfaGeom g;
  hd_status_t st = make_geom(B, L, n, Hq, Hkv, Dh, mode, mode == SFA_LOCAL ? 1 : 0, &g);
  if (st != HD_OK) return st;
  BwdWs ws;
  if ((st = split_ws(g, Dh, workspace, workspace_bytes, &ws)) != HD_OK) return st;
  return cuda_status(hdsfa::launch_sfa_bwd_finalize(dq, ws.dq, query_geom(g), Dh,
                                                    resolve_scale(softmax_scale, Dh), stream));
}

hd_status_t sfa_bwd(const void* q, const void* k, const void* v, const void* o, const float* lse,
                    const void* dout, void* dq, void* dk, void* dv, int B, int L, int n, int Hq,
                    int Hkv, int Dh, float softmax_scale, sfa_mode_t mode, int window,
                    void* workspace, size_t workspace_bytes, int32_t* dev_status,
                    cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_bwd");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(lse) ||
      !aligned16(dout) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv))
    return HD_ERR_INVALID_ARG;
  SfaGeom g;
  hd_status_t st = make_geom(B, L, n, Hq, Hkv, Dh, mode, window, &g);
  if (st != HD_OK) return st;
  BwdWs ws;
  if ((st = split_ws(g, Dh, workspace, workspace_bytes, &ws)) != HD_OK) return st;
  return cuda_status(backward(q, k, v, o, lse, dout, dq, dk, dv, ws, g, Dh, resolve_scale(softmax_scale, Dh), dev_status,
                              stream));
}

// Sizes of a decode step: max_tokens bounds every sequence's length and the cache
// capacity Lcap bounds max_tokens.
static hd_status_t decode_sizes(int B, int maxT, int Lcap, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode,
                                int window) {
  if (B <= 0 || maxT <= 0 || Lcap <= 0 || n <= 0 || Hq <= 0 || Hkv <= 0 || Dh <= 0) return HD_ERR_INVALID_ARG;
  if (Hq % Hkv != 0 || maxT > Lcap) return HD_ERR_INVALID_ARG;
  if (mode != SFA_WITHIN && mode != SFA_CROSS && mode != SFA_LOCAL) return HD_ERR_INVALID_ARG;
  if (mode == SFA_LOCAL && window <= 0) return HD_ERR_INVALID_ARG;
  if (Dh != 64 && Dh != 128 && Dh != 256) return HD_ERR_UNSUPPORTED;
  if ((long long)Lcap * n > (1LL << 30) || (long long)n * Hq > (1LL << 20)) return HD_ERR_UNSUPPORTED;
  return HD_OK;
}

size_t sfa_decode_workspace_bytes(int B, int max_tokens, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode,
                                  int window) {
  if (decode_sizes(B, max_tokens, max_tokens, n, Hq, Hkv, Dh, mode, window) != HD_OK) return 0;
  return hdsfa::decode_ws_bytes(hdsfa::decode_plan(B, max_tokens, n, Hq, Hkv, Dh, mode, window));
}

hd_status_t sfa_decode(const void* q, const void* k_cache, const void* v_cache, const int32_t* lens, void* o,
                       float* lse, int B, int max_tokens, int Lcap, int n, int Hq, int Hkv, int Dh,
                       float softmax_scale, sfa_mode_t mode, int window, void* workspace, size_t workspace_bytes,
                       int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_decode");
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(o)) return HD_ERR_INVALID_ARG;
  if (lens == nullptr || (reinterpret_cast<uintptr_t>(lens) & 3u) != 0) return HD_ERR_INVALID_ARG;
  if (lse != nullptr && (reinterpret_cast<uintptr_t>(lse) & 3u) != 0) return HD_ERR_INVALID_ARG;
  hd_status_t st = decode_sizes(B, max_tokens, Lcap, n, Hq, Hkv, Dh, mode, window);
  if (st != HD_OK) return st;
  const size_t need = sfa_decode_workspace_bytes(B, max_tokens, n, Hq, Hkv, Dh, mode, window);
  if (!aligned16(workspace) || workspace_bytes < need) return HD_ERR_WORKSPACE;
  return cuda_status(hdsfa::launch_sfa_decode(q, k_cache, v_cache, lens, o, lse, B, max_tokens, Lcap, n, Hq, Hkv,
                                              Dh, resolve_scale(softmax_scale, Dh), (int)mode,
                                              mode == SFA_LOCAL ? window : 0, workspace, dev_status, stream));
}

hd_status_t sfa_kv_append(const void* k_new, const void* v_new, void* k_cache, void* v_cache, const int32_t* lens,
                          int B, int Lcap, int n, int Hkv, int Dh, int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_kv_append");
  if (!aligned16(k_new) || !aligned16(v_new) || !aligned16(k_cache) || !aligned16(v_cache))
    return HD_ERR_INVALID_ARG;
  if (lens == nullptr || (reinterpret_cast<uintptr_t>(lens) & 3u) != 0) return HD_ERR_INVALID_ARG;
  if (B <= 0 || Lcap <= 0 || n <= 0 || Hkv <= 0 || Dh <= 0 || Dh % 8 != 0) return HD_ERR_INVALID_ARG;
  if ((long long)Lcap * n > (1LL << 30)) return HD_ERR_UNSUPPORTED;
  return cuda_status(hdsfa::launch_kv_append(k_new, v_new, k_cache, v_cache, lens, B, Lcap, n, Hkv, Dh,
                                             dev_status, stream));
}

// ---- packed prompts ----
// Geometry of N packed tokens (one sequence of them, of which the kernels take pieces), rows of an
// entry of their list and the most entries there can be.
static hd_status_t packed_sizes(int B, int N, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode, int window, SfaGeom* g,
                                int* tile_rows, long long* max_items) {
  if (B <= 0) return HD_ERR_INVALID_ARG;
  hd_status_t st = make_geom(1, N, n, Hq, Hkv, Dh, mode, window, g);
  if (st != HD_OK) return st;
  if (mode == SFA_WITHIN_NAIVE) return HD_ERR_UNSUPPORTED;
  *tile_rows = (Hq / Hkv) % 2 == 0 ? 128 : 256;  // two query tiles: of two heads, or of one
  *max_items = hdsfa::packed_max_items(B, N, n / g->ns, *tile_rows);
  // the entries of every head and stream are counted in 32 bits
  if (*max_items * Hq * g->ns >= (1LL << 30)) return HD_ERR_UNSUPPORTED;
  return HD_OK;
}

size_t sfa_fwd_packed_workspace_bytes(int B, int N, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode) {
  SfaGeom g;
  int rows;
  long long items;
  if (packed_sizes(B, N, n, Hq, Hkv, Dh, mode, mode == SFA_LOCAL ? 1 : 0, &g, &rows, &items) != HD_OK) return 0;
  return (size_t)(items + 1) * sizeof(hdsfa::PackedItem);
}

hd_status_t sfa_fwd_packed(const void* q, const void* k, const void* v, void* o, float* lse, const int32_t* offsets,
                           int B, int N, int n, int Hq, int Hkv, int Dh, float softmax_scale, sfa_mode_t mode, int window,
                           void* workspace, size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_fwd_packed");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(lse)) return HD_ERR_INVALID_ARG;
  if (!aligned_to(offsets, 4) || !aligned_or_null(dev_status, 4)) return HD_ERR_INVALID_ARG;
  SfaGeom g;
  int rows;
  long long items;
  hd_status_t st = packed_sizes(B, N, n, Hq, Hkv, Dh, mode, window, &g, &rows, &items);
  if (st != HD_OK) return st;
  if (!aligned16(workspace) || workspace_bytes < (size_t)(items + 1) * sizeof(hdsfa::PackedItem)) return HD_ERR_WORKSPACE;
  int32_t* count = static_cast<int32_t*>(workspace);
  hdsfa::PackedItem* list = static_cast<hdsfa::PackedItem*>(workspace) + 1;
  const bool shared = hdsfa::packed_shared(Dh, B, N, n / g.ns);
  cudaError_t e = hdsfa::launch_packed_plan(offsets, B, N, n / g.ns, rows, g.window, shared, list, count, dev_status, stream);
  if (e != cudaSuccess) return cuda_status(e);
  const float scale = resolve_scale(softmax_scale, Dh);
  const hdsfa::PackedList pl{list, count};
  if (Dh == 256) return cuda_status(hdsfa::launch_sfa_fwd_packed_tc256(q, k, v, o, lse, g, scale, pl, offsets, items, dev_status, stream));
  return cuda_status(hdsfa::launch_sfa_fwd_packed_tc(q, k, v, o, lse, g, Dh, scale, pl, offsets, shared, items, dev_status, stream));
}

// ---- paged cache ----
// Sizes of a pool and its tables; n = 1 where rows do not matter.
static hd_status_t page_sizes(int B, int max_pages, int num_pages, int P, int n) {
  if (B <= 0 || max_pages <= 0 || num_pages <= 0 || P <= 0 || n <= 0) return HD_ERR_INVALID_ARG;
  const long long prow = (long long)P * n;
  if (prow > (1LL << 30) || max_pages * prow > (1LL << 30) || num_pages * prow >= (1LL << 31) ||
      (long long)B * max_pages >= (1LL << 31))
    return HD_ERR_UNSUPPORTED;
  return HD_OK;
}

static hd_status_t append_paged(const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                                const int32_t* page_table, const int32_t* lens, const int32_t* offsets,
                                const int32_t* served, int B, int N, int num_pages, int page_tokens, int max_pages, int n,
                                int Hkv, int Dh, int32_t* dev_status, cudaStream_t stream) {
  if (!aligned16(k_pages) || !aligned16(v_pages)) return HD_ERR_INVALID_ARG;
  if (!aligned_to(page_table, 4) || !aligned_to(lens, 4) || !aligned_or_null(offsets, 4) || !aligned_or_null(dev_status, 4))
    return HD_ERR_INVALID_ARG;
  if (N < 0 || Hkv <= 0 || Dh <= 0 || Dh % 8 != 0 || (offsets == nullptr && N != B)) return HD_ERR_INVALID_ARG;
  hd_status_t st = page_sizes(B, max_pages, num_pages, page_tokens, n);
  if (st != HD_OK) return st;
  if ((long long)N * n >= (1LL << 31) || (long long)Hkv * Dh > (1LL << 24) || (long long)n * Hkv * Dh > (1LL << 24))
    return HD_ERR_UNSUPPORTED;
  if (N == 0) return HD_OK;
  if (!aligned16(k_new) || !aligned16(v_new)) return HD_ERR_INVALID_ARG;
  return cuda_status(hdsfa::launch_kv_append_paged(k_new, v_new, k_pages, v_pages, page_table, lens, offsets, served, B,
                                                   N, num_pages, page_tokens, max_pages, n, Hkv, Dh, dev_status, stream));
}

hd_status_t sfa_kv_append_paged(const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                                const int32_t* page_table, const int32_t* lens, const int32_t* offsets, int B, int N,
                                int num_pages, int page_tokens, int max_pages, int n, int Hkv, int Dh,
                                int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_kv_append_paged");
  return append_paged(k_new, v_new, k_pages, v_pages, page_table, lens, offsets, nullptr, B, N, num_pages, page_tokens,
                      max_pages, n, Hkv, Dh, dev_status, stream);
}

hd_status_t sfa_kv_append_paged_served(const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                                       const int32_t* page_table, const int32_t* lens, const int32_t* offsets,
                                       const int32_t* served, int B, int N, int num_pages, int page_tokens, int max_pages,
                                       int n, int Hkv, int Dh, int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_kv_append_paged_served");
  if (!aligned_to(served, 4)) return HD_ERR_INVALID_ARG;
  return append_paged(k_new, v_new, k_pages, v_pages, page_table, lens, offsets, served, B, N, num_pages, page_tokens,
                      max_pages, n, Hkv, Dh, dev_status, stream);
}

static hd_status_t decode_paged_sizes(int B, int maxT, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode, int window) {
  hd_status_t st = decode_sizes(B, maxT, maxT, n, Hq, Hkv, Dh, mode, window);
  if (st != HD_OK) return st;
  const long long groups = ((long long)n * (Hq / Hkv) + 31) / 32;  // a grid's limits
  return B > 65535 || Hkv * groups > 65535 ? HD_ERR_UNSUPPORTED : HD_OK;
}

// A window of every position sees them all: larger ones are cut to it, so that sums of a position
// and the window stay in 32 bits.
static int cut_window(sfa_mode_t mode, int window, long long positions) {
  return mode != SFA_LOCAL ? 0 : window < positions ? window : (int)positions;
}

size_t sfa_decode_paged_workspace_bytes(int B, int max_tokens, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode,
                                        int window) {
  if (decode_paged_sizes(B, max_tokens, n, Hq, Hkv, Dh, mode, window) != HD_OK) return 0;
  return hdsfa::decode_paged_ws_bytes(B, max_tokens, n, Hq, Hkv, Dh, mode,
                                      cut_window(mode, window, (long long)max_tokens * n));
}

hd_status_t sfa_decode_paged(const void* q, const void* k_pages, const void* v_pages, const int32_t* page_table,
                             const int32_t* lens, void* o, float* lse, int B, int max_tokens, int num_pages,
                             int page_tokens, int max_pages, int n, int Hq, int Hkv, int Dh, float softmax_scale,
                             sfa_mode_t mode, int window, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                             cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_decode_paged");
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(o)) return HD_ERR_INVALID_ARG;
  if (!aligned_to(page_table, 4) || !aligned_to(lens, 4) || !aligned_or_null(lse, 4) || !aligned_or_null(dev_status, 4))
    return HD_ERR_INVALID_ARG;
  hd_status_t st = decode_paged_sizes(B, max_tokens, n, Hq, Hkv, Dh, mode, window);
  if (st != HD_OK || (st = page_sizes(B, max_pages, num_pages, page_tokens, n)) != HD_OK) return st;
  if (max_tokens > max_pages * page_tokens) return HD_ERR_INVALID_ARG;
  const size_t need = sfa_decode_paged_workspace_bytes(B, max_tokens, n, Hq, Hkv, Dh, mode, window);
  if (!aligned16(workspace) || workspace_bytes < need) return HD_ERR_WORKSPACE;
  return cuda_status(hdsfa::launch_sfa_decode_paged(
      q, k_pages, v_pages, page_table, lens, o, lse, B, max_tokens, num_pages, page_tokens, max_pages, n, Hq, Hkv, Dh,
      resolve_scale(softmax_scale, Dh), (int)mode, cut_window(mode, window, (long long)max_tokens * n), workspace,
      workspace_bytes, dev_status, stream));
}

// ---- paged cache in 8 bits ----
static hd_status_t q8_sizes(int B, int max_pages, int num_pages, int P, int n, int Hkv, int Dh, int T) {
  if (Hkv <= 0 || Dh <= 0 || Dh % 16 != 0 || T <= 0) return HD_ERR_INVALID_ARG;
  hd_status_t st = page_sizes(B, max_pages, num_pages, P, n);
  if (st != HD_OK) return st;
  if (P % T != 0) return HD_ERR_INVALID_ARG;
  if ((long long)Hkv * Dh > (1LL << 24) || (long long)n * Hkv * Dh > (1LL << 24) || (long long)T * n * Dh > (1LL << 30) ||
      Hkv > 32767 || (long long)num_pages * P * n >= (1LL << 32) / Hkv)
    return HD_ERR_UNSUPPORTED;
  return HD_OK;
}

hd_status_t sfa_kv_append_paged_q8(const void* k_new, const void* v_new, void* k_pages, void* v_pages,
                                   uint8_t* k_scales, uint8_t* v_scales, const int32_t* page_table, const int32_t* lens,
                                   const int32_t* offsets, const int32_t* served, int B, int N, int num_pages,
                                   int page_tokens, int max_pages, int n, int Hkv, int Dh, int block_tokens,
                                   int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_kv_append_paged_q8");
  if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(k_scales) || !aligned16(v_scales)) return HD_ERR_INVALID_ARG;
  if (!aligned_to(page_table, 4) || !aligned_to(lens, 4) || !aligned_or_null(offsets, 4) || !aligned_or_null(served, 4) ||
      !aligned_or_null(dev_status, 4))
    return HD_ERR_INVALID_ARG;
  if (N < 0 || (offsets == nullptr && N != B)) return HD_ERR_INVALID_ARG;
  hd_status_t st = q8_sizes(B, max_pages, num_pages, page_tokens, n, Hkv, Dh, block_tokens);
  if (st != HD_OK) return st;
  if ((long long)N * n >= (1LL << 31)) return HD_ERR_UNSUPPORTED;
  if (N == 0) return HD_OK;
  if (!aligned16(k_new) || !aligned16(v_new)) return HD_ERR_INVALID_ARG;
  return cuda_status(hdsfa::launch_kv_append_paged_q8(k_new, v_new, k_pages, v_pages, k_scales, v_scales, page_table, lens,
                                                      offsets, served, B, N, num_pages, page_tokens, max_pages, n, Hkv, Dh,
                                                      block_tokens, dev_status, stream));
}

hd_status_t sfa_kv_read_paged_q8(const void* k_pages, const void* v_pages, const uint8_t* k_scales,
                                 const uint8_t* v_scales, const int32_t* page_table, const int32_t* lens,
                                 const int32_t* offsets, void* k, void* v, int B, int N, int num_pages, int page_tokens,
                                 int max_pages, int n, int Hkv, int Dh, int block_tokens, int32_t* dev_status,
                                 cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_kv_read_paged_q8");
  if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(k_scales) || !aligned16(v_scales)) return HD_ERR_INVALID_ARG;
  if (!aligned_to(page_table, 4) || !aligned_to(lens, 4) || !aligned_to(offsets, 4) || !aligned_or_null(dev_status, 4))
    return HD_ERR_INVALID_ARG;
  if (N < 0) return HD_ERR_INVALID_ARG;
  hd_status_t st = q8_sizes(B, max_pages, num_pages, page_tokens, n, Hkv, Dh, block_tokens);
  if (st != HD_OK) return st;
  if ((long long)N * n >= (1LL << 31)) return HD_ERR_UNSUPPORTED;
  if (N == 0) return HD_OK;
  if (!aligned16(k) || !aligned16(v)) return HD_ERR_INVALID_ARG;
  return cuda_status(hdsfa::launch_kv_read_paged_q8(k_pages, v_pages, k_scales, v_scales, page_table, lens, offsets, k, v, B,
                                                    N, num_pages, page_tokens, max_pages, n, Hkv, Dh, block_tokens,
                                                    dev_status, stream));
}

static hd_status_t decode_q8_sizes(int B, int maxT, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode, int window) {
  hd_status_t st = decode_paged_sizes(B, maxT, n, Hq, Hkv, Dh, mode, window);
  if (st != HD_OK) return st;
  const long long groups = ((long long)n * (Hq / Hkv) + 63) / 64;
  return (long long)B * Hkv * groups > (1LL << 30) ? HD_ERR_UNSUPPORTED : HD_OK;  // CTAs of one split
}

size_t sfa_decode_paged_q8_workspace_bytes(int B, int max_tokens, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode,
                                           int window) {
  if (decode_q8_sizes(B, max_tokens, n, Hq, Hkv, Dh, mode, window) != HD_OK) return 0;
  return hdsfa::decode_paged_q8_ws_bytes(B, max_tokens, n, Hq, Hkv, Dh, mode,
                                         cut_window(mode, window, (long long)max_tokens * n));
}

hd_status_t sfa_decode_paged_q8(const void* q, const void* k_pages, const void* v_pages, const uint8_t* k_scales,
                                const uint8_t* v_scales, const int32_t* page_table, const int32_t* lens, void* o,
                                float* lse, int B, int max_tokens, int num_pages, int page_tokens, int max_pages, int n,
                                int Hq, int Hkv, int Dh, int block_tokens, float softmax_scale, sfa_mode_t mode,
                                int window, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                                cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_decode_paged_q8");
  if (!aligned16(q) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(o) || !aligned16(k_scales) ||
      !aligned16(v_scales))
    return HD_ERR_INVALID_ARG;
  if (!aligned_to(page_table, 4) || !aligned_to(lens, 4) || !aligned_or_null(lse, 4) || !aligned_or_null(dev_status, 4))
    return HD_ERR_INVALID_ARG;
  hd_status_t st = decode_q8_sizes(B, max_tokens, n, Hq, Hkv, Dh, mode, window);
  if (st != HD_OK || (st = q8_sizes(B, max_pages, num_pages, page_tokens, n, Hkv, Dh, block_tokens)) != HD_OK) return st;
  if (max_tokens > max_pages * page_tokens) return HD_ERR_INVALID_ARG;
  const int w = cut_window(mode, window, (long long)max_tokens * n);
  const size_t need = hdsfa::decode_paged_q8_ws_bytes(B, max_tokens, n, Hq, Hkv, Dh, mode, w);
  if (!aligned16(workspace) || workspace_bytes < need) return HD_ERR_WORKSPACE;
  return cuda_status(hdsfa::launch_sfa_decode_paged_q8(
      q, k_pages, v_pages, k_scales, v_scales, page_table, lens, o, lse, B, max_tokens, num_pages, page_tokens, max_pages, n,
      Hq, Hkv, Dh, block_tokens, resolve_scale(softmax_scale, Dh), (int)mode, w, workspace, workspace_bytes, dev_status,
      stream));
}

hd_status_t hd_pages_copy_q8(void* k_pages, void* v_pages, uint8_t* k_scales, uint8_t* v_scales, const int32_t* copies,
                             int F, int num_pages, size_t page_bytes, size_t page_scales, int32_t* dev_status,
                             cudaStream_t stream) {
  HD_NVTX_RANGE("hd_pages_copy_q8");
  if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(k_scales) || !aligned16(v_scales) ||
      !aligned_or_null(dev_status, 4))
    return HD_ERR_INVALID_ARG;
  if (F < 0 || num_pages <= 0 || page_bytes == 0 || page_bytes % 16 != 0 || page_scales == 0) return HD_ERR_INVALID_ARG;
  if (page_bytes > (size_t)1 << 34 || page_scales > (size_t)1 << 30) return HD_ERR_UNSUPPORTED;
  if (F == 0) return HD_OK;
  if (!aligned_to(copies, 8)) return HD_ERR_INVALID_ARG;
  return cuda_status(hdsfa::launch_pages_copy_q8(k_pages, v_pages, k_scales, v_scales, copies, F, num_pages, page_bytes,
                                                 (int)page_scales, dev_status, stream));
}

// ---- who holds which page ----
static hd_status_t page_state_args(const int32_t* refs, const int32_t* table, const int32_t* lens, int B, int max_pages,
                                   int num_pages, int P, const int32_t* dev_status) {
  if (!aligned16(refs) || !aligned_to(table, 4) || !aligned_to(lens, 4) || !aligned_or_null(dev_status, 4))
    return HD_ERR_INVALID_ARG;
  return page_sizes(B, max_pages, num_pages, P, 1);
}

size_t hd_pages_workspace_bytes(int B, int num_pages) {
  return B <= 0 || num_pages <= 0 ? 0 : hdsfa::pages_ws_bytes(B, num_pages);
}

static hd_status_t pages_grow(int32_t* refs, int32_t* page_table, int32_t* lens, const int32_t* add, int32_t* served,
                              int B, int max_pages, int num_pages, int page_tokens, void* workspace,
                              size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream) {
  hd_status_t st = page_state_args(refs, page_table, lens, B, max_pages, num_pages, page_tokens, dev_status);
  if (st != HD_OK) return st;
  if (!aligned_to(add, 4)) return HD_ERR_INVALID_ARG;
  if (!aligned16(workspace) || workspace_bytes < hd_pages_workspace_bytes(B, num_pages)) return HD_ERR_WORKSPACE;
  return cuda_status(hdsfa::launch_pages_grow(refs, page_table, lens, add, served, B, max_pages, num_pages, page_tokens,
                                              workspace, dev_status, stream));
}

hd_status_t hd_pages_grow(int32_t* refs, int32_t* page_table, int32_t* lens, const int32_t* add, int B, int max_pages,
                          int num_pages, int page_tokens, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                          cudaStream_t stream) {
  HD_NVTX_RANGE("hd_pages_grow");
  return pages_grow(refs, page_table, lens, add, nullptr, B, max_pages, num_pages, page_tokens, workspace, workspace_bytes,
                    dev_status, stream);
}

hd_status_t hd_pages_grow_served(int32_t* refs, int32_t* page_table, int32_t* lens, const int32_t* add, int32_t* served,
                                 int B, int max_pages, int num_pages, int page_tokens, void* workspace,
                                 size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("hd_pages_grow_served");
  if (!aligned_to(served, 4)) return HD_ERR_INVALID_ARG;
  return pages_grow(refs, page_table, lens, add, served, B, max_pages, num_pages, page_tokens, workspace, workspace_bytes,
                    dev_status, stream);
}

hd_status_t hd_pages_fork(int32_t* refs, int32_t* page_table, int32_t* lens, const int32_t* src, const int32_t* dst,
                          const int32_t* tokens, int F, int32_t* copies, int B, int max_pages, int num_pages,
                          int page_tokens, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                          cudaStream_t stream) {
  HD_NVTX_RANGE("hd_pages_fork");
  hd_status_t st = page_state_args(refs, page_table, lens, B, max_pages, num_pages, page_tokens, dev_status);
  if (st != HD_OK) return st;
  if (F < 0 || F > B) return HD_ERR_INVALID_ARG;
  if (F == 0) return HD_OK;
  if (!aligned_to(src, 4) || !aligned_to(dst, 4) || !aligned_or_null(tokens, 4) || !aligned_to(copies, 8))
    return HD_ERR_INVALID_ARG;
  if (!aligned16(workspace) || workspace_bytes < hd_pages_workspace_bytes(B, num_pages)) return HD_ERR_WORKSPACE;
  return cuda_status(hdsfa::launch_pages_fork(refs, page_table, lens, src, dst, tokens, F, copies, B, max_pages,
                                              num_pages, page_tokens, workspace, dev_status, stream));
}

hd_status_t hd_pages_free(int32_t* refs, int32_t* page_table, int32_t* lens, const int32_t* seqs, int F, int B,
                          int max_pages, int num_pages, int page_tokens, int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("hd_pages_free");
  hd_status_t st = page_state_args(refs, page_table, lens, B, max_pages, num_pages, page_tokens, dev_status);
  if (st != HD_OK) return st;
  if (F < 0) return HD_ERR_INVALID_ARG;
  if (F == 0) return HD_OK;
  if (!aligned_to(seqs, 4)) return HD_ERR_INVALID_ARG;
  return cuda_status(hdsfa::launch_pages_free(refs, page_table, lens, seqs, F, B, max_pages, num_pages, page_tokens,
                                              dev_status, stream));
}

hd_status_t hd_pages_compact(const int32_t* refs, const int32_t* page_table, const int32_t* lens, int32_t* new_refs,
                             int32_t* new_table, int32_t* moves, int B, int max_pages, int num_pages, int page_tokens,
                             void* workspace, size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("hd_pages_compact");
  hd_status_t st = page_state_args(refs, page_table, lens, B, max_pages, num_pages, page_tokens, dev_status);
  if (st != HD_OK) return st;
  if (!aligned16(new_refs) || !aligned_to(new_table, 4) || !(num_pages < 2 ? true : aligned_to(moves, 8)))
    return HD_ERR_INVALID_ARG;
  if (!aligned16(workspace) || workspace_bytes < hd_pages_workspace_bytes(B, num_pages)) return HD_ERR_WORKSPACE;
  return cuda_status(hdsfa::launch_pages_compact(refs, page_table, lens, new_refs, new_table, moves, B, max_pages,
                                                 num_pages, page_tokens, workspace, dev_status, stream));
}

hd_status_t hd_pages_copy(void* k_pages, void* v_pages, const int32_t* copies, int F, int num_pages, size_t page_bytes,
                          int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("hd_pages_copy");
  if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned_or_null(dev_status, 4)) return HD_ERR_INVALID_ARG;
  if (F < 0 || num_pages <= 0 || page_bytes == 0 || page_bytes % 16 != 0) return HD_ERR_INVALID_ARG;
  if (page_bytes > (size_t)1 << 34) return HD_ERR_UNSUPPORTED;
  if (F == 0) return HD_OK;
  if (!aligned_to(copies, 8)) return HD_ERR_INVALID_ARG;
  return cuda_status(hdsfa::launch_pages_copy(k_pages, v_pages, copies, F, num_pages, (int)(page_bytes / 16), dev_status,
                                              stream));
}

// ---- final-stream problems (Eq. 2 rows; Sec. 3.1 final-stream-only layers) ----
hd_status_t sfa_fwd_final(const void* q, const void* k, const void* v, void* o, float* lse, int B, int L, int n,
                          int Hq, int Hkv, int Dh, float softmax_scale, sfa_mode_t mode, int window,
                          int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_fwd_final");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(lse))
    return HD_ERR_INVALID_ARG;
  SfaGeom g;
  hd_status_t st = make_final_geom(B, L, n, Hq, Hkv, Dh, mode, window, &g);
  if (st != HD_OK) return st;
  const float scale = resolve_scale(softmax_scale, Dh);
  if (Dh == 256) return cuda_status(hdsfa::launch_sfa_fwd_tc256(q, k, v, o, lse, g, scale, dev_status, stream));
  return cuda_status(hdsfa::launch_sfa_fwd_tc(q, k, v, o, lse, g, Dh, scale, dev_status, stream));
}

size_t sfa_bwd_final_workspace_bytes(int B, int L, int n, int Hq, int Hkv, int Dh, sfa_mode_t mode) {
  SfaGeom g;
  if (make_final_geom(B, L, n, Hq, Hkv, Dh, mode, mode == SFA_LOCAL ? 1 : 0, &g) != HD_OK) return 0;
  return ws_bytes(g, Dh);
}

hd_status_t sfa_bwd_final(const void* q, const void* k, const void* v, const void* o, const float* lse,
                          const void* dout, void* dq, void* dk, void* dv, int B, int L, int n, int Hq, int Hkv,
                          int Dh, float softmax_scale, sfa_mode_t mode, int window, void* workspace,
                          size_t workspace_bytes, int32_t* dev_status, cudaStream_t stream) {
  HD_NVTX_RANGE("sfa_bwd_final");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) || !aligned16(lse) ||
      !aligned16(dout) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv))
    return HD_ERR_INVALID_ARG;
  SfaGeom g;
  hd_status_t st = make_final_geom(B, L, n, Hq, Hkv, Dh, mode, window, &g);
  if (st != HD_OK) return st;

  BwdWs ws;
  if ((st = split_ws(g, Dh, workspace, workspace_bytes, &ws)) != HD_OK) return st;
  return cuda_status(backward(q, k, v, o, lse, dout, dq, dk, dv, ws, g, Dh, resolve_scale(softmax_scale, Dh), dev_status,
                              stream));
}

hd_status_t hd_selftest_bounded_wait(int32_t* dev_status, int32_t* dev_result, cudaStream_t stream) {
  HD_NVTX_RANGE("hd_selftest_bounded_wait");
  if (dev_result == nullptr || (reinterpret_cast<uintptr_t>(dev_result) & 3u) != 0) return HD_ERR_INVALID_ARG;
  if (dev_status != nullptr && (reinterpret_cast<uintptr_t>(dev_status) & 3u) != 0) return HD_ERR_INVALID_ARG;
  return cuda_status(hdsfa::launch_bounded_wait_selftest(dev_status, dev_result, stream));
}

const char* hd_status_string(hd_status_t s) {
  switch (s) {
    case HD_OK: return "HD_OK";
    case HD_ERR_INVALID_ARG: return "HD_ERR_INVALID_ARG: invalid argument";
    case HD_ERR_UNSUPPORTED: return "HD_ERR_UNSUPPORTED: configuration not supported";
    case HD_ERR_CUDA: return "HD_ERR_CUDA: CUDA launch or runtime error";
    case HD_ERR_WORKSPACE: return "HD_ERR_WORKSPACE: workspace missing, misaligned or too small";
    case HD_ERR_TIMEOUT: return "HD_ERR_TIMEOUT: bounded device wait expired";
    case HD_ERR_INDEX: return "HD_ERR_INDEX: index out of range";
    case HD_ERR_SCRATCH_LIMIT:
      return "HD_ERR_SCRATCH_LIMIT: sizes need more workspace than sfa_bwd_noalloc's fixed array";
  }
  return "unknown hd_status_t";
}

}  // extern "C"
