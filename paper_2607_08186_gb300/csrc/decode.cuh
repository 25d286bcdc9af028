// Shared by the kernels of the decoding step: its arguments, the split over a sequence's positions,
// and the settling of rows that are not finite.
#pragma once
#include "packed.cuh"
#include "pages.cuh"

namespace hdsfa {

typedef __nv_bfloat16 bf16;

namespace dec {
constexpr int NT = 128;      // 4 warps
constexpr int STAGES = 3;
// Head-dim split of the warps: at head dim 256 the four warps form two key groups x two
// halves of the head dim (a warp's O accumulator would not fit its registers whole);
// otherwise four key groups.  A stage holds 16 cached positions per key group.
template <int DH>
constexpr int dsplit() { return DH == 256 ? 2 : 1; }
template <int DH>
constexpr int ktile() { return 64 / dsplit<DH>(); }  // cached positions per pipeline stage
constexpr int RG = 32;       // query rows per CTA at most (two m16 tiles)
constexpr int kMaxSplit = 128;

struct DecodeArgs {
  const bf16* q;        // [B][n][Hq][Dh]
  const bf16* kc;       // [B][Lcap*n][Hkv][Dh]
  const bf16* vc;
  const int32_t* lens;  // [B] tokens in the cache
  bf16* o;              // [B][n][Hq][Dh]
  float* lse;           // [B][Hq][n] or null
  float* part_o;        // [B][Hkv][ngroups][nsplit][rg][Dh]
  float2* part_ml;      // [B][Hkv][ngroups][nsplit][rg]: (max in log2 units, sum)
  int32_t* status;
  int B, Lcap, maxT, n, Hq, Hkv, G, M, ngroups, nsplit, mode, window;
  int rg;               // query rows per row group (the partials' row pitch)
  float scale_log2;
  FastDiv d_nsplit;
  const int32_t* table;  // paged: [B][pg.max_pages]; kc, vc are the pools
  PageGeom pg;
  int tile, piece;       // paged: positions of a tile, in pieces of which none crosses a page
  int split_pages;       // paged: pages of a split of max_tokens tokens
  FastDiv d_G, d_n, d_tile;  // paged
};

// What a partial's (max, sum) says beyond that: the split met a page that is not in the pool.
constexpr float kBadPage = -1.f;  // as its sum

// Both kernels are launched early (launch_early's attribute): the decode kernel lets the
// combine kernel start at once, so the combine's launch and start overlap its tail.

// Visible position range [lo, hi) of a sequence of T tokens (the new token's rows
// see nothing outside it; per-row conditions are applied per element).
HD_DEVINLINE void seq_range(const DecodeArgs& a, int T, int& lo, int& hi) {
  hi = T * a.n;
  lo = a.mode == SFA_LOCAL ? max(0, (T - 1) * a.n - a.window + 1) : 0;
}

// One row's partial over the visible positions of [k0, k1), by one warp on the fp32 units: lane
// i holds DH/32 columns.  Only visible rows of K and V are read.
template <int DH>
__device__ __noinline__ void exact_row(const DecodeArgs& a, int b, int g, int r, int T, int k0, int k1, float* po,
                                       float2* pml) {
  constexpr int C = DH / 32;
  const int lane = threadIdx.x & 31, s = r / a.G, h = g * a.G + r % a.G, pq = (T - 1) * a.n + s;
  int p = a.mode == SFA_LOCAL ? max(k0, pq - a.window + 1) : k0, step = 1;
  if (a.mode == SFA_WITHIN) {
    step = a.n;
    p += (s + a.n - p % a.n) % a.n;
  }
  const int end = min(k1, pq + 1), keys = p < end ? (end - p + step - 1) / step : 0;
  float o[C], m, l;
  visible_row<DH>(a.q + (((long long)b * a.n + s) * a.Hq + h) * DH, a.kc + g * DH, a.vc + g * DH, (long long)a.Hkv * DH,
                  keys, [&](int i) { return (long long)page_row(a.pg, a.table + (long long)b * a.pg.max_pages, p + i * step); },
                  a.scale_log2, o, m, l);
#pragma unroll
  for (int c = 0; c < C; ++c) po[lane * C + c] = o[c];
  if (lane == 0) *pml = make_float2(m, l);
}

// Positions [k0, k1) of split c of a sequence of T tokens, in whole tiles of `kt`
// positions: the sequence's own range over all nsplit splits, not a share of max_tokens, so
// that a batch of different lengths keeps every CTA busy (16 sequences of 8k to 32k tokens,
// cross-stream: 815 -> 779 us).  Empty for lengths outside [1, max_tokens] and for splits
// past the range.  (32-bit with a multiplication for the division: in 64 bits this cost a
// 30 us step 3 us.)
// Paged, the first tile starts at a multiple of the tile (its positions before the window are
// masked), so that no piece of a tile crosses a page.
template <bool PAGED = false>
HD_DEVINLINE void split_range(const DecodeArgs& a, int T, int c, int kt, int& k0, int& k1) {
  k0 = k1 = 0;
  if (T < 1 || T > a.maxT) return;
  int lo, hi;
  seq_range(a, T, lo, hi);
  if (PAGED) lo = fast_div(lo, a.d_tile) * kt;
  const int tiles = PAGED ? fast_div(hi - lo + kt - 1, a.d_tile) : (hi - lo + kt - 1) / kt, per = fast_div(tiles + a.nsplit - 1, a.d_nsplit);
  if ((long long)c * per >= tiles) return;
  k0 = lo + c * per * kt;
  k1 = min(k0 + per * kt, hi);
}
}  // namespace dec

// The tcgen05 kernel over a paged cache (head dim 256), and the combine kernel after either.
cudaError_t launch_decode_paged_tc(const dec::DecodeArgs& a, cudaStream_t st);
cudaError_t launch_combine_paged(const dec::DecodeArgs& a, int Dh, cudaStream_t st);

}  // namespace hdsfa
