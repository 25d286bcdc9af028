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
  float* part_o;        // [B][Hkv][ngroups][nsplit][rg][Dh]; paged: [B * nsplit][Hkv][ngroups][rg][Dh]
  float2* part_ml;      // the same without [Dh]: (max in log2 units, sum)
  int32_t* status;
  int B, Lcap, maxT, n, Hq, Hkv, G, M, ngroups, nsplit, mode, window;
  int rg;               // query rows per row group (the partials' row pitch)
  float scale_log2;
  FastDiv d_nsplit;
  const int32_t* table;  // paged: [B][pg.max_pages]; kc, vc are the pools
  PageGeom pg;
  int tile, piece;       // paged: positions of a tile, in pieces of which none crosses a page
  FastDiv d_G, d_n, d_tile;  // paged
  // paged: the grid is linear, a split's K/V heads (x row groups) together, since their rows are
  FastDiv d_heads;
  // paged: the B * nsplit splits are shared out by the sequences' lengths (PagedSplit); share [B]: the
  // first split of each sequence and their number, for the combine kernel
  int balanced;
  int2* share;
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

// Split x of the B * nsplit of a paged batch (tensor-core kernel): sequence, its tokens and the
// positions [k0, k1), found by a whole warp.  In general split x is the (x mod nsplit)-th of sequence
// x / nsplit.  Balanced (several sequences, long splits), a split is `per` tiles of whichever sequence,
// with the least `per` (to 1/16) at which all splits suffice.
constexpr int kBalancedSeqs = 128;
struct PagedSplit {
  int b, T, k0, k1;
  HD_DEVINLINE PagedSplit(const DecodeArgs& a, int x, bool report) {
    k0 = k1 = 0;
    if (!a.balanced) {
      b = fast_div(x, a.d_nsplit);
      T = a.lens[b];
      split_range<true>(a, T, x - b * a.nsplit, a.tile, k0, k1);
      return;
    }
    constexpr int NI = kBalancedSeqs / 32;
    const int lane = threadIdx.x & 31, nb = (a.B + 31) / 32, S = a.B * a.nsplit;
    int len[NI], tiles[NI], total = 0, most = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int q = i * 32 + lane;
      len[i] = i < nb && q < a.B ? a.lens[q] : 0;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      tiles[i] = 0;
      if (len[i] >= 1 && len[i] <= a.maxT) {
        int lo, hi;
        seq_range(a, len[i], lo, hi);
        tiles[i] = fast_div(hi - fast_div(lo, a.d_tile) * a.tile + a.tile - 1, a.d_tile);
      }
      total += tiles[i];
      most = max(most, tiles[i]);
    }
    total = __reduce_add_sync(0xffffffffu, total);
    most = __reduce_max_sync(0xffffffffu, most);
    // the least `per` is between these two: sum ceil(tiles / per) <= total / per + B
    unsigned least = max(1u, max((total + (unsigned)S - 1) / S, (most + (unsigned)kMaxSplit - 1) / kMaxSplit));
    unsigned per = max(least, (total + (unsigned)(S - a.B) - 1) / (S - a.B));
    for (int step = 0; step < 4 && least < per; ++step) {
      const unsigned mid = (least + per) / 2;
      unsigned need = 0;
#pragma unroll
      for (int i = 0; i < NI; ++i)
        if (i < nb) need += (tiles[i] + mid - 1) / mid;
      if (__reduce_add_sync(0xffffffffu, need) <= (unsigned)S) per = mid;
      else least = mid + 1;
    }
    int before = 0;
    b = T = 0;
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      if (i >= nb) break;
      const int n = (int)((tiles[i] + per - 1) / per);
      int upto = n;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += y;
      }
      const int first = before + upto - n;
      if (report && i * 32 + lane < a.B) a.share[i * 32 + lane] = make_int2(first, n);
      const unsigned hit = __ballot_sync(0xffffffffu, first <= x && x < first + n);
      if (hit) {
        const int l = __ffs(hit) - 1;
        b = i * 32 + l;
        T = __shfl_sync(0xffffffffu, len[i], l);
        int lo, hi;
        seq_range(a, T, lo, hi);
        const int step = (int)per * a.tile;
        k0 = fast_div(lo, a.d_tile) * a.tile + (x - __shfl_sync(0xffffffffu, first, l)) * step;
        k1 = hi - k0 < step ? hi : k0 + step;
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
  }
};
}  // namespace dec

// The tcgen05 kernel over a paged cache (head dims 128 and 256) with the combine kernel, and the
// combine kernel alone.
cudaError_t launch_decode_paged_tc(const dec::DecodeArgs& a, int Dh, cudaStream_t st);
cudaError_t launch_combine_paged(const dec::DecodeArgs& a, int Dh, cudaStream_t st);

}  // namespace hdsfa
