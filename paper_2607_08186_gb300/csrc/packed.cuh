// Packed prompts: sequences of different lengths one behind another, and the list of their query
// tiles that the forward kernels work through.
#pragma once
#include <float.h>

#include "common.cuh"

namespace hdsfa {

// A query tile: `rows` virtual rows of a sequence (SfaGeom) that start at virtual row `first` of
// the packed tensors, and the tile's number among the sequence's.
struct PackedItem {
  int first, rows, tile, unused;
};
struct PackedList {
  const PackedItem* items;  // those with the most key tiles first
  const int32_t* count;
};
// Items that `tokens` packed tokens of B sequences make at most: sum of ceil(rows / tile_rows).
inline long long packed_max_items(int B, int tokens, int mult, int tile_rows) {
  return (long long)tokens * mult / tile_rows + (B < tokens ? B : tokens);
}
cudaError_t launch_packed_plan(const int32_t* offsets, int B, int N, int mult, int tile_rows, int window,
                               PackedItem* items, int32_t* count, int32_t* status, cudaStream_t st);

// What the forward kernels over packed prompts are given besides their tensor maps.
struct PackedArgs {
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* o;
  float* lse;
  SfaGeom g;  // of all packed rows: B = 1, Lv = Lq = rows of a stream's problem
  PackedList list;
  float scale_log2;
  int32_t* status;
  int head_pairs;  // 1: an entry's two query tiles are the same rows of two heads of one K/V group,
                   // 0: two tiles of a head
  int o_wide;      // o is 32-byte aligned
  int per;         // places of a list entry: head slots x streams
  FastDiv d_per, d_ns, d_grp;  // by per, streams, query heads of a K/V head
};
inline PackedArgs make_packed_args(const void* q, const void* k, const void* v, void* o, float* lse, const SfaGeom& g,
                                   float scale, const PackedList& list, int32_t* status) {
  PackedArgs a;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.k = static_cast<const __nv_bfloat16*>(k);
  a.v = static_cast<const __nv_bfloat16*>(v);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse;
  a.g = g;
  a.list = list;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.status = status;
  a.head_pairs = (g.Hq / g.Hkv) % 2 == 0;
  a.o_wide = (reinterpret_cast<uintptr_t>(o) & 31) == 0;
  a.per = (a.head_pairs ? g.Hq / 2 : g.Hq) * g.q_ns;
  a.d_per = make_fast_div((uint32_t)a.per);
  a.d_ns = make_fast_div((uint32_t)g.q_ns);
  a.d_grp = make_fast_div((uint32_t)(g.Hq / g.Hkv));
  return a;
}

// The work at place `pos` of the list (every entry stands for all head slots and streams).
struct PackedEntry {
  int first, rows;  // the sequence's first row and its rows
  int m0, head, stream;
  HD_DEVINLINE PackedEntry(const PackedArgs& a, int pos) {
    const int i = fast_div(pos, a.d_per);
    const PackedItem it = a.list.items[i];
    const int hs = pos - i * a.per, hx = fast_div(hs, a.d_ns);
    first = it.first;
    rows = it.rows;
    stream = hs - hx * a.g.q_ns;
    head = a.head_pairs ? 2 * hx : hx;
    m0 = it.tile * (a.head_pairs ? 128 : 256);
  }
  HD_DEVINLINE int head_of(const PackedArgs& a, int g) const { return a.head_pairs ? head + g : head; }
  HD_DEVINLINE int row0(const PackedArgs& a, int g) const { return a.head_pairs ? m0 : m0 + g * 128; }
};
// Key tiles of 128 [lo, hi] of the query tile at row r0 (hi < lo: no rows).
HD_DEVINLINE int packed_lo(const PackedArgs& a, int r0) { return a.g.window > 0 ? max(0, r0 - a.g.window + 1) / 128 : 0; }
HD_DEVINLINE int packed_hi(int r0, int rows) { return r0 >= rows ? -1 : (min(r0 + 128, rows) - 1) / 128; }
// The place of the k-th piece of work of one of `workers`: the list in rounds of one place each,
// every second round backwards, which evens out the descending sizes.
HD_DEVINLINE int packed_place(int k, int worker, int workers) {
  return k * workers + ((k & 1) ? workers - 1 - worker : worker);
}

// One query row against its visible key rows alone, by one warp on the fp32 units: row(i) is the
// tensor row of the i-th visible key, q, k and v start at the head; o: DH/32 columns a lane, not
// normalised, m: the maximum in log2 units (+inf if the sum l is NaN).
template <int DH, typename Row>
HD_DEVINLINE void visible_row(const __nv_bfloat16* q, const __nv_bfloat16* k, const __nv_bfloat16* v, long long pitch,
                              int keys, Row row, float scale_log2, float* o, float& m, float& l) {
  constexpr int C = DH / 32;
  const int lane = threadIdx.x & 31;
  float qf[C];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    qf[c] = __bfloat162float(q[lane * C + c]);
    o[c] = 0.f;
  }
  m = -INFINITY;
  l = 0.f;
  for (int i = 0; i < keys; ++i) {
    const long long r = row(i);
    if (r < 0) continue;
    const long long off = r * pitch + lane * C;
    float x = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) x += qf[c] * __bfloat162float(k[off + c]);
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    x *= scale_log2;
    const float mn = fmaxf(m, x), mu = mn == -INFINITY ? 0.f : mn, corr = exp2f(m - mu), w = exp2f(x - mu);
    m = mn;
    l = l * corr + w;
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] = o[c] * corr + w * __bfloat162float(v[off + c]);
  }
  if (l != l) m = INFINITY;
}

// A masked key has P = 0, and 0 times an infinity or a NaN of its V row is NaN: whether hidden key
// rows [k0, k1) hold one, so that a row that came out not finite has to be computed again from its
// visible keys.  By a warp.
template <int DH>
HD_DEVINLINE bool hides_not_finite(const __nv_bfloat16* v, long long pitch, int k0, int k1) {
  const int lane = threadIdx.x & 31;
  bool bad = false;
  for (int i = k0 * (DH / 8) + lane; i < k1 * (DH / 8); i += 32) {
    const uint4 x = *reinterpret_cast<const uint4*>(v + (long long)(i / (DH / 8)) * pitch + i % (DH / 8) * 8);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)  // an exponent of all ones in either half
      bad = bad || (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
  }
  return __any_sync(0xffffffffu, bad);
}

// The rows r0 + i (bits i of `rows`) of a query tile that came out not finite: computed again if keys
// of the tile's range [klo, khi) that they do not see hold an infinity or a NaN.  q, k, v, o and lse
// start at row 0 of the sequence (lse at row r0); rows lie qo_pitch, kv_pitch, lse_pitch apart.  One
// warp, which has written the rows before.
template <int DH>
__device__ __noinline__ void recompute_rows(const __nv_bfloat16* q, const __nv_bfloat16* k, const __nv_bfloat16* v,
                                            long long kv_pitch, __nv_bfloat16* o, long long qo_pitch, float* lse,
                                            long long lse_pitch, int r0, unsigned rows, int klo, int khi, int window,
                                            float scale_log2) {
  constexpr int C = DH / 32;
  const int lane = threadIdx.x & 31;
  __syncwarp();  // the rows' first results, stored by other lanes, come before these
  for (; rows; rows &= rows - 1) {
    const int i = __ffs(rows) - 1, r = r0 + i, first = window > 0 ? max(0, r - window + 1) : 0;
    if (!hides_not_finite<DH>(v, kv_pitch, r + 1, khi) && !hides_not_finite<DH>(v, kv_pitch, klo, first)) continue;
    float acc[C], m, l;
    visible_row<DH>(q + r * qo_pitch, k, v, kv_pitch, r + 1 - first, [&](int j) { return (long long)(first + j); },
                    scale_log2, acc, m, l);
    const float inv = 1.f / l;
#pragma unroll
    for (int c = 0; c < C; ++c) o[r * qo_pitch + lane * C + c] = __float2bfloat16_rn(acc[c] * inv);
    if (lane == 0) lse[i * lse_pitch] = (m + log2f(l)) * 0.6931471805599453f;
  }
}

}  // namespace hdsfa
