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
  for (int i0 = 0; i0 < keys; i0 += 4) {  // four keys' loads and sums in flight
    long long off[4];
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const long long r = i0 + e < keys ? row(i0 + e) : -1;
      off[e] = r < 0 ? -1 : r * pitch + lane * C;
      x[e] = 0.f;
      if (off[e] >= 0)
#pragma unroll
        for (int c = 0; c < C; ++c) x[e] += qf[c] * __bfloat162float(k[off[e] + c]);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] += __shfl_xor_sync(0xffffffffu, x[e], d);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (off[e] < 0) continue;
      x[e] *= scale_log2;
      const float mn = fmaxf(m, x[e]), mu = mn == -INFINITY ? 0.f : mn, corr = exp2f(m - mu), w = exp2f(x[e] - mu);
      m = mn;
      l = l * corr + w;
#pragma unroll
      for (int c = 0; c < C; ++c) o[c] = o[c] * corr + w * __bfloat162float(v[off[e] + c]);
    }
  }
  if (l != l) m = INFINITY;
}

// Eight bf16 values, all of them finite: no exponent is all ones.
HD_DEVINLINE bool finite8(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  bool bad = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) bad = bad || (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
  return !bad;
}

// A masked key has P = 0, and 0 times an infinity or a NaN of its V row is NaN: whether hidden key
// rows [k0, k1) hold one, so that a row that came out not finite has to be computed again from its
// visible keys.  By a warp.
template <int DH>
HD_DEVINLINE bool hides_not_finite(const __nv_bfloat16* v, long long pitch, int k0, int k1) {
  const int lane = threadIdx.x & 31;
  bool bad = false;
  const __nv_bfloat16* row = v + k0 * pitch;  // from here, within a tile: a sequence's rows times DH/8 may pass 31 bits
  for (int i = lane; i < (k1 - k0) * (DH / 8); i += 32)
    bad = bad || !finite8(*reinterpret_cast<const uint4*>(row + (long long)(i / (DH / 8)) * pitch + i % (DH / 8) * 8));
  return __any_sync(0xffffffffu, bad);
}

// The 32 query rows from row r0 of an entry's sequence, head and stream, whose results this warp and
// others of its CTA have stored: those that came out not finite are computed again if keys of their
// tile's range [klo, khi) that they do not see hold an infinity or a NaN.  By a warp, after the CTA's
// other work, since nobody waits for it then (a row takes as long as its sequence is).
template <int DH>
__device__ __noinline__ void settle_rows(const PackedArgs& a, const PackedEntry& w, int head, int r0, int klo, int khi) {
  constexpr int C = DH / 32;
  const int lane = threadIdx.x & 31, window = a.g.window;
  const long long qp = (long long)a.g.rs * a.g.Hq * DH, kp = (long long)a.g.rs * a.g.Hkv * DH;
  const long long tensor_row = (long long)w.first * a.g.rs + w.stream;
  const long long q0 = tensor_row * a.g.Hq * DH + (long long)head * DH;
  const long long k0 = tensor_row * a.g.Hkv * DH + (long long)fast_div(head, a.d_grp) * DH;
  float* lse = a.lse + (long long)head * a.g.q_nL + tensor_row;
  bool odd = false;
  if (r0 + lane < w.rows) {
    const __nv_bfloat16* o = a.o + q0 + (r0 + lane) * qp;
    for (int i = 0; i < DH; i += 8) odd = odd || !finite8(*reinterpret_cast<const uint4*>(o + i));
  }
  for (unsigned rows = __ballot_sync(0xffffffffu, odd); rows; rows &= rows - 1) {
    const int r = r0 + __ffs(rows) - 1, first = window > 0 ? max(0, r - window + 1) : 0;
    if (!hides_not_finite<DH>(a.v + k0, kp, r + 1, khi) && !hides_not_finite<DH>(a.v + k0, kp, klo, first)) continue;
    float acc[C], m, l;
    visible_row<DH>(a.q + q0 + r * qp, a.k + k0, a.v + k0, kp, r + 1 - first,
                    [&](int j) { return (long long)(first + j); }, a.scale_log2, acc, m, l);
    const float inv = 1.f / l;
#pragma unroll
    for (int c = 0; c < C; ++c) a.o[q0 + r * qp + lane * C + c] = __float2bfloat16_rn(acc[c] * inv);
    if (lane == 0) lse[(long long)r * a.g.rs] = (m + log2f(l)) * 0.6931471805599453f;
  }
}

}  // namespace hdsfa
