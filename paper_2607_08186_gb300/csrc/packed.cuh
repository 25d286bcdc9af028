// Packed prompts: sequences of different lengths one behind another, and the list of their query
// tiles that the forward kernels work through.
#pragma once
#include <float.h>
#include <limits.h>

#include "common.cuh"

namespace hdsfa {

// A query tile: `rows` virtual rows of a sequence (SfaGeom) that start at virtual row `first` of
// the packed tensors, and the tile's number among the sequence's.  Or a tile of short sequences (seqs
// > 0): the rows of sequences seq .. seq + seqs - 1 one behind another, at most a tile of them, in which
// a row's keys begin at its own sequence's first row.
struct PackedItem {
  int first, rows;
  int tile_or_seqs;  // the tile's number, or -seqs
  int seq;
};
constexpr int kShortRows = 48;  // a sequence of at most so many rows shares a tile with its neighbours
struct PackedList {
  const PackedItem* items;  // those with the most key tiles first
  const int32_t* count;
};
// Whether short neighbours share tiles.  It costs the softmax a register and a comparison a tile: at head
// dims 128 and 256 no time (200 sequences, 32 over 8 heads of 128, 4 streams, intra-stream: of 7 rows 359 -> 53
// us, 16: 97, 33: 177, 48: 244; 24 over 2 of 256: 357 -> 64, 118, 217, 295; 128 rows 381 / 394 and 558 / 561,
// 512 rows, 50 of them, 670 / 655 and 705 / 710), but at head dim 64, whose tiles have half the MMAs, about 6 %
// of every tile, so there it depends on an average sequence's rows (us apart / shared, 16 over 4 heads, 3
// streams, rows uniform around the average: 16: 217 / 65, 32: 216 / 150, 64: 112 / 109, 96: 104 / 106, 128: 96 /
// 103).  (The first row from shared memory instead of a register: 574 us for 200 of 128 rows at head dim 128.)
inline bool packed_shared(int Dh, int B, int tokens, int mult) { return Dh > 64 || (long long)tokens * mult <= 64LL * B; }
// Items that `tokens` packed tokens of B sequences make at most: sum of ceil(rows / tile_rows).
inline long long packed_max_items(int B, int tokens, int mult, int tile_rows) {
  return (long long)tokens * mult / tile_rows + (B < tokens ? B : tokens);
}
cudaError_t launch_packed_plan(const int32_t* offsets, int B, int N, int mult, int tile_rows, int window, bool shared,
                               PackedItem* items, int32_t* count, int32_t* status, cudaStream_t st);

// What the forward kernels over packed prompts are given besides their tensor maps.
struct PackedArgs {
  const __nv_bfloat16 *q, *k, *v;
  __nv_bfloat16* o;
  float* lse;
  SfaGeom g;  // of all packed rows: B = 1, Lv = Lq = rows of a stream's problem
  PackedList list;
  const int32_t* offsets;  // [B + 1], in tokens of `mult` rows
  int mult;
  float scale_log2;
  int32_t* status;
  int head_pairs;  // 1: an entry's two query tiles are the same rows of two heads of one K/V group,
                   // 0: two tiles of a head
  int o_wide;      // o is 32-byte aligned
  int per;         // places of a list entry: head slots x streams
  FastDiv d_per, d_ns, d_grp;  // by per, streams, query heads of a K/V head
};
inline PackedArgs make_packed_args(const void* q, const void* k, const void* v, void* o, float* lse, const SfaGeom& g,
                                   float scale, const PackedList& list, const int32_t* offsets, int32_t* status) {
  PackedArgs a;
  a.q = static_cast<const __nv_bfloat16*>(q);
  a.k = static_cast<const __nv_bfloat16*>(k);
  a.v = static_cast<const __nv_bfloat16*>(v);
  a.o = static_cast<__nv_bfloat16*>(o);
  a.lse = lse;
  a.g = g;
  a.list = list;
  a.offsets = offsets;
  a.mult = g.n / g.ns;
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
  int first, rows;  // the sequence's first row and its rows, or the short sequences'
  int m0, head, stream;
  int seq, seqs;  // short sequences of a shared tile (seqs = 0: one sequence)
  HD_DEVINLINE PackedEntry(const PackedArgs& a, int pos) {
    const int i = fast_div(pos, a.d_per);
    const PackedItem it = a.list.items[i];
    const int hs = pos - i * a.per, hx = fast_div(hs, a.d_ns);
    first = it.first;
    rows = it.rows;
    stream = hs - hx * a.g.q_ns;
    head = a.head_pairs ? 2 * hx : hx;
    m0 = max(it.tile_or_seqs, 0) * (a.head_pairs ? 128 : 256);
    seq = it.seq;
    seqs = max(-it.tile_or_seqs, 0);
  }
  HD_DEVINLINE int head_of(const PackedArgs& a, int g) const { return a.head_pairs ? head + g : head; }
  HD_DEVINLINE int row0(const PackedArgs& a, int g) const { return a.head_pairs ? m0 : m0 + g * 128; }
};
// Key tiles of 128 [lo, hi] of the query tile at row r0 (hi < lo: no rows).
HD_DEVINLINE int packed_lo(const PackedArgs& a, int r0) { return a.g.window > 0 ? max(0, r0 - a.g.window + 1) / 128 : 0; }
HD_DEVINLINE int packed_hi(int r0, int rows) { return r0 >= rows ? -1 : (min(r0 + 128, rows) - 1) / 128; }
// First row of the sequence that row r of an entry belongs to: 0, or one of up to 32 in a shared tile
// (empty ones among them hold no row).  By a whole warp.
HD_DEVINLINE int sequence_first(const PackedArgs& a, const PackedEntry& w, int r) {
  if (w.seqs == 0) return 0;
  const int lane = threadIdx.x & 31;
  const int at = lane < w.seqs ? a.offsets[w.seq + lane] * a.mult - w.first : INT_MAX;
  int s = 0;
#pragma unroll
  for (int d = 16; d; d >>= 1)
    if (__shfl_sync(0xffffffffu, at, s + d) <= r) s += d;
  return __shfl_sync(0xffffffffu, at, s);
}
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

// The 32 query rows from row r0 of an entry's sequence or sequences, head and stream, whose results this warp and
// others of its CTA have stored: those that came out not finite are computed again if keys of their
// tile's range [klo, khi) that they do not see hold an infinity or a NaN.  By a warp, after the CTA's
// other work, since nobody waits for it then (a row takes as long as its sequence is).
template <int DH, bool SHARED>
__device__ __noinline__ void settle_rows(const PackedArgs& a, const PackedEntry& w, int head, int r0, int klo, int khi) {
  constexpr int C = DH / 32;
  const int lane = threadIdx.x & 31, window = a.g.window;
  const long long qp = (long long)a.g.rs * a.g.Hq * DH, kp = (long long)a.g.rs * a.g.Hkv * DH;
  const long long tensor_row = (long long)w.first * a.g.rs + w.stream;
  const long long q0 = tensor_row * a.g.Hq * DH + (long long)head * DH;
  const long long k0 = tensor_row * a.g.Hkv * DH + (long long)fast_div(head, a.d_grp) * DH;
  float* lse = a.lse + (long long)head * a.g.q_nL + tensor_row;
  const int mine = SHARED ? sequence_first(a, w, r0 + lane) : 0;
  bool odd = false;
  __syncwarp();  // rows stored by single lanes, and by others below: votes and shuffles order no memory
  if (r0 + lane < w.rows) {
    const __nv_bfloat16* o = a.o + q0 + (r0 + lane) * qp;
    for (int i = 0; i < DH; i += 8) odd = odd || !finite8(*reinterpret_cast<const uint4*>(o + i));
  }
  __syncwarp();
  for (unsigned rows = __ballot_sync(0xffffffffu, odd); rows; rows &= rows - 1) {
    const int l = __ffs(rows) - 1, r = r0 + l;
    const int own = SHARED ? __shfl_sync(0xffffffffu, mine, l) : 0;
    const int first = max(own, window > 0 ? r - window + 1 : 0);
    if (!hides_not_finite<DH>(a.v + k0, kp, r + 1, khi) && !hides_not_finite<DH>(a.v + k0, kp, klo, first)) continue;
    float acc[C], m, sum;
    visible_row<DH>(a.q + q0 + r * qp, a.k + k0, a.v + k0, kp, r + 1 - first,
                    [&](int j) { return (long long)(first + j); }, a.scale_log2, acc, m, sum);
    const float inv = 1.f / sum;
#pragma unroll
    for (int c = 0; c < C; ++c) a.o[q0 + r * qp + lane * C + c] = __float2bfloat16_rn(acc[c] * inv);
    if (lane == 0) lse[(long long)r * a.g.rs] = (m + log2f(sum)) * 0.6931471805599453f;
  }
}

}  // namespace hdsfa
