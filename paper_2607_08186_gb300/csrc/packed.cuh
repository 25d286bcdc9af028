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
  const PackedItem* items;  // the longest sequences' tiles first, each sequence's last tile first
  const int32_t* count;
};
// Items that `tokens` packed tokens of B sequences make at most: sum of ceil(rows / tile_rows).
inline long long packed_max_items(int B, int tokens, int mult, int tile_rows) {
  return (long long)tokens * mult / tile_rows + (B < tokens ? B : tokens);
}
cudaError_t launch_packed_plan(const int32_t* offsets, int B, int N, int mult, int tile_rows, PackedItem* items,
                               int32_t* count, int32_t* status, cudaStream_t st);

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
