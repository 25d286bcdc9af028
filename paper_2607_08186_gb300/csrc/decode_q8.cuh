// Shared by the kernels that decode over the 8-bit paged cache (sfa_decode_q8.cu, sfa_decode_q8_tc.cu).
#pragma once
#include "decode.cuh"
#include "q8.cuh"
#include "tc_common.cuh"

namespace hdsfa {
namespace decq8 {
using dec::DecodeArgs;
using dec::kBadPage;

constexpr uint32_t kNoRow = 0xffffffffu;

// The softmax's sum counts P 2^-ev, and P is 2^(s + ev - m).  Where ev lies far below the largest that m has met, P leaves
// fp32's range before 2^-ev would bring it back (a block of zeros has ev = -64 whatever its neighbours hold), although
// the weight 2^s may count.  So from kFarSum binary orders on the partial's rows are computed again by exact_row.  (Up to
// there, what is flushed to 0, P < 2^-126, is a weight of less than 2^-35 of the row's largest.)
constexpr int kFarSum = 96;

// A query's codes (or its f16 form) miss its values far below its row's largest, which count where K's are as much larger.
// The row's sum of what they miss times K's largest value, 448 2^ek of its largest scale, bounds how far a score is off;
// rows whose bound passes kMissed (in log2 units) are computed again.  (Ordinary rows miss 2^-21 of their largest value
// in a column or none: 2^-14 of a score's unit where K's largest is 200 times a query's.)
constexpr float kMissed = 1.f / 256;

// The exponent of a partial's sum l, by which the partial is divided: l is a sum of P 2^-ev and P is relative to m, which
// counts ev, so between partials whose ev lie far apart the factors 2^(m - m') would leave fp32's range where the weights'
// do not.  Divided so, m is the logarithm of the partial's weight, to a binary order, and l lies in [1, 2).
HD_DEVINLINE int sum_exponent(float l) {
  const int e = (__float_as_int(l) >> 23) - 127;
  return l >= 1.17549435e-38f && e < 127 ? e : 0;  // (0, NaN and infinity as they are)
}
HD_DEVINLINE float two_to_minus(int e) { return __int_as_float((127 - e) << 23); }
// sum += x, the rounding error of the sum so far in `err` (Kahan).
HD_DEVINLINE void add_exactly(float& sum, float& err, float x) {
  const float y = x - err, t = sum + y;
  err = (t - sum) - y;
  sum = t;
}

struct Args : DecodeArgs {
  const uint8_t *kcodes, *vcodes, *kscale, *vscale;
  int blocks;       // blocks of a page
  FastDiv d_brow, d_blocks;  // rows of a block; blocks of a page
  int total;        // balanced: CTAs of a K/V head and row group
};
struct Params {
  CUtensorMap tm_k, tm_v;
  Args a;
};

// Row of position p >= 0 of K/V head g in the pools (of Dh codes each; below 2^32, checked on the host), kNoRow where
// the table names no page; and its block's scale.
HD_DEVINLINE uint32_t row_at(const Args& a, const int32_t* table, int g, int p, size_t* scale) {
  const int i = fast_div(p, a.pg.d_prow);
  if (i >= a.pg.max_pages) return kNoRow;
  const int id = table[i];
  if ((unsigned)id >= (unsigned)a.pg.num_pages) return kNoRow;
  const int off = p - i * a.pg.prow;
  const size_t ph = (size_t)id * a.Hkv + g;
  if (scale != nullptr) *scale = ph * a.blocks + fast_div(off, a.d_brow);
  return (uint32_t)(ph * a.pg.prow + off);
}

// A row's partial over the visible positions of [k0, k1), by one warp on the fp32 units: lane i holds DH/32 columns.
// Only visible rows are read: what a hidden NaN has made of the products' row is not.  The sums lose nothing of many small
// weights beside a large one; four positions' loads are in flight.
template <int DH>
__device__ __noinline__ void exact_row(const Args& a, int b, int g, int r, int T, int k0, int k1, float* po, float2* pml) {
  constexpr int C = DH / 32, NP = 4;
  const int lane = threadIdx.x & 31, s = r / a.G, h = g * a.G + r % a.G, pq = (T - 1) * a.n + s;
  const int32_t* table = a.table + (long long)b * a.pg.max_pages;
  int p = a.mode == SFA_LOCAL ? max(k0, pq - a.window + 1) : k0, step = 1;
  if (a.mode == SFA_WITHIN) {
    step = a.n;
    p += (s + a.n - p % a.n) % a.n;
  }
  const int end = min(k1, pq + 1);
  const bf16* q = a.q + (((long long)b * a.n + s) * a.Hq + h) * DH + lane * C;
  float qf[C], o[C], oe[C], m = -INFINITY, l = 0.f, le = 0.f;
#pragma unroll
  for (int c = 0; c < C; ++c) qf[c] = __bfloat162float(q[c]), o[c] = oe[c] = 0.f;
  for (; p < end; p += NP * step) {
    float x[NP], v[NP][C];
    bool in[NP];
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      const int at_p = p + e * step;
      size_t sc = 0;
      const uint32_t row = at_p < end ? row_at(a, table, g, at_p, &sc) : kNoRow;
      in[e] = row != kNoRow;
      x[e] = 0.f;
      if (!in[e]) continue;
      const size_t at = (size_t)row * DH;
      const float fk = q8::scale_of(q8::clamp_byte(a.kscale[sc])), fv = q8::scale_of(q8::clamp_byte(a.vscale[sc]));
#pragma unroll
      for (int c = 0; c < C; c += 2) {
        const float2 kv = q8::values2(*reinterpret_cast<const uint16_t*>(a.kcodes + at + lane * C + c));
        const float2 vv = q8::values2(*reinterpret_cast<const uint16_t*>(a.vcodes + at + lane * C + c));
        x[e] += qf[c] * (kv.x * fk) + qf[c + 1] * (kv.y * fk);  // (codes alone may pass fp32's range)
        v[e][c] = vv.x * fv, v[e][c + 1] = vv.y * fv;
      }
      x[e] *= a.scale_log2;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1)
#pragma unroll
      for (int e = 0; e < NP; ++e) x[e] += __shfl_xor_sync(0xffffffffu, x[e], d);
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      if (!in[e]) continue;
      const float mn = fmaxf(m, x[e]), mu = mn == -INFINITY ? 0.f : mn, corr = exp2f(m - mu), w = exp2f(x[e] - mu);
      m = mn;
      l *= corr, le *= corr;
      add_exactly(l, le, w);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        o[c] *= corr, oe[c] *= corr;
        add_exactly(o[c], oe[c], w * v[e][c]);
      }
    }
  }
  if (l != l) m = INFINITY;
#pragma unroll
  for (int c = 0; c < C; ++c) po[lane * C + c] = o[c];
  if (lane == 0) *pml = make_float2(m, l);
}

// A finished row by one warp: o / l and its LSE, or an empty row (l = 0).
template <int DH>
HD_DEVINLINE void store_row(const Args& a, int b, int g, int r, const float* o, float m, float l) {
  const int lane = threadIdx.x & 31, s = fast_div(r, a.d_G), h = g * a.G + r - s * a.G;
  const bool some = l != 0.f;
  const float inv = some ? 1.f / l : 0.f;
  bf16* to = a.o + (((long long)b * a.n + s) * a.Hq + h) * DH;
  for (int i = lane; i < DH / 4; i += 32) {
    uint2 w = make_uint2(0, 0);
    if (some) {
      const float4 x = *reinterpret_cast<const float4*>(o + i * 4);
      w = make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
    }
    *reinterpret_cast<uint2*>(to + i * 4) = w;
  }
  if (lane == 0 && a.lse != nullptr)
    a.lse[((long long)b * a.Hq + h) * a.n + s] = some ? (m + __log2f(l)) * 0.6931471805599453f : -INFINITY;
}
}  // namespace decq8

// The tcgen05 kernel (pages whose pieces TMA can bring): CTAs of so many query rows that an SM
// holds, and the launch without the combine kernel.
int decode_q8_tc_per_sm(int rows, int Dh);
cudaError_t launch_decode_q8_tc(decq8::Params& p, int Dh, cudaStream_t st);

}  // namespace hdsfa
