// Decoding over the 8-bit paged cache: softmax(q k^T) v over e4m3 codes with a power of two for each block of tokens
// and head (q8.cuh).
//
// The mathematics.  With K = 2^ek ck and V = 2^ev cv per position, a row's result is
//   o = sum_p 2^(s_p) 2^(ev_p) cv_p / sum_p 2^(s_p),   s_p = c (q . ck_p) 2^(ek_p)   (c: scale * log2 e).
// The codes go into the products as they are (e4m3 -> f16 is exact), ek multiplies a score, and ev is added to its
// exponent: with x_p = s_p + ev_p and m the running maximum of x (not of s), P_p = 2^(x_p - m + 15) is at most 2^15, f16
// holds it to 2^-11 of itself, below 2^-29 of the largest contribution to 2^-40 of that, and
//   o = sum P_p cv_p / sum P_p 2^(-ev_p):
// the sum's terms are one fused multiply-add each.  The queries are scaled by a power of two for each row, so that f16 holds
// them as bf16 did (a row's largest to 2^15; values from 2^-31 of it down lose bits, and vanish from 2^-39).  Where
// V's scales lie so far apart that weights that count lose bits (kFar) or leave fp32's range (kFarSum), or K is large where a
// query lost bits (kMissed), the rows are computed again in fp32, a position at a time (exact_row): right, and 40 to 200
// times as slow.
//
// This kernel takes what the tcgen05 kernel (sfa_decode_q8_tc.cu) does not: pages too small for TMA, and short ranges of few
// query rows, where it starts and ends sooner.  A warp takes 16 query rows and 32 of a tile's positions (16 with a single row
// tile at head dim 128); the warps of the row tiles share the tile in shared memory, so up to 64 rows of a K/V head's group read the cache once.  Tiles stream
// through a ring by 16-byte cp.async, whose rows the threads look up three tiles ahead.  mma.sync m16n8k16 (f16): a
// thread's four bytes of an ldmatrix row are k = 2t, 2t + 1, 2t + 8, 2t + 9 of the product, so q lies in that order; V's
// transposed loads bring pairs of head-dim columns for two keys, so even and odd columns are products of their own.
//
// Bound by the latency of a tile's chain (table entry, rows, scales, products, softmax) and by the instructions that
// turn codes into f16: 32 over 8 heads of 128, 4 streams, 4 sequences of 4000 tokens on pages of one token with a scale each
// take 42.2 us, 14.7 of them the bytes at the copy rate (64 over 8 58, 96 over 8 91.5).  Bringing larger pieces by TMA here
// with two sets of warps on alternate tiles gained nothing where this kernel runs (33 x 12 tokens 10.9 us and 10.0
// without, two sequences of 64 over heads of 64 6.5 and 6.1).
#include <float.h>

#include <algorithm>

#include "decode_plan.cuh"
#include "decode_q8.cuh"

namespace hdsfa {
namespace decq8 {
constexpr float kShift = 15.f;       // P's largest exponent
constexpr int kMaxRows = 64;         // query rows of a CTA at most (four row tiles)
// P in f16 is off by 2^-11 of P, or, below 2^-14, by up to 2^-25, 2^-40 of the row's largest.  A weight is P 2^-ev, so where V's
// scales lie no further apart than kFar binary orders, a position loses 2^-24 of the row's largest weight at most; further
// apart, all rows are computed again (exact_row), since a small block's columns in which larger blocks hold nothing may
// lose what they hold.  (V of the smallest scale, mostly zeros, counts only in the sum: kFarSum.)
constexpr int kFar = 16;

// Up to MT row tiles of 16 query rows; at head dim 256 a warp has half of the head dim, since O must fit its registers.  Two
// CTAs an SM while the queries leave room for three stages each: up to two row tiles, one at head dim 256; with four row
// tiles one.  At head dim 128 a single row tile leaves eight warps an SM so, so its warps take 16 positions of a tile and not
// 32, and four CTAs fit (pages of one token, 4 x 4000 tokens, 32 over 8 heads: 48.6 us
// for 41.3); at 64 three fit as it is.
template <int DH, int MT_>
struct Cfg {
  static constexpr int MT = MT_, WK = DH == 128 && MT == 1 ? 16 : 32;             // positions of a tile that a warp takes
  static constexpr int DS = DH == 256 ? 2 : 1, KW = 4 / DS, KT = WK * KW;         // head-dim parts, key groups, a tile
  static constexpr bool kWide = MT == 4;
  static constexpr int STAGES = !kWide ? 3 : DH == 256 ? 5 : 6;
  static constexpr int kPerSm = kWide ? 1 : WK == 16 ? 4 : 2;
  static constexpr int kWarps = 4 * MT, kThreads = kWarps * 32;
  static constexpr int kMergeRows = 16 * MT;  // rows of the partials at most
};
template <int DH, int MT>
struct Smem {
  using C = Cfg<DH, MT>;
  uint8_t k[C::STAGES][C::KT * DH];
  uint8_t v[C::STAGES][C::KT * DH];
  __half q[C::MT * 16 * DH];
  float4 scale[C::kWarps][C::WK];   // a warp's keys: 2^ek, ev, 2^-ev
  float qscale[C::MT * 16];
  unsigned missed;                      // the most that a row's f16 query misses (kMissed), as bits
  uint32_t row[4][C::KT];               // rows of the pool (kNoRow: none) of four tiles
  unsigned again[2];                    // rows of the merged partial (bits) that are not finite, which exact_row computes,
  int far;                              // and whether it computes all of them: V's scales lie far apart, or queries miss too much
  int bad_page;
};

// Byte offset of 16-byte chunk `c` of a row of a tile: blocks of [KT][128 bytes], at head dim 64 [KT][64], whose
// chunks are XORed with the row's number; conflict-free for ldmatrix.
template <int DH, int KT>
HD_DEVINLINE int chunk_at(int row, int c) {
  if (DH == 64) return row * 64 + ((c ^ ((row >> 1) & 3)) << 4);
  return (c >> 3) * (KT * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4);
}

HD_DEVINLINE void mma_f16_16816(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
HD_DEVINLINE uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Whether a query that misses `missed` 2^-ek is too far off at a position p, p + blockDim.x, ... < k1.  (Hardly ever called:
// f16 misses values 2^-31 of a row's largest and below.)
__device__ __noinline__ bool misses_keys(const Args& a, const int32_t* table, int g, int p, int k1, float missed) {
  bool r = false;
  for (; p < k1; p += blockDim.x) {
    size_t at = 0;
    if (row_at(a, table, g, p, &at) != kNoRow) r |= missed * q8::scale_of(q8::clamp_byte(a.kscale[at])) > kMissed;
  }
  return r;
}

template <int DH, int MT>
__global__ void __launch_bounds__(Cfg<DH, MT>::kThreads, Cfg<DH, MT>::kPerSm) decode_q8_kernel(const __grid_constant__ Args a) {
  using C = Cfg<DH, MT>;
  using Sm = Smem<DH, MT>;
  constexpr int KT = C::KT, STAGES = C::STAGES, WK = C::WK, NJ = WK / 8;  // NJ: tiles of 8 positions of a warp
  constexpr int KW = C::KW, DC = DH / C::DS, CPR = DH / 16;  // DC: O columns of a warp
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  {
    uint32_t dyn;
    asm("mov.u32 %0, %%dynamic_smem_size;\n" : "=r"(dyn));
    const uint32_t pad = (1024 - (smem_u32(smem_raw) & 1023)) & 1023;
    if (pad + sizeof(Sm) > dyn) {  // uniform: nothing touched yet
      if (threadIdx.x == 0) set_status(a.status, HD_DEVBIT_TIMEOUT);
      return;
    }
  }
  Sm& sm = *reinterpret_cast<Sm*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int split = fast_div((int)blockIdx.x, a.d_heads), head = (int)blockIdx.x - split * a.Hkv * a.ngroups;
  const int g = a.ngroups == 1 ? head : head / a.ngroups, rg = a.ngroups == 1 ? 0 : head % a.ngroups;
  const int tid = threadIdx.x, nt = blockDim.x, W = nt >> 5, warp = tid >> 5, lane = tid & 31, g4 = lane >> 2, t4 = lane & 3;
  const int mt = warp >> 2, kw = (warp & 3) % KW, dw = (warp & 3) / KW;  // row tile, key group and head-dim part
  const int R = a.rg;  // rows of the CTA
  const size_t pidx = blockIdx.x;
  float* po = a.part_o + pidx * R * DH;
  float2* pml = a.part_ml + pidx * R;
  const int tile = a.tile;
  if (tid == 0) {
    sm.bad_page = 0;
    sm.again[0] = sm.again[1] = 0;
    sm.far = 0;
    sm.missed = 0;
  }
  // this thread's query rows g4 and g4 + 8 of the row tile: their streams (-1: padding).  Where n divides a tile, which
  // of this thread's keys are of a row's stream is the same in every tile.
  int rs_[2];
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    const int r = rg * R + mt * 16 + g4 + 8 * hf;
    rs_[hf] = r < a.M ? fast_div(r, a.d_G) : -1;
  }
  const bool streams = a.mode == SFA_WITHIN && a.n > 1;
  const bool shifting = streams && tile - fast_div(tile, a.d_n) * a.n != 0;
  uint32_t mine = 0;  // bit hf*2*NJ + j*2 + e: the row may see key j*8 + 2*t4 + e
#pragma unroll
  for (int i = 0; i < 2 * NJ; ++i) {
    const int key = kw * WK + (i >> 1) * 8 + 2 * t4 + (i & 1);
    const int ks = streams && !shifting ? key - fast_div(key, a.d_n) * a.n : -1;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
      if (rs_[hf] >= 0 && key < tile && (ks < 0 || ks == rs_[hf])) mine |= 1u << (hf * 2 * NJ + i);
  }
  grid_dep_wait();
  grid_dep_launch();
  const int b = fast_div(split, a.d_nsplit), T = a.lens[b];
  const int32_t* table = a.table + (long long)b * a.pg.max_pages;
  int k0, k1;
  dec::split_range<true>(a, T, split - b * a.nsplit, tile, k0, k1);
  if (k0 >= k1) {  // nothing of this sequence in this split: an empty partial, or an empty result
    if (a.nsplit > 1) {
      for (int i = tid; i < R; i += nt) pml[i] = make_float2(-INFINITY, 0.f);
    } else {
      if (T != 0 && g == 0 && rg == 0 && tid == 0) set_status(a.status, HD_DEVBIT_INDEX);
      for (int row = warp; row < min(R, a.M - rg * R); row += W) store_row<DH>(a, b, g, rg * R + row, nullptr, -INFINITY, 0.f);
    }
    return;
  }
  const int nsub = fast_div(k1 - k0 + tile - 1, a.d_tile);

  // ---- the tiles' loads
  const int seen = a.mode == SFA_LOCAL ? (T - 1) * a.n - a.window + 1 : 0;  // first position any row sees
  // the pools' row of this thread's position of a tile
  auto row_of = [&](int it) {
    const int p = k0 + it * tile + tid;
    if (tid >= tile || p >= k1 || p < seen) return kNoRow;
    const uint32_t row = row_at(a, table, g, p, nullptr);
    if (row == kNoRow) sm.bad_page = 1;
    return row;
  };
  auto load_tile = [&](int it, int st) {  // tile `it` into stage st
    for (int i = tid; i < KT * CPR; i += nt) {
      const int rr = i / CPR, cc = i % CPR;
      const uint32_t row = rr < tile ? sm.row[it & 3][rr] : kNoRow;
      const size_t off = (row == kNoRow ? 0 : (size_t)row * DH) + cc * 16;
      cp_async_16(smem_u32(sm.k[st] + chunk_at<DH, KT>(rr, cc)), a.kcodes + off, row != kNoRow);
      cp_async_16(smem_u32(sm.v[st] + chunk_at<DH, KT>(rr, cc)), a.vcodes + off, row != kNoRow);
    }
  };
  // The scales of this warp's keys, a lane's key each: the page entry two tiles ahead, the bytes one ahead.  The
  // key's page and row there go on by a tile, without divisions.
  const int my_key = lane < WK ? kw * WK + lane : KT;
  const int step_pages = fast_div(tile, a.pg.d_prow), step_rows = tile - step_pages * a.pg.prow;
  int at_pos = k0 + my_key, at_page = fast_div(at_pos, a.pg.d_prow), at_row = at_pos - at_page * a.pg.prow;
  int next_entry = -1, next_row_in = 0;
  auto scale_entry = [&] {  // entry and row of the key in the next tile, whose number goes up by one
    next_entry = -1;
    next_row_in = at_row;
    if (my_key < tile && at_pos < k1 && at_pos >= seen && at_page < a.pg.max_pages) next_entry = table[at_page];
    at_pos += tile;
    at_page += step_pages;
    at_row += step_rows;
    if (at_row >= a.pg.prow) at_row -= a.pg.prow, ++at_page;
  };
  int kb = 127, vb = -1;
  unsigned ends = 0;  // V's largest so far << 16, and 255 less its smallest (the very smallest nearer, see kFar)
  auto scale_bytes = [&] {
    if ((unsigned)next_entry < (unsigned)a.pg.num_pages) {
      const size_t at = ((size_t)next_entry * a.Hkv + g) * a.blocks + fast_div(next_row_in, a.d_brow);
      kb = a.kscale[at];
      vb = a.vscale[at];
    }
  };
  {
    const uint32_t r0 = row_of(0), r1 = row_of(1), r2 = row_of(2);
    if (tid < tile) sm.row[0][tid] = r0, sm.row[1][tid] = r1, sm.row[2][tid] = r2;
  }
  __syncthreads();  // ... and the flags are set
  load_tile(0, 0);
  cp_async_commit();
  if (nsub > 1) load_tile(1, 1);
  cp_async_commit();
  scale_entry();
  scale_bytes();
  scale_entry();
  // The queries: a warp per row scales its row by a power of two, rounds it to f16 and lays it out in the products'
  // order: value 16i + 4t + j at column 16i + 2t + j (j < 2) or 16i + 6 + 2t + j.
  for (int rr = warp; rr < R; rr += W) {
    constexpr int NP = DH / 64;  // pairs of a lane
    const int r = rg * R + rr;
    uint32_t w[NP];
    uint32_t most = 0;
    if (r < a.M) {
      const int s = fast_div(r, a.d_G), h = g * a.G + r - s * a.G;
      const uint32_t* src = reinterpret_cast<const uint32_t*>(a.q + (((long long)b * a.n + s) * a.Hq + h) * DH) + lane * NP;
#pragma unroll
      for (int i = 0; i < NP; ++i) w[i] = src[i];
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) w[i] = 0;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) most = max(most, max(w[i] << 16 & 0x7fff0000u, w[i] & 0x7fff0000u));
    most = __reduce_max_sync(0xffffffffu, most);
    // the exponent field of the largest magnitude, kept where both powers are normal
    const int e = min(max((int)(most >> 23), 20), 254);
    const float to = __int_as_float(min(127 + 14 + 127 - e, 254) << 23);  // 2^(14 - (e - 127)), at most 2^127
    const float back = __int_as_float(max(e - 14, 1) << 23);              // 2^(e - 127 - 14)
    float miss = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int p = lane * NP + i, kk = p >> 3, t = (p >> 1) & 3, hi = p & 1;
      const float x0 = __uint_as_float(w[i] << 16) * to, x1 = __uint_as_float(w[i] & 0xffff0000u) * to;
      const __half2 u = __floats2half2_rn(x0, x1);
      const float2 y = __half22float2(u);
      miss += fabsf(x0 - y.x) + fabsf(x1 - y.y);
      *reinterpret_cast<__half2*>(sm.q + swz<DH>(rr, kk * 16 + hi * 8 + 2 * t)) = u;
    }
    if (lane == 0) sm.qscale[rr] = back * a.scale_log2;
    if (miss > 0.f) atomicMax(&sm.missed, __float_as_uint(miss * (32.f * 448.f) * fabsf(back * a.scale_log2)));  // (32 lanes')
  }
  __syncthreads();

  const float rowf[2] = {sm.qscale[mt * 16 + g4], sm.qscale[mt * 16 + g4 + 8]};
  const int own_lo = (T - 1) * a.n, win_hi = a.mode == SFA_LOCAL ? T * a.n - 1 - a.window : -1;
  float mx[2] = {-INFINITY, -INFINITY}, ls[2] = {0.f, 0.f}, oacc[DC / 8][4];
#pragma unroll
  for (int i = 0; i < DC / 8; ++i) oacc[i][0] = oacc[i][1] = oacc[i][2] = oacc[i][3] = 0.f;

  {  // a lane without a key holds another's byte, so that it does not count as one of its own
    const int some = __reduce_max_sync(0xffffffffu, vb);
    if (vb < 0) vb = some < 0 ? 127 : some;
  }
  for (int it = 0, st = 0; it < nsub; ++it) {
    const int base = k0 + it * tile;
    // this tile's scales into shared memory, the next ones' loads on their way
    {
      kb = q8::clamp_byte(kb);
      vb = q8::clamp_byte(vb);
      ends = __vmaxu2(ends, (unsigned)vb << 16 | (unsigned)(255 - (vb == q8::kMinByte ? vb + kFarSum - kFar : vb)));
      if (lane < WK) sm.scale[warp][lane] = make_float4(q8::scale_of(kb), (float)(vb - 127), q8::inverse_of(vb), 0.f);
      scale_bytes();
      scale_entry();
    }
    cp_async_wait<1>();  // stage `it` has landed
    __syncthreads();     // ... for every thread, and stage it - 1 is no longer read
    if (it + 2 < nsub) load_tile(it + 2, (it + 2) % STAGES);
    cp_async_commit();
    const uint32_t next_row = row_of(it + 3);  // the rows that the next iteration loads by
    const uint8_t *cK = sm.k[st], *cV = sm.v[st];

    // S = q ck^T: key tile j of 8 keys
    float sacc[NJ][4];
#pragma unroll
    for (int j = 0; j < NJ; ++j) sacc[j][0] = sacc[j][1] = sacc[j][2] = sacc[j][3] = 0.f;
#pragma unroll
    for (int kq = 0; kq < DH / 64; ++kq) {
      uint32_t qa[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        ldsm_x4(smem_u32(sm.q + swz<DH>(mt * 16 + (lane & 15), (kq * 4 + i) * 16 + (lane >> 4) * 8)), qa[i][0], qa[i][1],
                qa[i][2], qa[i][3]);
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        uint32_t c[4];
        ldsm_x4(smem_u32(cK + chunk_at<DH, KT>(kw * WK + j * 8 + (lane & 7), kq * 4 + (lane >> 3))), c[0], c[1], c[2],
                c[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t b0, b1;
          q8::f16x4_of(c[i], b0, b1);
          mma_f16_16816(sacc[j], qa[i], b0, b1);
        }
      }
    }
    // x = s + ev, the mask, and the online softmax in log2 units
    uint32_t vis = mine;
    const int kp = base + kw * WK + 2 * t4;
    if (base + tile - 1 > own_lo || base + tile > k1 || base <= win_hi || shifting) {
      // positions at the sequence's end, at the rows' windows, or streams that shift from tile to tile
#pragma unroll
      for (int i = 0; i < 4 * NJ; ++i) {
        const int hf = i / (2 * NJ), p = kp + ((i >> 1) % NJ) * 8 + (i & 1), pq = own_lo + rs_[hf];
        const bool in = p < k1 && p <= pq && (a.mode != SFA_LOCAL || p > pq - a.window) &&
                        (!shifting || p - fast_div(p, a.d_n) * a.n == rs_[hf]);
        if (!in) vis &= ~(1u << i);
      }
    }
    float tmax[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float4 sc = sm.scale[warp][j * 8 + 2 * t4 + e];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const float x = fmaf(sacc[j][hf * 2 + e] * rowf[hf], sc.x, sc.y);
          sacc[j][hf * 2 + e] = (vis >> (hf * 2 * NJ + j * 2 + e)) & 1u ? x : -INFINITY;
          tmax[hf] = fmaxf(tmax[hf], sacc[j][hf * 2 + e]);
        }
      }
    float corr[2], msub[2];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      tmax[hf] = fmaxf(tmax[hf], __shfl_xor_sync(0xffffffffu, tmax[hf], 1));
      tmax[hf] = fmaxf(tmax[hf], __shfl_xor_sync(0xffffffffu, tmax[hf], 2));
      const float mnew = fmaxf(mx[hf], tmax[hf]), mu = mnew == -INFINITY ? 0.f : mnew;
      corr[hf] = ex2_approx(0.5f * (mx[hf] - mu));  // (the root: the sum's range is wider than a power's)
      msub[hf] = mu - kShift;
      mx[hf] = mnew;
    }
    if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
      ls[0] = ls[0] * corr[0] * corr[0];
      ls[1] = ls[1] * corr[1] * corr[1];
      corr[0] *= corr[0];
      corr[1] *= corr[1];
#pragma unroll
      for (int i = 0; i < DC / 8; ++i) {
        oacc[i][0] *= corr[0];
        oacc[i][1] *= corr[0];
        oacc[i][2] *= corr[1];
        oacc[i][3] *= corr[1];
      }
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float inv = sm.scale[warp][j * 8 + 2 * t4 + e].z;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const float p = ex2_approx(sacc[j][hf * 2 + e] - msub[hf]);
          sacc[j][hf * 2 + e] = p;
          ls[hf] = fmaf(p, inv, ls[hf]);
        }
      }
    // O += P cv over this warp's keys, 16 at a time
#pragma unroll
    for (int u = 0; u < NJ / 2; ++u) {
      const uint32_t pa[4] = {pack_f16(sacc[2 * u][0], sacc[2 * u][1]), pack_f16(sacc[2 * u][2], sacc[2 * u][3]),
                              pack_f16(sacc[2 * u + 1][0], sacc[2 * u + 1][1]), pack_f16(sacc[2 * u + 1][2], sacc[2 * u + 1][3])};
#pragma unroll
      for (int c2 = 0; c2 < DC / 32; ++c2) {
        uint32_t r[4];
        ldsm_x4_t(smem_u32(cV + chunk_at<DH, KT>(kw * WK + u * 16 + (lane & 15), dw * (DC / 16) + c2 * 2 + (lane >> 4))),
                  r[0], r[1], r[2], r[3]);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t b0, b1, b2, b3;  // even columns of keys 2t, 2t+1 and 2t+8, 2t+9; odd columns
          q8::f16x4_of(__byte_perm(r[2 * c], 0, 0x3120), b0, b2);
          q8::f16x4_of(__byte_perm(r[2 * c + 1], 0, 0x3120), b1, b3);
          float(*acc)[4] = &oacc[(c2 * 2 + c) * 2];
          mma_f16_16816(acc[0], pa, b0, b1);
          mma_f16_16816(acc[1], pa, b2, b3);
        }
      }
    }
    __syncwarp();  // this tile's scales are read
    if (tid < tile) sm.row[(it + 3) & 3][tid] = next_row;
    if (++st == STAGES) st = 0;
  }
  cp_async_wait<0>();
  {
    const int most = (int)__reduce_max_sync(0xffffffffu, ends >> 16), least = 255 - (int)__reduce_max_sync(0xffffffffu, ends & 0xffff);
    if (most > least + kFar) sm.far = 1;
  }
  if (sm.missed != 0 && misses_keys(a, table, g, max(k0, seen) + tid, k1, __uint_as_float(sm.missed))) sm.far = 1;
  __syncthreads();

  // merge the key groups' partials in shared memory (the ring is free now): [KW][R][DH], then what the sums count
  // from, and the sums, each partial divided by its sum's power of two
  static_assert((KW * C::kMergeRows * DH + 2 * KW * C::kMergeRows) * 4 <= 2 * STAGES * KT * DH, "merge fits the ring");
  static_assert(kMaxRows <= 128, "one thread per row");
  float* sO = reinterpret_cast<float*>(sm.k[0]);
  float* sM = sO + KW * R * DH;  // [KW][R]
  float* sL = sM + KW * R;       // [KW][R]
#pragma unroll
  for (int hf = 0; hf < 2; ++hf) {
    ls[hf] += __shfl_xor_sync(0xffffffffu, ls[hf], 1);
    ls[hf] += __shfl_xor_sync(0xffffffffu, ls[hf], 2);
    const int row = kw * R + mt * 16 + g4 + 8 * hf, k = sum_exponent(ls[hf]);
    const float f = two_to_minus(k);
    if (t4 == 0 && dw == 0) {
      sM[row] = mx[hf] - kShift + (float)k;
      sL[row] = ls[hf] * f;
    }
#pragma unroll
    for (int c = 0; c < DC / 16; ++c)
      *reinterpret_cast<float4*>(sO + row * DH + dw * DC + c * 16 + 4 * t4) = make_float4(
          oacc[2 * c][2 * hf] * f, oacc[2 * c + 1][2 * hf] * f, oacc[2 * c][2 * hf + 1] * f, oacc[2 * c + 1][2 * hf + 1] * f);
  }
  __syncthreads();
  const bool bad = sm.bad_page != 0;
  if (tid < R) {  // one thread per row: its maximum and sum over the key groups, whose weights replace their maxima
    float m = -INFINITY, l = 0.f;
    for (int w = 0; w < KW; ++w) m = fmaxf(m, sM[w * R + tid]);
    const float mu = m == -INFINITY ? 0.f : m;
    for (int w = 0; w < KW; ++w) {
      const float f = exp2f(sM[w * R + tid] - mu);
      l += f * sL[w * R + tid];
      sM[w * R + tid] = f;
    }
    if (l != l) m = INFINITY;  // a visible score that is not finite: the combined row is NaN
    if (bad) m = -INFINITY, l = kBadPage;
    pml[tid] = make_float2(m, l);
    if (a.nsplit == 1 && bad && tid == 0) set_status(a.status, HD_DEVBIT_INDEX);
  }
  __syncthreads();
  for (int idx = tid; idx < R * (DH / 4); idx += nt) {
    const int row = idx / (DH / 4), c4 = idx % (DH / 4);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int w = 0; w < KW; ++w) {
      const float f = sM[w * R + row];
      const float4 v = *reinterpret_cast<const float4*>(sO + (w * R + row) * DH + c4 * 4);
      o.x += f * v.x;
      o.y += f * v.y;
      o.z += f * v.z;
      o.w += f * v.w;
    }
    *reinterpret_cast<float4*>(po + row * DH + c4 * 4) = o;
    if (!(fabsf(o.x) + fabsf(o.y) + fabsf(o.z) + fabsf(o.w) <= FLT_MAX)) atomicOr(&sm.again[row >> 5], 1u << (row & 31));
  }
  __syncthreads();
  if (!bad)
#pragma unroll
    for (int half = 0; half < 2; ++half)
      for (unsigned rows = sm.far ? 0xffffffffu : sm.again[half]; rows; rows &= rows - 1) {
        const int row = half * 32 + __ffs(rows) - 1;
        if (row % W == warp && row < R && rg * R + row < a.M)
          exact_row<DH>(a, b, g, rg * R + row, T, k0, k1, po + row * DH, pml + row);
      }
  if (a.nsplit > 1) return;
  // the only split: its rows are the results
  __syncthreads();
  for (int row = warp; row < min(R, a.M - rg * R); row += W) {
    const float2 ml = pml[row];
    store_row<DH>(a, b, g, rg * R + row, po + row * DH, ml.x, bad ? 0.f : ml.y);
  }
}

// The splits' partials of a query row together, a warp a row, where rows are many: a lane has DH / 32 columns of it, and the
// maximum and sum of each 32nd split; the splits' columns are asked for ahead of their weights.  Bound by latency.  The
// bf16 cache's combine kernel takes a CTA for a row, so fewer rounds over many splits but waves of CTAs over many rows:
// a step of 4 streams, CTA a row / warp a row, in us
//   128 rows   1 x 8192 tokens, 32 over 8 heads of 128 19.0 / 28.0;  384   4 x 8192, 24 over 2 of 256 30.2 / 40.3
//   512        4 x 4000, 32 over 8 28.9 / 33.3;  1024   8 x 16384 113.6 / 114.5;  2048   16 x 400 22.9 / 19.8
//   2560       20 x 2000 49.7 / 45.3;  8 x 8192, 96 over 8 101.5 / 96.0;  7680   20 x 2000, 96 over 8 87.0 / 73.1
template <int DH>
__global__ void __launch_bounds__(256) combine_rows_kernel(Args a) {
  constexpr int C = DH / 32, NB = DH == 256 ? 4 : 8, NW = dec::kMaxSplit / 32;  // columns, splits in flight, weights of a lane
  const int lane = threadIdx.x & 31, rows = min(a.rg, a.M);
  const int x = (int)blockIdx.x * 8 + (threadIdx.x >> 5), unit = x / rows, row = x - unit * rows;  // (b, g, row group), row
  const int heads = a.Hkv * a.ngroups, b = unit / heads, head = unit - b * heads, g = head / a.ngroups, rg = head - g * a.ngroups;
  const int r = rg * a.rg + row;
  grid_dep_wait();  // every partial of the decoding kernel is written
  if (b >= a.B) return;
  const int T = a.lens[b];
  const bool valid = T >= 1 && T <= a.maxT;
  if (!valid && T != 0 && head == 0 && row == 0 && lane == 0) set_status(a.status, HD_DEVBIT_INDEX);
  if (r >= a.M) return;  // the last row group may be short
  const int2 own = a.balanced ? a.share[b] : make_int2(b * a.nsplit, a.nsplit);
  const int n = valid ? own.y : 0;
  const size_t first = ((size_t)own.x * heads + head) * a.rg + row, step = (size_t)heads * a.rg;
  const float* po = a.part_o + first * DH + lane * C;
  auto load = [&](int i, float* v) {
#pragma unroll
    for (int c = 0; c < C; c += 2) {
      const float2 t = *reinterpret_cast<const float2*>(po + i * step * DH + c);
      v[c] = t.x, v[c + 1] = t.y;
    }
  };
  float v[NB][C];
#pragma unroll
  for (int k = 0; k < NB; ++k)
    if (k < n) load(k, v[k]);
  float2 ml[NW];
  float m = -INFINITY;
  bool bad = false;
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    ml[k] = lane + 32 * k < n ? a.part_ml[first + (lane + 32 * k) * step] : make_float2(-INFINITY, 0.f);
    m = fmaxf(m, ml[k].x);
    bad |= ml[k].y == kBadPage;
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  bad = __any_sync(0xffffffffu, bad);
  if (bad && lane == 0) set_status(a.status, HD_DEVBIT_INDEX);
  float w[NW], l = 0.f;
#pragma unroll
  for (int k = 0; k < NW; ++k) {
    w[k] = ml[k].x == -INFINITY ? 0.f : exp2f(ml[k].x - m);
    l += w[k] * ml[k].y;
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
  float o[C];
#pragma unroll
  for (int c = 0; c < C; ++c) o[c] = 0.f;
#pragma unroll
  for (int k = 0; k < NW; ++k)
#pragma unroll 1
    for (int i0 = 32 * k; i0 < min(n, 32 * (k + 1)); i0 += NB) {
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const float f = __shfl_sync(0xffffffffu, w[k], i0 + j & 31);
        if (i0 + j < n && f != 0.f)
#pragma unroll
          for (int c = 0; c < C; ++c) o[c] += f * v[j][c];
        if (i0 + j + NB < n) load(i0 + j + NB, v[j]);
      }
    }
  const bool ok = valid && !bad && l != 0.f;
  const float inv = ok ? 1.f / l : 0.f;
  const int s = fast_div(r, a.d_G), h = g * a.G + r - s * a.G;
  uint32_t* to = reinterpret_cast<uint32_t*>(a.o + (((long long)b * a.n + s) * a.Hq + h) * DH + lane * C);
#pragma unroll
  for (int c = 0; c < C; c += 2) to[c / 2] = ok ? pack_bf16(o[c] * inv, o[c + 1] * inv) : 0;
  if (lane == 0 && a.lse != nullptr)
    a.lse[((long long)b * a.Hq + h) * a.n + s] = ok ? (m + __log2f(l)) * 0.6931471805599453f : -INFINITY;
}
}  // namespace decq8

// ------------------------------------------------------------------ host side

namespace {
// The sequences' shares of a balanced batch's splits, in front of the partials.
constexpr size_t kShareBytes = dec::kBalancedSeqs * sizeof(int2);
struct Q8Plan {
  int G, M, ngroups, rg, nsplit, total;  // total: CTAs of a K/V head and row group where the batch is balanced, or 0
  size_t part_o_bytes, part_ml_bytes;
  size_t bytes() const { return kShareBytes + ((part_o_bytes + 255) & ~size_t(255)) + part_ml_bytes; }
};
}  // namespace

// Positions of a tile.
static int q8_tile(int Dh, int rg, bool tc) { return tc || Dh == 64 || (Dh == 128 && rg > 16) ? 128 : 64; }

// Splits of a step on the tensor cores (`tc`) or not: the fewest waves times (tiles of a CTA + about two tiles' time to
// start and end it), a combine kernel of about three tiles' time beside more than one split.  At most four waves of
// CTAs, which bounds the workspace: `bound` gives the most that any smaller maxT or window takes.
static Q8Plan q8_plan(int B, int maxT, int n, int Hq, int Hkv, int Dh, int mode, int window, bool tc, bool bound) {
  Q8Plan p = {};
  p.G = Hq / Hkv;
  p.M = n * p.G;
  p.ngroups = (p.M + decq8::kMaxRows - 1) / decq8::kMaxRows;
  p.rg = ((p.M + p.ngroups - 1) / p.ngroups + 15) / 16 * 16;
  const int KT = q8_tile(Dh, p.rg, tc);
  const long long tiles = (q8_range(maxT, n, mode, window) + KT - 1) / KT, ctas = (long long)B * Hkv * p.ngroups;
  int per_sm = tc ? decode_q8_tc_per_sm(p.rg, Dh) : p.rg > (Dh == 256 ? 16 : 32) ? 1 : p.rg > 16 || Dh == 256 ? 2 : Dh == 64 ? 3 : 4;
  // few tiles: fewer splits, which the combine kernel merges faster (1 x 8192 tokens, 4 streams, 32 over 8 heads of 128, 13
  // tiles an SM: two CTAs an SM 21.2 us, three 23.1; 8 x 2048, 27 tiles: 29.1 and 28.0; both before starts were shortened)
  if (tc && ctas * tiles < 20 * kSmCount) per_sm = std::min(per_sm, 2);
  const long long resident = (long long)kSmCount * per_sm;
  const long long most = std::min({tiles, (long long)dec::kMaxSplit, std::max(1LL, 4 * resident / ctas)});
  const int small = Dh * KT < 128 * 128 ? 2 : 1;  // tiles of half the bytes: twice as many in the time of a start
  long long best = 1, best_cost = -1;
  if (bound) {
    best = most;
  } else {
    for (long long ns = 1; ns <= most; ++ns) {
      const long long per = (tiles + ns - 1) / ns, used = (tiles + per - 1) / per;
      if (used != ns) continue;  // another ns gives the same chunks
      const long long cost = ((ctas * ns + resident - 1) / resident) * (per + 2 * small) + (ns > 1 ? 3 * small : 0);
      if (best_cost < 0 || cost < best_cost) {
        best = ns;
        best_cost = cost;
      }
    }
  }
  p.nsplit = (int)best;
  // Several sequences, long splits: a wave of CTAs shares their tiles equally, whatever the lengths; also where a CTA for
  // each head and sequence would be one wave of long ones, but not several waves, which even lengths out by themselves
  // and write results and not partials.  (One / the other, 4 streams and sequences of lengths from a quarter on, us: 96 over 8
  // heads of 128, 8 x 8192, 8 streams 494 / 340; 3 streams, 16 over 4 of 64, 100 x 2000 76 / 70.5; 96 over 8, 120 x 2000, seven
  // waves, 350 / 361; 60 x 400 68 / 78; 16 x 400, one wave of 13 tiles, 23.4 / 29.1.)
  const long long heads = (long long)Hkv * p.ngroups, range = q8_range(maxT, n, mode, window);
  const bool shared = best > 1 ? range / best >= 4 * 64 : ctas <= resident && tiles >= 32;
  if (tc && B > 1 && B <= dec::kBalancedSeqs && (bound || shared)) p.total = (int)std::max(1LL, resident / heads);
  const size_t parts = std::max((size_t)ctas * best, p.total > 0 ? (size_t)(p.total + B) * heads : 0);
  p.part_o_bytes = parts * p.rg * Dh * sizeof(float);
  p.part_ml_bytes = parts * p.rg * sizeof(float2);
  return p;
}

size_t decode_paged_q8_ws_bytes(int B, int maxT, int n, int Hq, int Hkv, int Dh, int mode, int window) {
  // either kernel's, whatever the pages
  const size_t x = q8_plan(B, maxT, n, Hq, Hkv, Dh, mode, window, false, true).bytes();
  return std::max(x, q8_plan(B, maxT, n, Hq, Hkv, Dh, mode, window, true, true).bytes());
}

template <int DH, int MT>
static cudaError_t launch_q8_t(const decq8::Args& a, cudaStream_t st) {
  using namespace decq8;
  const int smem = (int)sizeof(Smem<DH, MT>) + 1024;
  static_assert(Cfg<DH, MT>::kPerSm * (sizeof(Smem<DH, MT>) + 2048) <= 228 * 1024, "an SM's CTAs fit");
  cudaError_t e = cudaFuncSetAttribute(decode_q8_kernel<DH, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_kernel(true, decode_q8_kernel<DH, MT>, dim3((unsigned)a.nsplit * a.B * a.Hkv * a.ngroups),
                       (unsigned)a.rg / 16 * 128, smem, st, a);
}
static cudaError_t launch_q8(const decq8::Args& a, int Dh, cudaStream_t st) {
  if (Dh == 64) return a.rg <= 32 ? launch_q8_t<64, 2>(a, st) : launch_q8_t<64, 4>(a, st);
  if (Dh == 256) return a.rg <= 16 ? launch_q8_t<256, 1>(a, st) : launch_q8_t<256, 4>(a, st);
  return a.rg <= 16 ? launch_q8_t<128, 1>(a, st) : a.rg <= 32 ? launch_q8_t<128, 2>(a, st) : launch_q8_t<128, 4>(a, st);
}

static cudaError_t launch_combine_q8(const decq8::Args& a, int Dh, cudaStream_t st) {
  const long long rows = (long long)std::min(a.rg, a.M) * a.B * a.Hkv * a.ngroups;
  if (rows <= 8 * kSmCount) return launch_combine_paged(a, Dh, st);  // one wave of a CTA each
  const dim3 grid((unsigned)((rows + 7) / 8));
  if (Dh == 64) return launch_early(decq8::combine_rows_kernel<64>, grid, 256, st, a);
  if (Dh == 128) return launch_early(decq8::combine_rows_kernel<128>, grid, 256, st, a);
  return launch_early(decq8::combine_rows_kernel<256>, grid, 256, st, a);
}

cudaError_t launch_sfa_decode_paged_q8(const void* q, const void* kc, const void* vc, const uint8_t* ks, const uint8_t* vs,
                                       const int32_t* table, const int32_t* lens, void* o, float* lse, int B, int maxT,
                                       int num_pages, int P, int max_pages, int n, int Hq, int Hkv, int Dh, int T,
                                       float scale, int mode, int window, void* ws, size_t ws_bytes, int32_t* status,
                                       cudaStream_t st) {
  const long long range = q8_range(maxT, n, mode, window);
  const bool tc = q8_tc(Dh, P * n, n * (Hq / Hkv), range, (long long)B * Hkv);
  const Q8Plan plan = q8_plan(B, maxT, n, Hq, Hkv, Dh, mode, window, tc, false);
  if (plan.bytes() > ws_bytes) return cudaErrorInvalidValue;  // the bound says that it is not
  decq8::Params p = {};
  decq8::Args& a = p.a;
  a.q = (const bf16*)q;
  a.kcodes = (const uint8_t*)kc;
  a.vcodes = (const uint8_t*)vc;
  a.kscale = ks;
  a.vscale = vs;
  a.blocks = P / T;
  a.d_brow = make_fast_div((uint32_t)(T * n));
  a.d_blocks = make_fast_div((uint32_t)a.blocks);
  a.lens = lens;
  a.o = (bf16*)o;
  a.lse = lse;
  a.share = static_cast<int2*>(ws);
  a.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + kShareBytes);
  a.part_ml = reinterpret_cast<float2*>(static_cast<char*>(ws) + kShareBytes + ((plan.part_o_bytes + 255) & ~size_t(255)));
  a.status = status;
  a.B = B;
  a.maxT = maxT;
  a.n = n;
  a.Hq = Hq;
  a.Hkv = Hkv;
  a.G = plan.G;
  a.M = plan.M;
  a.ngroups = plan.ngroups;
  a.nsplit = plan.nsplit;
  a.rg = plan.rg;
  a.mode = mode;
  a.window = window;
  a.scale_log2 = scale * 1.4426950408889634f;
  a.d_nsplit = make_fast_div((uint32_t)plan.nsplit);
  a.table = table;
  a.pg = make_page_geom(num_pages, max_pages, P * n);
  a.d_G = make_fast_div((uint32_t)plan.G);
  a.d_n = make_fast_div((uint32_t)n);
  a.d_heads = make_fast_div((uint32_t)(Hkv * plan.ngroups));
  const int KT = q8_tile(Dh, plan.rg, tc);
  a.piece = paged_piece(a.pg.prow, KT);
  a.tile = tc ? KT / a.piece * a.piece : n <= KT ? KT / n * n : KT;  // whole pieces; whole tokens where a tile holds one
  a.d_tile = make_fast_div((uint32_t)a.tile);
  a.balanced = plan.total > 0;
  a.total = plan.total;
  if (tc && (!make_q8_tmap(&p.tm_k, kc, num_pages, Hkv, a.pg.prow, Dh, a.piece) ||
             !make_q8_tmap(&p.tm_v, vc, num_pages, Hkv, a.pg.prow, Dh, a.piece)))
    return cudaErrorInvalidValue;
  const cudaError_t e = tc ? launch_decode_q8_tc(p, Dh, st) : launch_q8(a, Dh, st);
  return e != cudaSuccess || (a.nsplit == 1 && !a.balanced) ? e : launch_combine_q8(a, Dh, st);
}

}  // namespace hdsfa
