// Decoding over a paged cache (where the tcgen05 kernel of sfa_decode.cu is not taken, see paged_tc):
// the decoding step's split over the cached positions and its warp-level products (mma.sync m16n8k16),
// with the rows found through a page table.
//
// Memory-bound: the K and V tiles of a split stream through a three-stage ring, and what a warp does
// beside its products must not hold the stream up.  So a tile is brought by TMA, in pieces that lie
// within a page: a page's rows as they are where a tile holds some, else the largest divisor of them
// (paged_tile); a tile ends with its last whole piece.  The four warps take turns at bringing tiles
// (issuing one takes a warp up to 1000 cycles) and meet on the stages' barriers alone.  Pieces of fewer than
// kTmaRows rows cost more to issue than to move (about 35 ns each), so such pages go through cp.async,
// 16 bytes a thread, with each row's place looked up a tile ahead.
// (By cp.async for all pages, 8 sequences of 8192 tokens, one stream, 32 over 8 heads: 57.7 us; so 47.)
//
// In shared memory a K or V tile is DH/64 blocks of [KT][64] with the 128-byte swizzle that TMA
// writes: conflict-free for ldmatrix as well.  Splits, partials and the combine kernel are those of
// the contiguous cache; a masked key's V row that is not finite is settled by exact_row.  P is rounded to
// bf16 for its product, whose operands have one type (at most 2^-8 of each term, as O's own rounding);
// maxima, sums, partials and LSE are fp32.
#include <float.h>

#include <algorithm>

#include "decode.cuh"
#include "decode_plan.cuh"
#include "tc_common.cuh"

namespace hdsfa {
namespace dec {
constexpr int kTmaRows = 8;

template <int DH, int MT>
struct PagedSmem {
  static constexpr int KT = ktile<DH>();
  bf16 k[STAGES][KT * DH];
  bf16 v[STAGES][KT * DH];
  bf16 q[MT * 16 * DH];
  int row[4][KT];  // cp.async: the pool rows of four tiles (of which three are loaded or about to be)
  uint64_t full[STAGES], empty[STAGES];
  int bad_page, abort;
  unsigned not_finite;  // a bit per row of the merged partial
};

struct PagedParams {
  CUtensorMap tm_k, tm_v;
  DecodeArgs a;
};

// Element offset of (row, col) in a tile of DH/64 swizzled blocks of [KT][64].
template <int KT>
HD_DEVINLINE int blk(int row, int col) {
  return (col >> 6) * (KT * 64) + row * 64 + ((((col >> 3) & 7) ^ (row & 7)) << 3) + (col & 7);
}

// A finished row by one warp: o / l and its LSE, or an empty row (l = 0).
template <int DH>
HD_DEVINLINE void store_row(const DecodeArgs& a, int b, int g, int r, const float* o, float m, float l) {
  const int lane = threadIdx.x & 31, s = r / a.G, h = g * a.G + r % a.G;
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

template <int DH, int MT, bool TMA>
__global__ void __launch_bounds__(NT, DH == 64 ? (MT == 1 ? 4 : 3) : 2)
    decode_paged_kernel(const __grid_constant__ PagedParams P) {
  constexpr int DS = dsplit<DH>(), KT = ktile<DH>(), KW = 4 / DS, DC = DH / DS;  // DC: O columns per warp
  constexpr int CPR = DH / 8;
  using Smem = PagedSmem<DH, MT>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const DecodeArgs& a = P.a;
  {
    uint32_t dyn;
    asm("mov.u32 %0, %%dynamic_smem_size;\n" : "=r"(dyn));
    const uint32_t pad = (1024 - (smem_u32(smem_raw) & 1023)) & 1023;
    if (pad + sizeof(Smem) > dyn) {  // uniform: nothing touched yet
      if (threadIdx.x == 0) set_status(a.status, HD_DEVBIT_TIMEOUT);
      return;
    }
  }
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int split = fast_div((int)blockIdx.x, a.d_heads), head = (int)blockIdx.x - split * a.Hkv * a.ngroups;
  const int g = a.ngroups == 1 ? head : head / a.ngroups, rg = a.ngroups == 1 ? 0 : head % a.ngroups;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g4 = lane >> 2, t4 = lane & 3;
  const int kw = warp / DS, dw = warp % DS;  // key group and head-dim part of this warp
  const size_t pidx = blockIdx.x;
  float* po = a.part_o + pidx * RG * DH;
  float2* pml = a.part_ml + pidx * RG;
  const int tile = a.tile;
  if (TMA && tid == 32) {
    tma_prefetch(&P.tm_k);
    tma_prefetch(&P.tm_v);
  }
  if (tid == 0) {
    sm.bad_page = sm.abort = 0;
    sm.not_finite = 0;
    if (TMA) {
      for (int i = 0; i < STAGES; ++i) {
        mbar_init(&sm.full[i], 1);
        mbar_init(&sm.empty[i], 4);  // one arrival per warp
      }
      fence_mbar_init();
    }
  }
  // rows that no piece fills: their P is zero, and their V must not be infinite or NaN
  if (TMA && tile < KT)
    for (int i = tid; i < STAGES * (DH / 64) * (KT - tile) * 8; i += NT) {
      const int blkno = i / ((KT - tile) * 8), e = i % ((KT - tile) * 8);
      reinterpret_cast<uint4*>(sm.v[0] + (size_t)blkno * KT * 64 + tile * 64)[e] = make_uint4(0, 0, 0, 0);
    }
  // What needs nothing from the kernels before this one.  This thread's query rows: (mt, half) -> local
  // row mt*16 + g4 + 8*half, its stream (-1: padding row).  Where n divides a tile, which of this
  // thread's keys are of a row's stream is the same in every tile.
  int rs_[MT][2];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int r = rg * RG + mt * 16 + g4 + 8 * hf;
      rs_[mt][hf] = r < a.M ? fast_div(r, a.d_G) : -1;
    }
  const bool streams = a.mode == SFA_WITHIN && a.n > 1;
  const bool shifting = streams && tile - fast_div(tile, a.d_n) * a.n != 0;
  uint32_t mine = 0;                            // bit mt*8 + hf*4 + j*2 + e: the row may see the key
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int key = kw * 16 + (i >> 1) * 8 + 2 * t4 + (i & 1);
    const int ks = streams && !shifting ? key - fast_div(key, a.d_n) * a.n : -1;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
        if (rs_[mt][hf] >= 0 && key < tile && (ks < 0 || ks == rs_[mt][hf])) mine |= 1u << (mt * 8 + hf * 4 + i);
  }
  grid_dep_wait();
  grid_dep_launch();
  const int b = fast_div(split, a.d_nsplit), T = a.lens[b];
  const int32_t* table = a.table + (long long)b * a.pg.max_pages;
  auto load_q = [&] {  // query rows of the group (rows past M zero-filled)
    for (int i = tid; i < MT * 16 * CPR; i += NT) {
      const int rr = i / CPR, cc = i % CPR, r = rg * RG + rr;
      const bool ok = r < a.M;
      const int s = ok ? fast_div(r, a.d_G) : 0, h = g * a.G + (ok ? r - s * a.G : 0);
      cp_async_16(smem_u32(sm.q + swz<DH>(rr, cc * 8)), a.q + (((long long)b * a.n + s) * a.Hq + h) * DH + cc * 8, ok);
    }
  };
  int k0, k1;
  split_range<true>(a, T, split - b * a.nsplit, tile, k0, k1);
  if (k0 >= k1) {  // nothing of this sequence in this split: an empty partial, or an empty result
    if (a.nsplit > 1) {
      for (int i = tid; i < RG; i += NT) pml[i] = make_float2(-INFINITY, 0.f);
    } else {
      if (T != 0 && g == 0 && rg == 0 && tid == 0) set_status(a.status, HD_DEVBIT_INDEX);
      for (int row = warp; row < min(MT * 16, a.M - rg * RG); row += 4)
        store_row<DH>(a, b, g, rg * RG + row, nullptr, -INFINITY, 0.f);
    }
    return;
  }
  const int nsub = fast_div(k1 - k0 + tile - 1, a.d_tile);
  __syncthreads();  // the barriers and flags are set

  // ---- the tiles' loads
  const int seen = a.mode == SFA_LOCAL ? (T - 1) * a.n - a.window + 1 : 0;  // first position any row sees
  // TMA: tile t is brought by warp (t + 2) & 3, two tiles ahead of the products; lane i brings piece i,
  // whose page entry it has looked up when it issued its last tile, four tiles before
  auto pos_of = [&](int t) {  // first position of this lane's piece of a tile, -1: none that a row sees
    const int p = lane * a.piece, pos = k0 + t * tile + p;
    return p >= tile || pos >= k1 || pos + a.piece <= seen ? -1 : pos;
  };
  int entry = 0;
  auto fetch = [&](int t) {
    const int pos = pos_of(t);
    if (pos >= 0) entry = table[fast_div(pos, a.pg.d_prow)];
  };
  // cp.async: pool row of this thread's position of a tile (-1: none that a row sees)
  auto row_of = [&](int it) {
    const int p = k0 + it * tile + tid;
    if (tid >= tile || p >= k1 || p < seen) return -1;
    const int row = page_row(a.pg, table, p);
    if (row < 0) sm.bad_page = 1;
    return row;
  };
  [[maybe_unused]] int brought = -1;  // TMA: the last tile that this warp brought
  auto load_tile = [&](int it) {
    const int st = it % STAGES;
    if constexpr (TMA) {
      brought = it;
      if (lane == 0) mbar_arrive_expect_tx(&sm.full[st], tile * DH * 2 * 2);
      __syncwarp();
      if (lane * a.piece < tile) {
        const int pos = pos_of(it);
        int row = a.pg.num_pages * a.pg.prow;  // behind the pool: zeros
        if (pos >= 0) {
          if ((unsigned)entry < (unsigned)a.pg.num_pages)
            row = entry * a.pg.prow + pos - fast_div(pos, a.pg.d_prow) * a.pg.prow;
          else
            sm.bad_page = 1;
        }
#pragma unroll
        for (int cb = 0; cb < DH / 64; ++cb) {
          tma_load_5d(sm.k[st] + cb * KT * 64 + lane * a.piece * 64, &P.tm_k, &sm.full[st], cb * 64, g, 0, row, 0);
          tma_load_5d(sm.v[st] + cb * KT * 64 + lane * a.piece * 64, &P.tm_v, &sm.full[st], cb * 64, g, 0, row, 0);
        }
      }
      __syncwarp();
      fetch(it + 4);
    } else {
      for (int i = tid; i < KT * CPR; i += NT) {
        const int rr = i / CPR, cc = i % CPR, row = rr < tile ? sm.row[it & 3][rr] : -1;
        const long long off = ((long long)max(row, 0) * a.Hkv + g) * DH + cc * 8;
        cp_async_16(smem_u32(sm.k[st] + blk<KT>(rr, cc * 8)), a.kc + off, row >= 0);
        cp_async_16(smem_u32(sm.v[st] + blk<KT>(rr, cc * 8)), a.vc + off, row >= 0);
      }
    }
  };
  if constexpr (TMA) {
    const int t = (warp + 2) & 3;  // this warp's first tile
    fetch(t);
    if (t < min(2, nsub)) load_tile(t);
    load_q();
    cp_async_commit();
    cp_async_wait<0>();
    __syncthreads();
  } else {
    const int r0 = row_of(0), r1 = row_of(1), r2 = row_of(2);
    if (tid < tile) sm.row[0][tid] = r0, sm.row[1][tid] = r1, sm.row[2][tid] = r2;
    __syncthreads();
    load_q();
    load_tile(0);
    cp_async_commit();
    if (nsub > 1) load_tile(1);
    cp_async_commit();
  }

  const int own_lo = (T - 1) * a.n, win_hi = a.mode == SFA_LOCAL ? T * a.n - 1 - a.window : -1;
  float mx[MT][2], ls[MT][2], oacc[MT][DC / 8][4];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    mx[mt][0] = mx[mt][1] = -INFINITY;
    ls[mt][0] = ls[mt][1] = 0.f;
#pragma unroll
    for (int i = 0; i < DC / 8; ++i) oacc[mt][i][0] = oacc[mt][i][1] = oacc[mt][i][2] = oacc[mt][i][3] = 0.f;
  }

  bool alive = true;
  for (int it = 0; it < nsub; ++it) {
    const int st = it % STAGES, base = k0 + it * tile;
    int next_row = -1;
    if constexpr (TMA) {
      // the warps meet on the stages' barriers alone: one that loads does not hold up the others
      if ((it & 3) == warp && it + 2 < nsub) {
        const int t = it + 2;
        if (t >= STAGES)
          alive = __all_sync(0xffffffffu, mbar_wait(&sm.empty[t % STAGES], (t / STAGES - 1) & 1, &sm.abort, a.status));
        if (alive) load_tile(t);
      }
      alive = alive && __all_sync(0xffffffffu, mbar_wait(&sm.full[st], (it / STAGES) & 1, &sm.abort, a.status));
      if (!alive) break;
      if (base + tile > k1) {  // cached rows behind the sequence's length may never have been written
        const int r0 = max(kw * 16, k1 - base), r1 = min(kw * 16 + 16, tile);
        for (int i = r0 * 8 + lane; i < r1 * 8; i += 32)
#pragma unroll
          for (int cb = 0; cb < DH / 64; ++cb) reinterpret_cast<uint4*>(sm.v[st] + cb * KT * 64)[i] = make_uint4(0, 0, 0, 0);
        __syncwarp();
      }
    } else {
      cp_async_wait<STAGES - 2>();  // stage `it` has landed
      __syncthreads();              // ... for every thread, and stage it-1 is no longer read
      if (it + 2 < nsub) load_tile(it + 2);
      cp_async_commit();
      next_row = row_of(it + 3);  // the rows that the next iteration loads by
    }
    const bf16 *cK = sm.k[st], *cV = sm.v[st];

    float sacc[MT][2][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int j = 0; j < 2; ++j) sacc[mt][j][0] = sacc[mt][j][1] = sacc[mt][j][2] = sacc[mt][j][3] = 0.f;
#pragma unroll
    for (int kk = 0; kk < DH / 16; ++kk) {
      uint32_t b0, b1, b2, b3;
      ldsm_x4(smem_u32(cK + blk<KT>(kw * 16 + (lane & 7) + (lane >> 4) * 8, kk * 16 + ((lane >> 3) & 1) * 8)), b0, b1, b2,
              b3);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        uint32_t qa[4];
        ldsm_x4(smem_u32(sm.q + swz<DH>(mt * 16 + (lane & 15), kk * 16 + (lane >> 4) * 8)), qa[0], qa[1], qa[2], qa[3]);
        mma_bf16_16816(sacc[mt][0], qa, b0, b1);
        mma_bf16_16816(sacc[mt][1], qa, b2, b3);
      }
    }
    // mask + online softmax (log2 domain)
    uint32_t vis = mine;
    const int kb = base + kw * 16 + 2 * t4;
    if (base + tile - 1 > own_lo || base + tile > k1 || base <= win_hi || shifting) {
      // positions at the sequence's end, at the rows' windows, or streams that shift from tile to tile
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int hf = i >> 2, p = kb + ((i >> 1) & 1) * 8 + (i & 1), pq = own_lo + rs_[mt][hf];
          const bool in = p < k1 && p <= pq && (a.mode != SFA_LOCAL || p > pq - a.window) &&
                          (!shifting || p - fast_div(p, a.d_n) * a.n == rs_[mt][hf]);
          if (!in) vis &= ~(1u << (mt * 8 + i));
        }
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      float tmax[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const int hf = e4 >> 1, bit = mt * 8 + hf * 4 + j * 2 + (e4 & 1);
          const float x = (vis >> bit) & 1u ? sacc[mt][j][e4] * a.scale_log2 : -INFINITY;
          sacc[mt][j][e4] = x;
          tmax[hf] = fmaxf(tmax[hf], x);
        }
      float corr[2], muse[2];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        tmax[hf] = fmaxf(tmax[hf], __shfl_xor_sync(0xffffffffu, tmax[hf], 1));
        tmax[hf] = fmaxf(tmax[hf], __shfl_xor_sync(0xffffffffu, tmax[hf], 2));
        const float mnew = fmaxf(mx[mt][hf], tmax[hf]);
        muse[hf] = mnew == -INFINITY ? 0.f : mnew;
        corr[hf] = ex2_approx(mx[mt][hf] - muse[hf]);
        mx[mt][hf] = mnew;
        ls[mt][hf] *= corr[hf];
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e4 = 0; e4 < 4; ++e4) {
          const float p = ex2_approx(sacc[mt][j][e4] - muse[e4 >> 1]);
          sacc[mt][j][e4] = p;
          ls[mt][e4 >> 1] += p;
        }
      if (__any_sync(0xffffffffu, corr[0] != 1.f || corr[1] != 1.f)) {
#pragma unroll
        for (int i = 0; i < DC / 8; ++i) {
          oacc[mt][i][0] *= corr[0];
          oacc[mt][i][1] *= corr[0];
          oacc[mt][i][2] *= corr[1];
          oacc[mt][i][3] *= corr[1];
        }
      }
    }
    // O += P V over this warp's 16 keys
    uint32_t pa[MT][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      pa[mt][0] = pack_bf16(sacc[mt][0][0], sacc[mt][0][1]);
      pa[mt][1] = pack_bf16(sacc[mt][0][2], sacc[mt][0][3]);
      pa[mt][2] = pack_bf16(sacc[mt][1][0], sacc[mt][1][1]);
      pa[mt][3] = pack_bf16(sacc[mt][1][2], sacc[mt][1][3]);
    }
#pragma unroll
    for (int dp = 0; dp < DC / 16; ++dp) {
      uint32_t b0, b1, b2, b3;
      ldsm_x4_t(smem_u32(cV + blk<KT>(kw * 16 + (lane & 7) + ((lane >> 3) & 1) * 8, dw * DC + dp * 16 + (lane >> 4) * 8)),
                b0, b1, b2, b3);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        mma_bf16_16816(oacc[mt][2 * dp], pa[mt], b0, b1);
        mma_bf16_16816(oacc[mt][2 * dp + 1], pa[mt], b2, b3);
      }
    }
    if constexpr (TMA) {
      __syncwarp();
      if (lane == 0) mbar_arrive(&sm.empty[st]);
    } else if (tid < tile) {
      sm.row[(it + 3) & 3][tid] = next_row;
    }
  }
  if constexpr (TMA) {
    // a wait gave up: the results are invalid.  A warp that goes on has seen every tile land; one that does not
    // waits (again with a limit) for the last that it brought, whose stage no earlier one can still be filling.
    if (!alive && brought >= 0 && lane == 0) mbar_drain(&sm.full[brought % STAGES], (brought / STAGES) & 1);
    if (__syncthreads_or(!alive)) return;
  }

  // merge the 4 warps' partials in shared memory (the K/V ring is free now)
  if (!TMA) {
    cp_async_wait<0>();
    __syncthreads();
  }
  // [KW][MT*16][DH]: key group kw's O, its head-dim parts side by side; then the key
  // groups' running max and sum (the DS warps of a key group hold the same ones)
  static_assert((KW * MT * 16 * DH + 2 * KW * MT * 16) * 4 <= 2 * STAGES * KT * DH * 2, "merge fits the ring");
  static_assert(MT * 16 <= NT, "one thread per row");
  float* sO = reinterpret_cast<float*>(sm.k[0]);
  float* sM = sO + KW * MT * 16 * DH;  // [KW][MT*16]
  float* sL = sM + KW * MT * 16;       // [KW][MT*16]
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      ls[mt][hf] += __shfl_xor_sync(0xffffffffu, ls[mt][hf], 1);
      ls[mt][hf] += __shfl_xor_sync(0xffffffffu, ls[mt][hf], 2);
      const int row = mt * 16 + g4 + 8 * hf;
      if (t4 == 0 && dw == 0) {
        sM[kw * MT * 16 + row] = mx[mt][hf];
        sL[kw * MT * 16 + row] = ls[mt][hf];
      }
    }
#pragma unroll
    for (int i = 0; i < DC / 8; ++i)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const int row = mt * 16 + g4 + 8 * hf, col = dw * DC + i * 8 + 2 * t4;
        *reinterpret_cast<float2*>(sO + (kw * MT * 16 + row) * DH + col) =
            make_float2(oacc[mt][i][2 * hf], oacc[mt][i][2 * hf + 1]);
      }
  }
  __syncthreads();
  const bool bad = sm.bad_page != 0;
  // one thread per row: its maximum and sum over the key groups, whose weights replace
  // their maxima
  if (tid < MT * 16) {
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int w = 0; w < KW; ++w) m = fmaxf(m, sM[w * MT * 16 + tid]);
    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const float f = exp2f(sM[w * MT * 16 + tid] - mu);
      l += f * sL[w * MT * 16 + tid];
      sM[w * MT * 16 + tid] = f;
    }
    if (l != l) m = INFINITY;  // a visible score that is not finite: the combined row is NaN
    if (bad) m = -INFINITY, l = kBadPage;
    pml[tid] = make_float2(m, l);
    if (a.nsplit == 1 && bad && tid == 0) set_status(a.status, HD_DEVBIT_INDEX);
  }
  __syncthreads();
  for (int idx = tid; idx < MT * 16 * (DH / 4); idx += NT) {
    const int row = idx / (DH / 4), c4 = idx % (DH / 4);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const float f = sM[w * MT * 16 + row];
      const float4 v = *reinterpret_cast<const float4*>(sO + (w * MT * 16 + row) * DH + c4 * 4);
      o.x += f * v.x;
      o.y += f * v.y;
      o.z += f * v.z;
      o.w += f * v.w;
    }
    *reinterpret_cast<float4*>(po + row * DH + c4 * 4) = o;
    if (!(fabsf(o.x) + fabsf(o.y) + fabsf(o.z) + fabsf(o.w) <= FLT_MAX)) atomicOr(&sm.not_finite, 1u << row);
  }
  __syncthreads();
  if (!bad)
    for (unsigned rows = sm.not_finite; rows; rows &= rows - 1) {
      const int row = __ffs(rows) - 1;
      if ((row & 3) == warp && rg * RG + row < a.M)
        exact_row<DH>(a, b, g, rg * RG + row, T, k0, k1, po + row * DH, pml + row);
    }
  if (a.nsplit > 1) return;
  // the only split: its rows are the results
  __syncthreads();
  for (int row = warp; row < min(MT * 16, a.M - rg * RG); row += 4) {
    const float2 ml = pml[row];
    store_row<DH>(a, b, g, rg * RG + row, po + row * DH, ml.x, bad ? 0.f : ml.y);
  }
}
}  // namespace dec

// ------------------------------------------------------------------ host side

// Positions that a step of maxT tokens reads at most.
static long long paged_range(int maxT, int n, int mode, int window) {
  return mode == SFA_LOCAL ? std::min<long long>((long long)maxT * n, (long long)window + n - 1) : (long long)maxT * n;
}

// The contiguous cache's plan, with the combine kernel (about three tiles' time, nothing to do for one
// split) in the cost: short sequences take one split, whose CTAs write the results.  (Four resident CTAs at
// head dim 64 are the contiguous kernel's and this one's for up to 16 query rows; with more rows its 158 to
// 160 registers leave room for three.)
static DecodePlan paged_plan(int B, int maxT, int n, int Hq, int Hkv, int Dh, int mode, int window,
                             TcDims tc_dims) {
  DecodePlan p = decode_plan(B, maxT, n, Hq, Hkv, Dh, mode, window, tc_dims);
  if (p.tc || p.nsplit == 1) return p;
  const long long range = paged_range(maxT, n, mode, window);
  const int KT = Dh == 256 ? dec::ktile<256>() : dec::ktile<128>();
  const long long tiles = (range + KT - 1) / KT, per = (tiles + p.nsplit - 1) / p.nsplit;
  const long long ctas = (long long)B * Hkv * p.ngroups, resident = 152LL * (Dh == 64 ? 4 : 2);
  const long long split = ((ctas * p.nsplit + resident - 1) / resident) * (per + 2) + 3,
                  whole = ((ctas + resident - 1) / resident) * (tiles + 2);
  if (whole <= split) p.nsplit = 1;
  return p;
}

// The sequences' shares of a balanced batch's splits, in front of the partials.
constexpr size_t kShareBytes = dec::kBalancedSeqs * sizeof(int2);

size_t decode_paged_ws_bytes(int B, int maxT, int n, int Hq, int Hkv, int Dh, int mode, int window) {
  // either kernel's, whatever the pages, and enough for every smaller maxT and window
  return std::max(decode_ws_bytes(decode_plan_bound(B, maxT, n, Hq, Hkv, Dh, mode, window, TcDims::kWith128)),
                  decode_ws_bytes(decode_plan_bound(B, maxT, n, Hq, Hkv, Dh, mode, window, TcDims::kNone))) + kShareBytes;
}

// A tile of at most `most` positions: whole pieces of pages.
static void paged_tile(dec::DecodeArgs& a, int most) {
  a.piece = paged_piece(a.pg.prow, most);
  a.tile = most / a.piece * a.piece;
  a.d_tile = make_fast_div((uint32_t)a.tile);
}

template <int DH, int MT, bool TMA>
static cudaError_t launch_paged_t(const dec::PagedParams& p, cudaStream_t st) {
  using namespace dec;
  // two CTAs fit an SM only without room to align the base at head dim 256, where it is aligned as it
  // is (checked on entry)
  const int smem = (int)sizeof(PagedSmem<DH, MT>) + (DH == 256 ? 0 : 1024);
  cudaError_t e = cudaFuncSetAttribute(decode_paged_kernel<DH, MT, TMA>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_kernel(true, decode_paged_kernel<DH, MT, TMA>, dim3((unsigned)p.a.nsplit * p.a.B * p.a.Hkv * p.a.ngroups), NT,
                       smem, st, p);
}

template <int DH, bool TMA>
static cudaError_t launch_paged_d(const dec::PagedParams& p, cudaStream_t st) {
  // a row group of more than 16 rows takes two m16 tiles
  return p.a.M > 16 ? launch_paged_t<DH, 2, TMA>(p, st) : launch_paged_t<DH, 1, TMA>(p, st);
}

cudaError_t launch_sfa_decode_paged(const void* q, const void* kp, const void* vp, const int32_t* table,
                                    const int32_t* lens, void* o, float* lse, int B, int maxT, int num_pages, int P,
                                    int max_pages, int n, int Hq, int Hkv, int Dh, float scale, int mode, int window,
                                    void* ws, size_t ws_bytes, int32_t* status, cudaStream_t st) {
  const long long range = paged_range(maxT, n, mode, window);
  const DecodePlan plan = paged_plan(B, maxT, n, Hq, Hkv, Dh, mode, window, paged_tc(B, n, Hq, Hkv, Dh, paged_piece(P * n, 128), range));
  if (kShareBytes + decode_ws_bytes(plan) > ws_bytes) return cudaErrorInvalidValue;  // the bound says that it is not
  dec::PagedParams p = {};
  dec::DecodeArgs& a = p.a;
  a.q = (const bf16*)q;
  a.kc = (const bf16*)kp;
  a.vc = (const bf16*)vp;
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
  if (plan.tc) {
    paged_tile(a, 128);
    // Splits shared out by length, where they are of some tiles (finding one takes about 0.5 us).  This
    // kernel has an SM to itself, so nobody takes up what a short sequence's split leaves: 7 sequences
    // of a quarter to all of 8192 tokens, 24 over 2 heads, 68.2 -> 60.9 us.  The other kernel's two
    // CTAs per SM do (4 and 16 such sequences 69.3 and 113 us, shared out 72.0 and 115).
    a.balanced = B > 1 && B <= dec::kBalancedSeqs && plan.nsplit > 1 && range / plan.nsplit >= 4 * 64 &&
                 B * (range / a.tile + 1) < (1LL << 30);  // the tiles of all sequences, counted in 32 bits
    return launch_decode_paged_tc(a, Dh, st);
  }
  const int KT = Dh == 256 ? dec::ktile<256>() : dec::ktile<128>();
  paged_tile(a, KT);
  const bool tma = a.piece >= dec::kTmaRows;
  if (tma) {
    SfaGeom gk = {};  // the pool as one problem of all its rows
    gk.B = 1;
    gk.nL = gk.Lv = a.pg.num_pages * a.pg.prow;
    gk.Hkv = Hkv;
    gk.ns = gk.rs = 1;
    if (!make_rows_tmap(&p.tm_k, kp, gk, Hkv, Dh, a.piece) || !make_rows_tmap(&p.tm_v, vp, gk, Hkv, Dh, a.piece))
      return cudaErrorInvalidValue;
  } else {
    a.tile = n <= KT ? KT / n * n : KT;  // any rows: whole tokens where a tile holds one
    a.d_tile = make_fast_div((uint32_t)a.tile);
  }
  cudaError_t e;
  if (Dh == 64)
    e = tma ? launch_paged_d<64, true>(p, st) : launch_paged_d<64, false>(p, st);
  else if (Dh == 128)
    e = tma ? launch_paged_d<128, true>(p, st) : launch_paged_d<128, false>(p, st);
  else
    e = tma ? launch_paged_d<256, true>(p, st) : launch_paged_d<256, false>(p, st);
  return e != cudaSuccess || a.nsplit == 1 ? e : launch_combine_paged(a, Dh, st);
}

}  // namespace hdsfa
