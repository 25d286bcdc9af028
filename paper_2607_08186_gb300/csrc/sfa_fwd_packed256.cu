// Attention over packed prompts of different lengths on the sm_103a tensor cores, head dim 256: the
// tile plan of the head-dim-256 forward (a pair of CTAs on two query tiles, each loading half of every
// K and V tile) in a persistent kernel over a list of query tiles, as for the smaller head dims: one
// pair on two SMs works through its places of the list, and the next entry's K and Q are loaded, and
// its first S is computed, while this one's last tile is finished and stored.
//   smem   Q (four [128][64] swizzle blocks, 64 KB), a ring of five 32 KB slots: of a K tile this CTA's
//          64 keys, of a V tile this CTA's 128 head-dim columns.
//   TMEM   S in two 128-column buffers (P packed bf16 over its S, each 64-key half at the start of its
//          own columns), O over columns 256..511.
//   issue  S of an entry's first tile, then per tile t: S(t+1), O += P(t) V(t).
// Tiles and ring units are counted through all entries, so barrier phases run on from one to the next.
// Roles per CTA (320 threads): warp 0 TMA producer; warp 1 MMA issuer (the pair's first CTA only) and
// TMEM owner; warps 2..9 online softmax, two threads per query row (TMEM lane), each half of a tile's
// keys; the two exchange their maximum through shared memory.  P is published in two parts.
// A full barrier lives in the first CTA and counts both CTAs' bytes; commits are multicast.  An
// entry's last V tile is loaded on a barrier of each CTA's own (v_tail), since its threads zero the
// rows behind the sequence (see the forward of the smaller head dims for why).
// Short sequences that lie together share a tile, as there.
// Before, as one pair per entry: 16000 cycles for an entry of one key tile, of which 2060 are MMAs.
// Every mbarrier wait is bounded.
#include "packed.cuh"
#include "tc_common.cuh"

namespace hdsfa {

typedef __nv_bfloat16 bf16;

namespace packed256 {
constexpr int DH = 256, BM = 128, BN = 128, NSLOT = 5, NTHREADS = 320;
constexpr int HB = 64;   // keys of a K tile that a CTA loads, and keys of one softmax thread
constexpr int PC = 128;  // head-dim columns of a V tile that a CTA loads, and of O per softmax thread
constexpr uint32_t COL_O = 256;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRescaleThreshold = 8.0f;  // log2 units: P stays <= 256 between O rescales

struct Smem {
  bf16 q[BM * DH];            // four [128 rows][64] swizzle blocks
  bf16 ring[NSLOT][HB * DH];  // K: four [64 keys][64] swizzle blocks; V: two [128 keys][64]
  float part[2][2][BM];       // by tile parity and key half: a row's maximum, at an entry's end its sum
  uint8_t odd[2][BM];         // at the end: whether a thread's half rows of O held a value that is not finite
  // S and PV of a tile complete: by tile mod 4, since the producer, which takes them as the release
  // of K and V, may be up to two tiles late; V(last) landed in this CTA, by entry mod 4 (the ring
  // holds the last V tiles of up to three entries)
  uint64_t s_full[4], pv_done[4], v_tail[4];
  uint64_t full[NSLOT], q_full[DH / 64], p_full[2][2], drain;
  int held[NSLOT];  // producer: the tile whose K (2 * tile) or V (2 * tile + 1) a slot holds
  uint32_t tmem_base;
  int abort;
};
// The layout needs 1024-byte alignment; the kernel checks the actual pad on entry.
constexpr int kSmemBytes = sizeof(Smem) + 1024 < 232448 ? (int)sizeof(Smem) + 1024 : 232448;
static_assert(sizeof(Smem) <= 232448, "shared memory exceeds 227 KB");

struct Params {
  CUtensorMap tm_q, tm_k, tm_v;  // boxes of 128 (Q, V) and 64 (K) rows x 64 columns
  PackedArgs a;
};

// First key tile of an entry and their number (>= 1).
HD_DEVINLINE void key_tiles(const PackedArgs& a, const PackedEntry& w, int& lo, int& T) {
  lo = packed_lo(a, w.m0);
  T = (min(w.m0 + (a.head_pairs ? BM : 2 * BM), w.rows) - 1) / BN - lo + 1;
}
HD_DEVINLINE int place_of(int k) { return packed_place(k, (int)(blockIdx.x >> 1), (int)(gridDim.x >> 1)); }

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(NTHREADS, 1)
    fwd_packed256_kernel(const __grid_constant__ Params P) {
  extern __shared__ uint8_t smem_raw[];
  const PackedArgs& A = P.a;
  {
    uint32_t dyn;
    asm("mov.u32 %0, %%dynamic_smem_size;\n" : "=r"(dyn));
    const uintptr_t base = reinterpret_cast<uintptr_t>(smem_raw);
    if (((base + 1023) & ~uintptr_t(1023)) - base + sizeof(Smem) > dyn) {  // uniform: nothing touched yet
      if (threadIdx.x == 0) set_status(A.status, HD_DEVBIT_TIMEOUT);
      return;
    }
  }
  Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = (int)(blockIdx.x & 1);  // = %cluster_ctarank
  if (threadIdx.x == 0) {
    for (int i = 0; i < NSLOT; ++i) mbar_init(&sm.full[i], 1);
    for (int i = 0; i < 4; ++i) {
      mbar_init(&sm.s_full[i], 1);
      mbar_init(&sm.pv_done[i], 1);
      mbar_init(&sm.v_tail[i], 1);
    }
    for (int i = 0; i < DH / 64; ++i) mbar_init(&sm.q_full[i], 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.p_full[i][0], 16);  // one arrival per softmax warp of the pair
      mbar_init(&sm.p_full[i][1], 16);
    }
    mbar_init(&sm.drain, 1);
    sm.abort = 0;
    fence_mbar_init();
  }
  __syncwarp();
  cluster_arrive();  // the barriers of this CTA are initialised
  if (warp == 1) {
    tma_prefetch(&P.tm_q);
    tma_prefetch(&P.tm_k);
    tma_prefetch(&P.tm_v);
    tmem_alloc_pair(&sm.tmem_base, 512);
    tc_fence_before();
  }
  grid_dep_wait();
  grid_dep_launch();  // at most one CTA per SM: the next kernel's find their places as these end
  const int total = *A.list.count * A.per;
  cluster_wait();
  uint32_t tmem = 0;
  if (warp != 0) {  // the producer does not wait for the TMEM allocation
    named_bar_sync(5, NTHREADS - 32);
    tc_fence_after();
    tmem = sm.tmem_base;
  }
  volatile int* abort = &sm.abort;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      // Units in the ring, entry after entry: K(0), then K(t+1), V(t) for each tile.  A slot is free
      // once the MMAs that read what it holds have completed.
      int units = 0, slot = 0, tiles = 0;  // ... and tiles of the entries before
      int queries = 0, tails = 0;          // entries whose Q, and whose last V, have been asked for
      bool ok = true;
      for (int k = 0, pos; ok && (pos = place_of(k)) < total; ++k) {
        const PackedEntry w(A, pos);
        int lo, T;
        key_tiles(A, w, lo, T);
        const int kvh = fast_div(w.head, A.d_grp);
        auto load_unit = [&](int t, bool is_v) {
          if (ok && units >= NSLOT) {
            const int h = sm.held[slot], tile = h >> 1;
            ok = mbar_wait((h & 1) ? &sm.pv_done[tile & 3] : &sm.s_full[tile & 3], (tile >> 2) & 1, abort, A.status);
          }
          if (!ok) return;
          sm.held[slot] = 2 * (tiles + t) + (is_v ? 1 : 0);
          const int r0 = w.first + (lo + t) * BN;
          if (is_v && t == T - 1) {
            if (rank == 0) mbar_arrive(&sm.full[slot]);  // nobody waits for this phase; the slot's go on
            uint64_t* bar = &sm.v_tail[k & 3];
            mbar_arrive_expect_tx(bar, BN * PC * 2);
            ++tails;
            for (int c = 0; c < PC / 64; ++c)
              tma_load_5d(sm.ring[slot] + c * BN * 64, &P.tm_v, bar, rank * PC + c * 64, kvh, w.stream, r0, 0);
          } else {
            if (rank == 0) mbar_arrive_expect_tx(&sm.full[slot], 2 * HB * DH * 2);
            const uint32_t lb = lead_addr(&sm.full[slot]);
            if (is_v) {
              for (int c = 0; c < PC / 64; ++c)
                tma_load_pair(sm.ring[slot] + c * BN * 64, &P.tm_v, lb, rank * PC + c * 64, kvh, w.stream, r0, 0);
            } else {
              for (int c = 0; c < DH / 64; ++c)
                tma_load_pair(sm.ring[slot] + c * HB * 64, &P.tm_k, lb, c * 64, kvh, w.stream, r0 + rank * HB, 0);
            }
          }
          ++units;
          if (++slot == NSLOT) slot = 0;
        };
        load_unit(0, false);
        // the last S of the entry before has read Q
        if (ok && k > 0) ok = mbar_wait(&sm.s_full[(tiles - 1) & 3], ((tiles - 1) >> 2) & 1, abort, A.status);
        if (!ok) break;
        ++queries;
        for (int c = 0; c < DH / 64; ++c) {
          if (rank == 0) mbar_arrive_expect_tx(&sm.q_full[c], 2 * BM * 64 * 2);
          tma_load_pair(sm.q + c * BM * 64, &P.tm_q, lead_addr(&sm.q_full[c]), c * 64, w.head_of(A, rank), w.stream,
                        w.first + w.row0(A, rank), 0);
        }
        for (int t = 0; ok && t < T; ++t) {
          if (t + 1 < T) load_unit(t + 1, false);
          load_unit(t, true);
        }
        tiles += T;
      }
      // Every copy that this thread started lands before the pair exits, also after a wait gave up (one limit for
      // all).  On the first CTA's barriers are both CTAs' bytes.
      const long long t0 = clock64();
      auto land = [&](uint64_t* bar, int par) {
        while (!mbar_try_wait(bar, par & 1) && clock64() - t0 < kWaitTimeoutCycles) {
        }
      };
      if (rank == 0) {
        for (int u = max(0, units - NSLOT); u < units; ++u) land(&sm.full[u % NSLOT], u / NSLOT);
        for (int c = 0; queries > 0 && c < DH / 64; ++c) land(&sm.q_full[c], queries - 1);
      }
      for (int k = max(0, tails - 4); k < tails; ++k) land(&sm.v_tail[k & 3], k >> 2);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer (first CTA)
    if (rank == 0) {
      constexpr uint32_t idS = idesc_bf16(2 * BM, BN, 0, 0);  // S = Q K^T, both K-major
      constexpr uint32_t idO = idesc_bf16(2 * BM, DH, 0, 1);  // O += P V: P in TMEM, V MN-major
      // descriptors encoded once; a block, slot or k-step adds its byte offset / 16
      const uint64_t qd = sdesc_sw128(smem_u32(sm.q), 16, 1024);
      const uint64_t kd0 = sdesc_sw128(smem_u32(sm.ring[0]), 16, 1024);
      const uint64_t vd0 = sdesc_sw128(smem_u32(sm.ring[0]), BN * 128, 1024);
      constexpr int SLOT16 = HB * DH * 2 / 16;
      auto wait_w = [&](uint64_t* bar, int par) -> bool {
        if (!__all_sync(0xffffffffu, mbar_wait(bar, par & 1, abort, A.status))) return false;
        tc_fence_after();
        return true;
      };
      auto issue_s = [&](int tile, int slot) {
        const uint64_t kd = kd0 + (uint64_t)(slot * SLOT16);
#pragma unroll
        for (int kk = 0; kk < DH / 16; ++kk)
          mma2_ss(tmem + (tile & 1) * BN, qd + (uint64_t)((kk >> 2) * (BM * 128 / 16) + (kk & 3) * 2),
                  kd + (uint64_t)((kk >> 2) * (HB * 128 / 16) + (kk & 3) * 2), idS, kk > 0 ? 1u : 0u);
        commit2(&sm.s_full[tile & 3]);
      };
      // The first part of P also says that V(t) and K(t+2) have landed.
      auto issue_pv = [&](int tile, bool first, int slot) -> bool {
        const uint64_t vd = vd0 + (uint64_t)(slot * SLOT16);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          if (!wait_w(&sm.p_full[tile & 1][part], tile >> 1)) return false;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            // part 0: keys 0..31 of each 64-key half, part 1: keys 32..63
            const int p = i >> 1, kh = 2 * part + (i & 1), kk = 4 * p + kh;
            mma2_ts(tmem + COL_O, tmem + (tile & 1) * BN + p * HB + kh * 8, vd + (uint64_t)(kk * 16 * 128 / 16), idO,
                    (!first || part > 0 || i > 0) ? 1u : 0u);
          }
        }
        commit2(&sm.pv_done[tile & 3]);
        return true;
      };
      auto next_slot = [](int s) { return s + 1 == NSLOT ? 0 : s + 1; };
      // an entry's first S, on the first 64 columns of Q as soon as they are there
      auto first_s = [&](int tile, int k, int slot) -> bool {
        const uint64_t kd = kd0 + (uint64_t)(slot * SLOT16);
#pragma unroll 1
        for (int c = 0; c < DH / 64; ++c) {
          if (!wait_w(&sm.q_full[c], k)) return false;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            mma2_ss(tmem + (tile & 1) * BN, qd + (uint64_t)(c * (BM * 128 / 16) + i * 2),
                    kd + (uint64_t)(c * (HB * 128 / 16) + i * 2), idS, c + i > 0 ? 1u : 0u);
        }
        commit2(&sm.s_full[tile & 3]);
        return true;
      };
      bool ok = true;
      int slot = 0, units = 0, tile = 0;
      int lo, T = 0;
      if (place_of(0) < total) {
        key_tiles(A, PackedEntry(A, place_of(0)), lo, T);
        ok = wait_w(&sm.full[0], 0) && first_s(0, 0, 0);
      }
      for (int k = 0; ok && place_of(k) < total; ++k) {
        const bool more = place_of(k + 1) < total;
        int nT;
        key_tiles(A, PackedEntry(A, more ? place_of(k + 1) : 0), lo, nT);
        slot = next_slot(slot);  // past K(0)
        if (T > 1) ok = wait_w(&sm.full[slot], (units + 1) / NSLOT);
        for (int t = 0; ok && t < T; ++t, ++tile) {
          // S(t+1) over P(t-1), which PV(t-1), issued before, has read
          if (t + 1 < T) {
            issue_s(tile + 1, slot);
            slot = next_slot(slot);
          }
          ok = issue_pv(tile, t == 0, slot);
          slot = next_slot(slot);
        }
        units += 2 * T;
        // the next entry's first S: the softmax finds it when it has stored O
        if (ok && more) ok = wait_w(&sm.full[slot], units / NSLOT) && first_s(tile, k + 1, slot);
        T = nT;
      }
      // every MMA issued above completes before TMEM / smem are released
      commit2(&sm.drain);
      mbar_drain(&sm.drain, 0);
    }
  } else {
    // ------------------------------------------------------------ softmax / epilogue
    const int q4 = warp & 3, hc = (warp - 2) >> 2;
    const int row = q4 * 32 + lane;
    const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16);
    const uint32_t tO = tl + COL_O + PC * hc;
    const float c2 = A.scale_log2;
    const uint64_t c2x2 = f2pack(c2, c2);
    int units = 0, tile = 0;
    bool ok = true, odd = false;  // odd: a row of this thread's came out not finite
    // (after a wait gave up, the warps go on through the entries: two of them meet on every tile)
    for (int k = 0, pos; (pos = place_of(k)) < total; ++k) {
      const PackedEntry w(A, pos);
      int lo, T;
      key_tiles(A, w, lo, T);
      const int row0 = w.row0(A, rank), r = row0 + row;  // first query row of the tile, the thread's
      const int own = sequence_first(A, w, r);           // first row of the sequence of the thread's row
      float m_run = -INFINITY, l_run = 0.f;              // m_run in raw score units
      for (int t = 0; t < T; ++t, ++tile) {
        const int j = lo + t;
        const uint32_t tS = tl + (uint32_t)((tile & 1) * BN + HB * hc);
        const uint32_t bar_p = lead_addr(sm.p_full[tile & 1]);
        if (ok && rank == 0 && warp == 2 && lane == 0) {
          // V(t) and K(t+2) have landed, before this thread's arrival on p_full
          const int uv = units + 2 * t + 2, uk = uv + 1;
          if (t + 1 < T) mbar_wait(&sm.full[uv % NSLOT], (uv / NSLOT) & 1, abort, A.status);
          if (t + 2 < T) mbar_wait(&sm.full[uk % NSLOT], (uk / NSLOT) & 1, abort, A.status);
        }
        __syncwarp();
        if (ok && t == T - 1) {  // under the S of the tile: this CTA's half of the last V has landed
          ok = __all_sync(0xffffffffu, mbar_wait(&sm.v_tail[k & 3], (k >> 2) & 1, abort, A.status));
          if (ok && (j + 1) * BN > w.rows) {  // its rows behind the sequence
            bf16* vt = sm.ring[(units + 2 * T - 1) % NSLOT];
            for (int e = (w.rows - j * BN) * 8 + hc * BM + row; e < BN * 8; e += 2 * BM)
#pragma unroll
              for (int c = 0; c < PC / 64; ++c) reinterpret_cast<uint4*>(vt + c * BN * 64)[e] = make_uint4(0, 0, 0, 0);
            fence_async_smem();
          }
        }
        // tcgen05.ld/st are warp-collective: every wait result is made warp-uniform
        ok = ok && __all_sync(0xffffffffu, mbar_wait(&sm.s_full[tile & 3], (tile >> 2) & 1, abort, A.status));
        float x[HB], tmax = -INFINITY;
        if (ok) {
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < HB / 32; ++c) tmem_ld32(tS + c * 32, reinterpret_cast<uint32_t*>(x) + c * 32);
          tmem_ld_wait();
          // tiles holding a key past the first query's key row (the diagonal band) or the sequence,
          // and (LOCAL) a key at or below the last query's window edge, or before a row's sequence.  All
          // conditions are the entry's: the warp goes on together to the tcgen05 instructions below.
          if ((j + 1) * BN - 1 > row0 || (j + 1) * BN > w.rows || w.seqs > 0 ||
              (A.g.window > 0 && j * BN <= min(row0 + BM, w.rows) - 1 - A.g.window)) {
            const int k0 = j * BN + HB * hc;
            const int e_hi = min(r, w.rows - 1) - k0;
#pragma unroll
            for (int e = 0; e < HB; ++e)
              if (e > e_hi) x[e] = -INFINITY;
            if (A.g.window > 0 || w.seqs > 0) {
              const int e_lo = max(own, A.g.window > 0 ? r - A.g.window + 1 : 0) - k0;
#pragma unroll
              for (int e = 0; e < HB; ++e)
                if (e < e_lo) x[e] = -INFINITY;
            }
          }
          float mx[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) mx[e] = x[e];
#pragma unroll
          for (int e = 4; e < HB; e += 2) mx[(e >> 1) & 3] = max3(mx[(e >> 1) & 3], x[e], x[e + 1]);
          tmax = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]);
          sm.part[tile & 1][hc][row] = tmax;
        }
        // the two warps of these 32 rows meet here on every tile, also after a wait gave up
        named_bar_sync(1 + q4, 64);
        if (!ok) continue;
        const float m_new = fmaxf(m_run, fmaxf(tmax, sm.part[tile & 1][hc ^ 1][row]));
        const bool rescale = (m_run == -INFINITY) || ((m_new - m_run) * c2 > kRescaleThreshold);
        const float m_use = rescale ? m_new : m_run;
        const float neg = (m_use == -INFINITY) ? 0.f : -m_use * c2;
        const uint64_t neg2 = f2pack(neg, neg);
        uint64_t sum2[4] = {0, 0, 0, 0};
        const bool mine = rescale && m_run != -INFINITY && t > 0;
#pragma unroll
        for (int c = 0; c < HB / 32; ++c) {
          uint32_t pk[16];
#pragma unroll
          for (int e = c * 32; e < c * 32 + 32; e += 2) {
            float a0, a1;
            f2unpack(ffma2(f2pack(x[e], x[e + 1]), c2x2, neg2), a0, a1);
            const float p0 = ex2_approx(a0), p1 = ex2_approx(a1);
            sum2[(e >> 1) & 3] = fadd2(sum2[(e >> 1) & 3], f2pack(p0, p1));
            pk[(e >> 1) & 15] = cvt_bf16x2(p0, p1);
          }
          tmem_st16(tS + c * 16, pk);
          if (c == 0 && __any_sync(0xffffffffu, mine)) {
            // O holds the PVs of every earlier tile only once PV(t-1) has completed (S(t) was
            // issued before it)
            if (!__all_sync(0xffffffffu, mbar_wait(&sm.pv_done[(tile - 1) & 3], ((tile - 1) >> 2) & 1, abort, A.status))) {
              ok = false;
              break;
            }
            tc_fence_after();
            const float alpha = mine ? ex2_approx((m_run - m_use) * c2) : 1.f;
            l_run *= alpha;
#pragma unroll
            for (int d = 0; d < PC / 16; ++d) {
              uint32_t o[16];
              tmem_ld16(tO + d * 16, o);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
              tmem_st16(tO + d * 16, o);
            }
          }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) arrive_lead(bar_p + 8 * c);
          if (c < HB / 32 - 1) __syncwarp();
        }
        float s0, s1, s2, s3;
        f2unpack(fadd2(sum2[0], sum2[1]), s0, s1);
        f2unpack(fadd2(sum2[2], sum2[3]), s2, s3);
        l_run += (s0 + s1) + (s2 + s3);
        m_run = m_use;
      }
      units += 2 * T;
      ok = ok && __all_sync(0xffffffffu, mbar_wait(&sm.pv_done[(tile - 1) & 3], ((tile - 1) >> 2) & 1, abort, A.status));
      // over the last tile's maxima, which the other warp has read where its P is in that PV; written
      // next behind the next tile's barrier
      sm.part[(tile - 1) & 1][hc][row] = l_run;
      named_bar_sync(1 + q4, 64);
      l_run += sm.part[(tile - 1) & 1][hc ^ 1][row];
      const int h = w.head_of(A, rank);
      const bool store = ok && r < w.rows;
      uint64_t zero2 = 0;
      if (ok) {
        tc_fence_after();
        const float inv = 1.f / l_run;
        const uint64_t inv2 = f2pack(inv, inv);
        // O leaves from registers, whole sectors of a row at a time: shared memory has the next
        // entry's Q in it.  The next entry's first P comes after these loads, so its PV finds O free.
        bf16* to = A.o + (((long long)(w.first + r) * A.g.q_rs + w.stream) * A.g.Hq + h) * DH + PC * hc;
#pragma unroll
        for (int c = 0; c < PC / 32; ++c) {
          uint32_t o[32], b[16];
          tmem_ld32(tO + c * 32, o);
          tmem_ld_wait();
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const uint64_t x2 = f2pack(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1]));
            zero2 = ffma2(x2, 0, zero2);  // 0 times an infinity or a NaN is NaN
            float a0, a1;
            f2unpack(fmul2(x2, inv2), a0, a1);
            b[e] = cvt_bf16x2(a0, a1);
          }
          if (store) {
            if (A.o_wide) {
              st_global_32(to + c * 32, b);
              st_global_32(to + c * 32 + 16, b + 8);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                reinterpret_cast<uint4*>(to + c * 32)[e] = make_uint4(b[4 * e], b[4 * e + 1], b[4 * e + 2], b[4 * e + 3]);
            }
          }
          __syncwarp();
        }
        tc_fence_before();  // ... before this thread's next arrival on p_full
      }
      if (hc == 0 && store)
        A.lse[(long long)h * A.g.q_nL + (long long)(w.first + r) * A.g.q_rs + w.stream] = (m_run * c2 + log2f(l_run)) * kLn2;
      float z0, z1;
      f2unpack(zero2, z0, z1);
      odd = odd || (store && !(z0 + z1 == 0.f));
    }
    sm.odd[hc][row] = odd;
    named_bar_sync(1 + q4, 64);  // both halves of the rows are stored, too
    if (ok && hc == 0 && __any_sync(0xffffffffu, sm.odd[0][row] | sm.odd[1][row])) {  // some row is not finite
      for (int k = 0, pos; (pos = place_of(k)) < total; ++k) {
        const PackedEntry w(A, pos);
        int lo, T;
        key_tiles(A, w, lo, T);
        settle_rows<DH, true>(A, w, w.head_of(A, rank), w.row0(A, rank) + q4 * 32, lo * BN, min((lo + T) * BN, w.rows));
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync();  // neither CTA's barriers or TMEM are used any more
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tmem, 512);
  }
}
}  // namespace packed256

cudaError_t launch_sfa_fwd_packed_tc256(const void* q, const void* k, const void* v, void* o, float* lse,
                                        const SfaGeom& g, float scale, const PackedList& list, const int32_t* offsets,
                                        long long max_items, int32_t* status, cudaStream_t st) {
  using namespace packed256;
  Params p;
  if (!make_rows_tmap(&p.tm_q, q, query_geom(g), g.Hq, DH, BM) || !make_rows_tmap(&p.tm_k, k, g, g.Hkv, DH, HB) ||
      !make_rows_tmap(&p.tm_v, v, g, g.Hkv, DH, BN))
    return cudaErrorInvalidValue;
  p.a = make_packed_args(q, k, v, o, lse, g, scale, list, offsets, status);
  cudaError_t e = cudaFuncSetAttribute(fwd_packed256_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
  if (e != cudaSuccess) return e;
  const long long work = max_items * p.a.per;
  return launch_kernel(true, fwd_packed256_kernel, dim3(2 * (unsigned)(work < kSmCount / 2 ? work : kSmCount / 2)),
                       NTHREADS, kSmemBytes, st, p);
}

}  // namespace hdsfa
