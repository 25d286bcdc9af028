// Attention over packed prompts of different lengths on the sm_103a tensor cores, head dims 64 and
// 128: the forward's problem and masks (Eq. 4, Fig. 2) for each sequence on its own, a run of rows
// of the packed tensors.
//
// Prompts are short beside training sequences, and a CTA that computes one query tile and ends spends
// 8500 cycles of start and end on a few key tiles of 2550.  So the kernel is persistent: one CTA per
// SM works through a list of query tiles (packed.cu), and what starts and ends a tile runs under its
// neighbours: the next Q and K are loaded while the last key tile is in use, the next S is computed
// while the softmax warps store O.  A CTA takes the list's entries in turn, every second round from
// the other end, which evens out the descending sizes.
//
// A CTA computes two query tiles of 128 rows (groups) that share their key tiles: the same rows of
// two heads of a K/V head where there is an even number of them, else 256 rows of one head.  Roles:
// warp 0 loads (TMA), warp 1 issues MMAs and owns TMEM, four warps per group do the online softmax, a
// thread per row.  Per key tile and group: S = Q K^T into 128 TMEM columns, P (bf16) over their first
// half, O += P V into DH columns.  P is rounded to bf16 because V is bf16 and an MMA's operands have one type:
// at most 2^-8 of each term, as O's own rounding; maxima, sums, O and LSE are fp32.
//
// Short sequences (at most kShortRows rows) that lie together share a tile: to a row of one, its
// neighbours' keys are masked, like those before a window, up to its own sequence's first row (SHARED;
// packed_shared has what it costs and brings).
//
// A key tile that reaches past its sequence holds rows of the next one, or memory behind the last:
// their scores are masked like later keys, and their V rows, which P = 0 would not silence if they
// held an infinity or a NaN, are zeroed in shared memory.  Later keys of the own sequence that are
// not finite are rare; rows that come out not finite with such keys about are computed again
// (settle_rows).  Every mbarrier wait is bounded.
#include "packed.cuh"
#include "tc_common.cuh"

namespace hdsfa {

typedef __nv_bfloat16 bf16;

namespace packed {
constexpr int BM = 128;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRescaleThreshold = 8.0f;  // log2 units: P stays <= 256 between O rescales

constexpr int BN = 128, NG = 2, NTHREADS = 64 + NG * 128;
constexpr uint32_t COL_O = NG * BN;  // TMEM: S_g at g*BN, O_g at COL_O + g*DH
// Parts in which P is published: at head dim 128 the PV of the first half runs while the second is
// computed; at 64 that saves 128 cycles of MMA and costs the issuer a wait of about as much (one part:
// 24 prompts of up to 701 tokens 84.4 -> 80.9 us).
template <int DH>
constexpr int parts() { return DH == 64 ? 1 : 2; }

template <int DH>
struct Smem {
  bf16 q[NG][BM * DH];  // per query tile: DH/64 swizzle blocks of [BM][64]
  static constexpr int NSLOT = DH == 64 ? 10 : 5;
  bf16 ring[NSLOT][BN * DH];  // one K or V tile each
  uint64_t q_full[NG], q_empty[NG], full[NSLOT], empty[NSLOT], s_full[NG], p_full[NG][2], o_done[NG], drain;
  uint32_t tmem_base;
  int abort;
};
// The layout needs 1024-byte alignment; the kernel checks the actual pad on entry.
template <int DH>
constexpr int smem_bytes() { return (int)sizeof(Smem<DH>) + 1024 < 232448 ? (int)sizeof(Smem<DH>) + 1024 : 232448; }
static_assert(sizeof(Smem<128>) <= 232448, "shared memory exceeds 227 KB");

struct Params {
  CUtensorMap tm_q, tm_k, tm_v;
  PackedArgs a;
};

// What the MMA issuer needs of an entry: the key tiles of its two query tiles.
struct Tiles {
  int lo[NG], hi[NG], n_lo, n_hi;
  HD_DEVINLINE Tiles(const PackedArgs& a, int pos) {
    const PackedEntry w(a, pos);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      lo[g] = packed_lo(a, w.row0(a, g));
      hi[g] = packed_hi(w.row0(a, g), w.rows);
    }
    n_lo = lo[0];
    n_hi = max(hi[0], hi[1]);
  }
};
HD_DEVINLINE int place_of(int k) { return packed_place(k, (int)blockIdx.x, (int)gridDim.x); }

// SHARED: the list may hold tiles of short sequences.
template <int DH, bool SHARED>
__global__ void __launch_bounds__(NTHREADS, 1) fwd_packed_kernel(const __grid_constant__ Params P) {
  constexpr int NSLOT = Smem<DH>::NSLOT;
  extern __shared__ uint8_t smem_raw[];
  {
    uint32_t dyn;
    asm("mov.u32 %0, %%dynamic_smem_size;\n" : "=r"(dyn));
    const uintptr_t base = reinterpret_cast<uintptr_t>(smem_raw);
    if (((base + 1023) & ~uintptr_t(1023)) - base + sizeof(Smem<DH>) > dyn) {  // uniform: nothing touched yet
      if (threadIdx.x == 0) set_status(P.a.status, HD_DEVBIT_TIMEOUT);
      return;
    }
  }
  Smem<DH>& sm = *reinterpret_cast<Smem<DH>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NSLOT; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], 1);
    }
    for (int g = 0; g < NG; ++g) {
      mbar_init(&sm.q_full[g], 1);
      mbar_init(&sm.q_empty[g], 1);
      mbar_init(&sm.s_full[g], 1);
      mbar_init(&sm.p_full[g][0], 4);  // one arrival per softmax warp of the group
      mbar_init(&sm.p_full[g][1], 4);
      mbar_init(&sm.o_done[g], 1);
    }
    mbar_init(&sm.drain, 1);
    sm.abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&sm.tmem_base, 512);
    tmem_relinquish();
    tc_fence_before();
  }
  grid_dep_wait();
  grid_dep_launch();  // at most one CTA per SM: the next kernel's find their places as these end
  volatile int* abort = &sm.abort;
  uint32_t tmem = 0;
  if (warp == 0) {
    named_bar_arrive(1, NTHREADS);  // the producer does not wait for the TMEM allocation
  } else {
    named_bar_sync(1, NTHREADS);
    tc_fence_after();
    tmem = sm.tmem_base;
  }
  const PackedArgs& A = P.a;
  const int total = *A.list.count * A.per;

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      tma_prefetch(&P.tm_q);
      tma_prefetch(&P.tm_k);
      tma_prefetch(&P.tm_v);
      int slot = 0, ph = 1;  // empty-barrier phase: the first lap does not wait
      uint32_t issued = 0;
      int used[NG] = {};  // entries in which each group took part
      bool ok = true;
      for (int k = 0, pos; ok && (pos = place_of(k)) < total; ++k) {
        const PackedEntry w(A, pos);
        const int kvh = fast_div(w.head, A.d_grp);
        auto load_tile = [&](const CUtensorMap* tm, int j) {
          if (!ok || !mbar_wait(&sm.empty[slot], ph, abort, P.a.status)) {
            ok = false;
            return;
          }
          mbar_arrive_expect_tx(&sm.full[slot], BN * DH * 2);
          for (int c = 0; c < DH / 64; ++c)
            tma_load_5d(sm.ring[slot] + c * BN * 64, tm, &sm.full[slot], c * 64, kvh, w.stream, w.first + j * BN, 0);
          ++issued;
          if (++slot == NSLOT) {
            slot = 0;
            ph ^= 1;
          }
        };
        const int n_lo = packed_lo(A, w.m0), n_hi = max(packed_hi(w.m0, w.rows), packed_hi(w.row0(A, 1), w.rows));
        load_tile(&P.tm_k, n_lo);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const int r0 = w.row0(A, g);
          if (!ok || r0 >= w.rows) continue;
          // the group's last S of its entry before has read Q
          if (used[g] > 0 && !mbar_wait(&sm.q_empty[g], (used[g] - 1) & 1, abort, P.a.status)) {
            ok = false;
            continue;
          }
          ++used[g];
          mbar_arrive_expect_tx(&sm.q_full[g], BM * DH * 2);
          for (int c = 0; c < DH / 64; ++c)
            tma_load_5d(sm.q[g] + c * BM * 64, &P.tm_q, &sm.q_full[g], c * 64, w.head_of(A, g), w.stream,
                        w.first + r0, 0);
        }
        for (int j = n_lo; ok && j <= n_hi; ++j) {
          load_tile(&P.tm_v, j);
          if (j < n_hi) load_tile(&P.tm_k, j + 1);
        }
      }
      // every copy this thread started lands before the CTA may exit
#pragma unroll
      for (int g = 0; g < NG; ++g)
        if (used[g] > 0) mbar_drain(&sm.q_full[g], (used[g] - 1) & 1);
      for (uint32_t u = issued > NSLOT ? issued - NSLOT : 0; u < issued; ++u)
        mbar_drain(&sm.full[u % NSLOT], (u / NSLOT) & 1);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA issuer
    // The whole warp runs the loop (warp-uniform operands); one elected lane issues.
    constexpr uint32_t idS = idesc_bf16(BM, BN, 0, 0);  // S[q][kv] = Q K^T (both K-major)
    constexpr uint32_t idO = idesc_bf16(BM, DH, 0, 1);  // O[q][d] += P V   (P in TMEM, V MN-major)
    // operand descriptors encoded once; a slot or k-step adds its byte offset / 16
    const uint64_t qd0 = sdesc_sw128(smem_u32(sm.q[0]), 16, 1024);
    const uint64_t kd0 = sdesc_sw128(smem_u32(sm.ring[0]), 16, 1024);
    const uint64_t vd0 = sdesc_sw128(smem_u32(sm.ring[0]), BN * 128, 1024);
    constexpr int TILE16 = BN * DH * 2 / 16;
    auto wait_w = [&](uint64_t* bar, int par) -> bool {
      if (!__all_sync(0xffffffffu, mbar_wait(bar, par & 1, abort, P.a.status))) return false;
      tc_fence_after();
      return true;
    };
    auto issue_s = [&](int g, int slot) {
      const uint64_t qd = qd0 + (uint64_t)(g * (BM * DH * 2 / 16)), kd = kd0 + (uint64_t)(slot * TILE16);
#pragma unroll
      for (int kk = 0; kk < DH / 16; ++kk)
        tc_mma_ss_w(tmem + g * BN, qd + (uint64_t)((kk >> 2) * (BM * 128 / 16) + (kk & 3) * 2),
                    kd + (uint64_t)((kk >> 2) * (BN * 128 / 16) + (kk & 3) * 2), idS, kk > 0 ? 1u : 0u);
      tc_commit_w(&sm.s_full[g]);
    };
    // The softmax publishes P(j) only after V(j) and K(j+1) have landed, so within an entry the
    // issuer waits for P alone; releases go where no wait follows at once.
    auto issue_pv = [&](int g, bool first, int count, int slot, int k_done) -> bool {
      const uint64_t vd = vd0 + (uint64_t)(slot * TILE16);
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        if (part < parts<DH>() && !wait_w(&sm.p_full[g][part], count)) return false;
#pragma unroll
        for (int kk = part * 4; kk < part * 4 + 4; ++kk)
          tc_mma_ts_w(tmem + COL_O + g * DH, tmem + g * BN + kk * 8, vd + (uint64_t)(kk * 16 * 128 / 16), idO,
                      (!first || kk > 0) ? 1u : 0u);
        if (part == 0 && k_done >= 0) tc_commit_w(&sm.empty[k_done]);
      }
      return true;
    };
    auto next_slot = [](int s) { return s + 1 == NSLOT ? 0 : s + 1; };
    bool ok = true;
    int k_slot = 0, k_par = 0;          // ring place of the entry's first K
    int used[NG] = {}, tiles[NG] = {};  // entries and key tiles of each group before
    Tiles e(A, place_of(0) < total ? place_of(0) : 0);
    auto first_s = [&](int g, const Tiles& t, int slot) {
      // over the S and P of the group's entry before, whose last PV was issued before
      if (t.hi[g] < 0) return;
      ok = ok && wait_w(&sm.q_full[g], used[g]++);
      if (ok && t.lo[g] <= t.n_lo) issue_s(g, slot);
    };
    if (place_of(0) < total) {
      ok = wait_w(&sm.full[0], 0);
#pragma unroll
      for (int g = 0; g < NG; ++g) first_s(g, e, 0);
    }
    for (int k = 0; ok && place_of(k) < total; ++k) {
      // The next entry's first S of a group follows the group's last PV of this one: the softmax
      // finds it when it has stored O.
      const bool more = place_of(k + 1) < total;
      const Tiles nx(A, more ? place_of(k + 1) : 0);
      const int slots = k_slot + 2 * (e.n_hi - e.n_lo + 1), nk_slot = slots % NSLOT, nk_par = k_par + slots / NSLOT;
      bool k_here = false;
      int k_done = k_slot, v_slot = next_slot(k_slot);
      for (int j = e.n_lo; ok && j <= e.n_hi; ++j) {
        const int k_next = next_slot(v_slot);  // K(j+1)
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const bool in = e.lo[g] <= j && j <= e.hi[g];
          if (ok && in) {
            ok = issue_pv(g, j == e.lo[g], tiles[g]++, v_slot, k_done);
            k_done = -1;
            if (ok && j == e.hi[g]) tc_commit_w(&sm.o_done[g]);
          }
          if (g == NG - 1) tc_commit_w(&sm.empty[v_slot]);
          // S of the next tile for this group reuses its S/P columns: issued after its PV
          if (ok && j + 1 <= e.hi[g] && e.lo[g] <= j + 1) issue_s(g, k_next);
          if (ok && in && j == e.hi[g] && more) {
            if (!k_here) ok = wait_w(&sm.full[nk_slot], nk_par);
            k_here = true;
            first_s(g, nx, nk_slot);
          }
        }
        k_done = k_next;
        v_slot = next_slot(k_next);
      }
      if (more) {
        if (ok && e.hi[NG - 1] < 0) first_s(NG - 1, nx, nk_slot);  // a group that had no rows here
        e = nx;
      }
      k_slot = nk_slot;
      k_par = nk_par;
    }
    // every MMA issued above completes before TMEM / smem are released
    tc_commit_w(&sm.drain);
    mbar_drain(&sm.drain, 0);
  } else {
    // ------------------------------------------------------------ softmax / epilogue
    const int g = (warp - 2) >> 2;
    const int q4 = warp & 3;
    const int row = q4 * 32 + lane;
    const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16);
    const uint32_t tS = tl + g * BN, tO = tl + COL_O + g * DH;
    const float c2 = A.scale_log2;
    const uint64_t c2x2 = f2pack(c2, c2);
    const bool lead = warp == 2 + 4 * g && lane == 0;
    uint32_t units = 0;
    int used = 0, tiles = 0;
    bool ok = true, odd = false;  // odd: a row of this thread's came out not finite
    // of an entry only this is held over the key tiles, whose scores take the registers
    int rows = 0, m0 = 0, n_lo = 0, n_hi = 0;
    bool apart = false;  // SHARED: the entry holds several sequences
    int own = 0;         // ... and the first row of that of this thread's row
    auto take = [&](const PackedEntry& w) {
      rows = w.rows;
      m0 = w.row0(A, g);
      n_lo = packed_lo(A, w.m0);
      n_hi = max(packed_hi(w.m0, rows), packed_hi(w.row0(A, 1), rows));
      if constexpr (SHARED) own = sequence_first(A, w, m0 + row), apart = w.seqs > 0;
    };
    int pos = place_of(0);
    if (pos < total) take(PackedEntry(A, pos));
    for (int k = 0; ok && pos < total; ++k) {
      const int r = m0 + row, lo = packed_lo(A, m0), hi = packed_hi(m0, rows);
      float m_run = -INFINITY, l_run = 0.f;  // m_run in raw score units
      for (int j = lo; j <= hi; ++j, ++tiles) {
        const int kb = j * BN;  // first key row of the tile
        const uint32_t u = units + 2 * (uint32_t)(j - n_lo) + 1;  // V(j)'s place in the ring's order
        // this thread's arrivals on p_full also say that V(j) and K(j+1) have landed (waited
        // for here, where the softmax waits for S anyway)
        if (lead) {
          mbar_wait(&sm.full[u % NSLOT], (u / NSLOT) & 1, abort, P.a.status);
          if (j < n_hi) mbar_wait(&sm.full[(u + 1) % NSLOT], ((u + 1) / NSLOT) & 1, abort, P.a.status);
        }
        __syncwarp();
        if (kb + BN > rows) {  // V rows behind the sequence (every group that reads them zeroes them);
                               // here, under the S of the tile
          if (!__all_sync(0xffffffffu, mbar_wait(&sm.full[u % NSLOT], (u / NSLOT) & 1, abort, P.a.status))) {
            ok = false;
            break;
          }
          for (int e = (rows - kb) * 8 + row; e < BN * 8; e += 128)
#pragma unroll
            for (int c = 0; c < DH / 64; ++c)
              reinterpret_cast<uint4*>(sm.ring[u % NSLOT] + c * BN * 64)[e] = make_uint4(0, 0, 0, 0);
          fence_async_smem();
        }
        // tcgen05.ld/st are warp-collective: every wait result is made warp-uniform
        if (!__all_sync(0xffffffffu, mbar_wait(&sm.s_full[g], tiles & 1, abort, P.a.status))) {
          ok = false;
          break;
        }
        tc_fence_after();
        mbar_arrive_if(lead && j == hi, &sm.q_empty[g]);  // the group's last S has read Q
        float x[BN];
#pragma unroll
        for (int c = 0; c < BN / 32; ++c) tmem_ld32(tS + c * 32, reinterpret_cast<uint32_t*>(x) + c * 32);
        tmem_ld_wait();
        // tiles holding a key past the first query's key row (the diagonal band) or the sequence,
        // and (LOCAL) a key at or below the last query's window edge, or one before a row's sequence.  All
        // conditions are the entry's, none a lane's: the warp goes on together to the tcgen05 instructions
        // below.  (With a vote on `own` and branches around the arrivals 4 prompts of 8B heads 684 us, so 661.)
        if (kb + BN - 1 > m0 || kb + BN > rows || (SHARED && apart) ||
            (A.g.window > 0 && kb <= min(m0 + BM, rows) - 1 - A.g.window)) {
          const int e_hi = min(r, rows - 1) - kb;
#pragma unroll
          for (int e = 0; e < BN; ++e)
            if (e > e_hi) x[e] = -INFINITY;
          if (A.g.window > 0 || (SHARED && apart)) {
            const int e_lo = (SHARED ? max(own, A.g.window > 0 ? r - A.g.window + 1 : 0) : r - A.g.window + 1) - kb;
#pragma unroll
            for (int e = 0; e < BN; ++e)
              if (e < e_lo) x[e] = -INFINITY;
          }
        }
        float mx[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) mx[e] = x[e];
#pragma unroll
        for (int e = 4; e < BN; e += 2) mx[(e >> 1) & 3] = max3(mx[(e >> 1) & 3], x[e], x[e + 1]);
        const float tmax = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]);
        const float m_new = fmaxf(m_run, tmax);
        const bool rescale = (m_run == -INFINITY) || ((m_new - m_run) * c2 > kRescaleThreshold);
        const float m_use = rescale ? m_new : m_run;
        const float neg = (m_use == -INFINITY) ? 0.f : -m_use * c2;
        const uint64_t neg2 = f2pack(neg, neg);
        // P (bf16 pairs) over the first half of this group's S columns
        uint64_t sum2[4] = {0, 0, 0, 0};
        const bool mine = rescale && m_run != -INFINITY && j > lo;
#pragma unroll
        for (int c = 0; c < BN / 32; ++c) {
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
          if (c & 1) {
            if (c == 1 && __any_sync(0xffffffffu, mine)) {
              // O_g already holds every earlier tile's PV (its S of this tile was issued after
              // them).  Looked at here, so that the vote does not delay the exponentials.
              const float alpha = mine ? ex2_approx((m_run - m_use) * c2) : 1.f;
              l_run *= alpha;
#pragma unroll
              for (int d = 0; d < DH / 16; ++d) {
                uint32_t o[16];
                tmem_ld16(tO + d * 16, o);
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                tmem_st16(tO + d * 16, o);
              }
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (parts<DH>() == 2 || c == 3) mbar_arrive_if(lane == 0, &sm.p_full[g][parts<DH>() == 2 ? c >> 1 : 0]);
          }
        }
        float s0, s1, s2, s3;
        f2unpack(fadd2(sum2[0], sum2[1]), s0, s1);
        f2unpack(fadd2(sum2[2], sum2[3]), s2, s3);
        l_run += (s0 + s1) + (s2 + s3);
        m_run = m_use;
      }
      units += 2 * (uint32_t)(n_hi - n_lo + 1);
      // looked up under the last PV: where the results go, and the next entry
      const PackedEntry w(A, pos);
      pos = place_of(k + 1);
      const PackedEntry nx(A, pos < total ? pos : 0);
      const int rows_now = rows;
      take(nx);
      if (!ok || hi < 0) continue;
      if (!__all_sync(0xffffffffu, mbar_wait(&sm.o_done[g], used++ & 1, abort, P.a.status))) {
        ok = false;
        continue;
      }
      tc_fence_after();
      // O leaves from registers, whole sectors of a row at a time: shared memory has the next entry's
      // Q in it.  The next entry's first P comes after these loads, so its PV finds O free.
      const float inv = 1.f / l_run;
      const int hd = w.head_of(A, g);
      const long long orow = ((long long)(w.first + r) * A.g.q_rs + w.stream) * A.g.Hq + hd;
      const bool store = r < rows_now;
      uint64_t zero2 = 0;
      const uint64_t inv2 = f2pack(inv, inv);
#pragma unroll
      for (int c = 0; c < DH / 32; ++c) {
        uint32_t o[32], h[16];
        tmem_ld32(tO + c * 32, o);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const uint64_t x2 = f2pack(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1]));
          zero2 = ffma2(x2, 0, zero2);  // 0 times an infinity or a NaN is NaN
          float a0, a1;
          f2unpack(fmul2(x2, inv2), a0, a1);
          h[e] = cvt_bf16x2(a0, a1);
        }
        if (store) {
          bf16* to = A.o + orow * DH + c * 32;
          if (A.o_wide) {
            st_global_32(to, h);
            st_global_32(to + 16, h + 8);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              reinterpret_cast<uint4*>(to)[e] = make_uint4(h[4 * e], h[4 * e + 1], h[4 * e + 2], h[4 * e + 3]);
          }
        }
        __syncwarp();
      }
      tc_fence_before();  // ... before this thread's next arrival on p_full
      if (store)
        A.lse[(long long)hd * A.g.q_nL + (long long)(w.first + r) * A.g.q_rs + w.stream] = (m_run * c2 + log2f(l_run)) * kLn2;
      float z0, z1;
      f2unpack(zero2, z0, z1);
      odd = odd || (store && !(z0 + z1 == 0.f));
    }
    if (ok && __any_sync(0xffffffffu, odd)) {  // some row of some entry is not finite
      for (int k = 0; (pos = place_of(k)) < total; ++k) {
        const PackedEntry w(A, pos);
        const int r0 = w.row0(A, g);
        settle_rows<DH, SHARED>(A, w, w.head_of(A, g), r0 + q4 * 32, packed_lo(A, r0) * BN, min((packed_hi(r0, w.rows) + 1) * BN, w.rows));
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

template <int DH, bool SHARED>
static cudaError_t launch(const Params& p, long long max_items, cudaStream_t st) {
  constexpr int smem = smem_bytes<DH>();
  cudaError_t e = cudaFuncSetAttribute(fwd_packed_kernel<DH, SHARED>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const long long work = max_items * p.a.per;
  return launch_kernel(true, fwd_packed_kernel<DH, SHARED>, dim3((unsigned)(work < kSmCount ? work : kSmCount)), NTHREADS, smem,
                       st, p);
}
}  // namespace packed

cudaError_t launch_sfa_fwd_packed_tc(const void* q, const void* k, const void* v, void* o, float* lse, const SfaGeom& g,
                                     int Dh, float scale, const PackedList& list, const int32_t* offsets,
                                     bool shared, long long max_items, int32_t* status, cudaStream_t st) {
  using namespace packed;
  Params p;
  if (!make_rows_tmap(&p.tm_q, q, query_geom(g), g.Hq, Dh, BM) || !make_rows_tmap(&p.tm_k, k, g, g.Hkv, Dh, BN) ||
      !make_rows_tmap(&p.tm_v, v, g, g.Hkv, Dh, BN))
    return cudaErrorInvalidValue;
  p.a = make_packed_args(q, k, v, o, lse, g, scale, list, offsets, status);
  if (Dh == 128) return launch<128, true>(p, max_items, st);
  return shared ? launch<64, true>(p, max_items, st) : launch<64, false>(p, max_items, st);
}

}  // namespace hdsfa
