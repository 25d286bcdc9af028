// Decoding over the 8-bit paged cache on the 5th-generation tensor cores (the mathematics of x, m and the scales:
// sfa_decode_q8.cu).
//
// K and V go from TMA to the products as the codes that they are; only scores pass through registers.  Both products
// have the cached positions or the head dim as their rows, and the few query rows as columns, so that no row of a
// tile is empty and a thread has one position:
//   S^T [128 positions x 2 R] = K (e4m3) * [q_hi | q_lo]^T (e4m3): a row's bf16 values, scaled by a power of two to [2^7,
//     2^8), are hi + lo / 16 in two codes, exact for values down to 2^-13 of the row's largest and to 2^-21 of it below (see
//     kMissed).  K is read from shared memory once.  Where tensor memory has no room for two columns a row (R = 32 and 64 at head dim
//     256), three e5m2 codes of the query's f16 form one after another instead, which read K three times.
//   O^T [Dh x 3 R] += V^T (e4m3) * [P_hi | P_mid | P_lo] (e5m2): three codes of three bits, so P is rounded to nine bits (of
//     its f16 form), half a step 2^-9 of it.  A row's largest P is 2^5 when its reference is set, and at most 2^15 before
//     it goes up; the third codes hold 64 times what they stand for, so steps end at 2^-22, 2^-27 of the row's largest
//     (see kFar).  The three columns are added at the end.
// A thread of a softmax warp takes its position's scores for its group's 16 rows: scales by 2^ek, adds ev, masks (what
// a position is visible to is a range of rows), and subtracts the row's reference.  References are the group's (a copy
// for each warp), and go up only when some P would pass 2^15 (a vote for each tile; every tile after the first few has
// none): then the rows' maxima are reduced over the four warps, and sums and O in tensor memory are rescaled.  (The vote as
// an arrival and a wait, with the exponentials between them, was slower: 96 rows of 8 heads 99 us for 96.)
//
// Warp 0 brings tiles (TMA, pieces of pages) into a ring of units of 128 columns, warp 1 issues the products, the
// others are R / 16 groups of four softmax warps, which first code the queries, four rows a warp.  S and P have two
// buffers, so S of the next tile is computed under this one's softmax and its P V under the next one's.  The first group
// brings the scales 384 blocks ahead, since a load behind a saturated memory's queue takes thousands of cycles.
//
// A batch of long sequences is one wave of CTAs, each with an equal share of all tiles (Work), because a CTA takes about
// 12000 cycles to start and 4000 to end, six to eight tiles' time: 8 x 8192 tokens, 96 over 8 heads of 128, 122 us with
// three waves of splits and 101 so.
//
// Bound by memory at 16 query rows, of 8 heads of 128: 16 sequences of 32768 tokens, 32 over 8 heads, 390 to 397 us (6.9
// TB/s of codes and scales; 400 at the copy rate), 8 of up to 16384 113 for 103.  With more rows by the softmax warps'
// chain, about 350 instructions for 16 rows of a warp's 32 positions, 2000 cycles a tile for each group at once (clock64,
// 48 rows: masks and scales 450, waiting for S 240, scores 430, vote 340, codes of P 380, fence 130): these
// lengths reach 0.86 of the copy rate at 32 rows (120 us), 0.61 at 48, 0.49 at 64; 48 of heads of 256 0.77 (67.5 for 52); more
// than 64 rows read the cache once for each group of 64 (8 x 8192, 96 rows, 340 for 104).  Three
// CTAs an SM at 16 rows (up to head dim 128) hide a tile's chain of barriers: 133 us with two, 114 with three.  Tried and
// dropped: warps of 24 to 48 rows (registers: fewer warps to hide the latency), two tiles in turn with an O each, two tiles for
// each vote (48 rows: 102 us for 96), queries in three codes everywhere (K's reads three times: bound by shared memory at
// 16 rows).
#include <float.h>

#include <algorithm>

#include "decode_plan.cuh"
#include "decode_q8.cuh"

namespace hdsfa {
namespace decq8tc {
using decq8::Args;
using decq8::Params;

constexpr int KT = 128;            // positions of a tile
constexpr int RW = 16;             // query rows of a warp group
constexpr float kTop = 15.f;       // P's largest exponent
constexpr float kSet = 5.f;        // the exponent of a row's largest P when its reference is set
constexpr float kLow = 64.f;       // P's third codes hold so many times what they stand for
constexpr float kLo = 16.f;        // a query's second e4m3 codes too
constexpr uint32_t kGaveUp = 1u << 31;
constexpr float kRedo = -2.f;      // as a partial's sum: the row is to be computed again (exact_row)
// P's codes are off by 2^-9 of P, or, where it is below 2^-14 (kExact), by up to 2^-23 (kStep), and a weight is P 2^-ev.  So
// blocks whose ev lies far below the largest (kFar binary orders, where 2^-23 is 2^-22 of the row's largest weight) may lose
// weight that counts, and with it what they hold in columns in which the larger blocks hold nothing.  What each row loses in
// such blocks is bounded tile by tile, and rows for which that passes kLost of their sum are computed again.
constexpr int kFar = 6;
constexpr float kExact = -14.f, kStep = -23.f;
constexpr float kLost = 1.f / 128;

// HV units of a K or V tile, of RB columns (128, or 64 at head dim 64) each: a ring slot.  R query rows: WG warp groups of RW.
template <int DH, int WG>
struct Cfg {
  static constexpr int R = RW * WG, kThreads = 64 + WG * 128;
  static constexpr int RB = DH < 128 ? DH : 128, HV = DH / RB, kUnit = KT * RB;
  // Queries in two e4m3 codes side by side (kPair: K is read once, S has two columns a row), or in three e5m2 codes one
  // after another (K is read three times) where tensor memory has no room for that.
  static constexpr bool kPair = 4 * R + 3 * HV * R <= (HV == 2 && R == 32 ? 256 : 512);
  static constexpr int SC = kPair ? 2 * R : R, QT = kPair ? 2 : 3;  // columns of S; codes of a query's value
  static constexpr int kCols = 2 * SC + 3 * HV * R;  // tensor memory: two S, three O
  static constexpr int kAlloc = kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
  static constexpr int kFixed = QT * R * DH + 6 * R * KT + 128 * (4 * 12 + 8 * 2) + 4 * 14 * R + 512;  // all but the ring
  static constexpr int kPerSm = kAlloc <= 128 && kFixed + 3 * kUnit <= 74 * 1024    ? 3
                                : kAlloc <= 256 && R <= 32 && kFixed + 3 * kUnit <= 112 * 1024 ? 2
                                                                                    : 1;
  static constexpr int kRoom = ((kPerSm == 3 ? 74 : kPerSm == 2 ? 112 : 226) * 1024 - kFixed) / kUnit;
  static constexpr int NSLOT = kRoom < 10 ? kRoom : 10;
};

template <int DH, int WG>
struct Smem {
  using C = Cfg<DH, WG>;
  uint8_t ring[C::NSLOT][C::kUnit];          // [128 positions][RB bytes], swizzled by 128 bytes (64)
  uint8_t q[C::HV][C::QT][C::R * C::RB];     // codes: [R rows][RB bytes], swizzled so too
  uint8_t p[2][3][C::R * KT];                // a buffer's hi, mid, lo: blocks of 16 rows, [128 positions][16 bytes]
  uint2 words[4][128];                       // of chunks: the words of K's and V's scales that hold a block's byte
  int entry[4][128];                         // its page entry
  uint16_t scale[8 * 128];                   // blocks' scale bytes, K's and V's above it
  float rowf[C::R];                          // a row's factor of q
  float missed[C::R];                        // what its codes miss (decq8::kMissed)
  float nref[4][C::R];                       // its reference, negated: a copy for each warp of the group; its sums at last
  float most[4][C::R];                       // a warp's maxima
  float lost[4][C::R];                       // a bound of what a warp's rounding has cost the row's sum
  uint64_t full[C::NSLOT], empty[C::NSLOT], s_full[2], s_free[2], p_full[2], pv_done[2], sc_full[8], q_full, drain;
  unsigned raise[4 * WG];                    // a warp's rows whose references go up, its largest scale byte << 16; kGaveUp
  uint32_t tmem_base;
  unsigned again[2];                         // rows of O that are not finite; whether there is one of them, or of too great
  int redo;                                  // a loss (kRedo)
  int most_kb[2][4];                         // K's largest scale byte of this sequence and the one before, by the first group's warps
  int abort, bad_page[16];                   // of the sequence with this number, mod 16 (the ring holds fewer)
};

// kind::f8f6f4, fp32 D: operand types 0 e4m3, 1 e5m2.
__host__ __device__ constexpr uint32_t idesc_f8(int M, int N, int a_type, int b_type, int a_mn, int b_mn) {
  return (1u << 4) | ((uint32_t)a_type << 7) | ((uint32_t)b_type << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) |
         ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// Matrix descriptor of rows of RB bytes, swizzled by as many: eight rows lie together.  K-major with a row to an index, or
// MN-major with a k to a row and RB indices in it.
template <int RB>
HD_DEVINLINE uint64_t sdesc_rows(uint32_t saddr) {
  if (RB == 128) return sdesc_sw128(saddr, 16, 1024);
  uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= 1ull << 16;
  d |= (uint64_t)(512 >> 4) << 32;
  d |= 1ull << 46;  // descriptor version for tcgen05
  d |= 4ull << 61;  // SWIZZLE_64B
  return d;
}
// Matrix descriptor without a swizzle, MN-major: 16 bytes of rows x 8 k lie together (128 bytes); the next 8 k are `kstep`
// bytes on, the next 16 rows `mstep`.
HD_DEVINLINE uint64_t sdesc_plain_mn(uint32_t saddr, uint32_t kstep, uint32_t mstep) {
  uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)((kstep >> 4) & 0x3FFFu) << 16;
  d |= (uint64_t)((mstep >> 4) & 0x3FFFu) << 32;
  d |= 1ull << 46;  // descriptor version for tcgen05
  return d;
}
HD_DEVINLINE void mma_f8_ss_w(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accum) {
  asm volatile(
      "{\n .reg .pred p, e;\n setp.ne.b32 p, %4, 0;\n elect.sync _|e, 0xffffffff;\n"
      " @e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accum));
}
// This warp's 32 lanes of N columns of tensor memory, STEP apart, times f twice.
template <int N, int STEP>
HD_DEVINLINE void tmem_scale(uint32_t taddr, float f) {
  float x[N];
#pragma unroll
  for (int i = 0; i < N; ++i)
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n" : "=f"(x[i]) : "r"(taddr + i * STEP));
  tmem_ld_wait();
#pragma unroll
  for (int i = 0; i < N; ++i)
    asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};\n" ::"r"(taddr + i * STEP), "f"(x[i] * f * f) : "memory");
}
// Whether `v` holds for a thread of the 128 on hardware barrier `id`.
HD_DEVINLINE bool group_any(int id, bool v) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n barrier.cta.red.or.pred q, %2, 128, p;\n selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"((uint32_t)v), "r"(id)
      : "memory");
  return r != 0;
}
// Floats as integers of the same order, and back.
HD_DEVINLINE int ordered(float x) {
  const int i = __float_as_int(x);
  return i ^ ((i >> 31) & 0x7fffffff);
}
HD_DEVINLINE float from_ordered(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7fffffff)); }
HD_DEVINLINE uint32_t hsub2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;\n" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// Bits [lo, hi) of RW, the range cut to them.
HD_DEVINLINE uint32_t bits(int lo, int hi) {
  lo = min(max(lo, 0), RW);
  hi = min(max(hi, 0), RW);
  return hi <= lo ? 0u : (1u << hi) - (1u << lo);
}
// `bytes` of four bytes, the others zero.
HD_DEVINLINE void cp_async_4(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;\n" ::"r"(dst), "l"(src), "r"(bytes));
}
// Three e5m2 codes of each of two f16: e5m2 is the upper byte of f16, so three bits, three of what is left, and the rest
// (times `f`, a power of two) to the nearest; each in the upper bytes of the halves.
template <bool SCALE>
HD_DEVINLINE void split3(uint32_t u, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  hi = u & 0xff00ff00u;
  const uint32_t v = hsub2(u, hi);
  mid = v & 0xff00ff00u;
  lo = hsub2(v, mid);
  if (SCALE) {
    const __half2 f = __float2half2_rn(kLow);
    asm("mul.rn.f16x2 %0, %0, %1;\n" : "+r"(lo) : "r"(*reinterpret_cast<const uint32_t*>(&f)));
  }
  lo += 0x00800080u;
}

// A thread's position's scores, as exponents of P.
struct Scores {
  float y[RW];
};
// Adds to the warp's bounds lost[RW] what the codes of this tile's P may cost each row's sum in blocks far below the
// largest.  By a whole warp; vis, vb: the rows that see the thread's position, its scale byte.  (A function of its own:
// inline, its registers cost every tile 2 %.)
__device__ __noinline__ void note_losses(Scores s, uint32_t vis, int vb, int top_vb, float* lost) {
  const int lane = threadIdx.x & 31;
  // (V of the smallest scale, mostly zeros, counts only in the sum: kFarSum)
  const bool far = vis != 0 && vb + kFar < top_vb, some = far && vb > q8::kMinByte;
  const unsigned low = __reduce_min_sync(0xffffffffu, some ? (unsigned)vb : (unsigned)q8::kMaxByte);
  unsigned mine = 0;  // lane r: row r's, in units of 2^-47 2^-low
#pragma unroll
  for (int r = 0; r < RW; ++r) {
    const bool loses = some && ((vis >> r) & 1u) && s.y[r] < kExact;
    const float x = loses ? ex2_approx(fminf(s.y[r], kStep) + 47.f + (float)((int)low - vb)) : 0.f;  // at most 2^24
    const unsigned sum = __reduce_add_sync(0xffffffffu, __float2uint_ru(x));
    if (lane == r) mine = sum;
  }
  float x = (float)mine * 0x1p-47f * q8::inverse_of((int)low);
  if (__any_sync(0xffffffffu, far && vb + decq8::kFarSum < top_vb)) x = 0x1p100f;  // above every sum
  if (lane < RW) lost[lane] += x;
  __syncwarp();
}

// What CTA x of a K/V head and row group works through: the x-th of nsplit parts of one sequence, or (SHARED) the x-th
// of `total` equal parts of the tiles of all sequences, one behind another, which may lie in several: then a partial is
// a CTA's of one sequence, with the number x + b (each differs from the one before in x or in b).  A sequence counts
// kStart tiles more in front of its own, for what a CTA takes to end one and start the next.  Found by a whole warp.
template <bool SHARED>
struct Work {
  static constexpr int kStart = 6;
  int x, b, T, k0, k1, slot, left;  // sequence, its tokens, positions [k0, k1), the partial's number; tiles after those
  // (Loops that are not unrolled, and inline: 2500 to 3000 cycles from the wait for the kernel before.  Unrolled over 128
  // sequences, in a function of its own with divisions in 64 bits, it took 7000 to 9000.)
  HD_DEVINLINE Work(const Args& a, int x_) : x(x_), b(0), T(0), k0(0), k1(0), slot(x_), left(0) {
    if constexpr (!SHARED) {
      b = fast_div(x, a.d_nsplit);
      T = a.lens[b];
      dec::split_range<true>(a, T, x - b * a.nsplit, a.tile, k0, k1);
    } else {
      const WaveParts whole = parts(a);
      const unsigned u0 = whole.begin(x), u1 = whole.begin(x + 1);
      if (x >= (int)whole.S || u0 >= u1) return;
      each(a, [&](int q, int len, unsigned first, unsigned size) {
        const unsigned hit = __ballot_sync(0xffffffffu, first <= u0 && u0 < first + size);
        if (hit == 0) return false;
        const int l = __ffs(hit) - 1;
        b = __shfl_sync(0xffffffffu, q, l);
        T = __shfl_sync(0xffffffffu, len, l);
        take(a, (int)(u0 - __shfl_sync(0xffffffffu, first, l)) - kStart, (int)(u1 - u0));
        return true;
      });
    }
  }
  // On to the next sequence; whether there is one.
  HD_DEVINLINE bool next(const Args& a) {
    if constexpr (SHARED) {
      if (left <= kStart) return false;
      do {
        if (++b >= a.B) return false;
        T = a.lens[b];
      } while (T < 1 || T > a.maxT);
      take(a, -kStart, left);
    }
    return SHARED;
  }
  // For the combine kernel, by one warp: each sequence's first partial, and their number.
  static HD_DEVINLINE void report(const Args& a) {
    const WaveParts whole = parts(a);
    each(a, [&](int q, int, unsigned first, unsigned size) {
      if (q < a.B) {
        const int x0 = size > 0 ? whole.of(first + kStart) : 0;
        a.share[q] = size > 0 ? make_int2(x0 + q, whole.of(first + size - 1) - x0 + 1) : make_int2(0, 0);
      }
      return false;
    });
  }

 private:
  static HD_DEVINLINE int tiles_of(const Args& a, int T) {
    int lo, hi;
    dec::seq_range(a, T, lo, hi);
    return fast_div(hi - fast_div(lo, a.d_tile) * a.tile + a.tile - 1, a.d_tile);
  }
  static HD_DEVINLINE unsigned size_of(const Args& a, int len) { return len >= 1 && len <= a.maxT ? tiles_of(a, len) + kStart : 0; }
  static HD_DEVINLINE WaveParts parts(const Args& a) {
    unsigned all = 0, most = 0;
#pragma unroll 1
    for (int q = threadIdx.x & 31; q < a.B; q += 32) {
      const unsigned size = size_of(a, a.lens[q]);
      all += size;
      most = max(most, size);
    }
    __syncwarp();
    all = __reduce_add_sync(0xffffffffu, all);
    most = __reduce_max_sync(0xffffffffu, most);
    return WaveParts(all, most, (unsigned)a.total, dec::kMaxSplit);
  }
  // f(sequence, its tokens, the tiles before its start, its own and its start's) for each lane's, until one returns true.
  template <class F>
  static HD_DEVINLINE void each(const Args& a, F f) {
    unsigned before = 0;
#pragma unroll 1
    for (int q0 = 0; q0 < a.B; q0 += 32) {
      const int lane = threadIdx.x & 31, q = q0 + lane, len = q < a.B ? a.lens[q] : 0;
      const unsigned size = size_of(a, len);
      unsigned upto = size;
#pragma unroll 1
      for (int d = 1; d < 32; d <<= 1) {
        const unsigned y = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += y;
      }
      if (f(q, len, before + upto - size, size)) return;
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
  }
  // Sequence b's tiles from `skip` on, `want` of them at most, its start's among them (which have numbers below 0).
  HD_DEVINLINE void take(const Args& a, int skip, int want) {
    want += min(skip, 0);
    skip = max(skip, 0);
    int lo, hi;
    dec::seq_range(a, T, lo, hi);
    const int n = min(want, tiles_of(a, T) - skip);  // (none, if that is the start alone)
    k0 = (fast_div(lo, a.d_tile) + skip) * a.tile;
    k1 = n > 0 ? min(hi, k0 + n * a.tile) : k0;
    slot = x + b;
    left = want - n;
  }
};

template <int DH, int WG, bool SHARED>
__global__ void __launch_bounds__(Cfg<DH, WG>::kThreads, Cfg<DH, WG>::kPerSm)
    decode_q8_tc_kernel(const __grid_constant__ Params P) {
  using C = Cfg<DH, WG>;
  using Sm = Smem<DH, WG>;
  constexpr int R = C::R, NSLOT = C::NSLOT, NT = C::kThreads, HV = C::HV, RB = C::RB, kUnit = C::kUnit;
  const Args& a = P.a;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Sm& sm = *reinterpret_cast<Sm*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int split = fast_div((int)blockIdx.x, a.d_heads), head = (int)blockIdx.x - split * a.Hkv * a.ngroups;
  const int g = a.ngroups == 1 ? head : head / a.ngroups, rg = a.ngroups == 1 ? 0 : head % a.ngroups;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int tile = a.tile, row0 = rg * R, rows = min(R, a.M - row0);
  // positions of a tile that no piece fills: their V must not be NaN, nor may their scales, which may not have come yet
  for (int i = tid; i < NSLOT * (KT - tile) * (RB / 16); i += NT) {
    const int per = (KT - tile) * (RB / 16);
    reinterpret_cast<uint4*>(sm.ring[i / per] + tile * RB)[i % per] = make_uint4(0, 0, 0, 0);
  }
  for (int i = tid; i < 512; i += NT) reinterpret_cast<uint32_t*>(sm.scale)[i] = 0;
  if (tid == 0) {
    for (int i = 0; i < NSLOT; ++i) {
      mbar_init(&sm.full[i], 1);
      mbar_init(&sm.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sm.s_full[i], 1);
      mbar_init(&sm.s_free[i], 4 * WG);
      mbar_init(&sm.p_full[i], 4 * WG);
      mbar_init(&sm.pv_done[i], 1);
    }
    for (int i = 0; i < 8; ++i) mbar_init(&sm.sc_full[i], 4);
    mbar_init(&sm.q_full, 4 * WG);
    mbar_init(&sm.drain, 1);
    sm.abort = 0;
    sm.again[0] = sm.again[1] = sm.redo = 0;
    fence_mbar_init();
  }
  if (warp == 0) {
    tmem_alloc(&sm.tmem_base, C::kAlloc);
    tmem_relinquish();
    if (lane == 0) {
      tma_prefetch(&P.tm_k);
      tma_prefetch(&P.tm_v);
    }
  }
  fence_async_smem();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sm.tmem_base;
  volatile int* abort = &sm.abort;
  grid_dep_wait();
  grid_dep_launch();
  Work<SHARED> work(a, split);
  auto tiles_here = [&] { return work.k0 < work.k1 ? fast_div(work.k1 - work.k0 + tile - 1, a.d_tile) : 0; };
  auto partial = [&] { return ((size_t)work.slot * a.Hkv * a.ngroups + head) * R; };  // its first row
  if (work.k0 >= work.k1) {  // nothing of this sequence in this split: an empty partial, or an empty result
    if (!SHARED) {
      if (a.nsplit > 1) {
        for (int i = tid; i < R; i += NT) a.part_ml[partial() + i] = make_float2(-INFINITY, 0.f);
      } else {
        if (work.T != 0 && g == 0 && rg == 0 && tid == 0) set_status(a.status, HD_DEVBIT_INDEX);
        for (int row = warp; row < rows; row += NT / 32)
          decq8::store_row<DH>(a, work.b, g, row0 + row, nullptr, -INFINITY, 0.f);
      }
    }
  } else if (warp == 0) {
    // ------------------------------------------------------------ TMA producer: K(0), then K(j + 1), V(j), of each sequence
    int issued = 0, slot = 0, lap = 0, seq = 0;
    auto load = [&](const CUtensorMap* tm, int2 x) -> bool {
#pragma unroll
      for (int hf = 0; hf < HV; ++hf) {
        if (lap > 0 && !__all_sync(0xffffffffu, mbar_wait(&sm.empty[slot], (lap - 1) & 1, abort, a.status))) return false;
        if (lane == 0) mbar_arrive_expect_tx(&sm.full[slot], tile * RB);
        __syncwarp();
        if (lane * a.piece < tile)
          tma_load_4d(sm.ring[slot] + lane * a.piece * RB, tm, &sm.full[slot], hf * RB, x.y, g, x.x);
        __syncwarp();
        ++issued;
        if (++slot == NSLOT) slot = 0, ++lap;
      }
      return true;
    };
    bool go = true;
    do {
      if (lane == 0) sm.bad_page[seq & 15] = 0;
      __syncwarp();
      const int b = work.b, T = work.T, k0 = work.k0, k1 = work.k1, nt = tiles_here();
      const int32_t* table = a.table + (long long)b * a.pg.max_pages;
      const int seen = a.mode == SFA_LOCAL ? (T - 1) * a.n - a.window + 1 : 0;  // first position any row sees
      // page and row there of this lane's piece of the tiles whose V (cur) and K (nxt) come next; the page entry of the
      // one after them is loaded a tile ahead
      auto pos_of = [&](int j) {  // first position of the piece, -1: none that a row sees
        const int p = lane * a.piece, pos = k0 + j * tile + p;
        return p >= tile || pos >= k1 || pos + a.piece <= seen ? -1 : pos;
      };
      int entry = 0;
      auto fetch = [&](int j) {
        const int pos = pos_of(j);
        if (pos >= 0) {
          const int i = fast_div(pos, a.pg.d_prow);
          entry = i < a.pg.max_pages ? table[i] : -1;
        }
      };
      auto place = [&](int j) {  // of the tile that was fetched: (page, row), behind the pool (zeros) where there is none
        const int pos = pos_of(j);
        int2 x = make_int2(a.pg.num_pages, 0);
        if (pos >= 0) {
          if ((unsigned)entry < (unsigned)a.pg.num_pages) x = make_int2(entry, pos - fast_div(pos, a.pg.d_prow) * a.pg.prow);
          else sm.bad_page[seq & 15] = 1;
        }
        return x;
      };
      fetch(0);
      int2 cur = place(0), nxt;
      fetch(1);
      go = load(&P.tm_k, cur);
      for (int j = 0; go && j < nt; ++j) {
        nxt = place(j + 1);
        fetch(j + 2);
        if (j + 1 < nt) go = load(&P.tm_k, nxt);
        go = go && load(&P.tm_v, cur);
        cur = nxt;
      }
      ++seq;
    } while (go && work.next(a));
    // (a wait that gave up ends the kernel's work, not its copies in flight)
    if (lane == 0)
      for (int u = max(0, issued - NSLOT); u < issued; ++u) mbar_drain(&sm.full[u % NSLOT], (u / NSLOT) & 1);
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ the products
    constexpr uint32_t idS = C::kPair ? idesc_f8(128, 2 * R, 0, 0, 0, 0) : idesc_f8(128, R, 0, 1, 0, 0);
    constexpr uint32_t idO = idesc_f8(RB, 3 * R, 0, 1, 1, 1);
    const uint64_t kd = sdesc_rows<RB>(smem_u32(sm.ring[0])), qd = sdesc_rows<RB>(smem_u32(sm.q[0][0]));
    const uint64_t pd = sdesc_plain_mn(smem_u32(sm.p[0][0]), 128, KT * 16);
    int slot = 0, lap = 0, done = 0, seq = 0;  // done: tiles of the sequences before
    bool ok = true;
    auto wait_unit = [&]() -> bool {
      if (!__all_sync(0xffffffffu, mbar_wait(&sm.full[slot], lap & 1, abort, a.status))) return false;
      tc_fence_after();
      return true;
    };
    auto done_unit = [&] {
      tc_commit_w(&sm.empty[slot]);
      if (++slot == NSLOT) slot = 0, ++lap;
    };
    auto issue_s = [&](int j) -> bool {
      const int at = done + j, sb = at & 1;
      if (at >= 2) {
        if (!__all_sync(0xffffffffu, mbar_wait(&sm.s_free[sb], ((at >> 1) - 1) & 1, abort, a.status))) return false;
        tc_fence_after();
      }
#pragma unroll
      for (int hf = 0; hf < HV; ++hf) {
        if (!wait_unit()) return false;
        const uint64_t kk = kd + (uint64_t)(slot * (kUnit / 16)), qq = qd + (uint64_t)(hf * (C::QT * R * RB / 16));
#pragma unroll
        for (int i = 0; i < RB / 32; ++i)
#pragma unroll
          for (int term = 0; term < (C::kPair ? 1 : 3); ++term)
            mma_f8_ss_w(tmem + sb * C::SC, kk + i * 2, qq + term * (R * RB / 16) + i * 2, idS, hf + i + term > 0 ? 1u : 0u);
        done_unit();
      }
      tc_commit_w(&sm.s_full[sb]);
      return true;
    };
    auto issue_pv = [&](int j) -> bool {
      const int at = done + j, pb = at & 1;
      if (!__all_sync(0xffffffffu, mbar_wait(&sm.p_full[pb], (at >> 1) & 1, abort, a.status))) return false;
      tc_fence_after();
#pragma unroll
      for (int hf = 0; hf < HV; ++hf) {
        if (!wait_unit()) return false;
        const uint64_t vv = kd + (uint64_t)(slot * (kUnit / 16)), pp = pd + (uint64_t)(pb * (3 * R * KT / 16));
#pragma unroll
        for (int i = 0; i < 4; ++i)
          mma_f8_ss_w(tmem + 2 * C::SC + hf * 3 * R, vv + i * (32 * RB / 16), pp + i * 32, idO, j > 0 || i > 0 ? 1u : 0u);
        done_unit();
      }
      tc_commit_w(&sm.pv_done[pb]);
      return true;
    };
    do {
      const int nt = tiles_here();
      ok = __all_sync(0xffffffffu, mbar_wait(&sm.q_full, seq++ & 1, abort, a.status));  // (and O of the one before is read)
      tc_fence_after();
      ok = ok && issue_s(0);
      for (int j = 0; ok && j < nt; ++j) {
        if (j + 1 < nt) ok = issue_s(j + 1);
        ok = ok && issue_pv(j);
      }
      done += nt;
    } while (ok && work.next(a));
    tc_commit_w(&sm.drain);
    mbar_drain(&sm.drain, 0);
  } else {
    // ------------------------------------------------------------ softmax: a thread per position
    const int wg = (warp - 2) >> 2, q4 = warp & 3, key = q4 * 32 + lane, r0 = wg * RW, bar = 1 + wg;
    const uint32_t tl = tmem + ((uint32_t)(q4 * 32) << 16), tO = tl + 2 * C::SC + r0;
    const uint32_t real = bits(0, rows - r0);
    bool ok = true;
    int done = 0, chunks = 0, seq = 0;  // tiles and chunks of the sequences before; their number
    do {
      const int b = work.b, T = work.T, k0 = work.k0, k1 = work.k1, nt = tiles_here();
      const int32_t* table = a.table + (long long)b * a.pg.max_pages;
      float* po = a.part_o + partial() * DH;
      float2* pml = a.part_ml + partial();
      const int own_lo = (T - 1) * a.n, win_hi = a.mode == SFA_LOCAL ? T * a.n - 1 - a.window : -1;
      const int seen = a.mode == SFA_LOCAL ? own_lo - a.window + 1 : 0;
      // The first group brings the scales, 128 blocks (a chunk) at a time, a thread each, by cp.async: behind a saturated
      // memory's queue a load takes thousands of cycles.  Blocks are counted from the split's first.  As chunk c is handed on,
      // the words that hold the bytes of chunk c + 3 are asked for (cut to the scales' array; a byte's place is kept), and
      // the page entries of chunk c + 6.
      const int b0 = fast_div(k0, a.d_brow), nblocks = fast_div(k1 - 1, a.d_brow) - b0 + 1;
      const int b_seen = seen <= 0 ? 0 : fast_div(seen, a.d_brow) - b0;  // the first that a row sees
      uint32_t places = 0;
      int handed = 0;  // chunks, from this sequence's first
      auto page_of = [&](int x, int& in) {  // of block x; -1: none that is needed
        if (x >= nblocks || x < b_seen) return -1;
        const int pg = fast_div(b0 + x, a.d_blocks);
        in = b0 + x - pg * a.blocks;
        return pg < a.pg.max_pages ? pg : -1;
      };
      auto chunk_words = [&](int c, int entry) {
        int in = 0;
        if (page_of(c * 128 + key, in) >= 0 && (unsigned)entry < (unsigned)a.pg.num_pages) {
          const size_t at = ((size_t)entry * a.Hkv + g) * a.blocks + in, word = at & ~(size_t)3;
          const int bytes = (int)min((size_t)a.pg.num_pages * a.Hkv * a.blocks - word, (size_t)4), sh = (c & 3) * 2;
          const uint32_t to = smem_u32(&sm.words[c & 3][key]);
          cp_async_4(to, a.kscale + word, bytes);
          cp_async_4(to + 4, a.vscale + word, bytes);
          places = (places & ~(3u << sh)) | (uint32_t)(at & 3) << sh;
        }
      };
      auto chunk_entries = [&](int c) {
        int in = 0;
        const int pg = page_of(c * 128 + key, in);
        if (pg >= 0) cp_async_4(smem_u32(&sm.entry[c & 3][key]), table + pg, 4);
      };
      auto hand_on = [&] {  // the next chunk's bytes
        cp_async_wait<2>();
        const int c = handed++;
        const uint2 x = sm.words[c & 3][key];
        const int sh = (places >> (c & 3) * 2 & 3) * 8;
        const int kb = q8::clamp_byte(x.x >> sh & 255), block = c * 128 + key;
        sm.scale[((chunks + c) & 7) * 128 + key] = (uint16_t)(kb | q8::clamp_byte(x.y >> sh & 255) << 8);
        const int most = (int)__reduce_max_sync(0xffffffffu, block >= b_seen && block < nblocks ? (unsigned)kb : 0u);
        if (lane == 0) sm.most_kb[seq & 1][q4] = max(c > 0 ? sm.most_kb[seq & 1][q4] : 0, most);
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.sc_full[(chunks + c) & 7]);
        chunk_words(c + 3, sm.entry[(c + 3) & 3][key]);
        chunk_entries(c + 6);
        cp_async_commit();
      };
      int first[3] = {-1, -1, -1};
      if (wg == 0) {
        int in = 0;
#pragma unroll
        for (int c = 0; c < 3; ++c) {
          const int pg = page_of(c * 128 + key, in);
          if (pg >= 0) first[c] = table[pg];
        }
      }
      {  // the queries: four rows a warp
        constexpr int NP = DH / 64;  // pairs of a lane
        uint32_t w[4][NP];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int rr = r0 + q4 * 4 + x;
#pragma unroll
          for (int i = 0; i < NP; ++i) w[x][i] = 0;
          if (rr < rows) {
            const int r = row0 + rr, s = fast_div(r, a.d_G), h = g * a.G + r - s * a.G;
            const uint32_t* src = reinterpret_cast<const uint32_t*>(a.q + (((long long)b * a.n + s) * a.Hq + h) * DH) + lane * NP;
#pragma unroll
            for (int i = 0; i < NP; ++i) w[x][i] = src[i];
          }
        }
        if (wg == 0) {
#pragma unroll
          for (int c = 0; c < 3; ++c) {
            chunk_words(c, first[c]);
            chunk_entries(c + 3);
            cp_async_commit();
          }
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int rr = r0 + q4 * 4 + x;
          uint32_t most = 0;
#pragma unroll
          for (int i = 0; i < NP; ++i) most = max(most, max(w[x][i] << 16 & 0x7fff0000u, w[x][i] & 0x7fff0000u));
          most = __reduce_max_sync(0xffffffffu, most);
          // the exponent field of the largest magnitude, kept where both powers are normal
          const int e = min(max((int)(most >> 23), 20), 254);
          constexpr int kUp = C::kPair ? 7 : 14;  // the largest to [2^kUp, 2^(kUp + 1))
          const float to = __int_as_float(min(127 + kUp + 127 - e, 254) << 23);  // 2^(kUp - (e - 127)), at most 2^127
          const float back = __int_as_float(max(e - kUp, 1) << 23);              // 2^(e - 127 - kUp)
          float miss = 0.f;  // at most 2^-14 a value (2^-17 where kUp is 14)
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            const float x0 = __uint_as_float(w[x][i] << 16) * to, x1 = __uint_as_float(w[x][i] & 0xffff0000u) * to;
            [[maybe_unused]] float2 left = make_float2(x0, x1);
            uint32_t t[3];
            if (C::kPair) {
              t[0] = q8::code2(x0, x1);
              const float2 y = q8::values2((uint16_t)t[0]);
              t[1] = q8::code2((x0 - y.x) * kLo, (x1 - y.y) * kLo);
              const float2 z = q8::values2((uint16_t)t[1]);
              miss += fabsf(x0 - y.x - z.x / kLo) + fabsf(x1 - y.y - z.y / kLo);
            } else {
              const __half2 u = __floats2half2_rn(x0, x1);
              split3<false>(*reinterpret_cast<const uint32_t*>(&u), t[0], t[1], t[2]);
#pragma unroll
              for (int y = 0; y < 3; ++y) {
                const uint32_t code = t[y] & 0xff00ff00u;
                const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&code));
                left.x -= z.x, left.y -= z.y;
                t[y] = __byte_perm(t[y], 0, 0x31);
              }
              miss += fabsf(left.x) + fabsf(left.y);
            }
            const int c = (lane * NP + i) * 2, at = (c % RB) >> 4, off = c & 15;  // column; its 16-byte chunk
            const int swizzled = RB == 64 ? at ^ (rr >> 1 & 3) : at ^ (rr & 7);
#pragma unroll
            for (int y = 0; y < C::QT; ++y)
              *reinterpret_cast<uint16_t*>(sm.q[c / RB][y] + rr * RB + swizzled * 16 + off) = (uint16_t)t[y];
          }
          constexpr float kUnit24 = C::kPair ? 0x1p36f : 0x1p39f;
          const unsigned missed = __reduce_add_sync(0xffffffffu, __float2uint_ru(miss * kUnit24));
          if (lane == 0) {
            sm.rowf[rr] = back * a.scale_log2;
            sm.missed[rr] = (float)missed / kUnit24 * 448.f * fabsf(back * a.scale_log2);
          }
        }
        if (lane < RW) sm.nref[q4][r0 + lane] = sm.lost[q4][r0 + lane] = 0.f;
        fence_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.q_full);
        named_bar_sync(bar, 128);  // the group's rows
      }
      uint64_t l[RW / 2];  // pairs of rows' sums over this thread's positions
#pragma unroll
      for (int r = 0; r < RW / 2; ++r) l[r] = 0;
      uint32_t set = 0;  // rows whose reference is set
      int top_vb = 0;    // V's largest scale byte in the tiles that set references: no row's sum is below 2^kSet 2^-ev of it
      const int brow = a.pg.prow / a.blocks;
      int waited = 0;                               // chunks that this warp has waited for
      long long scales_end = (long long)b0 * brow;  // the first position behind them
      // this key's block, from the split's first, and its row there; both go on by a tile
      const int step_blocks = fast_div(tile, a.d_brow), step_rows = tile - step_blocks * brow;
      int block = fast_div(k0 + key, a.d_brow) - b0, in_block = k0 + key - (block + b0) * brow;
      const int edge = tile < KT ? 0 : min(own_lo + 1, k1);  // tiles that end at or before it have no mask but WITHIN's
      for (int j = 0; j < nt; ++j) {
        const int at = done + j, sb = at & 1, base = k0 + j * tile, p = base + key;
        // the chunks of this tile's blocks: handed on by the first group, and waited for
        while (min(base + tile, k1) > scales_end) {
          if (wg == 0) hand_on();
          ok = ok && __all_sync(0xffffffffu, mbar_wait(&sm.sc_full[(chunks + waited) & 7], (chunks + waited) >> 3 & 1, abort, a.status));
          ++waited;
          scales_end += 128ll * brow;
        }
        // the rows that see this position: a range
        uint32_t vis = real;
        if (a.mode == SFA_WITHIN && a.n > 1) {
          const int s = p - fast_div(p, a.d_n) * a.n;
          vis &= bits(s * a.G - row0 - r0, (s + 1) * a.G - row0 - r0);
        }
        if (base + tile > edge || base <= win_hi) {
          // rows of the streams from p's own on, where p is the new token's
          const int first = max(p - own_lo, 0) * a.G - row0 - r0;
          const int last = a.mode == SFA_LOCAL ? (int)min(((long long)p - own_lo + a.window) * a.G - row0 - r0, (long long)RW) : RW;
          vis = key < tile && p < k1 ? vis & bits(p < own_lo ? 0 : first, last) : (uint32_t)0;
        }
        // (A wait that gave up: the warp goes on to the group's next vote, since the others may wait for it there, and all
        // leave after it.)
        ok = ok && __all_sync(0xffffffffu, mbar_wait(&sm.s_full[sb], (at >> 1) & 1, abort, a.status));
        tc_fence_after();
        const int sc = sm.scale[(chunks * 128 + min(block, nblocks - 1)) & 1023], kb = sc & 255, vb = sc >> 8;
        block += step_blocks;
        in_block += step_rows;
        if (in_block >= brow) in_block -= brow, ++block;
        const float kf = q8::scale_of(kb), ev = (float)(vb - 127), inv = q8::inverse_of(vb);
        const uint64_t kf2 = f2pack(kf, kf), ev2 = f2pack(ev, ev);
        float y[RW];
        {
          float low[RW];
          tmem_ld16(tl + sb * C::SC + r0, reinterpret_cast<uint32_t*>(y));
          if (C::kPair) tmem_ld16(tl + sb * C::SC + R + r0, reinterpret_cast<uint32_t*>(low));
          tmem_ld_wait();
          if (C::kPair)
#pragma unroll
            for (int r = 0; r < RW; r += 2)
              f2unpack(ffma2(f2pack(low[r], low[r + 1]), f2pack(1.f / kLo, 1.f / kLo), f2pack(y[r], y[r + 1])), y[r], y[r + 1]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.s_free[sb]);
#pragma unroll
        for (int c = 0; c < RW; c += 4) {
          const ulonglong2 f = *reinterpret_cast<const ulonglong2*>(sm.rowf + r0 + c);
          const ulonglong2 rf = *reinterpret_cast<const ulonglong2*>(sm.nref[q4] + r0 + c);
          f2unpack(ffma2(fmul2(f2pack(y[c], y[c + 1]), f.x), kf2, fadd2(ev2, rf.x)), y[c], y[c + 1]);
          f2unpack(ffma2(fmul2(f2pack(y[c + 2], y[c + 3]), f.y), kf2, fadd2(ev2, rf.y)), y[c + 2], y[c + 3]);
        }
        if (__any_sync(0xffffffffu, vis != real))
#pragma unroll
          for (int r = 0; r < RW; ++r)
            if (!((vis >> r) & 1u)) y[r] = -INFINITY;
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < RW; r += 2) top = max3(top, y[r], y[r + 1]);
        if (group_any(bar, !ok || top > kTop || (vis & ~set) != 0)) {
          // New references for the rows (of the whole group) of which some P would pass 2^kTop, or which have none yet:
          // their largest P to 2^kSet.
          uint32_t mask = vis & ~set;
          float m = 0.f;  // lane r: row r's
#pragma unroll
          for (int r = 0; r < RW; ++r) {
            if (y[r] > kTop) mask |= 1u << r;
            const int x = __reduce_max_sync(0xffffffffu, ordered(y[r] == y[r] ? y[r] : -INFINITY));
            if (lane == r) m = from_ordered(x);
          }
          mask = __reduce_or_sync(0xffffffffu, mask | (ok ? 0 : kGaveUp));
          const unsigned most_vb = __reduce_max_sync(0xffffffffu, vis != 0 ? (unsigned)vb : 0u);
          if (lane < RW) sm.most[q4][r0 + lane] = m;
          if (lane == 0) sm.raise[wg * 4 + q4] = mask | most_vb << 16;
          named_bar_sync(bar, 128);  // (the next vote lies before these are written again)
          mask = 0;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const unsigned x = sm.raise[wg * 4 + w];
            mask |= x & (0xffffu | kGaveUp);
            top_vb = max(top_vb, (int)(x >> 16 & 255));
          }
          if (mask & kGaveUp) {
            ok = false;
            break;
          }
          float down = 0.f, fac = 1.f;  // lane r: what row r's reference goes up by, negated; the root of 2^ that (a sum's
                                        // range is wider than a power's)
          if (lane < RW && (mask >> lane & 1u)) {
            const int r = r0 + lane;
            down = kSet - fmaxf(fmaxf(sm.most[0][r], sm.most[1][r]), fmaxf(sm.most[2][r], sm.most[3][r]));
            sm.nref[q4][r] += down;
            if (set >> lane & 1u) fac = ex2_approx(0.5f * down);
            sm.lost[q4][r] *= fac * fac;
          }
          __syncwarp();
#pragma unroll
          for (int r = 0; r < RW; r += 2) {
            const uint64_t root = f2pack(__shfl_sync(0xffffffffu, fac, r), __shfl_sync(0xffffffffu, fac, r + 1));
            l[r / 2] = fmul2(fmul2(l[r / 2], root), root);
            y[r] += __shfl_sync(0xffffffffu, down, r);
            y[r + 1] += __shfl_sync(0xffffffffu, down, r + 1);
          }
          if ((mask & set) != 0 && j > 0) {
            // (the products of the tile before the last are done, see below: so the wait is for the right phase)
            ok = __all_sync(0xffffffffu, mbar_wait(&sm.pv_done[(at - 1) & 1], ((at - 1) >> 1) & 1, abort, a.status));
            tc_fence_after();
            for (uint32_t left = mask & set; left; left &= left - 1) {
              const int r = __ffs(left) - 1;
              tmem_scale<3 * HV, R>(tO + r, __shfl_sync(0xffffffffu, fac, r));
            }
            tmem_st_wait();
          }
          set |= mask;
        }
        if (!ok) continue;
        if (__any_sync(0xffffffffu, vis != 0 && vb + kFar < top_vb)) {
          Scores x;
#pragma unroll
          for (int r = 0; r < RW; ++r) x.y[r] = y[r];
          note_losses(x, vis, vb, top_vb, &sm.lost[q4][r0]);
        }
        // S of this tile was issued behind the products of the tile before the last, so these are done: P's buffer is free
        const uint64_t inv2 = f2pack(inv, inv);
        {
          uint4 t[3];
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            uint32_t hi[2], mid[2], lo[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int r = h * 4 + i * 2;
              const float p0 = ex2_approx(y[r]), p1 = ex2_approx(y[r + 1]);
              l[r / 2] = ffma2(f2pack(p0, p1), inv2, l[r / 2]);
              const __half2 u = __floats2half2_rn(p0, p1);
              split3<true>(*reinterpret_cast<const uint32_t*>(&u), hi[i], mid[i], lo[i]);
            }
            (&t[0].x)[h] = __byte_perm(hi[0], hi[1], 0x7531);
            (&t[1].x)[h] = __byte_perm(mid[0], mid[1], 0x7531);
            (&t[2].x)[h] = __byte_perm(lo[0], lo[1], 0x7531);
          }
          const int to = wg * (KT * 16) + key * 16;
#pragma unroll
          for (int i = 0; i < 3; ++i) *reinterpret_cast<uint4*>(sm.p[sb][i] + to) = t[i];
        }
        // The sequence's last tile holds positions behind its length, which may never have been written: their P is 0, and
        // 0 times a NaN is NaN, so their V is zeroed before the product (which waits for this thread's arrival).
        if (base + tile > k1 && wg == 0) {
          // The ring's last units are this tile's V.  (A wait tells only a phase from the next: with the products of the
          // tile before done, all units but these have landed.)
          if (at >= 1) ok = __all_sync(0xffffffffu, mbar_wait(&sm.pv_done[(at - 1) & 1], ((at - 1) >> 1) & 1, abort, a.status));
          static_assert(NSLOT >= HV, "");
#pragma unroll
          for (int h = 0; h < HV; ++h) {
            const int u = 2 * HV * (at + 1) - HV + h;
            ok = ok && __all_sync(0xffffffffu, mbar_wait(&sm.full[u % NSLOT], (u / NSLOT) & 1, abort, a.status));
            if (ok && p >= k1)
#pragma unroll
              for (int c = 0; c < RB / 16; ++c) reinterpret_cast<uint4*>(sm.ring[u % NSLOT] + key * RB)[c] = make_uint4(0, 0, 0, 0);
          }
          __syncwarp();
          if (!ok) continue;
        }
        fence_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sm.p_full[sb]);
      }
      cp_async_wait<0>();
      float sum = 0.f;  // lane r: row r's over this warp's positions
#pragma unroll
      for (int r = 0; r < RW; ++r) {
        float x, other;
        if (r & 1) f2unpack(l[r / 2], other, x);
        else f2unpack(l[r / 2], x, other);
#pragma unroll
        for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        if (lane == r) sum = x;
      }
      // (this warp's references are its own to write over)
      const float ref = lane < RW ? sm.nref[q4][r0 + lane] : 0.f;
      if (lane < RW) sm.nref[q4][r0 + lane] = sum;
      ok = ok && __all_sync(0xffffffffu, mbar_wait(&sm.pv_done[(done + nt - 1) & 1], ((done + nt - 1) >> 1) & 1, abort, a.status));
      if (group_any(bar, !ok)) ok = false;  // (also: every warp's sums are written)
      if (ok) {
        int k = 0;  // lane r: the exponent of row r's sum, by which its partial is divided
        if (lane < RW) {
          const int r = r0 + lane;
          sum = (sm.nref[0][r] + sm.nref[1][r]) + (sm.nref[2][r] + sm.nref[3][r]);
          k = decq8::sum_exponent(sum);
        }
        const float part = decq8::two_to_minus(k);
        __syncwarp();  // (lanes' branches lie behind the accesses to tensor memory, here and below)
        tc_fence_after();
        const bool bad = *(volatile int*)&sm.bad_page[seq & 15] != 0;
        // this lane's row of O^T: all 128, or (a product of 64 rows) 16 of each 32
        const int column = RB == 128 ? key : lane < 16 ? q4 * 16 + lane : -1;
#pragma unroll
        for (int hf = 0; hf < HV; ++hf) {
          uint32_t o[3][16];
#pragma unroll
          for (int i = 0; i < 3; ++i) tmem_ld16(tO + (hf * 3 + i) * R, o[i]);
          tmem_ld_wait();
          uint32_t wrong = 0;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const float x = fmaf(__uint_as_float(o[2][e]), 1.f / kLow, __uint_as_float(o[0][e]) + __uint_as_float(o[1][e])) *
                            __shfl_sync(0xffffffffu, part, e);
            if (column < 0) continue;
            po[(size_t)(r0 + e) * DH + hf * RB + column] = x;
            if (!(fabsf(x) <= FLT_MAX)) wrong |= 1u << e;
          }
          wrong = __reduce_or_sync(0xffffffffu, wrong);
          if (wrong != 0 && lane == 0) atomicOr(&sm.again[r0 >> 5], wrong << (r0 & 31));
          __syncwarp();
        }
        named_bar_sync(bar, 128);
        if (key < RW) {
          const int r = r0 + key;
          const float lost = (sm.lost[0][r] + sm.lost[1][r]) + (sm.lost[2][r] + sm.lost[3][r]);
          const int* kb = sm.most_kb[seq & 1];
          const float missed = sm.missed[r] * q8::scale_of(max(max(kb[0], kb[1]), max(kb[2], kb[3])));
          const bool loss = (lost > kLost * sum || missed > decq8::kMissed) && (set >> key & 1u);
          sum *= part;
          float m = (set >> key) & 1u ? (float)k - ref : -INFINITY;
          if (sum != sum) m = INFINITY;  // a visible score that is not finite: the combined row is NaN
          if (bad) {
            m = -INFINITY, sum = decq8::kBadPage;
          } else if (r < rows && (loss || (sm.again[r >> 5] >> (r & 31) & 1u))) {
            sum = kRedo;
            sm.redo = 1;
          }
          pml[r] = make_float2(m, sum);
          if (!SHARED && a.nsplit == 1 && bad && key == 0) set_status(a.status, HD_DEVBIT_INDEX);
        }
        named_bar_sync(bar, 128);
        if (key == 0) atomicAnd(&sm.again[r0 >> 5], ~(0xffffu << (r0 & 31)));
      }
      done += nt;
      chunks += waited;
      ++seq;
    } while (ok && work.next(a));
    // Rows that came out not finite, by their visible keys alone: last, so that no other warp's bounded wait runs meanwhile.
    if (ok && *(volatile int*)&sm.redo) {
      if (SHARED) work = Work<SHARED>(a, split);
      do {
#pragma unroll 1
        for (int r = q4; r < RW; r += 4) {
          const size_t at = partial() + r0 + r;
          if (r0 + r < rows && a.part_ml[at].y == kRedo)
            decq8::exact_row<DH>(a, work.b, g, row0 + r0 + r, work.T, work.k0, work.k1, a.part_o + at * DH, a.part_ml + at);
        }
      } while (work.next(a));
    }
    if (!SHARED && ok && a.nsplit == 1) {  // the only split: its rows are the results
      __syncwarp();
      for (int r = r0 + q4; r < min(r0 + RW, rows); r += 4) {
        const size_t at = partial() + r;
        const float2 ml = a.part_ml[at];
        decq8::store_row<DH>(a, work.b, g, row0 + r, a.part_o + at * DH, ml.x, ml.y == decq8::kBadPage ? 0.f : ml.y);
      }
    }
  }
  if (SHARED && blockIdx.x == 0 && warp == 1) Work<SHARED>::report(a);
  tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, C::kAlloc);
  }
}
}  // namespace decq8tc

// ------------------------------------------------------------------ host side

template <int DH, int WG, bool SHARED>
static cudaError_t launch_s(const decq8::Params& p, unsigned parts, cudaStream_t st) {
  using namespace decq8tc;
  using C = Cfg<DH, WG>;
  const int smem = (int)sizeof(Smem<DH, WG>) + 1024;
  static_assert(sizeof(Smem<DH, WG>) + 1024 <= (C::kPerSm == 3 ? 75 : C::kPerSm == 2 ? 113 : 227) * 1024 && C::NSLOT >= 3 &&
                    C::kCols <= C::kAlloc && C::kPerSm * C::kAlloc <= 512,
                "an SM's CTAs fit");
  const auto kernel = decode_q8_tc_kernel<DH, WG, SHARED>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  return launch_kernel(true, kernel, dim3(parts * p.a.Hkv * p.a.ngroups), (unsigned)C::kThreads, smem, st, p);
}
template <int DH, int WG>
static cudaError_t launch_t(const decq8::Params& p, cudaStream_t st) {
  return p.a.balanced ? launch_s<DH, WG, true>(p, p.a.total, st) : launch_s<DH, WG, false>(p, p.a.nsplit * p.a.B, st);
}

template <int DH>
static int per_sm(int rows) {
  using namespace decq8tc;
  return rows <= 16   ? Cfg<DH, 1>::kPerSm
         : rows <= 32 ? Cfg<DH, 2>::kPerSm
         : rows <= 48 ? Cfg<DH, 3>::kPerSm
                      : Cfg<DH, 4>::kPerSm;
}
int decode_q8_tc_per_sm(int rows, int Dh) { return Dh == 64 ? per_sm<64>(rows) : Dh == 128 ? per_sm<128>(rows) : per_sm<256>(rows); }

template <int DH>
static cudaError_t launch_d(const decq8::Params& p, cudaStream_t st) {
  if (p.a.rg == 16) return launch_t<DH, 1>(p, st);
  if (p.a.rg == 32) return launch_t<DH, 2>(p, st);
  if (p.a.rg == 48) return launch_t<DH, 3>(p, st);
  return launch_t<DH, 4>(p, st);
}

cudaError_t launch_decode_q8_tc(decq8::Params& p, int Dh, cudaStream_t st) {
  return Dh == 64 ? launch_d<64>(p, st) : Dh == 128 ? launch_d<128>(p, st) : launch_d<256>(p, st);
}

}  // namespace hdsfa
