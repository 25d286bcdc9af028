// Rows into and out of the 8-bit paged cache, and copies of its pages.  All are bound by memory: a row's 2 bytes a
// value on the bf16 side, 1 on the cache's.
#include <algorithm>

#include "q8.cuh"

namespace hdsfa {
namespace q8 {

struct AppendArgs {
  const uint16_t *kn, *vn;  // bf16 bits: [B][n][Hkv][Dh], or packed [N*n][Hkv][Dh]
  uint8_t *kc, *vc, *ks, *vs;
  const int32_t *table, *lens, *offsets, *served;
  int B, N, cap;
  long long units;
  Geom g;
  FastDiv d_T, d_cpr;  // tokens of a block, 16-value chunks of a row
  int32_t* status;
};

// 32 bytes, a whole sector, in one load (p 32-byte aligned); two of 16 bytes take a sector twice (6 prompts of up to 4000
// tokens, 4 streams, 8 heads of 128, a scale a page, the CTA's teams: 42.7 -> 40.6 us, by now 39.7; the warps' spill with
// it: a scale a token 42.5 -> 49.9).
HD_DEVINLINE void ld_global_32(const void* p, uint32_t* r) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "l"(p)
               : "memory");
}

// Sixteen values of a row as 8 words of bf16 pairs.
struct Chunk {
  uint32_t w[8];
};
template <bool WHOLE>
HD_DEVINLINE Chunk load_chunk(const uint16_t* p) {
  Chunk c;
  if (WHOLE && (reinterpret_cast<uintptr_t>(p) & 31) == 0) {  // (a base need only be aligned to 16 bytes)
    ld_global_32(p, c.w);
    return c;
  }
  const uint4 a = reinterpret_cast<const uint4*>(p)[0], b = reinterpret_cast<const uint4*>(p)[1];
  c.w[0] = a.x, c.w[1] = a.y, c.w[2] = a.z, c.w[3] = a.w;
  c.w[4] = b.x, c.w[5] = b.y, c.w[6] = b.z, c.w[7] = b.w;
  return c;
}
// Largest finite magnitude, as bf16 bits.  Infinities become NaN, as their codes are: with a check for each value at its
// conversion instead, 24 short prompts with a scale a token took 11.5 us for 10.6, 6 of up to 4000 tokens 40.8 for 39.7.
HD_DEVINLINE uint32_t tame(Chunk& c) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = __vmaxu2(m, c.w[i] & 0x7fff7fffu);
  m = max(m & 0xffff, m >> 16);
  if (m < 0x7f80) return m;
  m = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const uint32_t x = (c.w[i >> 1] >> (i & 1) * 16) & 0x7fff;
    if (x < 0x7f80) m = max(m, x);
    else c.w[i >> 1] |= 0x7fffu << (i & 1) * 16;
  }
  return m;
}
// The codes of a tamed chunk.
HD_DEVINLINE uint4 codes_of(const Chunk& c, float inv) {
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t a = c.w[2 * i], b = c.w[2 * i + 1];
    r[i] = code2_sat(__uint_as_float(a << 16) * inv, __uint_as_float(a & 0xffff0000u) * inv) |
           code2_sat(__uint_as_float(b << 16) * inv, __uint_as_float(b & 0xffff0000u) * inv) << 16;
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}
// Codes of values divided by a power of two: exact but for results below 2^-6.
HD_DEVINLINE uint32_t recode4(uint32_t c, float f) {
  const float2 a = values2((uint16_t)c), b = values2((uint16_t)(c >> 16));
  return code2_sat(a.x * f, a.y * f) | code2_sat(b.x * f, b.y * f) << 16;
}

// The largest b < B with key(b) <= u, found by a warp with one load for each 5 bits of B; -1 if there is none.
template <class Key>
HD_DEVINLINE int last_not_above(int B, long long u, int lane, Key key) {
  int lo = 0, n = B;
  while (true) {
    const int step = (n + 31) / 32, i = lane * step;
    const unsigned le = __ballot_sync(0xffffffffu, i < n && key(lo + i) <= u);
    if (le == 0) return -1;
    const int l = 31 - __clz(le);
    lo += l * step;
    if (step == 1) return lo;
    n = min(step, n - l * step);
  }
}

constexpr int kHeld = 4;  // chunks that a thread holds from the maximum to the codes

// A unit is what a call appends to one block of tokens.  For each head and tensor (a pair, of which there are 2 Hkv) a team
// of threads finds the new rows' largest magnitude, which gives the scale, and codes the rows; they are read once where
// they fit kHeld chunks a thread.  A block that held tokens before keeps at least its scale, and where that grows the older
// rows are coded again, by the new rows' team (one token of 64 sequences, 8 heads of 128, 4 streams: 2.9 us where no block
// grows, 14 to 16 where some or all do with 16 tokens a block, 43 to 58 with 64).  A team is the CTA (a unit and pair each), or as many lanes of a warp as the rows need: then a warp
// takes a unit and finds its place once for all its pairs, or for one in gridDim.y of them where units are few.  (A warp
// for each unit and pair: 24 prompts of up to 701 tokens, 3 streams, 4 heads of 64, a scale a token 35.7 us.)
// With offsets, sequence b's units have the numbers from offsets[b] / T + 2 b on: x tokens touch at most x / T + 2
// blocks, and those numbers are at least as far apart.
template <int TEAM>
__global__ void __launch_bounds__(128, 6) append_q8_kernel(AppendArgs a) {
  static_assert(TEAM == 8 || TEAM == 16 || TEAM == 32 || TEAM == 128, "lanes of a warp, or the CTA");
  __shared__ uint32_t warp_most[4];
  const int lane = threadIdx.x & 31, tid = threadIdx.x % TEAM;
  const bool report = blockIdx.y == 0 && (TEAM == 128 ? threadIdx.x : lane) == 0;
  const Geom& g = a.g;
  const int n = g.n, Dh = g.Dh;
  grid_dep_wait();
  grid_dep_launch();
  if (a.offsets != nullptr && blockIdx.x == 0 && blockIdx.y == 0)
    for (int b = threadIdx.x; b < a.B; b += 128) {
      const int x = a.offsets[b], z = a.offsets[b + 1], L = a.lens[b];
      bool bad = x < 0 || z < x || z > a.N || L < 0 || L > a.cap;
      if (!bad) bad = z - x > L && (a.served == nullptr || a.served[b] >= z - x);
      if (bad) set_status(a.status, HD_DEVBIT_INDEX);
    }
  constexpr int kUnits = TEAM == 128 ? 1 : 4;        // of a CTA at a time
  constexpr int kTeams = TEAM == 128 ? 1 : 32 / TEAM;  // of a unit at a time
  for (long long u = (long long)blockIdx.x * kUnits + (TEAM == 128 ? 0 : threadIdx.x >> 5); u < a.units;
       u += (long long)gridDim.x * kUnits) {
    // the block's new tokens [t0, t1) of sequence b, t0's packed token i0, and the block's first token tb
    int b, t0, t1, tb;
    long long i0;
    if (a.offsets != nullptr) {
      b = last_not_above(a.B, u, lane, [&](int i) { return (long long)fast_div(max(a.offsets[i], 0), a.d_T) + 2ll * i; });
      if (b < 0) continue;
      const int x = a.offsets[b], z = a.offsets[b + 1], L = a.lens[b];
      if (x < 0 || z <= x || z > a.N || L > a.cap || z - x > L) continue;
      if (a.served != nullptr && a.served[b] < z - x) continue;
      const int first = L - (z - x);
      const long long j = u - fast_div(x, a.d_T) - 2ll * b, from = (long long)(fast_div(first, a.d_T) + j) * g.T;
      if (from >= L) continue;
      tb = (int)from;
      t0 = max(first, tb);
      t1 = L - tb < g.T ? L : tb + g.T;
      i0 = x + (t0 - first);
    } else {
      b = (int)u;
      const int L = a.lens[b];
      if (L < 0 || L > a.cap) {
        if (report) set_status(a.status, HD_DEVBIT_INDEX);
        continue;
      }
      if (L == 0 || (a.served != nullptr && a.served[b] < 1)) continue;
      t0 = L - 1;
      t1 = L;
      tb = fast_div(t0, a.d_T) * g.T;
      i0 = b;
    }
    const int row = page_row(g.pg, a.table + (long long)b * g.pg.max_pages, tb * n);
    if (row < 0) {
      if (report) set_status(a.status, HD_DEVBIT_INDEX);
      continue;
    }
    const int page = fast_div(row, g.pg.d_prow), off = row - page * g.pg.prow, block = fast_div(off, g.d_brow);
    const int cpr = Dh >> 4, chunks = (t1 - t0) * n * cpr;
    const size_t pitch = (size_t)g.Hkv * Dh;
    // (the same number of rounds for every team of a warp, whose lanes stay together)
    for (int first = (int)blockIdx.y * kTeams; first < 2 * g.Hkv; first += (int)gridDim.y * kTeams) {
      const int pair = first + (TEAM == 128 ? 0 : lane / TEAM);
      const bool mine = pair < 2 * g.Hkv, tensor = pair >= g.Hkv;
      const int h = mine ? pair - (tensor ? g.Hkv : 0) : 0, count = mine ? chunks : 0;
      uint8_t* codes = (tensor ? a.vc : a.kc) + (((size_t)page * g.Hkv + h) * g.pg.prow + off) * Dh;  // the block's rows
      uint8_t* scale = (tensor ? a.vs : a.ks) + scale_at(g, page, h, block);
      const uint16_t* rows = (tensor ? a.vn : a.kn) + (size_t)i0 * n * pitch + (size_t)h * Dh;
      auto at = [&](int c) {
        const int r = fast_div(c, a.d_cpr);
        return rows + r * pitch + (c - r * cpr) * 16;
      };
      const int had = mine && t0 > tb ? clamp_byte(*scale) : 0;
      Chunk held[kHeld];
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
        if (tid + k * TEAM < count) held[k] = load_chunk<TEAM == 128>(at(tid + k * TEAM));
      uint32_t most = 0;
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
        if (tid + k * TEAM < count) most = max(most, tame(held[k]));
      for (int c = tid + kHeld * TEAM; c < count; c += TEAM) {
        Chunk x = load_chunk<TEAM == 128>(at(c));
        most = max(most, tame(x));
      }
      if (TEAM >= 32) {
        most = __reduce_max_sync(0xffffffffu, most);
      } else {
#pragma unroll
        for (int d = TEAM / 2; d; d >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
      }
      if (TEAM == 128) {
        if (lane == 0) warp_most[threadIdx.x >> 5] = most;
        __syncthreads();
        most = max(max(warp_most[0], warp_most[1]), max(warp_most[2], warp_most[3]));
        __syncthreads();  // (also: every thread has read the block's old scale)
      }
      const int byte = max(scale_byte(most), had);
      const float inv = inverse_of(byte);
      uint4* to = reinterpret_cast<uint4*>(codes + (size_t)(t0 - tb) * n * Dh);
#pragma unroll
      for (int k = 0; k < kHeld; ++k)
        if (tid + k * TEAM < count) to[tid + k * TEAM] = codes_of(held[k], inv);
      for (int c = tid + kHeld * TEAM; c < count; c += TEAM) {
        Chunk x = load_chunk<TEAM == 128>(at(c));
        tame(x);
        to[c] = codes_of(x, inv);
      }
      if (mine && t0 > tb && byte > had) {
        const float f = scale_of(had - byte + 127);
        uint4* older = reinterpret_cast<uint4*>(codes);
        for (int c = tid; c < (t0 - tb) * n * cpr; c += TEAM) {
          const uint4 x = older[c];
          older[c] = make_uint4(recode4(x.x, f), recode4(x.y, f), recode4(x.z, f), recode4(x.w, f));
        }
      }
      if (TEAM < 128) __syncwarp();  // every lane has read the old scale
      if (mine && tid == 0) *scale = (uint8_t)byte;
    }
  }
}

struct ReadArgs {
  const uint8_t *kc, *vc, *ks, *vs;
  uint4 *kr, *vr;  // bf16 [N*n][Hkv][Dh]
  const int32_t *table, *lens, *offsets;
  int B, N, cap, pieces, chunks;  // 16-value chunks of a token, in pieces of kPiece
  Geom g;
  FastDiv d_cpr, d_Hkv;
  int32_t* status;
};
constexpr int kPiece = 128;

// Packed tokens out of the cache: a warp per token and piece (of its n * Hkv * Dh values, K's and V's), a lane's loads of 16
// codes ahead of its stores.  Bound by the latency of a warp's chain (search, page, loads, stores), with DRAM at 47 % and issue
// at 41 % under ncu (6 prompts of up to 4000 tokens, 4 streams, 8 heads of 128: 47.3 us, 5.2 TB/s; a warp that takes all of a
// token's pieces 53, pieces twice as large 57, stores of 32 bytes 50).
__global__ void __launch_bounds__(256) read_q8_kernel(ReadArgs a) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const bool report = blockIdx.y == 0;
  const Geom& g = a.g;
  const int cpr = g.Dh >> 4;
  const bool tensor = (int)blockIdx.y >= a.pieces;
  const int first = (tensor ? (int)blockIdx.y - a.pieces : (int)blockIdx.y) * kPiece;
  const uint4* pool = reinterpret_cast<const uint4*>(tensor ? a.vc : a.kc);
  const uint8_t* scales = tensor ? a.vs : a.ks;
  grid_dep_wait();
  grid_dep_launch();
  if (report && blockIdx.x == 0)
    for (int b = threadIdx.x; b < a.B; b += 256) {
      const int x = a.offsets[b], z = a.offsets[b + 1], L = a.lens[b];
      if (x < 0 || z < x || z > a.N || L < 0 || L > a.cap || z - x > L) set_status(a.status, HD_DEVBIT_INDEX);
    }
  for (long long w = (long long)blockIdx.x * 8 + warp; w < a.N; w += (long long)gridDim.x * 8) {
    const int b = last_not_above(a.B, w, lane, [&](int i) { return (long long)a.offsets[i]; });
    if (b < 0) continue;
    const int x = a.offsets[b], z = a.offsets[b + 1], L = a.lens[b];
    if (x < 0 || z <= w || z > a.N || L > a.cap || z - x > L) continue;
    const int t = L - z + (int)w;
    const int row = page_row(g.pg, a.table + (long long)b * g.pg.max_pages, t * g.n);
    if (row < 0) {
      if (report && lane == 0) set_status(a.status, HD_DEVBIT_INDEX);
      continue;
    }
    const int page = fast_div(row, g.pg.d_prow), off = row - page * g.pg.prow, block = fast_div(off, g.d_brow);
    uint4 code[kPiece / 32];
    int byte[kPiece / 32];
#pragma unroll
    for (int k = 0; k < kPiece / 32; ++k) {
      const int c = first + lane + k * 32;
      if (c < a.chunks) {
        const int sh = fast_div(c, a.d_cpr), s = fast_div(sh, a.d_Hkv), h = sh - s * g.Hkv;
        code[k] = pool[(((size_t)page * g.Hkv + h) * g.pg.prow + off + s) * cpr + c - sh * cpr];
        byte[k] = scales[scale_at(g, page, h, block)];
      }
    }
    uint4* to = (tensor ? a.vr : a.kr) + (size_t)w * a.chunks * 2;
#pragma unroll
    for (int k = 0; k < kPiece / 32; ++k) {
      const int c = first + lane + k * 32;
      if (c < a.chunks) {
        const float f = scale_of(clamp_byte(byte[k]));
        const uint32_t in[4] = {code[k].x, code[k].y, code[k].z, code[k].w};
        uint32_t r[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 v = values2((uint16_t)(in[i >> 1] >> (i & 1) * 16));
          r[i] = pack_bf16(v.x * f, v.y * f);  // exact
        }
        to[2 * c] = make_uint4(r[0], r[1], r[2], r[3]);
        to[2 * c + 1] = make_uint4(r[4], r[5], r[6], r[7]);
      }
    }
  }
}

// Pages and their scales copied within the pools: pair (a, b) is page a onto page b.  A warp takes 4 KB of codes at a
// time, or a page's scales; pairs of negative ids are left out.
__global__ void __launch_bounds__(256) copy_q8_kernel(uint4* kc, uint4* vc, uint8_t* ks, uint8_t* vs, const int2* copies,
                                                      long long units, int num_pages, size_t page16, int chunks,
                                                      int page_scales, int32_t* status) {
  const int lane = threadIdx.x & 31;
  grid_dep_wait();
  grid_dep_launch();
  for (long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += (long long)gridDim.x * 8) {
    const long long kv = u / (chunks + 1);  // pair * 2 + tensor
    const int c = (int)(u - kv * (chunks + 1));
    const int2 pr = copies[kv >> 1];
    if (pr.x < 0 && pr.y < 0) continue;
    if ((unsigned)pr.x >= (unsigned)num_pages || (unsigned)pr.y >= (unsigned)num_pages) {
      if (lane == 0) set_status(status, HD_DEVBIT_INDEX);
      continue;
    }
    if (c < chunks) {
      uint4* pool = (kv & 1) ? vc : kc;
      const size_t at = (size_t)c * 256;
      warp_copy(pool + pr.y * page16 + at, pool + pr.x * page16 + at, (int)min((size_t)256, page16 - at), lane);
    } else {
      uint8_t* s = (kv & 1) ? vs : ks;
      for (int i = lane; i < page_scales; i += 32) s[(size_t)pr.y * page_scales + i] = s[(size_t)pr.x * page_scales + i];
    }
  }
}
}  // namespace q8

// ------------------------------------------------------------------ host side

static q8::Geom q8_geom(int num_pages, int P, int max_pages, int n, int Hkv, int Dh, int T) {
  q8::Geom g;
  g.pg = make_page_geom(num_pages, max_pages, P * n);
  g.Hkv = Hkv;
  g.Dh = Dh;
  g.n = n;
  g.T = T;
  g.blocks = P / T;
  g.d_brow = make_fast_div((uint32_t)(T * n));
  return g;
}

cudaError_t launch_kv_append_paged_q8(const void* kn, const void* vn, void* kc, void* vc, uint8_t* ks, uint8_t* vs,
                                      const int32_t* table, const int32_t* lens, const int32_t* offsets,
                                      const int32_t* served, int B, int N, int num_pages, int P, int max_pages, int n,
                                      int Hkv, int Dh, int T, int32_t* status, cudaStream_t st) {
  q8::AppendArgs a = {};
  a.kn = (const uint16_t*)kn;
  a.vn = (const uint16_t*)vn;
  a.kc = (uint8_t*)kc;
  a.vc = (uint8_t*)vc;
  a.ks = ks;
  a.vs = vs;
  a.table = table;
  a.lens = lens;
  a.offsets = offsets;
  a.served = served;
  a.B = B;
  a.N = N;
  a.cap = max_pages * P;
  a.g = q8_geom(num_pages, P, max_pages, n, Hkv, Dh, T);
  a.d_T = make_fast_div((uint32_t)T);
  a.d_cpr = make_fast_div((uint32_t)(Dh / 16));
  a.status = status;
  a.units = offsets != nullptr ? (long long)N / T + 2ll * B : B;
  const long long values = (long long)(offsets != nullptr ? T : 1) * n * Dh;  // of a unit and pair, at most
  const int lanes = values <= 8 * 16 * q8::kHeld ? 8 : values <= 16 * 16 * q8::kHeld ? 16 : values <= 32 * 16 * q8::kHeld ? 32 : 128;
  // few units: their pairs are shared out, so that teams are a few for each place on the SMs (for CTAs 8 an SM take 62 us
  // where 24 take 42.7 and 96 take 41.5)
  const int rounds = lanes == 128 ? 2 * Hkv : (2 * Hkv * lanes + 31) / 32;
  const long long share = std::max(1LL, std::min<long long>(rounds, 24LL * kSmCount / a.units));
  if (lanes == 128)
    return launch_early(q8::append_q8_kernel<128>, dim3((unsigned)std::min<long long>(a.units, 1 << 20), (unsigned)share), 128, st, a);
  const dim3 grid((unsigned)std::min<long long>((a.units + 3) / 4, 1 << 20), (unsigned)share);
  return lanes == 8    ? launch_early(q8::append_q8_kernel<8>, grid, 128, st, a)
         : lanes == 16 ? launch_early(q8::append_q8_kernel<16>, grid, 128, st, a)
                       : launch_early(q8::append_q8_kernel<32>, grid, 128, st, a);
}

cudaError_t launch_kv_read_paged_q8(const void* kc, const void* vc, const uint8_t* ks, const uint8_t* vs,
                                    const int32_t* table, const int32_t* lens, const int32_t* offsets, void* k, void* v,
                                    int B, int N, int num_pages, int P, int max_pages, int n, int Hkv, int Dh, int T,
                                    int32_t* status, cudaStream_t st) {
  q8::ReadArgs a = {};
  a.kc = (const uint8_t*)kc;
  a.vc = (const uint8_t*)vc;
  a.ks = ks;
  a.vs = vs;
  a.kr = (uint4*)k;
  a.vr = (uint4*)v;
  a.table = table;
  a.lens = lens;
  a.offsets = offsets;
  a.B = B;
  a.N = N;
  a.cap = max_pages * P;
  a.chunks = n * Hkv * Dh / 16;
  a.pieces = (a.chunks + q8::kPiece - 1) / q8::kPiece;
  a.g = q8_geom(num_pages, P, max_pages, n, Hkv, Dh, T);
  a.d_cpr = make_fast_div((uint32_t)(Dh / 16));
  a.d_Hkv = make_fast_div((uint32_t)Hkv);
  a.status = status;
  const unsigned grid = (unsigned)std::min<long long>(((long long)N + 7) / 8, 64 * kSmCount);
  return launch_early(q8::read_q8_kernel, dim3(grid, 2 * a.pieces), 256, st, a);
}

cudaError_t launch_pages_copy_q8(void* kc, void* vc, uint8_t* ks, uint8_t* vs, const int32_t* copies, int F,
                                 int num_pages, size_t page_bytes, int page_scales, int32_t* status, cudaStream_t st) {
  const size_t page16 = page_bytes / 16;
  const int chunks = (int)((page16 + 255) / 256);
  const long long units = (long long)F * 2 * (chunks + 1);
  const unsigned grid = (unsigned)std::min<long long>((units + 7) / 8, 5 * kSmCount);
  return launch_early(q8::copy_q8_kernel, dim3(grid), 256, st, (uint4*)kc, (uint4*)vc, ks, vs, (const int2*)copies, units,
                      num_pages, page16, chunks, page_scales, status);
}

}  // namespace hdsfa
