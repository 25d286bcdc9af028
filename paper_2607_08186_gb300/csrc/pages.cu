// Pages of a K/V cache: who holds which page, copies of pages, and new rows into pages.
//
// State, all int32 in device memory of the caller: refs [num_pages] counts the sequences that
// hold a page (0: free), page_table [B][max_pages] lists a sequence's pages in order, lens [B]
// its tokens; a sequence of T tokens holds ceil(T / P) pages.  A page that two sequences share
// is full (hd_pages_fork copies the partly filled one), so a sequence that grow gave its pages appends to
// none that is shared.
// There is no list of free pages to keep: the lowest free ids are found by a scan of refs,
// which makes every result a function of the state alone.
//
// The bookkeeping is bound by latency (4 bytes a page and table entry), so it is few launches,
// each free to start under the one before it; the copies are bound by HBM.
#include <limits.h>

#include <algorithm>

#include "pages.cuh"

namespace hdsfa {
namespace pages {
constexpr int NT = 1024;

struct State {
  int32_t* refs;
  int32_t* table;
  int32_t* lens;
  int B, max_pages, num_pages, P, cap;  // cap: tokens a sequence's table has entries for
  FastDiv d_p;
  int32_t* status;
};

HD_DEVINLINE int pages_of(const State& s, int tokens) { return fast_div(tokens + s.P - 1, s.d_p); }

// Exclusive prefix sum of v over the CTA's NT threads; `total` is the sum.
HD_DEVINLINE int block_scan(int v, int* sh, int& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) sh[warp] = x;
  __syncthreads();
  if (warp == 0) {
    int t = sh[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, t, d);
      if (lane >= d) t += y;
    }
    sh[lane] = t;
  }
  __syncthreads();
  total = sh[31];
  const int before = warp > 0 ? sh[warp - 1] : 0;
  __syncthreads();  // sh may be written again
  return before + x - v;
}

// Counts of pages id .. id + 3 (id a multiple of 4); `none` for those behind the pool.
HD_DEVINLINE void load_refs(const int32_t* refs, int num_pages, int id, int none, int* r) {
  if (id + 3 < num_pages) {
    const int4 q = *reinterpret_cast<const int4*>(refs + id);
    r[0] = q.x, r[1] = q.y, r[2] = q.z, r[3] = q.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = id + e < num_pages ? refs[id + e] : none;
  }
}

// The free pages' ids, ascending, into list[0, want), as far as there are as many; returns how
// many were written.
HD_DEVINLINE int list_free(const State& s, int want, int32_t* list, int* sh) {
  int found = 0;
  for (int p0 = 0; p0 < s.num_pages && found < want; p0 += 4 * NT) {
    const int id = p0 + 4 * (int)threadIdx.x;
    int r[4];
    load_refs(s.refs, s.num_pages, id, 1, r);
    int total;
    int at = found + block_scan((r[0] == 0) + (r[1] == 0) + (r[2] == 0) + (r[3] == 0), sh, total);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (r[e] == 0) {
        if (at < want) list[at] = id + e;
        ++at;
      }
    found += total;
  }
  __syncthreads();
  return min(found, want);
}

// Pages for add[b] more tokens of each sequence: ids ascending, sequences ascending.  served (or null): the
// tokens that each got.
__global__ void __launch_bounds__(NT) grow_kernel(State s, const int32_t* add, int32_t* served, int32_t* base,
                                                  int32_t* list) {
  __shared__ int sh[32];
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto need_of = [&](int T, int x) {
    return T < 0 || T > s.cap || x < 0 || x > s.cap - T ? -1 : pages_of(s, T + x) - pages_of(s, T);
  };
  int total = 0;
  for (int b0 = 0; b0 < s.B; b0 += NT) {
    const int b = b0 + (int)threadIdx.x;
    const int need = b < s.B ? need_of(s.lens[b], add[b]) : 0;
    if (need < 0) set_status(s.status, HD_DEVBIT_INDEX);
    int sum;
    const int at = total + block_scan(max(need, 0), sh, sum);
    if (b < s.B) base[b] = at;
    total += sum;
  }
  const int avail = list_free(s, total, list, sh);  // its barrier also orders base
  for (int b = warp; b < s.B; b += NT / 32) {
    const int T = s.lens[b], x = add[b], need = need_of(T, x), at = base[b];
    const bool none = need > 0 && at + need > avail;
    if (lane == 0 && served != nullptr) served[b] = need < 0 || none ? 0 : x;
    if (need < 0 || x == 0) continue;
    if (none) {
      if (lane == 0) set_status(s.status, HD_DEVBIT_PAGES);
      continue;
    }
    int32_t* row = s.table + (long long)b * s.max_pages + pages_of(s, T);
    for (int i = lane; i < need; i += 32) {
      const int id = list[at + i];
      row[i] = id;
      s.refs[id] = 1;
    }
    __syncwarp();
    if (lane == 0) s.lens[b] = T + x;
  }
}

// Each fork: the full pages of the prefix shared, the partly filled one new and listed for a copy.
// claim [B]: the first fork that names a destination; tok [F]: its tokens, -1 if refused.
//
// One CTA, a warp per fork: bound by the latency of the entries' loads and their refs', so a lane keeps
// kForkLoads of each in flight.  One at a time 64 forks of 512 pages took 31.4 us and of 2000 pages 103
// us; so 25.2 and 72.3 (16 of 512 pages 17.1 -> 12.9, 4 of 64 pages 8.9 -> 8.8).
constexpr int kForkLoads = 8;
__global__ void __launch_bounds__(NT) fork_kernel(State s, const int32_t* src, const int32_t* dst, const int32_t* tokens,
                                                  int F, int2* copies, int32_t* claim, int32_t* tok, int32_t* base,
                                                  int32_t* list) {
  __shared__ int sh[32];
  grid_dep_wait();
  grid_dep_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int i = threadIdx.x; i < F; i += NT)
    if ((unsigned)dst[i] < (unsigned)s.B) claim[dst[i]] = INT_MAX;
  __syncthreads();
  for (int i = threadIdx.x; i < F; i += NT)
    if ((unsigned)dst[i] < (unsigned)s.B) atomicMin(claim + dst[i], i);
  __syncthreads();
  for (int i = warp; i < F; i += NT / 32) {
    const int a = src[i], b = dst[i];
    bool ok = (unsigned)a < (unsigned)s.B && (unsigned)b < (unsigned)s.B && a != b;
    int t = 0;
    if (ok) {
      const int T = s.lens[a];
      t = tokens != nullptr ? tokens[i] : T;
      ok = T >= 0 && T <= s.cap && t >= 0 && t <= T && s.lens[b] == 0 && claim[b] == i;
    }
    const int held = ok ? pages_of(s, t) : 0;
    const int32_t* row = s.table + (long long)(ok ? a : 0) * s.max_pages;
    for (int j0 = lane; j0 < held; j0 += 32 * kForkLoads) {
      int id[kForkLoads], r[kForkLoads];
#pragma unroll
      for (int u = 0; u < kForkLoads; ++u) id[u] = j0 + 32 * u < held ? row[j0 + 32 * u] : row[j0];
#pragma unroll
      for (int u = 0; u < kForkLoads; ++u) r[u] = (unsigned)id[u] < (unsigned)s.num_pages ? s.refs[id[u]] : 0;
#pragma unroll
      for (int u = 0; u < kForkLoads; ++u) ok = ok && r[u] > 0;
    }
    ok = __all_sync(0xffffffffu, ok);
    if (lane == 0) {
      tok[i] = ok ? t : -1;
      if (!ok) set_status(s.status, HD_DEVBIT_INDEX);
    }
  }
  __syncthreads();
  int total = 0;
  for (int i0 = 0; i0 < F; i0 += NT) {
    const int i = i0 + (int)threadIdx.x;
    const int t = i < F ? tok[i] : 0;
    int sum;
    const int at = total + block_scan(t > 0 && pages_of(s, t) * s.P != t, sh, sum);
    if (i < F) base[i] = at;
    total += sum;
  }
  const int avail = list_free(s, total, list, sh);
  for (int i = warp; i < F; i += NT / 32) {
    const int t = tok[i];
    const int full = t > 0 ? fast_div(t, s.d_p) : 0;
    const bool part = t > 0 && full * s.P != t;
    int2 pair = make_int2(-1, -1);
    if (t > 0 && part && base[i] >= avail) {
      if (lane == 0) set_status(s.status, HD_DEVBIT_PAGES);
    } else if (t > 0) {
      const int32_t* from = s.table + (long long)src[i] * s.max_pages;
      int32_t* to = s.table + (long long)dst[i] * s.max_pages;
      for (int j0 = lane; j0 < full; j0 += 32 * kForkLoads) {
        int id[kForkLoads];
#pragma unroll
        for (int u = 0; u < kForkLoads; ++u) id[u] = j0 + 32 * u < full ? from[j0 + 32 * u] : -1;
#pragma unroll
        for (int u = 0; u < kForkLoads; ++u)
          if (id[u] >= 0) {
            to[j0 + 32 * u] = id[u];
            atomicAdd(s.refs + id[u], 1);
          }
      }
      if (lane == 0) {
        if (part) {
          pair = make_int2(from[full], list[base[i]]);
          to[full] = pair.y;
          s.refs[pair.y] = 1;
        }
        s.lens[dst[i]] = t;
      }
    }
    if (lane == 0) copies[i] = pair;
  }
}

// One CTA per entry of seqs.  The sequence is taken by exchanging its length, so an entry that
// comes twice frees nothing the second time.
__global__ void __launch_bounds__(256) free_kernel(State s, const int32_t* seqs) {
  __shared__ int taken;
  grid_dep_wait();
  grid_dep_launch();
  const int b = seqs[blockIdx.x];
  if ((unsigned)b >= (unsigned)s.B) {
    if (threadIdx.x == 0) set_status(s.status, HD_DEVBIT_INDEX);
    return;
  }
  if (threadIdx.x == 0) taken = atomicExch(s.lens + b, 0);
  __syncthreads();
  const int T = taken;
  if (T < 0 || T > s.cap) {
    if (threadIdx.x == 0) set_status(s.status, HD_DEVBIT_INDEX);
    return;
  }
  int32_t* row = s.table + (long long)b * s.max_pages;
  for (int i = threadIdx.x; i < pages_of(s, T); i += 256) {
    const int id = row[i];
    row[i] = -1;
    bool ok = (unsigned)id < (unsigned)s.num_pages;
    if (ok && atomicSub(s.refs + id, 1) <= 0) {  // a free page in a table: its count stays
      atomicAdd(s.refs + id, 1);
      ok = false;
    }
    if (!ok) set_status(s.status, HD_DEVBIT_INDEX);
  }
}

// Compaction, first part: with K pages live, the j-th live page with an id >= K moves to the
// j-th free id below K.  low, high: these ids; map: every live page's new id, -1
// for the others; count: K, moves.
__global__ void __launch_bounds__(NT) compact_plan_kernel(const int32_t* refs, int num_pages, int32_t* low,
                                                          int32_t* high, int32_t* map, int32_t* count) {
  __shared__ int sh[32];
  grid_dep_wait();
  grid_dep_launch();
  int live = 0;
  for (int p0 = 0; p0 < num_pages; p0 += 4 * NT) {
    int r[4];
    load_refs(refs, num_pages, p0 + 4 * (int)threadIdx.x, 0, r);
    live += (r[0] > 0) + (r[1] > 0) + (r[2] > 0) + (r[3] > 0);
  }
  int K;
  block_scan(live, sh, K);
  int nlow = 0, nhigh = 0;
  for (int p0 = 0; p0 < num_pages; p0 += 4 * NT) {
    const int p = p0 + 4 * (int)threadIdx.x;
    int r[4], both = 0;
    load_refs(refs, num_pages, p, 0, r);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (p + e < num_pages) both += r[e] > 0 ? (int)(p + e >= K) << 16 : (int)(p + e < K);
    int sum;  // a chunk's two counts in one scan, 16 bits each (at most 4 * NT of both)
    const int at = block_scan(both, sh, sum);
    int lo = nlow + (at & 0xffff), hi = nhigh + (at >> 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (p + e >= num_pages) continue;
      const bool on = r[e] > 0;
      if (on && p + e >= K) {
        high[hi++] = p + e;
      } else {
        map[p + e] = on ? p + e : -1;
        if (!on && p + e < K) low[lo++] = p + e;
      }
    }
    nlow += sum & 0xffff;
    nhigh += sum >> 16;
  }
  __syncthreads();
  for (int j = threadIdx.x; j < nhigh; j += NT) map[high[j]] = low[j];  // nlow == nhigh
  if (threadIdx.x == 0) {
    count[0] = K;
    count[1] = nhigh;
  }
}

// Second part: counts, tables and the list of moves.  Each element is read and written by one
// thread, so the new arrays may be the old ones.
__global__ void __launch_bounds__(256) compact_apply_kernel(State s, int32_t* new_refs, int32_t* new_table, int2* moves,
                                                            int max_moves, const int32_t* low, const int32_t* high,
                                                            const int32_t* map, const int32_t* count) {
  const long long step = (long long)gridDim.x * 256, first = (long long)blockIdx.x * 256 + threadIdx.x;
  grid_dep_wait();
  grid_dep_launch();
  const int K = count[0], nmoves = count[1];
  for (long long j = first; j < max_moves; j += step) {
    int2 mv = make_int2(-1, -1);
    if (j < nmoves) {
      mv = make_int2(high[j], low[j]);
      const int r = s.refs[mv.x];
      new_refs[mv.y] = r;
      new_refs[mv.x] = 0;
    }
    moves[j] = mv;
  }
  for (long long p = first; p < s.num_pages; p += step) {  // the pages that no move names
    const int to = map[p];
    if (to == p) new_refs[p] = s.refs[p];
    else if (to < 0 && p >= K) new_refs[p] = 0;
  }
  for (long long e = first; e < (long long)s.B * s.max_pages; e += step) {
    const int b = (int)(e / s.max_pages), i = (int)(e - (long long)b * s.max_pages);
    const int T = s.lens[b];
    const bool sane = T >= 0 && T <= s.cap;
    int id = -1;
    if (sane && i < pages_of(s, T)) {
      const int old = s.table[e];
      if ((unsigned)old < (unsigned)s.num_pages) id = map[old];
      if (id < 0) set_status(s.status, HD_DEVBIT_INDEX);  // no page, or by its count a free one
    } else if (!sane && i == 0) {
      set_status(s.status, HD_DEVBIT_INDEX);
    }
    new_table[e] = id;
  }
}

// Pages copied within both pools: pair (a, b) is page a onto page b.  A warp takes 4 KB of a page
// at a time; pairs of negative ids are left out.
__global__ void __launch_bounds__(256, 5) copy_kernel(uint4* kp, uint4* vp, const int2* copies, long long units,
                                                      int num_pages, int page16, int chunks, int32_t* status) {
  const int lane = threadIdx.x & 31;
  const long long step = (long long)gridDim.x * 8;
  grid_dep_wait();
  grid_dep_launch();
  for (long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += step) {
    const long long kv = u / chunks;  // pair * 2 + tensor
    const int c = (int)(u - kv * chunks);
    const int2 pr = copies[kv >> 1];
    if (pr.x < 0 && pr.y < 0) continue;
    if ((unsigned)pr.x >= (unsigned)num_pages || (unsigned)pr.y >= (unsigned)num_pages) {
      if (lane == 0) set_status(status, HD_DEVBIT_INDEX);
      continue;
    }
    uint4* pool = (kv & 1) ? vp : kp;
    warp_copy(pool + (long long)pr.y * page16 + c * 256, pool + (long long)pr.x * page16 + c * 256,
              min(256, page16 - c * 256), lane);
  }
}

// The sequence of packed token w: the largest b with offsets[b] <= w, found by a warp with one
// load for each 5 bits of B; -1 if there is none.
HD_DEVINLINE int find_sequence(const int32_t* offsets, int B, int w, int lane) {
  int lo = 0, n = B;
  while (true) {
    const int step = (n + 31) / 32, i = lane * step;
    const unsigned le = __ballot_sync(0xffffffffu, i < n && offsets[lo + i] <= w);
    if (le == 0) return -1;
    const int l = 31 - __clz(le);
    lo += l * step;
    if (step == 1) return lo;
    n = min(step, n - l * step);
  }
}

// New tokens' K and V rows (blockIdx.y: tensor, 4 KB piece) into pages: a warp per token, whose n
// rows lie together on both sides.  Without offsets token b is sequence b's one new token; with
// them sequence b's are the packed tokens offsets[b] .. offsets[b + 1].  served (or null): the tokens that
// grow gave each sequence; one that got fewer than it brings is left out, since its last tokens' rows are
// others', in a page that it may share.
__global__ void __launch_bounds__(256, 5) append_paged_kernel(const uint4* kn, const uint4* vn, uint4* kp, uint4* vp,
                                                              const int32_t* page_table, const int32_t* lens,
                                                              const int32_t* offsets, const int32_t* served, int B,
                                                              int N, int n, int cap, PageGeom g, int tok16, int chunks, int32_t* status) {
  const int lane = threadIdx.x & 31;
  const bool first = blockIdx.y == 0;  // reports errors
  const int piece = (int)blockIdx.y % chunks * 256;
  const uint4* src = (int)blockIdx.y < chunks ? kn : vn;
  uint4* pool = (int)blockIdx.y < chunks ? kp : vp;
  grid_dep_wait();  // an earlier step may still read the cache, or write what is read here
  grid_dep_launch();
  if (offsets != nullptr && blockIdx.x == 0 && first)
    for (int b = threadIdx.x; b < B; b += 256) {
      const int a = offsets[b], z = offsets[b + 1], T = lens[b];
      bool bad = a < 0 || z < a || z > N || T < 0 || T > cap;
      if (!bad) bad = z - a > T && (served == nullptr || served[b] >= z - a);
      if (bad) set_status(status, HD_DEVBIT_INDEX);
    }
  for (long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); w < N; w += (long long)gridDim.x * 8) {
    int b = (int)w, t;
    if (offsets != nullptr) {
      b = find_sequence(offsets, B, (int)w, lane);
      if (b < 0) continue;
      const int a = offsets[b], z = offsets[b + 1], T = lens[b];
      if (a < 0 || z <= w || z > N || T > cap || z - a > T) continue;
      if (served != nullptr && served[b] < z - a) continue;
      t = T - z + (int)w;
    } else {
      const int T = lens[b];
      if (T < 0 || T > cap) {
        if (lane == 0 && first) set_status(status, HD_DEVBIT_INDEX);
        continue;
      }
      t = T - 1;
      if (t < 0 || (served != nullptr && served[b] < 1)) continue;  // an idle slot, or one that grow refused
    }
    const int row = page_row(g, page_table + (long long)b * g.max_pages, t * n);
    if (row < 0) {
      if (lane == 0 && first) set_status(status, HD_DEVBIT_INDEX);
      continue;
    }
    warp_copy(pool + (long long)(row / n) * tok16 + piece, src + w * tok16 + piece, min(256, tok16 - piece), lane);
  }
}
}  // namespace pages

// ------------------------------------------------------------------ host side

static pages::State page_state(int32_t* refs, int32_t* table, int32_t* lens, int B, int max_pages, int num_pages, int P,
                               int32_t* status) {
  pages::State s;
  s.refs = refs;
  s.table = table;
  s.lens = lens;
  s.B = B;
  s.max_pages = max_pages;
  s.num_pages = num_pages;
  s.P = P;
  s.cap = max_pages * P;
  s.d_p = make_fast_div((uint32_t)P);
  s.status = status;
  return s;
}

// Workspace, in int32: three arrays of B (fork's claim, tok; a prefix sum), three of num_pages
// (free or low ids, high ids, the map), two counts.
size_t pages_ws_bytes(int B, int num_pages) { return ((size_t)3 * B + (size_t)3 * num_pages + 2) * sizeof(int32_t); }

cudaError_t launch_pages_grow(int32_t* refs, int32_t* table, int32_t* lens, const int32_t* add, int32_t* served, int B,
                              int max_pages, int num_pages, int P, void* ws, int32_t* status, cudaStream_t st) {
  const pages::State s = page_state(refs, table, lens, B, max_pages, num_pages, P, status);
  int32_t* w = static_cast<int32_t*>(ws);
  return launch_early(pages::grow_kernel, dim3(1), pages::NT, st, s, add, served, w, w + (size_t)3 * B);
}

cudaError_t launch_pages_fork(int32_t* refs, int32_t* table, int32_t* lens, const int32_t* src, const int32_t* dst,
                              const int32_t* tokens, int F, int32_t* copies, int B, int max_pages, int num_pages, int P,
                              void* ws, int32_t* status, cudaStream_t st) {
  const pages::State s = page_state(refs, table, lens, B, max_pages, num_pages, P, status);
  int32_t* w = static_cast<int32_t*>(ws);
  return launch_early(pages::fork_kernel, dim3(1), pages::NT, st, s, src, dst, tokens, F, (int2*)copies, w, w + B,
                      w + (size_t)2 * B, w + (size_t)3 * B);
}

cudaError_t launch_pages_free(int32_t* refs, int32_t* table, int32_t* lens, const int32_t* seqs, int F, int B,
                              int max_pages, int num_pages, int P, int32_t* status, cudaStream_t st) {
  const pages::State s = page_state(refs, table, lens, B, max_pages, num_pages, P, status);
  return launch_early(pages::free_kernel, dim3((unsigned)F), 256, st, s, seqs);
}

cudaError_t launch_pages_compact(const int32_t* refs, const int32_t* table, const int32_t* lens, int32_t* new_refs,
                                 int32_t* new_table, int32_t* moves, int B, int max_pages, int num_pages, int P,
                                 void* ws, int32_t* status, cudaStream_t st) {
  const pages::State s = page_state(const_cast<int32_t*>(refs), const_cast<int32_t*>(table), const_cast<int32_t*>(lens), B,
                                    max_pages, num_pages, P, status);
  int32_t *low = static_cast<int32_t*>(ws) + (size_t)3 * B, *high = low + num_pages, *map = high + num_pages,
          *count = map + num_pages;
  cudaError_t e = launch_early(pages::compact_plan_kernel, dim3(1), pages::NT, st, refs, num_pages, low, high, map, count);
  if (e != cudaSuccess) return e;
  const long long most = std::max<long long>((long long)B * max_pages, num_pages);
  const unsigned grid = (unsigned)std::min<long long>((most + 255) / 256, 4 * kSmCount);
  return launch_early(pages::compact_apply_kernel, dim3(grid), 256, st, s, new_refs, new_table, (int2*)moves,
                      num_pages / 2, low, high, map, count);
}

cudaError_t launch_pages_copy(void* kp, void* vp, const int32_t* copies, int F, int num_pages, int page16,
                              int32_t* status, cudaStream_t st) {
  const int chunks = (page16 + 255) / 256;
  const long long units = (long long)F * 2 * chunks;
  const unsigned grid = (unsigned)std::min<long long>((units + 7) / 8, 5 * kSmCount);
  return launch_early(pages::copy_kernel, dim3(grid), 256, st, (uint4*)kp, (uint4*)vp, (const int2*)copies, units,
                      num_pages, page16, chunks, status);
}

cudaError_t launch_kv_append_paged(const void* kn, const void* vn, void* kp, void* vp, const int32_t* table,
                                   const int32_t* lens, const int32_t* offsets, const int32_t* served, int B, int N,
                                   int num_pages, int P, int max_pages, int n, int Hkv, int Dh, int32_t* status,
                                   cudaStream_t st) {
  const int tok16 = n * Hkv * Dh / 8, chunks = (tok16 + 255) / 256;
  const PageGeom g = make_page_geom(num_pages, max_pages, P * n);
  const unsigned grid = (unsigned)std::min<long long>(((long long)N + 7) / 8, 64 * kSmCount);
  return launch_early(pages::append_paged_kernel, dim3(grid, 2 * chunks), 256, st, (const uint4*)kn, (const uint4*)vn,
                      (uint4*)kp, (uint4*)vp, table, lens, offsets, served, B, N, n, max_pages * P, g, tok16, chunks, status);
}

}  // namespace hdsfa
