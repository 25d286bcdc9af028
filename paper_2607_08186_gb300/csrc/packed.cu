// The list of query tiles of packed prompts.  One CTA: a few KB of work that starts while the kernel
// before it ends, and under which the attention kernel starts (about 4 us alone).
#include "packed.cuh"

namespace hdsfa {
namespace packed {
constexpr int NT = 1024;

// items: every sequence's tiles, by their number of key tiles, most first (a counting sort by the
// tile's number, capped where the window or the number of classes ends the growth), so that the long
// ones start first and the short ones fill the end.  The order within a class depends on the atomics
// and changes no result.  Offsets that descend or leave [0, N] make no items at all.
// Shared: neighbours of at most `most` = kShortRows rows share a tile where they start in the same run of tile_rows -
// kShortRows rows, so that their last one ends within tile_rows of the first one's start: a rule that
// every sequence can follow by itself.  At most 32 of them, which a warp's lanes hold.
__global__ void __launch_bounds__(NT) packed_plan_kernel(const int32_t* offsets, int B, int N, int mult, FastDiv d_tile, FastDiv d_run,
                                                         int tile_rows, int most, int top, PackedItem* items, int32_t* count,
                                                         int32_t* status) {
  __shared__ int place[NT], sums[32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  place[tid] = 0;
  grid_dep_wait();
  grid_dep_launch();
  bool bad = false;
  for (int b = tid; b < B; b += NT) bad = bad || offsets[b] < 0 || offsets[b + 1] < offsets[b] || offsets[b + 1] > N;
  if (__syncthreads_or(bad)) {
    if (tid == 0) {
      *count = 0;
      set_status(status, HD_DEVBIT_INDEX);
    }
    return;
  }
  // f(first row, rows, tile or -sequences, sequence) for every tile: a thread takes its sequences' first
  // tiles, its warp the rest
  auto for_tiles = [&](auto f) {
    constexpr int OWN = 8;
    for (int b0 = 0; b0 < B; b0 += NT) {
      const int b = b0 + tid;
      const int first = b < B ? offsets[b] * mult : 0, end = b < B ? offsets[b + 1] * mult : 0, own = end - first;
      // the short sequences of this warp that share a tile: the first of them takes it
      const int run = b < B && own <= most ? fast_div(first, d_run) : -1;
      const int left = __shfl_up_sync(0xffffffffu, run, 1);
      const unsigned heads = __ballot_sync(0xffffffffu, lane == 0 || run < 0 || left != run);
      const unsigned later = heads & (0xfffffffeu << lane);
      const int upto = later ? __ffs(later) - 1 : 32;
      const bool head = (heads >> lane) & 1u;
      const int seqs = head && upto - lane > 1 ? upto - lane : 0;
      const int shared_end = __shfl_sync(0xffffffffu, end, upto - 1);
      const int rows = !head ? 0 : seqs > 0 ? shared_end - first : own;
      const int tiles = fast_div(rows + tile_rows - 1, d_tile);
      if (seqs > 0) {
        if (rows > 0) f(first, rows, -seqs, b);
      } else {
        for (int t = 0; t < min(tiles, OWN); ++t) f(first, rows, t, b);
      }
      for (unsigned more = __ballot_sync(0xffffffffu, tiles > OWN); more; more &= more - 1) {
        const int l = __ffs(more) - 1, fl = __shfl_sync(0xffffffffu, first, l), rl = __shfl_sync(0xffffffffu, rows, l),
                  tl = __shfl_sync(0xffffffffu, tiles, l);
        for (int t = OWN + lane; t < tl; t += 32) f(fl, rl, t, 0);
      }
    }
  };
  auto place_of = [&](int tile) { return place + NT - 1 - min(max(tile, 0), top); };
  for_tiles([&](int, int, int t, int) { atomicAdd(place_of(t), 1); });
  __syncthreads();
  const int mine = place[tid];  // exclusive prefix sum over the classes
  int x = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, d);
    if (lane >= d) x += y;
  }
  if (lane == 31) sums[warp] = x;
  __syncthreads();
  int before = 0;
  for (int w = 0; w < warp; ++w) before += sums[w];
  place[tid] = before + x - mine;
  if (tid == NT - 1) *count = before + x;
  __syncthreads();
  for_tiles([&](int first, int rows, int t, int b) { items[atomicAdd(place_of(t), 1)] = PackedItem{first, rows, t, b}; });
}
}  // namespace packed

cudaError_t launch_packed_plan(const int32_t* offsets, int B, int N, int mult, int tile_rows, int window, bool shared,
                               PackedItem* items, int32_t* count, int32_t* status, cudaStream_t st) {
  const int top = window > 0 && window / tile_rows < packed::NT - 2 ? window / tile_rows + 1 : packed::NT - 1;
  return launch_early(packed::packed_plan_kernel, dim3(1), packed::NT, st, offsets, B, N, mult,
                      make_fast_div((uint32_t)tile_rows), make_fast_div((uint32_t)(tile_rows - kShortRows)), tile_rows,
                      shared ? kShortRows : -1, top, items, count, status);
}

}  // namespace hdsfa
