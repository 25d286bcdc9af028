// The list of query tiles of packed prompts.  One CTA: it is a few KB of work that every layer of
// a batch repeats, under the start of the attention kernel (about 4 us alone).
#include "packed.cuh"

namespace hdsfa {
namespace packed {
constexpr int NT = 1024;

// Sequences by number of tiles, most first: one class each up to 511 tiles, then one for 512.
HD_DEVINLINE int size_class(int tiles) { return NT - 1 - (tiles < 512 ? tiles : min(NT - 1, 512 + (tiles >> 9))); }

// items: every sequence's tiles, its last (the most keys) first; classes in order of size, so that
// the longest work starts first and the shortest ends the launch.  Which sequence of a class comes
// first depends on the atomics and changes no result.  Offsets that descend or leave [0, N] make no
// items at all.
__global__ void __launch_bounds__(NT) packed_plan_kernel(const int32_t* offsets, int B, int N, int mult, FastDiv d_tile,
                                                         int tile_rows, PackedItem* items, int32_t* count,
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
  auto tiles_of = [&](int b) { return fast_div((offsets[b + 1] - offsets[b]) * mult + tile_rows - 1, d_tile); };
  for (int b = tid; b < B; b += NT) {
    const int t = tiles_of(b);
    if (t > 0) atomicAdd(place + size_class(t), t);
  }
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
  for (int b = warp; b < B; b += NT / 32) {
    const int t = tiles_of(b);
    if (t == 0) continue;
    int at = lane == 0 ? atomicAdd(place + size_class(t), t) : 0;
    at = __shfl_sync(0xffffffffu, at, 0);
    const int first = offsets[b] * mult, rows = (offsets[b + 1] - offsets[b]) * mult;
    for (int i = lane; i < t; i += 32) items[at + i] = PackedItem{first, rows, t - 1 - i, 0};
  }
}
}  // namespace packed

cudaError_t launch_packed_plan(const int32_t* offsets, int B, int N, int mult, int tile_rows, PackedItem* items,
                               int32_t* count, int32_t* status, cudaStream_t st) {
  return launch_early(packed::packed_plan_kernel, dim3(1), packed::NT, st, offsets, B, N, mult,
                      make_fast_div((uint32_t)tile_rows), tile_rows, items, count, status);
}

}  // namespace hdsfa
