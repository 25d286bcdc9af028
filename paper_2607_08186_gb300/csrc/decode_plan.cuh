// Host-side work split of the decoding step, shared by its kernels' file and the C ABI.
#pragma once
#include <stddef.h>

#include "common.cuh"

namespace hdsfa {

// Head dims at which the tcgen05 kernel may be taken.
enum class TcDims { kNone, k256, kWith128 };

struct DecodePlan {
  int G, M, ngroups, nsplit, rg;
  bool tc;  // the tcgen05 kernel: <= 128 query rows per K/V head at head dim 256 (128: see TcDims, and > 32)
  size_t part_o_bytes, part_ml_bytes;
};
DecodePlan decode_plan(int B, int maxT, int n, int Hq, int Hkv, int Dh, int mode, int window, TcDims tc_dims = TcDims::k256);
DecodePlan decode_plan_bound(int B, int maxT, int n, int Hq, int Hkv, int Dh, int mode, int window, TcDims tc_dims);
size_t decode_paged_ws_bytes(int B, int maxT, int n, int Hq, int Hkv, int Dh, int mode, int window);
size_t decode_ws_bytes(const DecodePlan& p);

// Rows of a piece of a page in a tile of at most `most` positions, the largest that no page boundary cuts: a
// page's rows, or their largest divisor that a tile holds.
inline int paged_piece(int prow, int most) {
  int d = prow < most ? prow : most;
  while (prow % d) --d;
  return d;
}

// Which kernel reads the pages, by query rows per K/V head and rows per piece of a page in a tile of 128.  The
// tensor-core kernel reads the cache once for up to 128 rows, but by TMA alone, which small pieces make slow
// (those of small pages, and of large ones without a divisor that a tile holds: of 262 rows come 2 at a time, with
// which 4 sequences of 8192 tokens, 2 streams, 24 over 2 heads of 256, take 118 us here and 42 there); the
// other one reads it once for each 32 rows, by cp.async where pieces are small.  Measured on pages of so many
// rows in us, tensor cores / the other (at head
// dim 256 4 sequences of 8192 tokens, 2 K/V heads; at 128 8 of 2048, 8 K/V heads; n streams):
//   <= 16 query rows   never    256: 16 rows a page 23.8 / 19.0 (n 1), 64: 51.6 / 48.6 (n 4), 128: 22.0 / 18.8 (n 1);
//                               only lengths of a quarter to all 58.3 / 65.4 (7 sequences, n 4)
//   <= 32, 256 only    from 12  8 rows a page 79 / 69, 9: 80 / 61, 10: 96 / 83, 12: 70.7 / 75.6, 16: 56.3 / 60.9
//   <= 64              from 5   256: 3 rows a page 130 / 105, 4: 126 / 125, 5: 136 / 158, 6: 81 / 101
//                               128: 3 rows a page 158 / 110, 4: 159 / 139, 5: 175 / 174, 6: 98 / 109, 8: 103 / 128, 64: 57 / 95
//   <= 128             from 4   256: 2 rows a page 72 / 58 (n 1), 3: 65 / 57 (n 1), 4: 45 / 57 (n 1)
//                               128: 3 rows a page 168 / 155 (n 3), 4: 55 / 69 (n 1), 164 / 191 (n 4)
// And it takes longer to start and end, one CTA per SM, so a range of few positions is the other one's (4
// streams, pages of 64 rows; B sequences of so many tokens):
//   128, > 32 rows   B 4: 50 tokens 13.7 / 11.6, 150: 14.5 / 16.3; B 16 (128 CTAs): 50: 27.6 / 14.8, 400: 41.6 /
//                    39.0, 1000: 64 / 79; B 64: 12: 97 / 41, 150: 122 / 81, 400: 164 / 145, 1000: 275 / 357
//   256, > 32 rows   B 4: 50: 13.1 / 10.6, 150: 13.2 / 12.9, 400: 13.8 / 15.5; B 33: 50: 22 / 20, 150: 28 / 34
//   256, <= 32 rows  B 4: 50: 12.9 / 10.0, 400: 13.9 / 14.4; B 33: 50: 19.3 / 18.2, 400: 35.2 / 36.7
inline TcDims paged_tc(int B, int n, int Hq, int Hkv, int Dh, int piece, long long range) {
  const int M = n * (Hq / Hkv);
  if (M <= 16) return TcDims::kNone;
  const int few = M <= 32 ? 1200 : Dh == 128 && (long long)B * Hkv > kSmCount / 4 ? 2000 : 400;
  if (range < few) return TcDims::kNone;
  if (M <= 32) return piece < 12 ? TcDims::kNone : TcDims::k256;
  return piece < (M <= 64 ? 5 : 4) ? TcDims::kNone : TcDims::kWith128;
}

// Positions that a step of maxT tokens over the 8-bit cache reads at most.
inline long long q8_range(int maxT, int n, int mode, int window) {
  const long long all = (long long)maxT * n, seen = (long long)window + n - 1;
  return mode == SFA_LOCAL && seen < all ? seen : all;
}

// Whether the tcgen05 kernel takes a step over the 8-bit cache.  It reads tiles by TMA alone, in pieces of at least
// kQ8TmaRows rows of a page that start on 128 bytes of shared memory, and takes longer to start and end, so up to 16 query
// rows leave it short ranges; at head dim 64, where a tile has half the bytes for the same softmax, all but a million
// positions over the heads.
// Measured (replayed from a graph, us, tcgen05 / mma.sync; sequences x tokens x streams):
//   16 over 4 of 64     4 x 400 x 3 11.2 / 9.3, 33 x 700 x 3 24.4 / 16.9, 2 x 8192 x 1 14.2 / 10.8, 4 x 6000 x 3 22.4 / 18.0, 8 x
//                       8192 x 3 34.5 / 32.4, 33 x 3000 x 3 (1.2 M positions over the heads) 45.6 / 46.3, 100 x 3000 x 3 98 / 122
//   32 over 8 of 128    33 x 12 x 4 11.6 / 9.4, 4 x 25 x 4 8.0 / 8.9, 33 x 25 x 4 11.3 / 10.6, 4 x 50 x 4 9.2 / 10.6, 4 x 1000 x 4
//                       17.0 / 18.4, 16 x 1000 x 4 28.0 / 40.4
//   24 over 2 of 256    33 x 20 x 1 10.0 / 8.9, 4 x 400 x 1 12.7 / 9.6, 4 x 1000 x 1 10.3 / 10.3, 33 x 1000 x 1 15.3 / 18.1
//   more than 16 rows   24 over 2 of 256, 4 x 50 x 4 13.8 / 22.0; 96 over 8 of 128, 16 x 50 x 4 12.5 / 14.2
constexpr int kQ8TmaRows = 8;
inline bool q8_tc(int Dh, int prow, int rows, long long range, long long heads) {
  const int piece = paged_piece(prow, 128);
  if (piece < kQ8TmaRows || (Dh == 64 && piece % 2 != 0)) return false;
  return rows > 16 || (Dh == 64 ? range * heads > 1 << 20 : range > (Dh == 128 ? 64 : 512));
}

// The parts that one wave of CTAs makes of a batch's `all` units (tiles and starts), the longest sequence of `most` units:
// at most `total` parts, none empty, and no sequence in more than max_split of them.  Part x begins at unit x * all / S.
struct WaveParts {
  unsigned all, S;
  __host__ __device__ WaveParts(unsigned all_, unsigned most, unsigned total, unsigned max_split) : all(all_) {
    S = total < all ? total : all;
    if (S < 1) S = 1;
    if ((unsigned long long)most * S > (max_split - 2ull) * all) S = (unsigned)((max_split - 2ull) * all / most);
  }
  // (S and x are hundreds at most)
  __host__ __device__ unsigned begin(unsigned x) const {
    const unsigned per = all / S;
    return x * per + x * (all - per * S) / S;
  }
  __host__ __device__ int of(unsigned u) const { return (int)(((u + 1ull) * S - 1) / all); }  // the part that holds unit u
};

}  // namespace hdsfa
