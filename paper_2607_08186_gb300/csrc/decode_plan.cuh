// Host-side work split of the decoding step, shared by its kernels' file and the C ABI.
#pragma once
#include <stddef.h>

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

}  // namespace hdsfa
