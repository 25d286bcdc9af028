// The 8-bit paged cache: where codes and scales lie and how values become codes, shared by the kernels that
// write, read and attend to it.
//
// A pool holds e4m3 codes [num_pages][Hkv][prow][Dh] (prow = P tokens x n streams): a page's rows of one head lie
// together, so that what one decoding CTA reads is whole runs of a page (prow * Dh bytes) and not rows of Dh bytes
// Hkv * Dh apart.  Each block of T tokens (brow = T * n rows) of a page and head has one scale, a power of two 2^e
// stored as the byte e + 127 in [num_pages][Hkv][P / T].  A code c stands for c * 2^e, which bf16 holds exactly.
//
// Powers of two lose nothing against other scales (e4m3 has its own exponent; a block's values span 17 binades before
// the smallest lose bits), and with them a block whose e grows is coded again without error but for values that
// become subnormal, and everything about a code is exact arithmetic in any precision.
#pragma once
#include <cuda_fp16.h>

#include "pages.cuh"

namespace hdsfa {
namespace q8 {

// e lies in [-64, 50].  Values below 2^-74 become 0, values above 448 * 2^50 (5e17) saturate.  Within these bounds
// the products of the decoding kernel stay in fp32's range whatever the blocks' scales are.
constexpr int kMinByte = 63, kMaxByte = 177;

// The byte of a block whose largest finite magnitude has these bf16 bits: the smallest e with value <= 448 * 2^e;
// value = 1.m * 2^(E - 127) and 448 = 1.75 * 2^8.
__host__ __device__ inline int scale_byte(uint32_t most) {
  const int b = (int)(most >> 7) - 8 + ((most & 0x7f) > 0x60 ? 1 : 0);
  return b < kMinByte ? kMinByte : b > kMaxByte ? kMaxByte : b;
}
__host__ __device__ inline int clamp_byte(int b) { return b < kMinByte ? kMinByte : b > kMaxByte ? kMaxByte : b; }
HD_DEVINLINE float scale_of(int byte) { return __int_as_float(byte << 23); }               // 2^e
HD_DEVINLINE float inverse_of(int byte) { return __int_as_float((254 - byte) << 23); }     // 2^-e

// Pool geometry.
struct Geom {
  PageGeom pg;
  int Hkv, Dh, n, T, blocks;  // T tokens a block, blocks of a page
  FastDiv d_brow;             // T * n rows
};

// Offset of a block's scale.
HD_DEVINLINE size_t scale_at(const Geom& g, int page, int h, int block) {
  return ((size_t)page * g.Hkv + h) * g.blocks + block;
}

// Two codes (lo, hi) of two values, to the nearest, ties to even; beyond 448 they saturate, NaN stays NaN.
HD_DEVINLINE uint32_t code2_sat(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;\n" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
// ... where infinities become NaN too (e4m3 has none).
HD_DEVINLINE uint32_t code2(float lo, float hi) {
  return code2_sat(fabsf(lo) <= 3.4e38f ? lo : NAN, fabsf(hi) <= 3.4e38f ? hi : NAN);
}
// The values of two codes, exactly.
HD_DEVINLINE uint32_t f16x2_of(uint16_t codes) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;\n" : "=r"(r) : "h"(codes));
  return r;
}
// ... of the four codes of a word.  (One asm statement: the conversions take the word's halves as they lie.)
HD_DEVINLINE void f16x4_of(uint32_t codes, uint32_t& lo, uint32_t& hi) {
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}\n"
      : "=r"(lo), "=r"(hi)
      : "r"(codes));
}
HD_DEVINLINE float2 values2(uint16_t codes) {
  const uint32_t r = f16x2_of(codes);
  return __half22float2(*reinterpret_cast<const __half2*>(&r));
}

}  // namespace q8
}  // namespace hdsfa
