// The 4-bit key/value cache (MXFP4): 32 consecutive values of one head's row
// share a power of two 2^e, stored as the byte e + 127 (255: the block holds a
// value that is not finite); each value is an E2M1 code, one of
// 0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign, two to a byte, the earlier one low.
//
// Layout: codes [pages, heads, page_size, 2, d / 2], scales [pages, heads,
// page_size, 2, d / 32]; index 2 is 0 for the key and 1 for the value. A
// slot's key and value lie side by side (128 bytes for d = 128, one cache
// line), so reading single slots wastes nothing; a head's page is contiguous.
//
// Why this format: gfx950 converts E2M1 with its scale in one instruction for
// two values, and E2M1 * 2^e is exact in bfloat16, so products formed from
// the decoded values carry no rounding beyond the cache's own.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lt {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

struct Cache4 {
  int64_t num_pages;
  int shift;  // log2 of the page size
  int hkv, d;
  // Row (slot, head) of codes and scales, in slots.
  __device__ __forceinline__ int64_t row(int64_t slot, int h) const {
    const int64_t page = slot >> shift;
    return ((page * hkv + h) << shift) + (slot & ((1 << shift) - 1));
  }
};

// Scale byte of a block whose largest magnitude has the bits `top`: the
// smallest e with top <= 7 * 2^e (7 rounds to 6, the largest code), not below
// -127 and not above 125, where 6 * 2^e is still finite. 7 * 2^e has the mantissa 0x600000, so adding 0x1FFFFF carries into the
// exponent exactly where e has to be one larger.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7F800000u) return 255u;
  const uint32_t e = (top + 0x1FFFFFu) >> 23;
  return e > 2u ? min(e - 2u, 252u) : 0u;
}

// Eight codes times the scale (its exponent field is what counts; 255 gives
// NaN). The conversion is exact.
__device__ __forceinline__ bf16x8_t decode8(uint32_t w, float s) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

}  // namespace lt
