// 8-bit matrices (als_fp8): scales and conversion on the device, checks on the host.
#pragma once
#include "common.h"

namespace als {

// Both formats' largest value is 1.75 * 2^t, t = 8 (e4m3) and 15 (e5m2).  amax = m 2^k with 1 <= m < 2 is at most that value times 2^e from
// e = k - t on if m <= 1.75, from k - t + 1 on else: the scale's byte e + 127 comes from the bits of amax alone.  0 is a block without finite magnitudes.
__device__ __forceinline__ int fp8_scale_byte(unsigned u, int format) {   // u: bits of amax
  const int b = (int)(u >> 23) - (format == ALS_FP8_E4M3 ? 8 : 15) + ((u & 0x7fffff) > 0x600000);
  return u == 0 ? 127 : (b < 0 ? 0 : b);
}
// the scale as fp32 bits for the conversions below, which take the exponent alone: 2^-127 needs no other form
__device__ __forceinline__ float fp8_scale(int byte) { return __builtin_bit_cast(float, (unsigned)byte << 23); }
// the largest of 16 neighbouring lanes' (rows of the DPP operations), bits of numbers that are not negative
__device__ __forceinline__ unsigned lanes16_max(unsigned m) {
#define ALS_DPP_MAX(CTRL)                                                                                      \
  {                                                                                                            \
    const unsigned o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)m, CTRL, 0xf, 0xf, true);                 \
    m = m > o ? m : o;                                                                                         \
  }
  ALS_DPP_MAX(0xB1)    // lanes 1 0 3 2
  ALS_DPP_MAX(0x4E)    // lanes 2 3 0 1
  ALS_DPP_MAX(0x141)   // 8 lanes mirrored
  ALS_DPP_MAX(0x140)   // 16 lanes mirrored
#undef ALS_DPP_MAX
  return m;
}
// the largest of 32
__device__ __forceinline__ unsigned lanes32_max(unsigned m) {
  m = lanes16_max(m);
  auto a = __builtin_amdgcn_permlane16_swap(m, m, false, false);
  return a[0] > a[1] ? a[0] : a[1];
}
// bits of |v|, 0 for what is not finite
__device__ __forceinline__ unsigned fp8_magnitude(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}
// four values, divided by the scale, to four bytes
__device__ __forceinline__ unsigned fp8_pack4(float a, float b, float c, float d, float scale, int format) {
  typedef short s16x2 __attribute__((ext_vector_type(2)));
  s16x2 v = {0, 0};
  if (format == ALS_FP8_E4M3) {
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, a, b, scale, false);
    v = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(v, c, d, scale, true);
  } else {
    v = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(v, a, b, scale, false);
    v = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(v, c, d, scale, true);
  }
  return __builtin_bit_cast(unsigned, v);
}

// Non-temporal: what a pass over memory writes is no use in the caches that hold what it reads (quantiser of 16384 x 3584 bf16 in both
// orientations 55.5 to 51.5 us, norms 7 to 10 %; loads gain nothing).
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
// Four consecutive elements to p, at any address of their type; only the first n.
__device__ __forceinline__ void store4(float* p, int n, const float (&v)[4]) {
  if (n >= 4) {
    __builtin_nontemporal_store((f32x4_any){v[0], v[1], v[2], v[3]}, reinterpret_cast<f32x4_any*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (i < n) p[i] = v[i];
  }
}
__device__ __forceinline__ void store4(bf16* p, int n, const float (&v)[4]) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  if (n >= 4) {
    bf16x4 a;
#pragma unroll
    for (int i = 0; i < 4; i++) a[i] = (bf16)v[i];
    __builtin_nontemporal_store((u32x2_any)__builtin_bit_cast(u32x2, a), reinterpret_cast<u32x2_any*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (i < n) p[i] = (bf16)v[i];
  }
}
// four bytes to p, which is 4-byte aligned; only the first n of them
__device__ __forceinline__ void store4_bytes(uint8_t* p, int n, unsigned v) {
  if (n >= 4) {
    __builtin_nontemporal_store(v, reinterpret_cast<unsigned*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (i < n) p[i] = (uint8_t)(v >> (8 * i));
  }
}
// eight bytes to p, which is 8-byte aligned; only the first n of them
__device__ __forceinline__ void store8_bytes(uint8_t* p, int n, unsigned lo, unsigned hi) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  if (n >= 8) {
    __builtin_nontemporal_store((u32x2){lo, hi}, reinterpret_cast<u32x2*>(p));
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < n) p[i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
  }
}

inline int64_t fp8_blocks(int64_t cols) { return (cols + 127) / 128; }
// what als.h asks of a matrix in 8 bits; `what` names it in the error
inline int check_fp8(const als_fp8* f, int64_t rows, int64_t cols, const char* what) {
  if (f->format != ALS_FP8_E4M3 && f->format != ALS_FP8_E5M2) return set_error(ALS_ERR_INVALID, "%s: unknown 8-bit format %d", what, f->format);
  if (f->block_rows != 1 && f->block_rows != 128) return set_error(ALS_ERR_INVALID, "%s: block_rows must be 1 or 128", what);
  if (rows == 0 || cols == 0) return ALS_OK;
  if (!f->data || !f->scale) return set_error(ALS_ERR_INVALID, "%s: null data or scale", what);
  if (f->ld < cols || f->ld % 16 || f->ld_scale < fp8_blocks(cols) || f->ld_scale % 4)
    return set_error(ALS_ERR_INVALID, "%s: ld must be a multiple of 16 and at least %lld, ld_scale of 4 and at least %lld", what, (long long)cols, (long long)fp8_blocks(cols));
  if ((uintptr_t)f->data % 16 || (uintptr_t)f->scale % 4) return set_error(ALS_ERR_INVALID, "%s: data must be 16-byte aligned, scale 4-byte", what);
  return ALS_OK;
}
inline int check_dtype(int dtype, const char* what) {
  if (dtype != ALS_DTYPE_F32 && dtype != ALS_DTYPE_BF16) return set_error(ALS_ERR_INVALID, "%s: unknown dtype %d", what, dtype);
  return ALS_OK;
}

}  // namespace als
