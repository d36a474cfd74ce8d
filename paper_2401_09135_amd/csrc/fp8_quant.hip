// A matrix to 8 bits with a power-of-two scale for each block (als_k_quant_fp8): as it is, transposed, or both from one reading.
//
// Memory bounds it: 4 or 2 bytes read and 1 written for each orientation and element.  A workgroup of 256 threads owns a tile of 128 x 128, whole blocks of
// both orientations; a thread has 8 rows of 8 columns of it in registers, so that a row's largest magnitude is 16 neighbouring lanes' and the bytes of
// a thread are 8 in a row of either orientation.  The transposed bytes go through LDS (16 KB) to be written as whole rows of 128.
#include "fp8.h"

namespace als {

namespace {

struct Fp8Out { uint8_t* data; uint8_t* scale; int64_t ld, ld_scale; int format, block_rows; };

__device__ __forceinline__ float lanes16_max(float v) {
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

template <typename T, bool VEC, bool Q, bool QT>
__global__ __launch_bounds__(256) void quant_fp8_kernel(const T* __restrict__ x, int rows, int cols, int64_t ldx, Fp8Out q, Fp8Out qt, int tiles_c) {
  __shared__ float cmax[QT ? 4 : 1][QT ? 128 : 1];
  __shared__ float wmax[4];
  __shared__ __attribute__((aligned(16))) uint8_t tile[QT ? 128 * 128 : 16];
  const int tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
  const int row0 = tr * 128, col0 = tc * 128;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
  const int c = col0 + 8 * cx, r0 = row0 + 8 * ry;
  const int left = cols - c;   // columns of this thread that exist, if below 8
  float v[8][8];
#pragma unroll
  for (int i = 0; i < 8; i++) load8<VEC>(x + (int64_t)(r0 + i) * ldx + c, r0 + i < rows ? left : 0, v[i]);

  const bool whole = (Q && q.block_rows == 128) || (QT && qt.block_rows == 128);   // a block is the tile
  float amax_tile = 0.0f;
  if (whole) {
#pragma unroll
    for (int i = 0; i < 8; i++)
#pragma unroll
      for (int j = 0; j < 8; j++) amax_tile = fmaxf(amax_tile, fp8_magnitude(v[i][j]));
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) amax_tile = fmaxf(amax_tile, __shfl_xor(amax_tile, o, 64));
    if (lane == 0) wmax[wave] = amax_tile;
  }
  if (QT && qt.block_rows == 1) {
#pragma unroll
    for (int j = 0; j < 8; j++) {
      float m = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; i++) m = fmaxf(m, fp8_magnitude(v[i][j]));
      m = fmaxf(m, __shfl_xor(m, 16, 64));
      m = fmaxf(m, __shfl_xor(m, 32, 64));
      if (lane < 16) cmax[wave][8 * cx + j] = m;
    }
  }
  if (whole || QT) __syncthreads();
  if (whole) amax_tile = fmaxf(fmaxf(wmax[0], wmax[1]), fmaxf(wmax[2], wmax[3]));

  if (Q) {
    const int bt = q.block_rows == 128 ? fp8_scale_byte(amax_tile, q.format) : 0;
    if (q.block_rows == 128 && threadIdx.x == 0) q.scale[(int64_t)tr * q.ld_scale + tc] = (uint8_t)bt;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      int b = bt;
      if (q.block_rows == 1) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; j++) m = fmaxf(m, fp8_magnitude(v[i][j]));
        b = fp8_scale_byte(lanes16_max(m), q.format);
        if (cx == 0 && r0 + i < rows) q.scale[(int64_t)(r0 + i) * q.ld_scale + tc] = (uint8_t)b;
      }
      const float s = fp8_inv_scale(b);
      const unsigned lo = fp8_pack4(v[i][0] * s, v[i][1] * s, v[i][2] * s, v[i][3] * s, q.format);
      const unsigned hi = fp8_pack4(v[i][4] * s, v[i][5] * s, v[i][6] * s, v[i][7] * s, q.format);
      if (r0 + i < rows && left > 0) store8_bytes(q.data + (int64_t)(r0 + i) * q.ld + c, left, lo, hi);
    }
  }
  if (QT) {
    const int bt = qt.block_rows == 128 ? fp8_scale_byte(amax_tile, qt.format) : 0;
    if (qt.block_rows == 128 && threadIdx.x == 0) qt.scale[(int64_t)tc * qt.ld_scale + tr] = (uint8_t)bt;
    // column 8 cx + j of the tile is row 8 cx + j of 128 bytes in LDS; its 8-byte piece ry lies at piece ry ^ cx, so that 16 columns' pieces
    // fall into 16 different pairs of banks
#pragma unroll
    for (int j = 0; j < 8; j++) {
      int b = bt;
      if (qt.block_rows == 1) {
        const int cc = 8 * cx + j;
        b = fp8_scale_byte(fmaxf(fmaxf(cmax[0][cc], cmax[1][cc]), fmaxf(cmax[2][cc], cmax[3][cc])), qt.format);
        if (ry == 0 && j < left) qt.scale[(int64_t)(c + j) * qt.ld_scale + tr] = (uint8_t)b;
      }
      const float s = fp8_inv_scale(b);
      const unsigned lo = fp8_pack4(v[0][j] * s, v[1][j] * s, v[2][j] * s, v[3][j] * s, qt.format);
      const unsigned hi = fp8_pack4(v[4][j] * s, v[5][j] * s, v[6][j] * s, v[7][j] * s, qt.format);
      *reinterpret_cast<uint2*>(tile + (8 * cx + j) * 128 + (ry ^ cx) * 8) = make_uint2(lo, hi);
    }
    __syncthreads();
#pragma unroll
    for (int p = 0; p < 4; p++) {
      const int cc = p * 32 + (threadIdx.x >> 3), k = threadIdx.x & 7, sw = cc >> 3;   // sw: the cx that wrote it
      uint4 d = *reinterpret_cast<const uint4*>(tile + cc * 128 + (k ^ (sw >> 1)) * 16);
      if (sw & 1) d = make_uint4(d.z, d.w, d.x, d.y);
      const int r = row0 + 16 * k;
      if (col0 + cc < cols && r < rows) {
        uint8_t* o = qt.data + (int64_t)(col0 + cc) * qt.ld + r;
        if (rows - r >= 16) {
          *reinterpret_cast<uint4*>(o) = d;
        } else {
          store8_bytes(o, rows - r, d.x, d.y);
          if (rows - r > 8) store8_bytes(o + 8, rows - r - 8, d.z, d.w);
        }
      }
    }
  }
}

template <typename T>
int launch_quant(const T* x, int rows, int cols, int64_t ldx, const als_fp8* q, const als_fp8* qt, hipStream_t st) {
  auto out = [](const als_fp8* f) {
    return f ? Fp8Out{(uint8_t*)f->data, f->scale, f->ld, f->ld_scale, f->format, f->block_rows} : Fp8Out{};
  };
  const bool vec = (uintptr_t)x % 16 == 0 && ldx * sizeof(T) % 16 == 0;
  const int64_t tr = fp8_blocks(rows), tc = fp8_blocks(cols);
  if (tr * tc > 0x7fffffff) return set_error(ALS_ERR_INVALID, "als_k_quant_fp8: matrix too large");
#define ALS_QUANT(V, A, B) hipLaunchKernelGGL((quant_fp8_kernel<T, V, A, B>), dim3((unsigned)(tr * tc)), dim3(256), 0, st, x, rows, cols, ldx, out(q), out(qt), (int)tc)
  if (q && qt) { if (vec) ALS_QUANT(true, true, true); else ALS_QUANT(false, true, true); }
  else if (q) { if (vec) ALS_QUANT(true, true, false); else ALS_QUANT(false, true, false); }
  else { if (vec) ALS_QUANT(true, false, true); else ALS_QUANT(false, false, true); }
#undef ALS_QUANT
  ALS_CHECK_LAUNCH();
  return ALS_OK;
}

}  // namespace

}  // namespace als

using namespace als;

extern "C" int als_k_quant_fp8(const void* x, int dtype, int rows, int cols, int64_t ldx, const als_fp8* q, const als_fp8* qt, void* stream) {
  if (!q && !qt) return set_error(ALS_ERR_INVALID, "als_k_quant_fp8: no output");
  if (rows < 0 || cols < 0 || rows > 1 << 30 || cols > 1 << 30) return set_error(ALS_ERR_INVALID, "als_k_quant_fp8: rows, cols must be in 0..2^30");
  int rc = check_dtype(dtype, "als_k_quant_fp8");
  if (!rc && q) rc = check_fp8(q, rows, cols, "als_k_quant_fp8, q");
  if (!rc && qt) rc = check_fp8(qt, cols, rows, "als_k_quant_fp8, qt");
  if (rc) return rc;
  if (rows == 0 || cols == 0) return ALS_OK;
  if (!x || ldx < cols) return set_error(ALS_ERR_INVALID, "als_k_quant_fp8: null x or ldx below cols");
  if ((uintptr_t)x % (dtype == ALS_DTYPE_BF16 ? 2 : 4)) return set_error(ALS_ERR_INVALID, "als_k_quant_fp8: x is not aligned to its type");
  if (dtype == ALS_DTYPE_BF16) return launch_quant((const bf16*)x, rows, cols, ldx, q, qt, (hipStream_t)stream);
  return launch_quant((const float*)x, rows, cols, ldx, q, qt, (hipStream_t)stream);
}
