// A matrix to 8 bits with a power-of-two scale for each block (als_k_quant_fp8): as it is, transposed, or both from one reading.
//
// Memory bounds it: 4 or 2 bytes read and 1 written for each orientation and element.  A workgroup of 256 threads owns a tile of 128 x 128, whole blocks of
// both orientations; a thread has 8 rows of 8 columns of it in registers, so that a row's largest magnitude is 16 neighbouring lanes' and the bytes of
// a thread are 8 in a row of either orientation.  The transposed bytes go through LDS (16 KB) to be written as whole rows of 128.
// Magnitudes are compared as whole numbers, two bf16 at a time, and the conversion divides by the scale: 3 vector instructions an element in bf16 and both
// orientations.  Scales are written as single bytes, a tile's rows and columns in one store each (1.5 us of 51 less), which meet their neighbours in an L2: every XCD has a run of
// neighbouring tiles.
// 16384 x 3584 bf16, both orientations: 51 us with a scale a row (4.6 TB/s, a copy of that size 5.4), 48.5 with one a tile; one orientation 35.5; fp32 72 and 69, 56 for one orientation
// (5.2 TB/s).  With magnitudes in floating point,
// products by 1 / scale, tiles dealt to the XCDs in turn and ordinary stores bf16 took 70 and 55.  Bands of tiles column by column, for the transposed scales, gain 1 us of 56, but with
// 4096 columns take 74 instead of 67.
#include "fp8.h"

namespace als {

namespace {

struct Fp8Out { uint8_t* data; uint8_t* scale; int64_t ld, ld_scale; int format, block_rows; };
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ unsigned pk_max(unsigned a, unsigned b) {   // of two pairs of 16 bits
  return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// the largest over the four groups of 16 lanes, lane by lane
template <typename F>
__device__ __forceinline__ unsigned groups4_max(unsigned m, F f) {
  auto a = __builtin_amdgcn_permlane16_swap(m, m, false, false);
  m = f(a[0], a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(m, m, false, false);
  return f(b[0], b[1]);
}

// A thread's 8 x 8 elements: fp32 one a word, bf16 two.
template <typename T>
struct Elements {
  static constexpr int W = sizeof(T) == 4 ? 8 : 4;
  unsigned w[8][W];
  // row i from p; n: how many exist
  __device__ __forceinline__ void load(int i, const T* p, int n) {
    if (n >= 8) {
      __builtin_memcpy(w[i], p, 8 * sizeof(T));
    } else {
#pragma unroll
      for (int k = 0; k < W; k++) w[i][k] = 0;
#pragma unroll
      for (int j = 0; j < 8; j++)
        if (j < n) {
          if constexpr (sizeof(T) == 4) w[i][j] = __builtin_bit_cast(unsigned, p[j]);
          else w[i][j / 2] |= (unsigned)__builtin_bit_cast(unsigned short, p[j]) << (16 * (j & 1));
        }
    }
  }
  __device__ __forceinline__ float at(int i, int j) const {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i][j]);
    else return __builtin_bit_cast(float, j & 1 ? w[i][j / 2] & 0xffff0000u : w[i][j / 2] << 16);
  }
  // bits of the largest finite magnitude of each row and column of these
  __device__ __forceinline__ void maxima(unsigned (&row)[8], unsigned (&col)[8]) const {
    unsigned any;
    if constexpr (sizeof(T) == 4) {
      any = 0;
#pragma unroll
      for (int j = 0; j < 8; j++) col[j] = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        row[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const unsigned m = w[i][j] & 0x7fffffffu;
          row[i] = max(row[i], m);
          col[j] = max(col[j], m);
        }
        any = max(any, row[i]);
      }
    } else {
      unsigned c[4] = {0, 0, 0, 0}, all = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        unsigned r = 0;
#pragma unroll
        for (int k = 0; k < 4; k++) {
          const unsigned m = w[i][k] & 0x7fff7fffu;
          r = pk_max(r, m);
          c[k] = pk_max(c[k], m);
        }
        row[i] = max(r & 0xffff0000u, r << 16);
        all = pk_max(all, r);
      }
#pragma unroll
      for (int k = 0; k < 4; k++) {
        col[2 * k] = c[k] << 16;
        col[2 * k + 1] = c[k] & 0xffff0000u;
      }
      any = max(all & 0xffff0000u, all << 16);
    }
    if (any >= 0x7f800000u) {   // an infinity or a NaN among them: once more, without those
#pragma unroll
      for (int j = 0; j < 8; j++) col[j] = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) {
        row[i] = 0;
#pragma unroll
        for (int j = 0; j < 8; j++) {
          const unsigned m = fp8_magnitude(at(i, j));
          row[i] = max(row[i], m);
          col[j] = max(col[j], m);
        }
      }
    }
  }
  // elements 4 h .. + 3 of row i, and of column j, as bytes
  __device__ __forceinline__ unsigned row4(int i, int h, float scale, int format) const {
    if constexpr (sizeof(T) == 4) return fp8_pack4(at(i, 4 * h), at(i, 4 * h + 1), at(i, 4 * h + 2), at(i, 4 * h + 3), scale, format);
    else return pairs4(w[i][2 * h], w[i][2 * h + 1], scale, format);
  }
  __device__ __forceinline__ unsigned col4(int j, int h, float scale, int format) const {
    if constexpr (sizeof(T) == 4) return fp8_pack4(at(4 * h, j), at(4 * h + 1, j), at(4 * h + 2, j), at(4 * h + 3, j), scale, format);
    else {
      const int sel = j & 1 ? 0x07060302 : 0x05040100;   // the upper or the lower halves of two words
      return pairs4(__builtin_amdgcn_perm(w[4 * h + 1][j / 2], w[4 * h][j / 2], sel), __builtin_amdgcn_perm(w[4 * h + 3][j / 2], w[4 * h + 2][j / 2], sel), scale, format);
    }
  }
  static __device__ __forceinline__ unsigned pairs4(unsigned a, unsigned b, float scale, int format) {
    s16x2 v = {0, 0};
    if (format == ALS_FP8_E4M3) {
      v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2, a), scale, false);
      v = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(v, __builtin_bit_cast(bf16x2, b), scale, true);
    } else {
      v = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(v, __builtin_bit_cast(bf16x2, a), scale, false);
      v = __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(v, __builtin_bit_cast(bf16x2, b), scale, true);
    }
    return __builtin_bit_cast(unsigned, v);
  }
};

template <typename T, bool Q, bool QT>
__global__ __launch_bounds__(256) void quant_fp8_kernel(const T* __restrict__ x, int rows, int cols, int64_t ldx, Fp8Out q, Fp8Out qt, int tiles_c) {
  __shared__ __attribute__((aligned(16))) unsigned cmax[QT ? 4 : 1][QT ? 128 : 4];
  __shared__ unsigned wmax[4];
  __shared__ uint8_t scales[2][128];   // of the tile's rows and columns, written together: a thread each
  __shared__ __attribute__((aligned(16))) uint8_t tile[QT ? 128 * 128 : 16];
  const int total = gridDim.x, base = total / 8, rem = total % 8, xcd = blockIdx.x & 7;
  const int id = xcd * base + (xcd < rem ? xcd : rem) + (blockIdx.x >> 3);
  const int tr = id / tiles_c, tc = id - tr * tiles_c;
  const int row0 = tr * 128, col0 = tc * 128;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, cx = threadIdx.x & 15, ry = threadIdx.x >> 4;
  const int c = col0 + 8 * cx, r0 = row0 + 8 * ry;
  const int left = cols - c;   // columns of this thread that exist, if below 8
  Elements<T> v;
#pragma unroll
  for (int i = 0; i < 8; i++) v.load(i, x + (int64_t)(r0 + i) * ldx + c, r0 + i < rows ? left : 0);
  unsigned rmax[8], cm[8];
  v.maxima(rmax, cm);

  auto larger = [](unsigned a, unsigned b) { return a > b ? a : b; };
  const bool whole = (Q && q.block_rows == 128) || (QT && qt.block_rows == 128);   // a block is the tile
  unsigned amax_tile = 0;
  if (whole) {
#pragma unroll
    for (int i = 0; i < 8; i++) amax_tile = max(amax_tile, rmax[i]);
    amax_tile = groups4_max(lanes16_max(amax_tile), larger);
    if (lane == 0) wmax[wave] = amax_tile;
  }
  if (QT && qt.block_rows == 1) {
#pragma unroll
    for (int j = 0; j < 8; j++) cm[j] = groups4_max(cm[j], larger);
    if (lane < 16) {
      *reinterpret_cast<u32x4*>(&cmax[wave][8 * cx]) = (u32x4){cm[0], cm[1], cm[2], cm[3]};
      *reinterpret_cast<u32x4*>(&cmax[wave][8 * cx + 4]) = (u32x4){cm[4], cm[5], cm[6], cm[7]};
    }
  }
  if (whole || QT) __syncthreads();
  if (whole) amax_tile = max(max(wmax[0], wmax[1]), max(wmax[2], wmax[3]));

  if (Q) {
    const int bt = q.block_rows == 128 ? fp8_scale_byte(amax_tile, q.format) : 0;
    if (q.block_rows == 128 && threadIdx.x == 0) q.scale[(int64_t)tr * q.ld_scale + tc] = (uint8_t)bt;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      int b = bt;
      if (q.block_rows == 1) {
        b = fp8_scale_byte(lanes16_max(rmax[i]), q.format);
        if (cx == 0) scales[0][8 * ry + i] = (uint8_t)b;
      }
      const float s = fp8_scale(b);
      const unsigned lo = v.row4(i, 0, s, q.format), hi = v.row4(i, 1, s, q.format);
      if (r0 + i < rows && left > 0) store8_bytes(q.data + (int64_t)(r0 + i) * q.ld + c, left, lo, hi);
    }
  }
  if (QT) {
    const int bt = qt.block_rows == 128 ? fp8_scale_byte(amax_tile, qt.format) : 0;
    if (qt.block_rows == 128 && threadIdx.x == 0) qt.scale[(int64_t)tc * qt.ld_scale + tr] = (uint8_t)bt;
    if (qt.block_rows == 1) {
#pragma unroll
      for (int h = 0; h < 2; h++) {
        u32x4 m = *reinterpret_cast<const u32x4*>(&cmax[0][8 * cx + 4 * h]);
#pragma unroll
        for (int w = 1; w < 4; w++) m = __builtin_elementwise_max(m, *reinterpret_cast<const u32x4*>(&cmax[w][8 * cx + 4 * h]));
#pragma unroll
        for (int j = 0; j < 4; j++) cm[4 * h + j] = m[j];
      }
    }
    // column 8 cx + j of the tile is row 8 cx + j of 128 bytes in LDS; its 8-byte piece ry lies at piece ry ^ cx, so that 16 columns' pieces
    // fall into 16 different pairs of banks
#pragma unroll
    for (int j = 0; j < 8; j++) {
      int b = bt;
      if (qt.block_rows == 1) {
        b = fp8_scale_byte(cm[j], qt.format);
        if (ry == 0) scales[1][8 * cx + j] = (uint8_t)b;
      }
      const float s = fp8_scale(b);
      *reinterpret_cast<uint2*>(tile + (8 * cx + j) * 128 + (ry ^ cx) * 8) = make_uint2(v.col4(j, 0, s, qt.format), v.col4(j, 1, s, qt.format));
    }
  }
  if (QT || q.block_rows == 1) __syncthreads();
  const int line = threadIdx.x & 127;
  if (Q && q.block_rows == 1 && threadIdx.x < 128 && row0 + line < rows) q.scale[(int64_t)(row0 + line) * q.ld_scale + tc] = scales[0][line];
  if (QT && qt.block_rows == 1 && threadIdx.x >= 128 && col0 + line < cols) qt.scale[(int64_t)(col0 + line) * qt.ld_scale + tr] = scales[1][line];
  if (QT) {
#pragma unroll
    for (int p = 0; p < 4; p++) {
      const int cc = p * 32 + (threadIdx.x >> 3), k = threadIdx.x & 7, sw = cc >> 3;   // sw: the cx that wrote it
      uint4 d = *reinterpret_cast<const uint4*>(tile + cc * 128 + (k ^ (sw >> 1)) * 16);
      if (sw & 1) d = make_uint4(d.z, d.w, d.x, d.y);
      const int rt = row0 + 16 * k;
      if (col0 + cc < cols && rt < rows) {
        uint8_t* o = qt.data + (int64_t)(col0 + cc) * qt.ld + rt;
        if (rows - rt >= 16) {
          __builtin_nontemporal_store(__builtin_bit_cast(u32x4, d), reinterpret_cast<u32x4*>(o));
        } else {
          store8_bytes(o, rows - rt, d.x, d.y);
          if (rows - rt > 8) store8_bytes(o + 8, rows - rt - 8, d.z, d.w);
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
  const int64_t tr = fp8_blocks(rows), tc = fp8_blocks(cols);
  if (tr * tc >= 1 << 24) return set_error(ALS_ERR_INVALID, "als_k_quant_fp8: matrix of 2^24 blocks of 128 x 128 or more");
#define ALS_QUANT(A, B) hipLaunchKernelGGL((quant_fp8_kernel<T, A, B>), dim3((unsigned)(tr * tc)), dim3(256), 0, st, x, rows, cols, ldx, out(q), out(qt), (int)tc)
  if (q && qt) ALS_QUANT(true, true);
  else if (q) ALS_QUANT(true, false);
  else ALS_QUANT(false, true);
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
