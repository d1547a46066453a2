// Operands of nt.h made from row-major matrices and from 4-bit ones, and the epilogues that write results
// back.  Part of layers.hip and orthogonalize.hip.
#pragma once

#include "nt.h"

namespace vcr {

inline int64_t blocks_of(int64_t n, int64_t b) { return (n + b - 1) / b; }

// go(first, count) for stretches of `wgs` workgroups whose threads a launch can count (32 bits)
template <class F>
hipError_t launch_stretches(int64_t wgs, F &&go) {
  constexpr int64_t MOST = 1 << 22;
  for (int64_t first = 0; first < wgs; first += MOST) {
    go(first, dim3((unsigned)std::min(MOST, wgs - first)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// A row-major matrix on the device: type 0 float32, 1 bf16 (VCR_F32, VCR_BF16)
struct DevMat {
  const void *p;
  int32_t bf16;
  int64_t rows, cols, ld;
  int64_t stride;   // elements from one matrix of a batch to the next
};

__device__ __forceinline__ float bf16_value(uint16_t u) { return __builtin_bit_cast(float, (uint32_t)u << 16); }
__device__ __forceinline__ uint16_t bf16_round(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// whether whole 16-byte loads of rows are aligned
__host__ __device__ inline bool rows_aligned(const void *p, int64_t ld, int bytes) {
  return ((uintptr_t)p & 15) == 0 && (ld * bytes & 15) == 0;
}

// element (r, c), zero outside
template <bool BF>
__device__ __forceinline__ float mat_at(const DevMat &x, int64_t base, int64_t r, int64_t c) {
  if (r >= x.rows || c >= x.cols) return 0.f;
  if constexpr (BF) return bf16_value(static_cast<const uint16_t *>(x.p)[base + r * x.ld + c]);
  else return static_cast<const float *>(x.p)[base + r * x.ld + c];
}

// eight consecutive elements of row r from column c on, zeros outside
template <bool BF>
__device__ __forceinline__ void mat_row8(const DevMat &x, int64_t base, int64_t r, int64_t c, bool vec, float (&v)[8]) {
  if (vec && r < x.rows && c + 8 <= x.cols) {
    if constexpr (BF) {
      const uint4 q = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(x.p) + base + r * x.ld + c);
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_value((uint16_t)w[i]);
        v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
      }
    } else {
      const float4 *q = reinterpret_cast<const float4 *>(static_cast<const float *>(x.p) + base + r * x.ld + c);
      const float4 a = q[0], b = q[1];
      v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = mat_at<BF>(x, base, r, c + i);
}

// The parts of two values, P of them.  A value that is infinite or NaN has no small parts; one that only
// rounds to infinity in bf16 (from 2^128 - 2^119 on) has the largest bf16 value as its large part.
template <int P>
__device__ __forceinline__ void parts_of(float x0, float x1, uint32_t (&out)[P]) {
  auto cut = [](float x) {   // the large part of a value that rounds to infinity: truncated
    return __builtin_bit_cast(uint32_t, x) >> 16;
  };
  typedef float f32v2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  auto pack = [](float a, float b) {
    const f32v2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  };
  uint32_t h = pack(x0, x1);
  if constexpr (P > 1) {
    auto inf = [](float x) { return fabsf(x) >= 0x1.ffp127f; };   // (NaN: false)
    if (__builtin_expect(inf(x0) || inf(x1) || x0 != x0 || x1 != x1, 0)) {
      if (inf(x0)) h = (h & 0xffff0000u) | cut(x0);
      if (inf(x1)) h = (h & 0xffffu) | cut(x1) << 16;
      // what remains of infinite and NaN values is nothing
      const float m0 = __builtin_bit_cast(float, h << 16), m1 = __builtin_bit_cast(float, h & 0xffff0000u);
      x0 = fabsf(x0) < __builtin_huge_valf() ? x0 - m0 : 0.f;
      x1 = fabsf(x1) < __builtin_huge_valf() ? x1 - m1 : 0.f;
    } else {
      x0 -= __builtin_bit_cast(float, h << 16);
      x1 -= __builtin_bit_cast(float, h & 0xffff0000u);
    }
  }
  out[0] = h;
#pragma unroll
  for (int p = 1; p < P; ++p) {
    out[p] = pack(x0, x1);
    x0 -= __builtin_bit_cast(float, out[p] << 16);
    x1 -= __builtin_bit_cast(float, out[p] & 0xffff0000u);
  }
}

// 16 bytes of each part from eight values: slot of fragment (row block, chunk), lane l
template <int P>
__device__ __forceinline__ void store_slot(uint8_t *planes, int64_t frag, int l, const float (&v)[8]) {
  uint32_t w[4][P];
#pragma unroll
  for (int i = 0; i < 4; ++i) parts_of<P>(v[2 * i], v[2 * i + 1], w[i]);
#pragma unroll
  for (int p = 0; p < P; ++p)
    *reinterpret_cast<uint4 *>(planes + (frag * P + p) * FRAG + l * 16) = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
}

// Operands made from a matrix, its rows and its columns in one pass (either may be null): a workgroup takes 64 x 64 values, a
// wave 16 rows of them as the fragments of its row block, the transposed ones from LDS.  Bound by memory.
//   x      rows x cols of it, or only those where y > 0; times `scale`
//   rows   operand of x's rows, row_chunks chunks of 32 columns
//   cols   operand of x's columns, col_chunks chunks of 32 rows
//   sums   [64-row group][cols]: column sums (null: none)
// Chunks beyond x hold zeros; row blocks beyond x's rows or columns, rounded up to 16, are not written unless they are
// below row_blocks, col_blocks.
struct PlanesArgs {
  DevMat x, y;
  int32_t vec;
  uint8_t *rows, *cols;
  int64_t row_blocks, row_chunks, col_blocks, col_chunks;
  float *sums;
  int32_t grouped;   // rows: chunks in the order of 4-bit operands (NT_MIXED); row_chunks is a multiple of 4
};
// A factor that float32 may not hold: powers of two, applied first (exactly), and a rest
struct PlanesScale {
  float two[2], rest;
};
template <int P, bool BF>
__device__ __forceinline__ void planes_tile(const PlanesArgs &g, int64_t base, int64_t tr, int64_t tc, PlanesScale scale, float (&tile)[64][65]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, oct = lane >> 4;
  const int64_t rb = tr * 4 + wave, row = rb * 16 + r;
  float v[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t col = tc * 64 + h * 32 + oct * 8;
    mat_row8<BF>(g.x, base, row, col, g.vec, v[h]);
    if (g.y.p) {
      float m[8];
      mat_row8<BF>(g.y, base, row, col, g.vec, m);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[h][i] = m[i] > 0.f ? v[h][i] : 0.f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[h][i] = v[h][i] * scale.two[0] * scale.two[1] * scale.rest;
    const int64_t ch = tc * 2 + h;   // 32 columns
    if (g.rows && rb < g.row_blocks && ch < g.row_chunks) {
      if (g.grouped) store_slot<P>(g.rows, rb * g.row_chunks + (ch & ~(int64_t)3) + oct, (int)(ch & 3) * 16 + r, v[h]);
      else store_slot<P>(g.rows, rb * g.row_chunks + ch, lane, v[h]);
    }
  }
  if (!g.cols && !g.sums) return;   // uniform
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 8; ++i) tile[wave * 16 + r][h * 32 + oct * 8 + i] = v[h][i];
  __syncthreads();
  // wave: 16 columns; lane: column r, rows 32 h + 8 oct ..
  float s = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      t[i] = tile[h * 32 + oct * 8 + i][wave * 16 + r];
      s += t[i];
    }
    const int64_t cb = tc * 4 + wave, ch = tr * 2 + h;
    if (g.cols && cb < g.col_blocks && ch < g.col_chunks) store_slot<P>(g.cols, cb * g.col_chunks + ch, lane, t);
  }
  if (g.sums) {
    s += __shfl_xor(s, 16);
    s += __shfl_xor(s, 32);
    const int64_t col = tc * 64 + wave * 16 + r;
    if (oct == 0 && col < g.x.cols) g.sums[tr * g.x.cols + col] = s;
  }
}

// Four consecutive k of one row, into an operand of P parts with so many chunks
template <int P>
__device__ __forceinline__ void store_quad(uint8_t *planes, int64_t row, int64_t k, int64_t chunks, f32v4 v) {
  uint32_t a[P], b[P];
  parts_of<P>(v[0], v[1], a);
  parts_of<P>(v[2], v[3], b);
  uint8_t *d = planes + ((row >> 4) * chunks + (k >> 5)) * P * FRAG + (((k & 31) >> 3) * 16 + (row & 15)) * 16 + (k & 4) * 2;
#pragma unroll
  for (int p = 0; p < P; ++p) *reinterpret_cast<uint2 *>(d + p * FRAG) = make_uint2(a[p], b[p]);
}
template <int P>
__device__ __forceinline__ f32v4 load_quad(const uint8_t *planes, int64_t row, int64_t k, int64_t chunks) {
  const uint8_t *d = planes + ((row >> 4) * chunks + (k >> 5)) * P * FRAG + (((k & 31) >> 3) * 16 + (row & 15)) * 16 + (k & 4) * 2;
  f32v4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int p = P - 1; p >= 0; --p) {
    const uint2 q = *reinterpret_cast<const uint2 *>(d + p * FRAG);
    v[0] += __builtin_bit_cast(float, q.x << 16);
    v[1] += __builtin_bit_cast(float, q.x & 0xffff0000u);
    v[2] += __builtin_bit_cast(float, q.y << 16);
    v[3] += __builtin_bit_cast(float, q.y & 0xffff0000u);
  }
  return v;
}

// Four consecutive columns of a row of a matrix, those inside it (vec: rows_aligned)
__device__ __forceinline__ void store_row4(void *p, int bf16, int64_t ld, int64_t rows, int64_t cols, bool vec, int64_t r,
                                           int64_t c, f32v4 v) {
  if (r >= rows || c >= cols) return;
  if (bf16) {
    uint16_t *d = static_cast<uint16_t *>(p) + r * ld + c;
    const uint16_t q[4] = {bf16_round(v[0]), bf16_round(v[1]), bf16_round(v[2]), bf16_round(v[3])};
    if (vec && c + 4 <= cols) {
      *reinterpret_cast<uint2 *>(d) = make_uint2(q[0] | (uint32_t)q[1] << 16, q[2] | (uint32_t)q[3] << 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < cols) d[i] = q[i];
    }
  } else {
    float *d = static_cast<float *>(p) + r * ld + c;
    if (vec && c + 4 <= cols) {
      *reinterpret_cast<f32v4 *>(d) = v;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < cols) d[i] = v[i];
    }
  }
}

}  // namespace vcr
