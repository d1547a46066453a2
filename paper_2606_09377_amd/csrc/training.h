// What the epilogues and gradients of float layers share: matrices of either type by eight columns, dropout's
// random bits, activations and their slopes.  Part of dense.hip, dropout.hip and loss.hip.
#pragma once

#include <cmath>

#include "layers.h"
#include "planes.h"

namespace vcr {

// ---- matrices -------------------------------------------------------------------------------
struct MatRef {
  void *p;             // null: none
  int32_t bf16, vec;   // vec: rows are 16-byte aligned
  int64_t ld;
};
inline MatRef mat_ref(const vcr_mat *m) {
  if (!m) return MatRef{nullptr, 0, 0, 0};
  return MatRef{m->p, m->type == VCR_BF16, rows_aligned(m->p, m->ld, m->type == VCR_BF16 ? 2 : 4), m->ld};
}
__device__ __forceinline__ void unpack8(const uint4 &q, float (&v)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __builtin_bit_cast(float, w[i] << 16);
    v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef float f32v2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32v2{a, b}), bf16x2));
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Columns c .. c + 7 of row r, those below cols (the others are 0)
__device__ __forceinline__ void load8(const MatRef &m, int64_t r, int64_t c, int64_t cols, float (&v)[8]) {
  const int64_t at = r * m.ld + c;
  if (m.vec && c + 8 <= cols) {
    if (m.bf16) {
      unpack8(*reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(m.p) + at), v);
    } else {
      const f32v4 *s = reinterpret_cast<const f32v4 *>(static_cast<const float *>(m.p) + at);
      const f32v4 a = s[0], b = s[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    v[i] = c + i >= cols ? 0.f : m.bf16 ? bf16_value(static_cast<const uint16_t *>(m.p)[at + i]) : static_cast<const float *>(m.p)[at + i];
}
// (those below cols)
__device__ __forceinline__ void save8(const MatRef &m, int64_t r, int64_t c, int64_t cols, const float (&v)[8]) {
  const int64_t at = r * m.ld + c;
  if (m.vec && c + 8 <= cols) {
    if (m.bf16) {
      *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(m.p) + at) = pack8(v);
    } else {
      f32v4 *d = reinterpret_cast<f32v4 *>(static_cast<float *>(m.p) + at);
      d[0] = f32v4{v[0], v[1], v[2], v[3]};
      d[1] = f32v4{v[4], v[5], v[6], v[7]};
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (c + i >= cols) continue;
    if (m.bf16) static_cast<uint16_t *>(m.p)[at + i] = bf16_round(v[i]);
    else static_cast<float *>(m.p)[at + i] = v[i];
  }
}

// ---- dropout --------------------------------------------------------------------------------
// Sixteen bits a value: one Philox output serves eight columns.  Its twenty 32 x 32 -> 64-bit products are a quarter of the
// vector units' rate, so with 32 bits a value the random numbers of a bf16 matrix would take about as long as its
// bytes; p in steps of 2^-16 is what that costs, and the factor is that of the p taken.
struct DropDev {
  uint32_t k;   // 0: none
  float factor;
  uint32_t key0, key1;
  uint64_t offset;
  const uint64_t *step;
};
// (p has been checked)
inline DropDev drop_dev(const vcr_drop *d) {
  if (!d) return DropDev{0, 1.f, 0, 0, 0, nullptr};
  const uint32_t k = (uint32_t)std::lrint((double)d->p * 65536.0);
  return DropDev{k, (float)(65536.0 / (65536 - k)), (uint32_t)d->seed, (uint32_t)(d->seed >> 32), d->offset, d->step};
}
inline vcr_status check_drop(vcr_ctx *c, const vcr_drop *d) {
  if (!d) return VCR_OK;
  if (!(d->p >= 0.f && d->p < 1.f) || std::lrint((double)d->p * 65536.0) > 65535)
    return fail(c, VCR_ERR_ARG, "dropout: p = %g is not in [0, 1) by steps of 2^-16", (double)d->p);
  if ((reinterpret_cast<uintptr_t>(d->step) & 7) != 0) return fail(c, VCR_ERR_ARG, "dropout: step is not 8-byte aligned");
  return VCR_OK;
}
__device__ __forceinline__ uint64_t drop_offset(const DropDev &d) { return d.step ? d.offset + *d.step : d.offset; }
// Philox 4x32-10: ten rounds of two multiplications each, whose high words meet the other two words and the round's key
__device__ __forceinline__ void philox(uint32_t (&c)[4], uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)0xD2511F53u * c[0], b = (uint64_t)0xCD9E8D57u * c[2];
    c[0] = (uint32_t)(b >> 32) ^ c[1] ^ k0;
    c[1] = (uint32_t)b;
    c[2] = (uint32_t)(a >> 32) ^ c[3] ^ k1;
    c[3] = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
}
// Zeros in the place of the dropped ones of columns c .. c + 7 (c a multiple of 8) of row r
__device__ __forceinline__ void drop8(const DropDev &d, uint64_t offset, int64_t r, int64_t c, float (&v)[8]) {
  uint32_t w[4] = {(uint32_t)(c >> 3), (uint32_t)r, (uint32_t)offset, (uint32_t)(offset >> 32)};
  philox(w, d.key0, d.key1);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = (w[i] & 0xffff) >= d.k ? v[2 * i] : 0.f;
    v[2 * i + 1] = w[i] >> 16 >= d.k ? v[2 * i + 1] : 0.f;
  }
}

// ---- activations ----------------------------------------------------------------------------
// Phi(z) = erfc(-z / sqrt 2) / 2 keeps its relative accuracy for negative z, as exp(-|z|) does 1 / (1 + exp(-z)).
__device__ __forceinline__ float act_value(int act, float z) {
  if (act == VCR_ACT_RELU) return z < 0.f ? 0.f : z;   // NaN stays
  if (act == VCR_ACT_GELU) return 0.5f * z * erfcf(z * -0.70710678118654752f);
  if (act == VCR_ACT_SILU) {
    const float t = expf(-fabsf(z));
    return z * ((z < 0.f ? t : 1.f) / (1.f + t));
  }
  return z;
}
__device__ __forceinline__ float act_slope(int act, float z) {
  if (act == VCR_ACT_GELU) return 0.5f * erfcf(z * -0.70710678118654752f) + z * (0.39894228040143268f * expf(-0.5f * z * z));
  const float t = expf(-fabsf(z)), d = 1.f / (1.f + t);   // VCR_ACT_SILU
  return z < 0.f ? t * d * (1.f + z * d) : d * (1.f + z * (t * d));
}

}  // namespace vcr
