// Layers whose weights are held in microscaled 4-bit floating point: quantisation and its reverse, products of
// 4-bit rows and of float rows with 4-bit weights, and the latter's gradients.  vcr_mx_* of vcrown.h.
//
// Format.  32 consecutive values of a row share a power of two: e = floor(log2 max |x|) - 2, within
// [-127, 127], kept as the byte e + 127 (255: the block held an infinity or NaN, and reads as NaN), and
// each is a 4-bit float x 2^-e: sign, two exponent bits, one mantissa bit, i.e. +-{0, .5, 1, 1.5, 2, 3, 4,
// 6}, rounded to nearest, ties to an even code, 6 above 6.  Storage is in the order of the matrix
// instructions (nt.h): codes [rows / 16][cols / 128][64 lanes][16 bytes], lane 16 g + r holding the
// block of columns 32 g .. 32 g + 31 of row r, the first value in the low bits; scales [rows /
// 16][cols / 512][64 lanes][4 groups of 128 columns].  Rows are padded to 16 and columns to 128 with zeros.
#include <algorithm>
#include <type_traits>

#include "ctx.h"
#include "layers.h"
#include "planes.h"

namespace vcr {

// ---- 4-bit values ---------------------------------------------------------------------------
__host__ __device__ inline int64_t mx_groups(int64_t cols) { return (cols + 127) / 128; }

// the float of a scale byte, as the conversions take it
__device__ __forceinline__ float mx_scale(uint32_t byte) {
  return __builtin_bit_cast(float, byte == 255 ? 0x7fc00000u : byte == 0 ? 0x00400000u : byte << 23);
}

struct MxDev {
  const uint8_t *codes, *scales;
  int64_t rows, cols;
};
__device__ __forceinline__ int64_t mx_scale_at(int64_t rb, int64_t group, int64_t groups, int lane) {
  return ((rb * ((groups + 3) >> 2) + (group >> 2)) * 64 + lane) * 4 + (group & 3);
}

// Quantisation: a thread per block.  A workgroup takes 16 rows by 512 columns, a wave one group of
// 128 columns in lane order.
template <bool BF>
__global__ __launch_bounds__(256) void k_mx_quantize(DevMat x, int vec, uint8_t *codes, uint8_t *scales) {
  __shared__ uint8_t sb[256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t groups = mx_groups(x.cols), n4 = (groups + 3) >> 2;
  const int64_t rb = blockIdx.x / n4, c4 = blockIdx.x - rb * n4, grp = c4 * 4 + wave;
  const int64_t row = rb * 16 + (lane & 15), col = grp * 128 + (lane >> 4) * 32;
  uint32_t byte = 0;
  if (grp < groups) {
    float v[4][8];
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      mat_row8<BF>(x, 0, row, col + 8 * q, vec, v[q]);
#pragma unroll
      for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, v[q][i]) & 0x7fffffffu);
    }
    const uint32_t e = top >> 23;
    byte = e == 255 ? 255 : e > 2 ? e - 2 : 0;
    const float s = mx_scale(byte == 255 ? 127 : byte);
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      uint32_t u = 0;
      u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[q][0], v[q][1], s, 0);
      u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[q][2], v[q][3], s, 1);
      u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[q][4], v[q][5], s, 2);
      u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[q][6], v[q][7], s, 3);
      w[q] = u;
    }
    *reinterpret_cast<uint4 *>(codes + ((rb * groups + grp) * 64 + lane) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
  }
  sb[lane * 4 + wave] = (uint8_t)byte;
  __syncthreads();
  if (wave == 0)
    *reinterpret_cast<uint32_t *>(scales + (rb * n4 + c4) * 256 + lane * 4) = *reinterpret_cast<uint32_t *>(sb + lane * 4);
}

// The values of a lane's block: 32 consecutive ones of a row
__device__ __forceinline__ void mx_block(const MxDev &w, int64_t rb, int64_t grp, int64_t groups, int lane, uint4 &q,
                                         float &s) {
  q = *reinterpret_cast<const uint4 *>(w.codes + ((rb * groups + grp) * 64 + lane) * 16);
  s = mx_scale(w.scales[mx_scale_at(rb, grp, groups, lane)]);
}
__device__ __forceinline__ uint4 mx_to_bf16(uint32_t u, float s) {   // eight values
  auto c = [](auto v) { return __builtin_bit_cast(uint32_t, v); };
  return make_uint4(c(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 0)), c(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 1)),
                    c(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 2)), c(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, s, 3)));
}

template <bool BF>
__global__ __launch_bounds__(256) void k_mx_dequantize(MxDev w, void *y, int64_t ld, int vec) {
  const int lane = threadIdx.x & 63;
  const int64_t groups = mx_groups(w.cols), id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t rb = id / groups, grp = id - rb * groups, row = rb * 16 + (lane & 15), col = grp * 128 + (lane >> 4) * 32;
  if (row >= w.rows) return;
  uint4 q;
  float s;
  mx_block(w, rb, grp, groups, lane, q, s);
  const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint4 b = mx_to_bf16(u[i], s);
    const uint32_t h[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const f32v4 v = {__builtin_bit_cast(float, h[2 * k] << 16), __builtin_bit_cast(float, h[2 * k] & 0xffff0000u),
                       __builtin_bit_cast(float, h[2 * k + 1] << 16), __builtin_bit_cast(float, h[2 * k + 1] & 0xffff0000u)};
      store_row4(y, BF, ld, w.rows, w.cols, vec, row, col + 8 * i + 4 * k, v);
    }
  }
}

// ---- operands of the bf16 products ------------------------------------------------------------
// x, or x where y > 0 (mask), in P parts: a wave per (row block, chunk)
template <int P, bool BF>
__global__ __launch_bounds__(256) void k_planes(DevMat x, DevMat y, int vec, int64_t chunks, uint8_t *out) {
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), rb = id / chunks, ch = id - rb * chunks;
  const int64_t row = rb * 16 + (lane & 15), col = ch * 32 + (lane >> 4) * 8;
  if (rb * 16 >= x.rows) return;
  float v[8];
  mat_row8<BF>(x, 0, row, col, vec, v);
  if (y.p) {
    float m[8];
    mat_row8<BF>(y, 0, row, col, vec, m);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = m[i] > 0.f ? v[i] : 0.f;
  }
  store_slot<P>(out, id, lane, v);
}

// The same transposed (rows of the operand: columns of x), and the column sums of every 32 rows: a
// wave reads 8 rows of 64 columns, a workgroup 32.
template <int P, bool BF>
__global__ __launch_bounds__(256) void k_planes_t(DevMat x, DevMat y, int64_t chunks, uint8_t *out, float *sums) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t nc = (x.cols + 63) / 64, ch = blockIdx.x / nc, col = (blockIdx.x - ch * nc) * 64 + lane;
  float v[8], s = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t r = ch * 32 + wave * 8 + i;
    v[i] = mat_at<BF>(x, 0, r, col);
    if (y.p) v[i] = mat_at<BF>(y, 0, r, col) > 0.f ? v[i] : 0.f;
    s += v[i];
  }
  if (out && col < (x.cols + 15) / 16 * 16) store_slot<P>(out, (col >> 4) * chunks + ch, wave * 16 + (int)(col & 15), v);
  if (!sums) return;   // uniform
  part[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < x.cols) sums[ch * x.cols + col] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
}

__global__ __launch_bounds__(256) void k_column_sums(const float *sums, int64_t parts, int64_t cols, float *out) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  float s = 0.f;
  for (int64_t p = 0; p < parts; ++p) s += sums[p * cols + c];
  out[c] = s;
}

// 4-bit weights as a bf16 operand (exact): a thread per block
__global__ __launch_bounds__(256) void k_mx_planes(MxDev w, uint8_t *out) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int64_t groups = mx_groups(w.cols), id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t rb = id / groups, grp = id - rb * groups;
  if (rb * 16 >= w.rows) return;
  uint4 q;
  float s;
  mx_block(w, rb, grp, groups, lane, q, s);
  const uint32_t u[4] = {q.x, q.y, q.z, q.w};
  uint8_t *d = out + (rb * groups * 4 + grp * 4 + g) * FRAG + r * 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4 *>(d + i * 256) = mx_to_bf16(u[i], s);
}

// The transposed weights as a bf16 operand, rows k and contraction n: a thread per 32 k of 8 rows n
__global__ __launch_bounds__(256) void k_mx_planes_t(MxDev w, int64_t chunks, int64_t row_blocks, uint8_t *out) {
  const int64_t groups = mx_groups(w.cols), octets = chunks * 4;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t o = id % octets, gk = id / octets, grp = gk >> 2;   // 32 k from 32 gk on
  if (grp >= groups) return;
  uint4 q[8];
  float s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t n = o * 8 + i;
    q[i] = make_uint4(0, 0, 0, 0);
    s[i] = 1.f;
    if (n < w.rows) mx_block(w, n >> 4, grp, groups, (int)((gk & 3) * 16 + (n & 15)), q[i], s[i]);
  }
  const int lane0 = (int)(o & 3) * 16;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint4 b[8];   // 8 k of every n
#pragma unroll
    for (int n = 0; n < 8; ++n) b[n] = mx_to_bf16(i == 0 ? q[n].x : i == 1 ? q[n].y : i == 2 ? q[n].z : q[n].w, s[n]);
    const int64_t rb = gk * 2 + (i >> 1);
    if (rb >= row_blocks) return;
    uint8_t *d = out + (rb * chunks + (o >> 2)) * FRAG + (lane0 + (i & 1) * 8) * 16;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      uint32_t h[8];
#pragma unroll
      for (int n = 0; n < 8; ++n) {
        const uint32_t p = k < 2 ? b[n].x : k < 4 ? b[n].y : k < 6 ? b[n].z : b[n].w;
        h[n] = k & 1 ? p >> 16 : p & 0xffffu;
      }
      *reinterpret_cast<uint4 *>(d + k * 16) =
          make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
    }
  }
}

// ---- epilogues --------------------------------------------------------------------------------
struct OutMat {
  void *p;
  int32_t bf16, vec;
  int64_t rows, cols, ld;
  const float *bias;   // or null
  int32_t relu;
  __device__ __forceinline__ void put(int64_t m, int64_t n, f32v4 v) const {
    if (bias) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] += n + q < cols ? bias[n + q] : 0.f;
    }
    if (relu) {
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = v[q] < 0.f ? 0.f : v[q];   // NaN stays
    }
    store_row4(p, bf16, ld, rows, cols, vec, m, n, v);
  }
};
struct EpiOut {
  OutMat o;
  __device__ __forceinline__ void store(int, int, int m, int n, f32v4 v, int) const { o.put(m, n, v); }
};
// sums over one part of the contraction, [parts][rows][ld]
struct EpiPart {
  float *p;
  int64_t rows, ld;
  __device__ __forceinline__ void store(int, int z, int m, int n, f32v4 v, int) const {
    if (m < rows && n < ld) *reinterpret_cast<f32v4 *>(p + (z * rows + m) * ld + n) = v;
  }
};
__global__ __launch_bounds__(256) void k_join(const float *p, int parts, int64_t rows, int64_t ld, OutMat o) {
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, per = ld / 4, m = id / per, n = (id - m * per) * 4;
  if (m >= rows) return;
  f32v4 v = {0.f, 0.f, 0.f, 0.f};
  for (int z = 0; z < parts; ++z) v += *reinterpret_cast<const f32v4 *>(p + (z * rows + m) * ld + n);
  o.put(m, n, v);
}

// ---- choice of tiles --------------------------------------------------------------------------
template <int PA, int PB, bool FP4>
struct Tiles {
  static constexpr int KS = PA == 1 ? 2 : 1;
  typedef std::conditional_t<PA == 3, NtTile<4, 4, 4, 2, PA, PB, KS, FP4>, NtTile<8, 4, 2, 4, PA, PB, KS, FP4>> L;
  typedef std::conditional_t<PB == 3, NtTile<4, 2, 2, 4, PA, PB, KS, FP4>, NtTile<4, 4, 2, 2, PA, PB, KS, FP4>> M;
  typedef NtTile<2, 2, 2, 2, PA, PB, KS, FP4> S;
};
static int64_t tiles_of(int64_t m, int64_t n, int bm, int bn) { return blocks_of(m, bm) * blocks_of(n, bn); }

// 0: L, 1: M, 2: S; parts of the contraction (S only)
struct NtPlan {
  int kind, parts;
  size_t part_bytes(int64_t M, int64_t N) const { return parts > 1 ? (size_t)parts * M * blocks_of(N, 4) * 16 : 0; }
};
template <int PA, int PB, bool FP4>
static NtPlan nt_plan(int64_t M, int64_t N, int64_t chunks) {
  typedef Tiles<PA, PB, FP4> TS;
  if (tiles_of(M, N, TS::L::BM, TS::L::BN) >= 200) return {0, 1};
  if (tiles_of(M, N, TS::M::BM, TS::M::BN) >= 200) return {1, 1};
  const int64_t t = tiles_of(M, N, TS::S::BM, TS::S::BN), steps = blocks_of(chunks, TS::S::KS);
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(512 / t, steps / 8));
  return {2, (int)parts};
}
template <int PA, int PB, bool FP4, class EPI>
static hipError_t nt_kind(int kind, const NtArgs &g, int64_t M, int64_t N, int parts, const EPI &e, hipStream_t s) {
  typedef Tiles<PA, PB, FP4> TS;
  if (kind == 0) return launch_nt<typename TS::L>(g, M, N, 1, parts, e, s);
  if (kind == 1) return launch_nt<typename TS::M>(g, M, N, 1, parts, e, s);
  return launch_nt<typename TS::S>(g, M, N, 1, parts, e, s);
}
// D = A B^T into o; part: room for nt_plan's partial sums
template <int PA, int PB, bool FP4>
static hipError_t nt_product(const NtArgs &g, const OutMat &o, float *part, hipStream_t s) {
  const NtPlan p = nt_plan<PA, PB, FP4>(o.rows, o.cols, g.chunks);
  if (p.parts == 1) return nt_kind<PA, PB, FP4>(p.kind, g, o.rows, o.cols, 1, EpiOut{o}, s);
  const int64_t ld = blocks_of(o.cols, 4) * 4;
  const hipError_t e = nt_kind<PA, PB, FP4>(p.kind, g, o.rows, o.cols, p.parts, EpiPart{part, o.rows, ld}, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_join, dim3((unsigned)blocks_of(o.rows * (ld / 4), 256)), dim3(256), 0, s, part, p.parts, o.rows, ld, o);
  return hipGetLastError();
}

static hipError_t launch_planes(const DevMat &x, const DevMat &y, int parts, int64_t chunks, uint8_t *out, hipStream_t s) {
  const int bytes = x.bf16 ? 2 : 4;
  const int vec = rows_aligned(x.p, x.ld, bytes) && (!y.p || rows_aligned(y.p, y.ld, bytes));
  const dim3 grid((unsigned)blocks_of(blocks_of(x.rows, 16) * chunks, 4));
  if (x.bf16) hipLaunchKernelGGL((k_planes<1, true>), grid, dim3(256), 0, s, x, y, vec, chunks, out);
  else hipLaunchKernelGGL((k_planes<3, false>), grid, dim3(256), 0, s, x, y, vec, chunks, out);
  (void)parts;
  return hipGetLastError();
}
static hipError_t launch_planes_t(const DevMat &x, const DevMat &y, int64_t chunks, uint8_t *out, float *sums, hipStream_t s) {
  const dim3 grid((unsigned)(chunks * blocks_of(x.cols, 64)));
  if (x.bf16) hipLaunchKernelGGL((k_planes_t<1, true>), grid, dim3(256), 0, s, x, y, chunks, out, sums);
  else hipLaunchKernelGGL((k_planes_t<3, false>), grid, dim3(256), 0, s, x, y, chunks, out, sums);
  return hipGetLastError();
}

}  // namespace vcr

using namespace vcr;

// ---- the context's room for these calls -------------------------------------------------------
vcr_status op_space(vcr_ctx *c, size_t bytes, Workspace **out) {
  vcr_internal::OpSpace *sp = nullptr;
  for (auto &o : c->op_spaces)
    if (o.stream == c->stream) sp = &o;
  if (!sp) {
    c->op_spaces.emplace_back();
    sp = &c->op_spaces.back();
    sp->stream = c->stream;
  }
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(c->stream, &cap) != hipSuccess) (void)hipGetLastError();
  const bool capturing = cap != hipStreamCaptureStatusNone;
  sp->w.used = 0;
  *out = &sp->w;
  if (sp->w.cap < bytes) {
    if (c->ws_cap > 0 && bytes > c->ws_cap)
      return fail(c, VCR_ERR_OOM, "the call needs %llu bytes of workspace, the cap is %llu", (unsigned long long)bytes,
                  (unsigned long long)c->ws_cap);
    if (capturing)
      return fail(c, VCR_ERR_STATE, "no workspace can be made while the stream is recorded: make the call once before");
    if (sp->w.base) {
      if (sp->held) {
        c->op_retired.push_back(sp->w.base);   // a recorded graph uses it
      } else {
        HIP_TRY(c, hipStreamSynchronize(c->stream));
        (void)hipFree(sp->w.base);
      }
    }
    sp->w = Workspace{};
    sp->held = false;
    void *p = nullptr;
    const hipError_t e = device_alloc(c, &p, bytes);
    if (e != hipSuccess)
      return fail(c, VCR_ERR_OOM, "hipMalloc(%llu) failed: %s", (unsigned long long)bytes, hipGetErrorString(e));
    sp->w.base = static_cast<char *>(p);
    sp->w.cap = bytes;
    uint64_t all = c->ws.cap;
    for (auto &o : c->op_spaces) all += o.w.cap;
    c->peak_ws = std::max<uint64_t>(c->peak_ws, all);
  }
  sp->held |= capturing;
  return VCR_OK;
}

vcr_status op_begin(vcr_ctx *c) {
  if (c->device < 0) return fail(c, VCR_ERR_STATE, "validation-only context");
  HIP_TRY(c, hipSetDevice(c->device));
  return VCR_OK;
}
vcr_status op_end(vcr_ctx *c) {
  if (c->sync_check) HIP_TRY(c, hipStreamSynchronize(c->stream));
  return VCR_OK;
}

vcr_status check_mat(vcr_ctx *c, const vcr_mat *m, const char *name) {
  if (!m) return fail(c, VCR_ERR_ARG, "%s: null", name);
  if (m->type != VCR_F32 && m->type != VCR_BF16) return fail(c, VCR_ERR_ARG, "%s: type %d is not one of VCR_F32, VCR_BF16", name, m->type);
  if (m->rows < 0 || m->cols <= 0 || m->rows > VCR_MAX_NODE_ELEMENTS || m->cols > VCR_MAX_NODE_ELEMENTS)
    return fail(c, VCR_ERR_SHAPE, "%s: %lld x %lld", name, (long long)m->rows, (long long)m->cols);
  if (m->ld < m->cols || m->ld > VCR_MAX_LAYER_WEIGHTS)
    return fail(c, VCR_ERR_SHAPE, "%s: rows of %lld elements with a pitch of %lld", name, (long long)m->cols, (long long)m->ld);
  if (m->rows > 0 && !m->p) return fail(c, VCR_ERR_ARG, "%s: null pointer", name);
  if ((reinterpret_cast<uintptr_t>(m->p) & (m->type == VCR_F32 ? 3 : 1)) != 0)
    return fail(c, VCR_ERR_ARG, "%s: pointer not aligned to its type", name);
  return VCR_OK;
}
static vcr_status check_mx(vcr_ctx *c, const vcr_mx *m, const char *name) {
  if (!m) return fail(c, VCR_ERR_ARG, "%s: null", name);
  if (m->rows < 0 || m->cols <= 0 || m->rows > VCR_MAX_NODE_ELEMENTS || m->cols > VCR_MAX_NODE_ELEMENTS ||
      m->rows * m->cols > VCR_MAX_LAYER_WEIGHTS)
    return fail(c, VCR_ERR_SHAPE, "%s: %lld x %lld", name, (long long)m->rows, (long long)m->cols);
  if (m->rows > 0 && (!m->codes || !m->scales)) return fail(c, VCR_ERR_ARG, "%s: null pointer", name);
  if (((reinterpret_cast<uintptr_t>(m->codes) | reinterpret_cast<uintptr_t>(m->scales)) & 15) != 0)
    return fail(c, VCR_ERR_ARG, "%s: pointers must be 16-byte aligned", name);
  return VCR_OK;
}
static vcr_status check_bias(vcr_ctx *c, const float *b, const char *name) {
  if ((reinterpret_cast<uintptr_t>(b) & 3) != 0) return fail(c, VCR_ERR_ARG, "%s: pointer not aligned to its type", name);
  return VCR_OK;
}
static DevMat dev(const vcr_mat *m) {
  if (!m) return DevMat{nullptr, 0, 0, 0, 0, 0};
  return DevMat{m->p, m->type == VCR_BF16, m->rows, m->cols, m->ld, 0};
}
static MxDev dev(const vcr_mx *m) { return MxDev{m->codes, m->scales, m->rows, m->cols}; }
static OutMat out_mat(const vcr_mat *y, const float *bias, int relu) {
  const int bytes = y->type == VCR_BF16 ? 2 : 4;   // four columns a store
  const bool vec = (reinterpret_cast<uintptr_t>(y->p) & (4 * bytes - 1)) == 0 && y->ld % 4 == 0;
  return OutMat{y->p, y->type == VCR_BF16, vec, y->rows, y->cols, y->ld, bias, relu};
}
#define TRY(expr)                       \
  do {                                  \
    const vcr_status st_ = (expr);      \
    if (st_ != VCR_OK) return st_;      \
  } while (0)

extern "C" {

vcr_status vcr_mx_bytes(int64_t rows, int64_t cols, uint64_t *codes, uint64_t *scales) {
  if (rows < 0 || cols <= 0 || rows > VCR_MAX_NODE_ELEMENTS || cols > VCR_MAX_NODE_ELEMENTS || !codes || !scales)
    return VCR_ERR_ARG;
  const uint64_t rb = (uint64_t)blocks_of(rows, 16), groups = (uint64_t)mx_groups(cols);
  *codes = rb * groups * 1024;
  *scales = rb * ((groups + 3) / 4) * 256;
  return VCR_OK;
}

vcr_status vcr_mx_quantize(vcr_ctx *c, const vcr_mat *x, const vcr_mx *q) {
  if (!c) return VCR_ERR_ARG;
  TRY(check_mat(c, x, "x"));
  TRY(check_mx(c, q, "q"));
  if (x->rows != q->rows || x->cols != q->cols) return fail(c, VCR_ERR_SHAPE, "x and q differ in shape");
  TRY(op_begin(c));
  if (x->rows == 0) return VCR_OK;
  const DevMat d = dev(x);
  const int vec = rows_aligned(d.p, d.ld, d.bf16 ? 2 : 4);
  const int64_t wg = blocks_of(x->rows, 16) * blocks_of(mx_groups(x->cols), 4);
  if (d.bf16) hipLaunchKernelGGL((k_mx_quantize<true>), dim3((unsigned)wg), dim3(256), 0, c->stream, d, vec, q->codes, q->scales);
  else hipLaunchKernelGGL((k_mx_quantize<false>), dim3((unsigned)wg), dim3(256), 0, c->stream, d, vec, q->codes, q->scales);
  HIP_TRY(c, hipGetLastError());
  return op_end(c);
}

vcr_status vcr_mx_dequantize(vcr_ctx *c, const vcr_mx *q, const vcr_mat *y) {
  if (!c) return VCR_ERR_ARG;
  TRY(check_mx(c, q, "q"));
  TRY(check_mat(c, y, "y"));
  if (y->rows != q->rows || y->cols != q->cols) return fail(c, VCR_ERR_SHAPE, "q and y differ in shape");
  TRY(op_begin(c));
  if (y->rows == 0) return VCR_OK;
  const OutMat o = out_mat(y, nullptr, 0);
  const int64_t wg = blocks_of(blocks_of(y->rows, 16) * mx_groups(y->cols), 4);
  if (o.bf16) hipLaunchKernelGGL((k_mx_dequantize<true>), dim3((unsigned)wg), dim3(256), 0, c->stream, dev(q), y->p, y->ld, o.vec);
  else hipLaunchKernelGGL((k_mx_dequantize<false>), dim3((unsigned)wg), dim3(256), 0, c->stream, dev(q), y->p, y->ld, o.vec);
  HIP_TRY(c, hipGetLastError());
  return op_end(c);
}

vcr_status vcr_mx_product(vcr_ctx *c, const vcr_mx *a, const vcr_mx *w, const float *bias, int32_t relu, const vcr_mat *y) {
  if (!c) return VCR_ERR_ARG;
  TRY(check_mx(c, a, "a"));
  TRY(check_mx(c, w, "w"));
  TRY(check_bias(c, bias, "bias"));
  TRY(check_mat(c, y, "y"));
  if (w->rows == 0) return fail(c, VCR_ERR_SHAPE, "w has no rows");
  if (a->cols != w->cols || y->rows != a->rows || y->cols != w->rows)
    return fail(c, VCR_ERR_SHAPE, "y (%lld x %lld) is not a (%lld x %lld) times the transpose of w (%lld x %lld)", (long long)y->rows,
                (long long)y->cols, (long long)a->rows, (long long)a->cols, (long long)w->rows, (long long)w->cols);
  TRY(op_begin(c));
  if (y->rows == 0) return VCR_OK;
  NtArgs g{};
  g.A = NtOperand{a->codes, a->scales, (int32_t)blocks_of(a->rows, 16), 0};
  g.B = NtOperand{w->codes, w->scales, (int32_t)blocks_of(w->rows, 16), 0};
  g.chunks = (int32_t)mx_groups(a->cols);
  Workspace *ws = nullptr;
  const size_t room = nt_plan<1, 1, true>(y->rows, y->cols, g.chunks).part_bytes(y->rows, y->cols);
  TRY(op_space(c, room, &ws));
  HIP_TRY(c, (nt_product<1, 1, true>(g, out_mat(y, bias, relu != 0), reinterpret_cast<float *>(ws->base), c->stream)));
  return op_end(c);
}

vcr_status vcr_mx_linear(vcr_ctx *c, const vcr_mat *x, const vcr_mx *w, const float *bias, int32_t relu, const vcr_mat *y) {
  if (!c) return VCR_ERR_ARG;
  TRY(check_mat(c, x, "x"));
  TRY(check_mx(c, w, "w"));
  TRY(check_bias(c, bias, "bias"));
  TRY(check_mat(c, y, "y"));
  if (w->rows == 0) return fail(c, VCR_ERR_SHAPE, "w has no rows");
  if (x->cols != w->cols || y->rows != x->rows || y->cols != w->rows)
    return fail(c, VCR_ERR_SHAPE, "y (%lld x %lld) is not x (%lld x %lld) times the transpose of w (%lld x %lld)", (long long)y->rows,
                (long long)y->cols, (long long)x->rows, (long long)x->cols, (long long)w->rows, (long long)w->cols);
  TRY(op_begin(c));
  if (y->rows == 0) return VCR_OK;
  const DevMat d = dev(x);
  const int P = d.bf16 ? 1 : 3;
  const int64_t chunks = 4 * mx_groups(x->cols), rb = blocks_of(x->rows, 16), wb = blocks_of(w->rows, 16);
  const NtPlan plan = d.bf16 ? nt_plan<1, 1, false>(y->rows, y->cols, chunks) : nt_plan<3, 1, false>(y->rows, y->cols, chunks);
  const size_t xb = (size_t)rb * chunks * P * FRAG, wbytes = (size_t)wb * chunks * FRAG;
  Workspace *ws = nullptr;
  TRY(op_space(c, al(xb) + al(wbytes) + al(plan.part_bytes(y->rows, y->cols)), &ws));
  uint8_t *xp = take<uint8_t>(*ws, xb), *wp = take<uint8_t>(*ws, wbytes);
  float *part = reinterpret_cast<float *>(ws->base + ws->used);
  HIP_TRY(c, launch_planes(d, dev(static_cast<const vcr_mat *>(nullptr)), P, chunks, xp, c->stream));
  hipLaunchKernelGGL(k_mx_planes, dim3((unsigned)blocks_of(wb * (chunks / 4), 4)), dim3(256), 0, c->stream, dev(w), wp);
  HIP_TRY(c, hipGetLastError());
  NtArgs g{};
  g.A = NtOperand{xp, nullptr, (int32_t)rb, 0};
  g.B = NtOperand{wp, nullptr, (int32_t)wb, 0};
  g.chunks = (int32_t)chunks;
  const OutMat o = out_mat(y, bias, relu != 0);
  if (d.bf16) HIP_TRY(c, (nt_product<1, 1, false>(g, o, part, c->stream)));
  else HIP_TRY(c, (nt_product<3, 1, false>(g, o, part, c->stream)));
  return op_end(c);
}

vcr_status vcr_mx_linear_grad(vcr_ctx *c, const vcr_mat *dy, const vcr_mat *y, const vcr_mat *x, const vcr_mx *w, const vcr_mat *dx,
                              const vcr_mat *dw, float *db) {
  if (!c) return VCR_ERR_ARG;
  TRY(check_mat(c, dy, "dy"));
  if (y) TRY(check_mat(c, y, "y"));
  if (dw && !x) return fail(c, VCR_ERR_ARG, "dw needs x");
  if (dx && !w) return fail(c, VCR_ERR_ARG, "dx needs w");
  if (x) TRY(check_mat(c, x, "x"));
  if (w) TRY(check_mx(c, w, "w"));
  if (dx) TRY(check_mat(c, dx, "dx"));
  if (dw) TRY(check_mat(c, dw, "dw"));
  TRY(check_bias(c, db, "db"));
  const int64_t M = dy->rows, N = dy->cols;
  if (y && (y->rows != M || y->cols != N)) return fail(c, VCR_ERR_SHAPE, "y and dy differ in shape");
  if (y && y->type != dy->type) return fail(c, VCR_ERR_ARG, "y and dy differ in type");
  if (dx && (w->rows != N || dx->rows != M || dx->cols != w->cols)) return fail(c, VCR_ERR_SHAPE, "dx is not dy times w");
  if (dw && (x->rows != M || dw->rows != N || dw->cols != x->cols)) return fail(c, VCR_ERR_SHAPE, "dw is not the transpose of dy times x");
  if (dw && x->type != dy->type) return fail(c, VCR_ERR_ARG, "x and dy differ in type");
  TRY(op_begin(c));
  const DevMat g = dev(dy), mask = dev(y);
  const int P = g.bf16 ? 1 : 3;
  const hipStream_t s = c->stream;
  const int64_t nch = blocks_of(N, 32), mch = blocks_of(std::max<int64_t>(M, 1), 32), mb = blocks_of(M, 16), nb = blocks_of(N, 16);
  const int64_t kx = dx ? w->cols : 1, kw = dw ? x->cols : 1, kxb = blocks_of(kx, 16), kwb = blocks_of(kw, 16);
  const bool has_dx = dx && M > 0;
  size_t b_g = 0, b_wt = 0, b_gt = 0, b_xt = 0, b_sums = 0, b_part = 0;
  if (has_dx) {
    b_g = (size_t)mb * nch * P * FRAG;
    b_wt = (size_t)kxb * nch * FRAG;
    b_part = (P == 1 ? nt_plan<1, 1, false>(M, kx, nch) : nt_plan<3, 1, false>(M, kx, nch)).part_bytes(M, kx);
  }
  if (dw) {
    b_gt = (size_t)nb * mch * P * FRAG;
    b_xt = (size_t)kwb * mch * P * FRAG;
    b_part = std::max(b_part, (P == 1 ? nt_plan<1, 1, false>(N, kw, mch) : nt_plan<3, 3, false>(N, kw, mch)).part_bytes(N, kw));
  }
  if (db) b_sums = (size_t)mch * N * 4;
  Workspace *ws = nullptr;
  TRY(op_space(c, al(b_g) + al(b_wt) + al(b_gt) + al(b_xt) + al(b_sums) + al(b_part) + 6 * 256, &ws));
  uint8_t *gp = take<uint8_t>(*ws, b_g), *wt = take<uint8_t>(*ws, b_wt), *gt = take<uint8_t>(*ws, b_gt), *xt = take<uint8_t>(*ws, b_xt);
  float *sums = take<float>(*ws, b_sums / 4), *part = take<float>(*ws, b_part / 4);
  const DevMat none = dev(static_cast<const vcr_mat *>(nullptr));
  if (has_dx) {
    HIP_TRY(c, launch_planes(g, mask, P, nch, gp, s));
    hipLaunchKernelGGL(k_mx_planes_t, dim3((unsigned)blocks_of(4 * nch * 4 * mx_groups(kx), 256)), dim3(256), 0, s, dev(w), nch, kxb, wt);
    HIP_TRY(c, hipGetLastError());
    NtArgs a{};
    a.A = NtOperand{gp, nullptr, (int32_t)mb, 0};
    a.B = NtOperand{wt, nullptr, (int32_t)kxb, 0};
    a.chunks = (int32_t)nch;
    const OutMat o = out_mat(dx, nullptr, 0);
    if (P == 1) HIP_TRY(c, (nt_product<1, 1, false>(a, o, part, s)));
    else HIP_TRY(c, (nt_product<3, 1, false>(a, o, part, s)));
  }
  if (dw || db) {
    HIP_TRY(c, launch_planes_t(g, mask, mch, dw ? gt : nullptr, db ? sums : nullptr, s));
    if (db) {
      hipLaunchKernelGGL(k_column_sums, dim3((unsigned)blocks_of(N, 256)), dim3(256), 0, s, sums, mch, N, db);
      HIP_TRY(c, hipGetLastError());
    }
  }
  if (dw) {
    HIP_TRY(c, launch_planes_t(dev(x), none, mch, xt, nullptr, s));
    NtArgs a{};
    a.A = NtOperand{gt, nullptr, (int32_t)nb, 0};
    a.B = NtOperand{xt, nullptr, (int32_t)kwb, 0};
    a.chunks = (int32_t)mch;
    const OutMat o = out_mat(dw, nullptr, 0);
    if (P == 1) HIP_TRY(c, (nt_product<1, 1, false>(a, o, part, s)));
    else HIP_TRY(c, (nt_product<3, 3, false>(a, o, part, s)));
  }
  return op_end(c);
}

}  // extern "C"
