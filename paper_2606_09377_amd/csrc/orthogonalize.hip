// Orthogonalised updates of layers' weights by Newton-Schulz products: vcr_orthogonalize of vcrown.h.
//
// With X = G / (|G| + eps) (Frobenius norm; G transposed where it is taller than wide, so X is m x n, m <= n),
// every step is  A = X X^T,  Q = a I + b A + c A A,  X <- Q X,  which takes each singular value s of X to
// s (a + b s^2 + c s^4) and so all of them towards 1.
//
// A and Q are symmetric: of their 16 x 16 blocks those on and below the diagonal are computed and
// stored twice.  A step is 3 m^2 n + m^3 multiply-adds that way (of 4 m^2 n + 2 m^3).  All three products
// contract the contiguous axes of operands in the layout of nt.h: X (rows m) and its transpose (rows
// n) are both kept, written by the epilogue that makes them.  X, A and Q are held in three bf16 parts, float32's accuracy, whatever
// the result's type: what one step rounds, the later ones raise by up to a = 3.4 each in the directions that the update has little
// or nothing of.  (With two parts, 2^-17, a bf16 result of a 300 x 500 update of rank 1 is off by 2.8e-3 after five steps and
// 6e-2 after eight, where its own rounding is 1.7e-3.)
//
// A bf16 update is exact in one part, times a power of two: the first step multiplies one part where the later ones take three.
//
// Bound by the matrix instructions where the update is large (8192 x 8192, bf16, five steps in 44 to 45 ms: 60 TFLOP of partial
// products at 1.33 to 1.36 PFLOP/s), by the operands the epilogues write and the tiles' last rounds at 1024 (five float32 1024 x 1024 in 0.75 ms: a
// step's three launches take 43, 46 and 62 us, of which 12 write X twice), and by the starts and ends of fifteen launches of 12
// to 21 us on 777 x 1500.
#include <algorithm>
#include <cmath>

#include "layers.h"
#include "planes.h"

namespace vcr {

constexpr int NORM_PARTS = 1024;   // partial sums of a matrix's squares
constexpr int P = 3;               // parts of X, A and Q
constexpr int first_parts(bool bf16) { return bf16 ? 1 : P; }   // of the first step's X

// Sums of squares in 64 bits (float32's range does not hold the squares of all its values): a wave per stretch of 512
// columns of a row.  Bound by memory: a bf16 8192 x 8192 update, 134 MB, in 32 us.
template <bool BF>
__global__ __launch_bounds__(256) void k_ns_norm(DevMat g, int vec, double *part) {
  __shared__ double sh[4];
  const int lane = threadIdx.x & 63;
  const int64_t base = (int64_t)blockIdx.y * g.stride, per = (g.cols + 511) / 512, total = g.rows * per;
  double s = 0.0;
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < total; i += NORM_PARTS * 4) {
    const int64_t r = i / per;
    float v[8];
    mat_row8<BF>(g, base, r, (i - r * per) * 512 + lane * 8, vec, v);
#pragma unroll
    for (int q = 0; q < 8; ++q) s = fma((double)v[q], (double)v[q], s);
  }
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if (lane == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) part[blockIdx.y * NORM_PARTS + blockIdx.x] = (sh[0] + sh[1]) + (sh[2] + sh[3]);
}
// 1 / (norm + eps) = two[0] two[1] rest, by every wave: powers of two, whose product float32 may not hold (norms of finite
// matrices lie in 2^-149 .. 2^144), and a rest in [1, 2).  Where it is no finite number above 0 it is the rest.
struct NsScale {
  float two[2], rest;
};
__device__ __forceinline__ NsScale ns_scale(const double *part, int batch, float eps) {
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < NORM_PARTS / 64; ++i) s += part[batch * NORM_PARTS + i * 64 + (threadIdx.x & 63)];
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  const double f = 1.0 / (sqrt(s) + (double)eps);
  if (!(f > 0.0 && f <= 0x1p200)) return NsScale{{1.f, 1.f}, (float)f};
  const int e = ilogb(f), e0 = min(max(e, -100), 100);
  return NsScale{{ldexpf(1.f, e0), ldexpf(1.f, e - e0)}, (float)ldexp(f, -e)};
}

// X's parts from G, its rows' and its columns' (bf16 8192 x 8192, 403 MB with what it writes, in
// 95 to 104 us).  A bf16 G as it is, times the power of two that brings its norm near 1: exact in one part, so that the first step
// multiplies one part; the rest of the factor is left to its epilogues (scale[batch]).
template <bool BF>
__global__ __launch_bounds__(256) void k_ns_planes(PlanesArgs g, int64_t col_tiles, const double *part, float eps, float *scale) {
  constexpr int P0 = first_parts(BF);
  __shared__ float tile[64][65];
  const NsScale sc = ns_scale(part, blockIdx.y, eps);
  if (BF && blockIdx.x == 0 && threadIdx.x == 0) scale[blockIdx.y] = sc.rest;
  const int64_t tr = blockIdx.x / col_tiles, bytes = g.row_blocks * g.row_chunks * P0 * FRAG;   // of either
  g.rows += blockIdx.y * bytes;
  g.cols += blockIdx.y * bytes;
  planes_tile<P0, BF>(g, (int64_t)blockIdx.y * g.x.stride, tr, blockIdx.x - tr * col_tiles,
                      PlanesScale{{sc.two[0], sc.two[1]}, BF ? 1.f : sc.rest}, tile);
}

enum NsMode : int32_t { NS_GRAM = 0, NS_POLY = 1, NS_UPDATE = 2, NS_OUT = 3 };

// Epilogue of a step's three products; mp x np the padded sizes
struct NsEpilogue {
  int32_t mp, np;
  uint8_t *dst, *dst_t;        // [mp][mp] (gram, poly); X [mp][np] and its transpose (update)
  const uint8_t *gram;         // poly
  float a, b, c;
  // out = keep base + gain X, transposed back where the update is
  DevMat base;
  void *out;
  int64_t out_rows, out_cols, out_ld, out_stride;
  float keep, gain;
  int32_t out_bf16, vec, transposed;
  const float *scale;   // FIRST: of X in its product (gram: of both factors)
};
template <int MODE, bool FIRST = false>
struct EpiNs : NsEpilogue {
  __device__ __forceinline__ void store(int batch, int, int m, int n, f32v4 v, int lane) const {
    const int bm = m >> 4, bn = n >> 4, r = lane & 15;
    // after a transposition the lane holds row nt, columns mt .. mt + 3
    const int nt = n + (r & 3), mt = (m & ~3);
    if constexpr (FIRST && MODE != NS_POLY) {
      const float s = scale[batch];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = MODE == NS_GRAM ? v[i] * s * s : v[i] * s;
    }
    if constexpr (MODE <= NS_POLY) {
      if (bm * 16 >= mp || bn > bm) return;   // wave-uniform
      const int64_t off = (int64_t)batch * (mp / 16) * (mp / 32) * P * FRAG;
      if constexpr (MODE == NS_POLY) {
        const f32v4 q = load_quad<P>(gram + off, m, n, mp / 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fmaf(c, v[i], fmaf(b, q[i], m == n + i ? a : 0.f));
      }
      store_quad<P>(dst + off, m, n, mp / 32, v);
      if (bm != bn) store_quad<P>(dst + off, nt, mt, mp / 32, quad_transpose(v, lane));
    } else if (bm * 16 >= mp || bn * 16 >= np) {
      return;
    } else if constexpr (MODE == NS_UPDATE) {
      const int64_t off = (int64_t)batch * (mp / 16) * (np / 32) * P * FRAG;
      store_quad<P>(dst + off, m, n, np / 32, v);
      store_quad<P>(dst_t + off, nt, mt, mp / 32, quad_transpose(v, lane));
    } else {
      if (transposed) v = quad_transpose(v, lane);
      const int64_t row = transposed ? nt : m, col = transposed ? mt : n;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] *= gain;
        if (base.p && row < out_rows && col + i < out_cols) {
          const int64_t at = batch * base.stride + row * base.ld + col + i;
          const float w = base.bf16 ? bf16_value(static_cast<const uint16_t *>(base.p)[at]) : static_cast<const float *>(base.p)[at];
          v[i] = fmaf(keep, w, v[i]);
        }
      }
      store_row4(static_cast<char *>(out) + batch * out_stride * (out_bf16 ? 2 : 4), out_bf16, out_ld, out_rows, out_cols, vec, row, col, v);
    }
  }
};

struct NsSpace {
  double *norm;
  float *scale;
  uint8_t *x, *xt, *x2, *xt2, *gram, *poly;
};
static NsSpace ns_carve(Workspace &w, int64_t mp, int64_t np, int batch) {
  NsSpace s;
  const size_t bx = (size_t)batch * mp * np * 2 * P, bg = (size_t)batch * mp * mp * 2 * P;
  s.norm = take<double>(w, (size_t)batch * NORM_PARTS);
  s.scale = take<float>(w, (size_t)batch);
  s.x = take<uint8_t>(w, bx);
  s.xt = take<uint8_t>(w, bx);
  s.x2 = take<uint8_t>(w, bx);
  s.xt2 = take<uint8_t>(w, bx);
  s.gram = take<uint8_t>(w, bg);
  s.poly = take<uint8_t>(w, bg);
  return s;
}

template <bool BF>
static hipError_t ns_run(const DevMat &g, int batch, int64_t mp, int64_t np, bool transposed, int steps, NsEpilogue e, float eps,
                         NsSpace sp, hipStream_t s) {
  const int vec = rows_aligned(g.p, g.ld, BF ? 2 : 4) && (g.stride * (BF ? 2 : 4)) % 16 == 0;
  hipLaunchKernelGGL((k_ns_norm<BF>), dim3(NORM_PARTS, batch), dim3(256), 0, s, g, vec, sp.norm);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  // G's rows padded to rp, its columns to cp
  const int64_t rp = transposed ? np : mp, cp = transposed ? mp : np;
  uint8_t *rows = transposed ? sp.xt : sp.x, *cols = transposed ? sp.x : sp.xt;
  PlanesArgs pl{};
  pl.x = g;
  pl.vec = vec;
  pl.rows = rows;
  pl.row_blocks = rp / 16;
  pl.row_chunks = cp / 32;
  pl.cols = cols;
  pl.col_blocks = cp / 16;
  pl.col_chunks = rp / 32;
  const int64_t ct = blocks_of(cp, 64);
  constexpr int P0 = first_parts(BF);
  hipLaunchKernelGGL((k_ns_planes<BF>), dim3((unsigned)(blocks_of(rp, 64) * ct), batch), dim3(256), 0, s, pl, ct, sp.norm, eps, sp.scale);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  e.mp = (int32_t)mp;
  e.np = (int32_t)np;
  e.scale = sp.scale;
  const int64_t sg = mp * mp * 2 * P;
  auto step = [&](auto first, bool last) {   // first: of a bf16 G, whose X has one part
    constexpr bool FIRST = decltype(first)::value;
    constexpr int PX = FIRST ? P0 : P;
    const int64_t sx0 = mp * np * 2 * PX;
    hipError_t err;
    NtArgs a{};
    a.A = a.B = NtOperand{sp.x, nullptr, (int32_t)(mp / 16), sx0};
    a.chunks = (int32_t)(np / 32);
    a.tri = 1;
    e.dst = sp.gram;
    if ((err = launch_nt_plan<NtTiles<PX, PX, NT_BF16>>(a, mp, mp, batch, 4.f * P, EpiNs<NS_GRAM, FIRST>{e}, s)) != hipSuccess) return err;
    a.A = a.B = NtOperand{sp.gram, nullptr, (int32_t)(mp / 16), sg};
    a.chunks = (int32_t)(mp / 32);
    e.gram = sp.gram;
    e.dst = sp.poly;
    if ((err = launch_nt_plan<NtTiles<P, P, NT_BF16>>(a, mp, mp, batch, 4.f * P, EpiNs<NS_POLY>{e}, s)) != hipSuccess) return err;
    a.A = NtOperand{sp.poly, nullptr, (int32_t)(mp / 16), sg};
    a.B = NtOperand{sp.xt, nullptr, (int32_t)(np / 16), sx0};
    a.tri = 0;
    e.dst = sp.x2;
    e.dst_t = sp.xt2;
    std::swap(sp.x, sp.x2);
    std::swap(sp.xt, sp.xt2);
    return last ? launch_nt_plan<NtTiles<P, PX, NT_BF16>>(a, mp, np, batch, e.base.p ? 8.f : 4.f, EpiNs<NS_OUT, FIRST>{e}, s)
                : launch_nt_plan<NtTiles<P, PX, NT_BF16>>(a, mp, np, batch, 4.f * P, EpiNs<NS_UPDATE, FIRST>{e}, s);
  };
  for (int i = 0; i < steps; ++i) {
    err = BF && i == 0 ? step(std::integral_constant<bool, BF>{}, i + 1 == steps) : step(std::false_type{}, i + 1 == steps);
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace vcr

using namespace vcr;

extern "C" vcr_status vcr_orthogonalize(vcr_ctx *c, const vcr_mat *g, int32_t count, int64_t g_stride, const vcr_ns_opts *o,
                                        const vcr_mat *base, int64_t base_stride, const vcr_mat *out, int64_t out_stride) {
  if (!c) return VCR_ERR_ARG;
  vcr_status st;
  if ((st = check_mat(c, g, "g")) != VCR_OK || (st = check_mat(c, out, "out")) != VCR_OK) return st;
  if (base && (st = check_mat(c, base, "base")) != VCR_OK) return st;
  if (!o) return fail(c, VCR_ERR_ARG, "opts: null");
  if (count < 0 || count > 65535) return fail(c, VCR_ERR_ARG, "count %d is not in [0, 65535]", count);
  if (o->steps < 1 || o->steps > 100) return fail(c, VCR_ERR_ARG, "steps %d is not in [1, 100]", o->steps);
  const float vals[] = {o->a, o->b, o->c, o->eps, o->gain, o->keep};
  for (float v : vals)
    if (!std::isfinite(v)) return fail(c, VCR_ERR_ARG, "an option is not finite");
  if (o->eps < 0.f) return fail(c, VCR_ERR_ARG, "eps < 0");
  if (out->rows != g->rows || out->cols != g->cols || (base && (base->rows != g->rows || base->cols != g->cols)))
    return fail(c, VCR_ERR_SHAPE, "g, base and out differ in shape");
  if (g->rows * g->cols > VCR_MAX_LAYER_WEIGHTS)
    return fail(c, VCR_ERR_SHAPE, "%lld x %lld exceeds the limit of %lld weights", (long long)g->rows, (long long)g->cols,
                (long long)VCR_MAX_LAYER_WEIGHTS);
  if ((st = check_contraction(c, std::max(g->rows, g->cols))) != VCR_OK) return st;
  auto span = [](const vcr_mat *m) { return m->rows > 0 ? (m->rows - 1) * m->ld + m->cols : 0; };
  if (count > 1 && (g_stride < span(g) || out_stride < span(out) || (base && base_stride < span(base))))
    return fail(c, VCR_ERR_SHAPE, "matrices of a batch overlap");
  if ((st = op_begin(c)) != VCR_OK) return st;
  if (count == 0 || g->rows == 0) return VCR_OK;
  const bool tr = g->rows > g->cols, bf = g->type == VCR_BF16;
  const int64_t mp = blocks_of(std::min(g->rows, g->cols), 32) * 32, np = blocks_of(std::max(g->rows, g->cols), 32) * 32;
  Workspace size;
  (void)ns_carve(size, mp, np, count);
  Workspace *ws = nullptr;
  if ((st = op_space(c, size.used, &ws)) != VCR_OK) return st;
  const NsSpace sp = ns_carve(*ws, mp, np, count);
  const DevMat d{g->p, bf, g->rows, g->cols, g->ld, g_stride};
  NsEpilogue e{};
  e.a = o->a;
  e.b = o->b;
  e.c = o->c;
  e.base = base ? DevMat{base->p, base->type == VCR_BF16, base->rows, base->cols, base->ld, base_stride} : DevMat{};
  e.out = out->p;
  e.out_rows = out->rows;
  e.out_cols = out->cols;
  e.out_ld = out->ld;
  e.out_stride = out_stride;
  e.keep = o->keep;
  e.gain = o->gain;
  e.out_bf16 = out->type == VCR_BF16;
  e.vec = (reinterpret_cast<uintptr_t>(out->p) & (e.out_bf16 ? 7 : 15)) == 0 && out->ld % 4 == 0 && out_stride % 4 == 0;
  e.transposed = tr;
  HIP_TRY(c, bf ? ns_run<true>(d, count, mp, np, tr, o->steps, e, o->eps, sp, c->stream)
                : ns_run<false>(d, count, mp, np, tr, o->steps, e, o->eps, sp, c->stream));
  return op_end(c);
}
