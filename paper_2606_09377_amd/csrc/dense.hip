// Layers in float: the product with its bias, activation, dropout and residual, and its gradients.  vcr_linear and
// vcr_linear_grad of vcrown.h.
//
//   z = x w^T + b,  y = D(act(z)) + residual;   g = D(dy) act'(z),  dx = g w + add,  dw = g^T x,  db = sum g.
//
// The products are nt.h's, on matrix instructions.  bf16 matrices go into the tiles as they are stored (rows aligned to 16 bytes; the
// gradients' operands are transposed on the way out of LDS), others are laid out in the instructions' order first, bf16 values in one part,
// float32 ones in three (their six partial products keep float32's accuracy).  Dropout's factor is left out of g and
// multiplies the sums, so that a bf16 g is dy itself or zero behind ReLU.  Behind GELU and SiLU g = dy act'(z) has more bits than dy, and is rounded to bf16 for both
// products, as dy was when its layer wrote it: results are then off by 2.3e-3 of themselves instead of the 1.7e-3 that their own rounding costs.  In two
// parts it would double the products' instructions, which are what bounds them; float32 operands keep all bits.  db takes g unrounded.
//
// 4096 x 8192 x 8192 in bf16 is bound by the matrix instructions and what feeds them: y alone 364 us (1.51 PFLOP/s; a library product 345), with all that the
// epilogue does 434; dx 371 and dw 399 (library 396 and 471), both with db behind ReLU and dropout 818.  Few rows are bound by reading the weights: one bf16 row of
// 8192 x 8192 takes 22 us in the kernel, 6.1 TB/s.
#include <algorithm>

#include "products.h"
#include "training.h"

namespace vcr {

// ---- where results go -------------------------------------------------------------------------
// Eight columns of a row at a time, from a tile's rows in LDS (nt.h), so that every access is 16 or 32 bytes.  The sums are rounded once, to y (and z); bias,
// activation, dropout and residual cost no pass of their own.  (4096 x 8192 x 8192 in bf16: 364 us with nothing here, 370 with bias and ReLU, 406 with
// bias and GELU, whose error function no product hides, since a large tile has its compute unit to itself; 434 with bias, ReLU, dropout,
// residual and z, 134 MB more and 4 M Philox outputs.)
struct DenseOut {
  static constexpr bool STAGED = true;
  MatRef y, z, res;
  const float *bias;   // or null
  int64_t rows, cols;
  int32_t act;
  float factor;        // of the sums
  DropDev drop;
  float bytes() const { return (y.bf16 ? 2.f : 4.f) + (z.p ? z.bf16 ? 2.f : 4.f : 0.f) + (res.p ? res.bf16 ? 2.f : 4.f : 0.f); }
  struct Col {
    float bias[8];
    uint64_t offset;
  };
  __device__ __forceinline__ Col col(int64_t n) const {
    Col c;
#pragma unroll
    for (int i = 0; i < 8; ++i) c.bias[i] = 0.f;
    if (bias) {
      if (n + 8 <= cols) {
        __builtin_memcpy(c.bias, __builtin_assume_aligned(bias + n, 4), 32);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (n + i < cols) c.bias[i] = bias[n + i];
      }
    }
    c.offset = drop.k ? drop_offset(drop) : 0;
    return c;
  }
  __device__ __forceinline__ void store8(int64_t m, int64_t n, float (&v)[8], const Col &c) const {
    if (m >= rows || n >= cols) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf(v[i], factor, c.bias[i]);
    if (z.p) save8(z, m, n, cols, v);
    if (act != VCR_ACT_NONE) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = act_value(act, v[i]);
    }
    if (drop.k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= drop.factor;
      drop8(drop, c.offset, m, n, v);
    }
    if (res.p) {
      float a[8];
      load8(res, m, n, cols, a);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += a[i];
    }
    save8(y, m, n, cols, v);
  }
};

// ---- operands ---------------------------------------------------------------------------------
// Up to three matrices of one type laid out in a launch, 64 x 64 values a workgroup; the first one may be a gradient, whose
// values are those kept by dropout times the activation's slope.  Bound by memory: float32 2001 x 1000 and 1500 x 1000, 14 MB in and 21 MB out, 8.5 us.
struct GradSource {
  MatRef z;
  int32_t act;
  DropDev drop;
};
struct PlanesOf {
  PlanesArgs p;
  int64_t col_tiles, tiles;
};
template <int P, bool BF>
__global__ __launch_bounds__(256) void k_dense_planes(PlanesOf a, PlanesOf b, PlanesOf c, GradSource src, int64_t first) {
  __shared__ float tile[64][65];
  int64_t id = first + blockIdx.x;
  const bool is_a = id < a.tiles, is_b = !is_a && id < a.tiles + b.tiles;   // uniform
  id -= is_a ? 0 : is_b ? a.tiles : a.tiles + b.tiles;
  const PlanesArgs &p = is_a ? a.p : is_b ? b.p : c.p;
  const int64_t ct = is_a ? a.col_tiles : is_b ? b.col_tiles : c.col_tiles, tr = id / ct, tc = id - tr * ct;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t row = (tr * 4 + wave) * 16 + (lane & 15);
  float v[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t col = tc * 64 + h * 32 + (lane >> 4) * 8;
    mat_row8<BF>(p.x, 0, row, col, p.vec, v[h]);
    if (is_a && row < p.x.rows && col < p.x.cols) {
      if (src.act != VCR_ACT_NONE) {
        float z[8];
        load8(src.z, row, col, p.x.cols, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[h][i] = src.act == VCR_ACT_RELU ? (z[i] > 0.f ? v[h][i] : 0.f) : v[h][i] * act_slope(src.act, z[i]);
      }
      if (src.drop.k) drop8(src.drop, drop_offset(src.drop), row, col, v[h]);
    }
    planes_rows<P>(p, tr, tc, h, v[h]);
  }
  planes_cols<P>(p, tr, tc, v, tile);
}
// g = the kept values of dy times the activation's slope as rows of bf16 (out null: not stored), and the sums of its columns over every 64
// rows, sums [group][cols] (null: none; of one group: times `factor`, what is asked for).  A workgroup takes 64 x 64 values, a
// thread eight columns of two rows.  Bound by memory: 4096 x 8192 with ReLU and dropout, 201 MB, 49 us (4.1 TB/s).
__global__ __launch_bounds__(256) void k_grad_rows(DevMat dy, int vec, GradSource src, uint16_t *out, int64_t pitch, float *sums, float factor, int64_t first) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, oct = threadIdx.x & 7;
  const int64_t ct = (dy.cols + 63) / 64, id = first + blockIdx.x, tr = id / ct, tc = id - tr * ct, col = tc * 64 + oct * 8, row0 = tr * 64 + (threadIdx.x >> 3);
  float v[2][8], z[2][8];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    mat_row8<true>(dy, 0, row0 + 32 * i, col, vec, v[i]);
    if (src.act != VCR_ACT_NONE && row0 + 32 * i < dy.rows && col < dy.cols) load8(src.z, row0 + 32 * i, col, dy.cols, z[i]);
  }
  const uint64_t offset = src.drop.k ? drop_offset(src.drop) : 0;
  float s[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) s[k] = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int64_t row = row0 + 32 * i;
    if (row >= dy.rows || col >= dy.cols) continue;
    if (src.act != VCR_ACT_NONE) {
#pragma unroll
      for (int k = 0; k < 8; ++k) v[i][k] = src.act == VCR_ACT_RELU ? (z[i][k] > 0.f ? v[i][k] : 0.f) : v[i][k] * act_slope(src.act, z[i][k]);
    }
    if (src.drop.k) drop8(src.drop, offset, row, col, v[i]);
    if (out) *reinterpret_cast<uint4 *>(out + row * pitch + col) = pack8(v[i]);   // (zeros beyond the columns, up to the pitch)
#pragma unroll
    for (int k = 0; k < 8; ++k) s[k] += v[i][k];
  }
  if (!sums) return;   // uniform
#pragma unroll
  for (int k = 0; k < 8; ++k) {   // over a wave's 8 rows
    s[k] += __shfl_xor(s[k], 8);
    s[k] += __shfl_xor(s[k], 16);
    s[k] += __shfl_xor(s[k], 32);
  }
  if (lane < 8) {
#pragma unroll
    for (int k = 0; k < 8; ++k) part[wave][lane * 8 + k] = s[k];
  }
  __syncthreads();
  const int64_t c = tc * 64 + threadIdx.x;
  if (threadIdx.x < 64 && c < dy.cols)
    sums[tr * dy.cols + c] = factor * ((part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]));
}
static PlanesOf planes_of(const PlanesArgs *p) {
  PlanesOf o{};
  if (!p) return o;
  o.p = *p;
  o.p.vec = rows_aligned(p->x.p, p->x.ld, p->x.bf16 ? 2 : 4);
  // tiles of 64 rows and columns, those of the padding among them
  o.col_tiles = std::max(blocks_of(p->x.cols, 64), p->rows ? blocks_of(p->row_chunks, 2) : 0);
  o.tiles = std::max(blocks_of(p->x.rows, 64), p->cols ? blocks_of(p->col_chunks, 2) : 0) * o.col_tiles;
  return o;
}
static hipError_t launch_dense_planes(const PlanesArgs *a, const PlanesArgs *b, const PlanesArgs *c, const GradSource &src, bool bf16, hipStream_t s) {
  const PlanesOf pa = planes_of(a), pb = planes_of(b), pc = planes_of(c);
  return launch_stretches(pa.tiles + pb.tiles + pc.tiles, [&](int64_t first, dim3 grid) {
    if (bf16) hipLaunchKernelGGL((k_dense_planes<1, true>), grid, dim3(256), 0, s, pa, pb, pc, src, first);
    else hipLaunchKernelGGL((k_dense_planes<3, false>), grid, dim3(256), 0, s, pa, pb, pc, src, first);
  });
}

// Three parts of eight values, plainly split; `top` is raised to their largest magnitude.  The plain split is wrong where a finite value rounds to
// infinity alone (an infinite or NaN one makes its small products NaN, and the large one, which is then infinite or NaN, is the result):
// a wave that finds `top` so large takes its sums again with ANY, parts_of<3>.  (A question with every eight values, and the other way's code beside each,
// outgrew the instruction cache: 64 x 1024 x 1024 took 16 us asked for every pair, its dx 14.5 asked for every eight.)
constexpr float PLAIN_SPLIT = 0x1.ffp127f;   // below
template <bool ANY>
__device__ __forceinline__ void parts8(const float (&v)[8], bf16x8 (&out)[3], float &top) {
  uint32_t w[4][3];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (ANY) {
      parts_of<3>(v[2 * i], v[2 * i + 1], w[i]);
    } else {
      top = fmaxf(fmaxf(fabsf(v[2 * i]), fabsf(v[2 * i + 1])), top);
      split_pair(v[2 * i], v[2 * i + 1], w[i][0], w[i][1], w[i][2]);
    }
  }
#pragma unroll
  for (int p = 0; p < 3; ++p) out[p] = __builtin_bit_cast(bf16x8, make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]));
}
// db = factor times the sums of the columns' groups of 64 rows: a workgroup takes 64 columns, a wave every fourth group (64 groups of 8192 columns: 5 us,
// a launch and its reads' latency)
struct ColumnSums {
  const float *sums;
  int64_t groups, cols;
  float factor;
  float *out;   // or null
};
__device__ __forceinline__ void column_sums(const ColumnSums &g, int64_t block, float *lds) {   // lds: 256 floats (waves beyond four have nothing to do)
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = block * 64 + lane;
  float s = 0.f;
  if (wave < 4) {
#pragma unroll 8
    for (int64_t p = wave; p < g.groups; p += 4) s += c < g.cols ? g.sums[p * g.cols + c] : 0.f;
    lds[threadIdx.x] = s;
  }
  __syncthreads();
  if (wave == 0 && c < g.cols) g.out[c] = g.factor * ((lds[lane] + lds[64 + lane]) + (lds[128 + lane] + lds[192 + lane]));
}
__global__ __launch_bounds__(256) void k_dense_sums(ColumnSums g) {
  __shared__ float lds[256];
  column_sums(g, blockIdx.x, lds);
}

// ---- both gradients in one launch -------------------------------------------------------------
// Two products of small tiles and the columns' sums, where the launches would take longer than their work: workgroups
// of one after those of the other.  (us a call, together and apart: bf16 512 x 1024 x 1024 15.0 and 21.1, 512 x 2048 x 2048 32.7 and 28.3; float32
// 128 x 2048 x 2048 36.4 and 38.7, 128 x 4096 x 4096 117.8 and 108.4.)
template <class TA, class TB>
__global__ __launch_bounds__(TA::T, 2) void k_dense_pair(const NtArgs ga, const EpiOut<DenseOut> ea, int na, const NtArgs gb, const EpiOut<DenseOut> eb, int nb,
                                                         ColumnSums sums) {
  static_assert(TA::T == 256 && TB::T == 256, "workgroups of both");
  __shared__ __attribute__((aligned(16))) uint8_t lds[TA::LDS > TB::LDS ? TA::LDS : TB::LDS];
  const int id = blockIdx.x;
  if (id < na) nt_run<TA>(ga, ea, lds, id, na, 0);
  else if (id < na + nb) nt_run<TB>(gb, eb, lds, id - na, nb, 0);
  else column_sums(sums, id - na - nb, reinterpret_cast<float *>(lds));
}
// dx of up to 64 float32 rows (MT row blocks) from g's rows as an operand and w as it is stored: laid out for the tiles, w would be moved four times.  A
// workgroup takes 32 columns of w and all its rows, its 8 waves chunks of 32 rows in turn, each with the next one's loads in flight.  A lane has two
// columns of eight rows, which are the even and the odd columns of two blocks of the matrix instruction: it reads them
// across the rows, 128 bytes of each together, and splits them in registers.  Sums of the waves are added in LDS, in order.
// 64 x 1024 x 1024 takes 11.4 us, dw's tiles and db in the same launch (12.3 with 4 waves): a wave's chunks one after another, each 48
// matrix instructions and two splits behind its loads.
template <int MT>
__device__ __forceinline__ void few_dx(const uint8_t *gp, int nch, const DevMat &w, const DenseOut &o, uint8_t *lds, int64_t block) {
  const int lane = threadIdx.x & 63, r16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (two columns or more: vcr_linear_grad.  Columns beyond the last lie where they are read without a branch and are not stored)
  const int K = (int)w.cols, N = (int)w.rows, k0 = (int)block * 32, kc = min(k0 + 2 * r16, K - 2);
  const bool second = k0 + 2 * r16 == K - 1;   // the first of the lane's columns is the second one read
  const float *wp = static_cast<const float *>(w.p) + kc;
  struct Chunk {
    float w[8][2];
    bf16x8 a[MT][3];
  };
  auto load = [&](Chunk &q, int ch) {
#pragma unroll
    for (int e = 0; e < 8; ++e) __builtin_memcpy(q.w[e], __builtin_assume_aligned(wp + min(ch * 32 + 8 * g4 + e, N - 1) * w.ld, 4), 8);
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int p = 0; p < 3; ++p) q.a[t][p] = *reinterpret_cast<const bf16x8 *>(gp + (((int64_t)t * nch + ch) * 3 + p) * FRAG + lane * 16);
  };
  f32v4 hi[MT][2], lo[MT][2];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int b = 0; b < 2; ++b) hi[t][b] = lo[t][b] = f32v4{0.f, 0.f, 0.f, 0.f};
  float top = 0.f;
  auto use = [&](const Chunk &q, int ch, auto any) {
    const int left = N - ch * 32 - 8 * g4;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      float c[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = e < left ? b == 0 && !second ? q.w[e][0] : q.w[e][1] : 0.f;
      bf16x8 v[3];
      parts8<decltype(any)::value>(c, v, top);
      constexpr int pa[5] = {0, 2, 1, 0, 1}, pb[5] = {2, 0, 1, 1, 0};   // (nt.h)
#pragma unroll
      for (int p = 0; p < 5; ++p)   // (the row blocks' sums in turn: one's would wait for each other)
#pragma unroll
        for (int t = 0; t < MT; ++t) lo[t][b] = mfma_bf16(v[pb[p]], q.a[t][pa[p]], lo[t][b]);
#pragma unroll
      for (int t = 0; t < MT; ++t) hi[t][b] = mfma_bf16(v[0], q.a[t][0], hi[t][b]);
    }
  };
  const std::false_type plain{};
  Chunk q[2];
  int ch = wave;
  if (ch < nch) load(q[0], ch);
  for (; ch < nch; ch += 16) {
    if (ch + 8 < nch) load(q[1], ch + 8);
    use(q[0], ch, plain);
    if (ch + 16 < nch) load(q[0], ch + 16);
    if (ch + 8 < nch) use(q[1], ch + 8, plain);
  }
  if (__builtin_expect(__any(top >= PLAIN_SPLIT), 0)) {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int b = 0; b < 2; ++b) hi[t][b] = lo[t][b] = f32v4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (ch = wave; ch < nch; ch += 8) {
      load(q[0], ch);
      use(q[0], ch, std::true_type{});
    }
  }
  f32v4 *red = reinterpret_cast<f32v4 *>(lds);   // [wave][row block][block][lane]
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      f32v4 v = hi[t][b];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = fabsf(v[i]) < __builtin_huge_valf() ? v[i] + lo[t][b][i] : v[i];
      red[((wave * MT + t) * 2 + b) * 64 + lane] = v;
    }
  __syncthreads();
  for (int it = threadIdx.x; it < (int)o.rows * 4; it += 512) {
    const int m = it >> 2, j = it & 3, at = (m >> 4) * 128 + (m & 15) + 16 * j;
    f32v4 v[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      v[b] = red[at + 64 * b];
#pragma unroll
      for (int k = 1; k < 8; ++k) v[b] += red[k * MT * 128 + at + 64 * b];
    }
    float x[8] = {v[0][0], v[1][0], v[0][1], v[1][1], v[0][2], v[1][2], v[0][3], v[1][3]};
    o.store8(m, k0 + 8 * j, x, o.col(k0 + 8 * j));
  }
}
// dw's tiles beside it: at most two chunks
typedef NtTile<NT_BF16, 2, 2, 2, 4, 1, 3, 3, 1, 2> FewTile;
template <int MT>
__global__ __launch_bounds__(512) void k_dense_few(const uint8_t *gp, int nch, DevMat w, const DenseOut oa, int na, const NtArgs gb, const EpiOut<DenseOut> eb, int nb,
                                                      ColumnSums sums) {
  typedef FewTile TB;
  static_assert(TB::T == 512 && TB::LDS >= 8 * MT * 2 * 1024, "workgroups of both");
  __shared__ __attribute__((aligned(16))) uint8_t lds[TB::LDS];
  const int id = blockIdx.x;
  if (id < na) few_dx<MT>(gp, nch, w, oa, lds, id);
  else if (id < na + nb) nt_run<TB>(gb, eb, lds, id - na, nb, 0);
  else column_sums(sums, id - na - nb, reinterpret_cast<float *>(lds));
}
// b: dw's product, if it goes along (nb tiles)
static hipError_t launch_few(const uint8_t *gp, int64_t nch, const DevMat &w, const DenseOut &a, NtArgs gb, const DenseOut &b, int64_t nb, const ColumnSums &sums,
                             hipStream_t s) {
  if (nb) {
    const hipError_t e = nt_args<FewTile>(gb, b.rows, b.cols, FewTile::BM, FewTile::BN, 0, nb, 1);
    if (e != hipSuccess) return e;
  }
  const int64_t na = blocks_of(a.cols, 32), ns = sums.out ? blocks_of(sums.cols, 64) : 0;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)(na + nb + ns)), dim3(512), 0, s, gp, (int)nch, w, a, (int)na, gb, EpiOut<DenseOut>{b}, (int)nb, sums);
    return hipGetLastError();
  };
  return a.rows <= 16 ? go(k_dense_few<1>) : a.rows <= 32 ? go(k_dense_few<2>) : go(k_dense_few<4>);
}

// Whether that pays: on narrow layers few workgroups go through a long chain of chunks (us, left), where the other way moves w four times.  (us a call
// this way and by tiles: 16 x 1024 x 1024 15.0 and 21.1, 64 x 1024 x 1024 17.2 and 22.7, 32 x 256 x 2048 17.3 and 23.0, 32 x 2048 x 8192 77 and 86,
// 64 x 8192 x 8192 229 and 394; 64 x 256 x 8192 58.7 and 33.7, 1 x 1024 x 8192 58.7 and 53.6, 64 x 512 x 65536 628 and 233.)
static bool few_pays(int64_t M, int64_t N, int64_t K) {
  return K > 1 && M <= 64 && (float)blocks_of(N, 256) * (.8f + .013f * (float)M) < 10.f + 1.8e-6f * (float)N * (float)K;
}

template <int P, int KIND>
struct PairTile {   // 32 x 64 outputs
  typedef typename NtTiles<P, P, KIND>::T4 T;
};
// By the plan's figures for that shape, its longest chain of chunks or its work on all compute units, whichever is longer (P parts; KA, KB: kinds of dx and dw)
template <int P, int KA, int KB>
static bool pair_pays(const DenseOut &a, int64_t ca, const DenseOut &b, int64_t cb) {
  const NtShape &x = NtTiles<P, P, KA>::shapes[4];
  const int64_t na = nt_tiles(a.rows, a.cols, 32, 64, false), nb = nt_tiles(b.rows, b.cols, 32, 64, false);
  if (na + nb > 1 << 20) return false;
  const float chain = x.us1 * (float)std::max(ca, cb) + NT_ROUND_US;
  const float work = (.5f * x.us2 * (float)(na * ca + nb * cb) + .5f * NT_ROUND_US * (float)(na + nb)) / NT_CUS;
  return NT_LAUNCH_US + std::max(chain, work) <
         product_us<P, P, KA, 32>(a.rows, a.cols, ca, a.bytes()) + product_us<P, P, KB, 32>(b.rows, b.cols, cb, b.bytes());
}
template <int P, int KA, int KB>
static hipError_t launch_pair(NtArgs ga, const DenseOut &a, NtArgs gb, const DenseOut &b, const ColumnSums &sums, hipStream_t s) {
  typedef typename PairTile<P, KA>::T TA;
  typedef typename PairTile<P, KB>::T TB;
  static_assert(TA::BM == 32 && TA::BN == 64 && TB::BM == 32 && TB::BN == 64, "the shape of pair_pays");
  const int64_t na = nt_tiles(a.rows, a.cols, 32, 64, false), nb = nt_tiles(b.rows, b.cols, 32, 64, false);
  hipError_t e = nt_args<TA>(ga, a.rows, a.cols, 32, 64, 0, na, 1);
  if (e == hipSuccess) e = nt_args<TB>(gb, b.rows, b.cols, 32, 64, 0, nb, 1);
  if (e != hipSuccess) return e;
  const int64_t ns = sums.out ? blocks_of(sums.cols, 64) : 0;
  hipLaunchKernelGGL((k_dense_pair<TA, TB>), dim3((unsigned)(na + nb + ns)), dim3(256), 0, s, ga, EpiOut<DenseOut>{a}, (int)na, gb, EpiOut<DenseOut>{b}, (int)nb,
                     sums);
  return hipGetLastError();
}

// ---- few rows ---------------------------------------------------------------------------------
// y for up to 64 rows of x, from x and w as they are stored: bound by reading the weights once.  A workgroup takes NB row blocks of w (16
// rows), its 8 waves go through groups of U chunks of 32 columns in turn, each with the next group's loads in flight, and their sums are added in LDS in wave order.
// A lane reads its row's eight columns of a chunk as the matrix instruction takes them, of w and of x alike (x comes from L2: laid out
// in LDS it would have to wait there for the slowest wave); float32 values are split into their parts in registers.  Rows beyond
// the last read that one, and their results are not stored.  Float32 8192 x 8192: one row 51 us (5.2 TB/s), 64 rows 98 to 104 us, in which the splits of x,
// anew for every 32 rows of w, take as long as the loads (ten of that variant's registers wait in scratch memory outside the
// loop, none is fetched in it).  (Laid out for the tiles instead, us a call: float32 16 x 1024 x 1024 15.0, 8.0 here;
// 64 x 8192 x 8192 230 and 100; bf16 rows of no alignment, 64 x 1024 x 1024 12.9 and 11.6, 64 x 8192 x 8192 155 and 103.)
template <bool BF>
struct Raw8 {   // eight columns of a row as stored
  uint4 q[BF ? 1 : 2];
};
template <bool BF>
__device__ __forceinline__ Raw8<BF> raw_load(const uint8_t *p) {   // (rows may be aligned to their element alone)
  Raw8<BF> r;
  __builtin_memcpy(&r, __builtin_assume_aligned(p, BF ? 2 : 4), sizeof(r));
  return r;
}
template <bool BF>
__device__ __forceinline__ Raw8<BF> raw_edge(const uint8_t *p, int n) {   // the first n of them, zeros beyond
  Raw8<BF> r;
  uint32_t *w = reinterpret_cast<uint32_t *>(&r);
#pragma unroll
  for (int i = 0; i < (BF ? 4 : 8); ++i) {
    if constexpr (BF) {
      const uint16_t *s = reinterpret_cast<const uint16_t *>(p) + 2 * i;
      w[i] = (2 * i < n ? s[0] : 0u) | (2 * i + 1 < n ? (uint32_t)s[1] << 16 : 0u);
    } else {
      w[i] = i < n ? reinterpret_cast<const uint32_t *>(p)[i] : 0u;
    }
  }
  return r;
}
template <bool BF>
struct Parts8 {
  bf16x8 p[BF ? 1 : 3];
};
template <bool BF, bool ANY>
__device__ __forceinline__ Parts8<BF> raw_parts(const Raw8<BF> &r, float &top) {
  Parts8<BF> o;
  if constexpr (BF) {
    o.p[0] = __builtin_bit_cast(bf16x8, r.q[0]);
  } else {
    const float v[8] = {__builtin_bit_cast(float, r.q[0].x), __builtin_bit_cast(float, r.q[0].y), __builtin_bit_cast(float, r.q[0].z),
                        __builtin_bit_cast(float, r.q[0].w), __builtin_bit_cast(float, r.q[1].x), __builtin_bit_cast(float, r.q[1].y),
                        __builtin_bit_cast(float, r.q[1].z), __builtin_bit_cast(float, r.q[1].w)};
    parts8<ANY>(v, o.p, top);
  }
  return o;
}
template <bool BF, int MT, int NB, int U>
__global__ __launch_bounds__(512) void k_dense_rows(DevMat x, DevMat w, DenseOut o, float *part, int z_groups) {
  constexpr int ES = BF ? 2 : 4;
  __shared__ f32v4 red[8][MT * NB][64];
  const int lane = threadIdx.x & 63, r16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NB);
  const int M = (int)x.rows, K = (int)w.cols, whole = K / (32 * U), groups = (K + 32 * U - 1) / (32 * U);
  const int g0 = blockIdx.y * z_groups, g1 = min(groups, g0 + z_groups), gw = min(whole, g1);
  const uint8_t *wp[NB], *xp[MT];
#pragma unroll
  for (int b = 0; b < NB; ++b) wp[b] = static_cast<const uint8_t *>(w.p) + (min(n0 + 16 * b + r16, w.rows - 1) * w.ld + 8 * g4) * ES;
#pragma unroll
  for (int t = 0; t < MT; ++t) xp[t] = static_cast<const uint8_t *>(x.p) + (min(16 * t + r16, M - 1) * x.ld + 8 * g4) * ES;
  struct Group {
    Raw8<BF> w[U][NB], x[U][MT];
  };
  auto load = [&](Group &q, int gi) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t at = ((int64_t)gi * U + u) * (32 * ES);
#pragma unroll
      for (int b = 0; b < NB; ++b) q.w[u][b] = raw_load<BF>(wp[b] + at);
#pragma unroll
      for (int t = 0; t < MT; ++t) q.x[u][t] = raw_load<BF>(xp[t] + at);
    }
  };
  f32v4 hi[MT][NB], lo[BF ? 1 : MT][BF ? 1 : NB];
  auto clear = [&] {
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        hi[t][b] = f32v4{0.f, 0.f, 0.f, 0.f};
        if constexpr (!BF) lo[t][b] = f32v4{0.f, 0.f, 0.f, 0.f};
      }
  };
  clear();
  float top = 0.f;
  const std::false_type plain{};
  auto multiply = [&](const Raw8<BF> (&rw)[NB], const Raw8<BF> (&rx)[MT], auto any) {
    constexpr bool ANY = decltype(any)::value;
    Parts8<BF> a[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) a[t] = raw_parts<BF, ANY>(rx[t], top);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const Parts8<BF> v = raw_parts<BF, ANY>(rw[b], top);
      if constexpr (!BF) {   // (nt.h: the small products, in order of their size, in an accumulator of their own; the row blocks' in turn, since one's wait for each other)
        constexpr int pa[5] = {0, 2, 1, 0, 1}, pb[5] = {2, 0, 1, 1, 0};
#pragma unroll
        for (int p = 0; p < 5; ++p)
#pragma unroll
          for (int t = 0; t < MT; ++t) lo[t][b] = mfma_bf16(v.p[pb[p]], a[t].p[pa[p]], lo[t][b]);
      }
#pragma unroll
      for (int t = 0; t < MT; ++t) hi[t][b] = mfma_bf16(v.p[0], a[t].p[0], hi[t][b]);
    }
  };
  auto use = [&](const Group &q) {
#pragma unroll
    for (int u = 0; u < U; ++u) multiply(q.w[u], q.x[u], plain);
  };
  Group q[2];
  int gi = g0 + wave;
  if (gi < gw) load(q[0], gi);
  for (; gi < gw; gi += 16) {
    if (gi + 8 < gw) load(q[1], gi + 8);
    use(q[0]);
    if (gi + 16 < gw) load(q[0], gi + 16);
    if (gi + 8 < gw) use(q[1]);
  }
  auto chunk = [&](int c, auto any) {   // one that may lie beyond the columns in part
    const int n = max(0, min(8, K - 32 * c - 8 * g4));
    const int64_t at = (int64_t)c * (32 * ES);
    Raw8<BF> ew[NB], ex[MT];
#pragma unroll
    for (int b = 0; b < NB; ++b) ew[b] = raw_edge<BF>(wp[b] + at, n);
#pragma unroll
    for (int t = 0; t < MT; ++t) ex[t] = raw_edge<BF>(xp[t] + at, n);
    multiply(ew, ex, any);
  };
  if (groups > whole && g1 == groups && wave == (whole - g0) % 8) {   // the columns beyond whole groups
#pragma unroll 1
    for (int c = whole * U; c * 32 < K; ++c) chunk(c, plain);
  }
  if constexpr (!BF) {
    if (__builtin_expect(__any(top >= PLAIN_SPLIT), 0)) {   // (groups of this wave, as above)
      clear();
#pragma unroll 1
      for (gi = g0 + wave; gi < g1; gi += 8)
#pragma unroll 1
        for (int c = gi * U; c < (gi + 1) * U && c * 32 < K; ++c) chunk(c, std::true_type{});
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      f32v4 v = hi[t][b];
      if constexpr (!BF) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fabsf(v[i]) < __builtin_huge_valf() ? v[i] + lo[t][b][i] : v[i];
      }
      red[wave][t * NB + b][lane] = v;
    }
  __syncthreads();
  for (int it = threadIdx.x; it < M * NB * 2; it += 512) {
    const int m = it / (NB * 2), oct = it - m * (NB * 2), blk = (m >> 4) * NB + (oct >> 1), l = (m & 15) + 32 * (oct & 1);
    f32v4 a = red[0][blk][l], b = red[0][blk][l + 16];
#pragma unroll
    for (int k = 1; k < 8; ++k) a += red[k][blk][l], b += red[k][blk][l + 16];
    const int64_t n = n0 + oct * 8;
    if (part) {
      f32v4 *d = reinterpret_cast<f32v4 *>(part + ((int64_t)blockIdx.y * M + m) * (gridDim.x * (16 * NB)) + n);
      d[0] = a;
      d[1] = b;
    } else {
      float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
      o.store8(m, n, v, o.col(n));
    }
  }
}
// Two row blocks a workgroup halve what is read and split of x, where enough workgroups are left (us with one and two: float32 64 x 4096 x 8192 82.6 and
// 55.0, 16 x 4096 x 8192 38.7 and 35.6, 8 x 8192 x 8192 61.8 and 76.9; bf16 8 x 8192 x 8192 63.5 and 53.4, 1 x 4096 x 8192 23.4 and 25.3).  The
// columns are divided among idle compute units where that saves more than the launch that joins the parts, of which it takes more than 64 too long
// to read (us whole and in parts: float32 1 x 2048 x 256 8.3 and 11.3, 1 x 8192 x 256 22.6 and 11.2, 64 x 784 x 1024 10.0 and 11.3,
// 64 x 2048 x 256 22.2 and 11.2, 64 x 65536 x 64 563 and 27; 1 x 262144 x 16 in 64 parts 21, in 256 34).
struct DenseRows {
  int nb, u, parts, z_groups;
  int64_t wgs;
  size_t part_bytes;
};
static DenseRows dense_rows(bool bf16, int64_t M, int64_t N, int64_t K) {
  DenseRows p{};
  const int64_t blocks = blocks_of(N, 16);
  p.nb = M > (bf16 ? 4 : 8) && blocks >= 512 ? 2 : 1;
  p.u = bf16 ? (M <= 16 ? 4 : 2) : M <= 16 ? 2 : 1;
  p.wgs = blocks_of(blocks, p.nb);
  const int64_t groups = blocks_of(K, 32 * p.u);
  int64_t z = std::min<int64_t>({256 / p.wgs, groups / 8, 64});
  const float chain = (2.f + .1f * (float)M) * (1.f / 1024) * (float)K;   // us of a workgroup with all columns
  if (z < 2 || chain - chain / (float)z < 5.f) z = 1;
  p.z_groups = (int)blocks_of(groups, z);
  p.parts = (int)blocks_of(groups, p.z_groups);
  p.part_bytes = p.parts > 1 ? (size_t)p.parts * M * p.wgs * p.nb * 64 : 0;
  return p;
}
template <bool BF>
static hipError_t launch_dense_rows(const DevMat &x, const DevMat &w, const DenseRows &p, const DenseOut &o, float *part, hipStream_t s) {
  if (p.parts == 1) part = nullptr;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)p.wgs, (unsigned)p.parts), dim3(512), 0, s, x, w, o, part, p.z_groups); };
  constexpr int U1 = BF ? 4 : 2, U2 = BF ? 2 : 1;
  if (x.rows <= 16) p.nb == 2 ? go(k_dense_rows<BF, 1, 2, U1>) : go(k_dense_rows<BF, 1, 1, U1>);
  else if (x.rows <= 32) p.nb == 2 ? go(k_dense_rows<BF, 2, 2, U2>) : go(k_dense_rows<BF, 2, 1, U2>);
  else p.nb == 2 ? go(k_dense_rows<BF, 4, 2, U2>) : go(k_dense_rows<BF, 4, 1, U2>);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !part) return e;
  const int64_t ld = p.wgs * p.nb * 16;
  hipLaunchKernelGGL((k_join<DenseOut>), dim3((unsigned)blocks_of(o.rows * (ld / 8), 256)), dim3(256), 0, s, part, p.parts, o.rows, ld, o);
  return hipGetLastError();
}

static DevMat dev(const vcr_mat *m) { return DevMat{m->p, m->type == VCR_BF16, m->rows, m->cols, m->ld, 0}; }
static size_t room(bool bf16, int64_t M, int64_t N, int64_t chunks) {
  return bf16 ? part_bytes<1, 1, NT_BF16, 32>(M, N, chunks) : part_bytes<3, 3, NT_BF16_DENSE, 32>(M, N, chunks);
}
static hipError_t product(bool bf16, const NtArgs &g, const DenseOut &o, float *part, hipStream_t s) {
  return bf16 ? nt_product<1, 1, NT_BF16, 32>(g, o, part, s) : nt_product<3, 3, NT_BF16_DENSE, 32>(g, o, part, s);
}

// Up to 64 rows of bf16: tiles of all the rows and 32 columns, whose waves divide the contraction, with as many stages in flight as memory takes to answer
struct SkinnyTiles {
  typedef NtTile<NT_ROWS, 1, 2, 1, 1, 4, 1, 1, 4, 6> R16;
  typedef NtTile<NT_ROWS, 2, 2, 1, 1, 4, 1, 1, 4, 6> R32;
  typedef NtTile<NT_ROWS, 4, 2, 1, 1, 4, 1, 1, 4, 4> R64;
};
// Taken where there are about enough such tiles for the chip, so that dividing the contraction would only add a launch, or where the
// contraction is short (this way and by the plan, us a call with weights from memory: 1 x 8192 x 8192 29.0 and 31.3, 64 x 8192 x 8192 34.4 and 36.7,
// 64 x 4096 x 4096 16.8 and 18.1, 16 x 2048 x 2048 7.9 and 10.4; 16 x 8192 x 2048 17.6 and 12.5, 64 x 1024 x 65536 54 and 30).
static bool skinny(int64_t M, int64_t N, int64_t K) {
  const int64_t tiles = blocks_of(N, 32);
  return M <= 64 && (tiles >= 128 || K <= 2048) && (tiles <= 512 || M <= 16);
}
static hipError_t skinny_product(const NtArgs &g, const DenseOut &o, hipStream_t s) {
  auto go = [&](auto t) {
    typedef decltype(t) T;
    return launch_nt<T>(g, o.rows, o.cols, T::BM, T::BN, 0, nt_tiles(o.rows, o.cols, T::BM, T::BN, false), 1, EpiOut<DenseOut>{o}, s);
  };
  return o.rows <= 16 ? go(SkinnyTiles::R16{}) : o.rows <= 32 ? go(SkinnyTiles::R32{}) : go(SkinnyTiles::R64{});
}
// bf16 matrices that the tiles take as they are (nt.h)
static bool rows_operand(const vcr_mat *m) { return m->cols % 8 == 0 && rows_aligned(m->p, m->ld, 2) && m->ld < (int64_t)1 << 22; }
static bool rows_product(const vcr_mat *x, const vcr_mat *w) { return rows_operand(x) && rows_operand(w); }

}  // namespace vcr

using namespace vcr;
#define TRY(expr)                       \
  do {                                  \
    const vcr_status st_ = (expr);      \
    if (st_ != VCR_OK) return st_;      \
  } while (0)

static vcr_status check_opts(vcr_ctx *c, const vcr_linear_opts *o) {
  if (o->act < VCR_ACT_NONE || o->act > VCR_ACT_SILU) return fail(c, VCR_ERR_ARG, "act: %d is not one of VCR_ACT_*", o->act);
  return check_drop(c, o->drop);
}
static vcr_status check_like(vcr_ctx *c, const vcr_mat *m, int64_t rows, int64_t cols, const char *name) {
  TRY(check_mat(c, m, name));
  if (m->rows != rows || m->cols != cols)
    return fail(c, VCR_ERR_SHAPE, "%s is %lld x %lld, not %lld x %lld", name, (long long)m->rows, (long long)m->cols, (long long)rows,
                (long long)cols);
  return VCR_OK;
}
static vcr_status check_rows(vcr_ctx *c, int64_t rows) {
  if (rows > VCR_MAX_LINEAR_ROWS)
    return fail(c, VCR_ERR_UNSUPPORTED, "%lld rows exceed the limit of %lld", (long long)rows, (long long)VCR_MAX_LINEAR_ROWS);
  return VCR_OK;
}

// The gradients of bf16 matrices that the tiles take as they are, M > 0: g is written out where it is not dy itself
static vcr_status grad_of_rows(vcr_ctx *c, const vcr_mat *dy, const vcr_mat *x, const vcr_mat *w, const vcr_linear_opts &o, const vcr_mat *add,
                               const vcr_mat *dx, const vcr_mat *dw, float *db) {
  const int64_t M = dy->rows, N = dy->cols, K = dx ? w->cols : dw ? x->cols : 1, mg = blocks_of(M, 64), nch = blocks_of(N, 32), mch = blocks_of(M, 32);
  const DropDev drop = drop_dev(o.drop), none = drop_dev(nullptr);
  const bool store = (dx || dw) && (o.act != VCR_ACT_NONE || drop.k || !rows_operand(dy));
  const int64_t pitch = store ? blocks_of(N, 8) * 8 : dy->ld;
  const size_t b_g = store ? (size_t)M * pitch * 2 : 0, b_sums = db && mg > 1 ? (size_t)mg * N * 4 : 0;
  const size_t b_part = std::max(dx ? part_bytes<1, 1, NT_RT, 32>(M, K, nch) : 0, dw ? part_bytes<1, 1, NT_TT, 32>(N, K, mch) : 0);
  Workspace *ws = nullptr;
  TRY(op_space(c, al(b_g) + al(b_sums) + al(b_part) + 3 * 256, &ws));
  uint16_t *g = take<uint16_t>(*ws, b_g / 2);
  float *sums = take<float>(*ws, b_sums / 4), *part = take<float>(*ws, b_part / 4);
  const hipStream_t s = c->stream;
  if (store || db) {
    const GradSource src{mat_ref(o.act != VCR_ACT_NONE ? o.z : nullptr), o.act, drop};
    const hipError_t e = launch_stretches(mg * blocks_of(N, 64), [&](int64_t first, dim3 grid) {
      hipLaunchKernelGGL(k_grad_rows, grid, dim3(256), 0, s, dev(dy), rows_aligned(dy->p, dy->ld, 2), src, store ? g : nullptr, pitch,
                         db ? mg > 1 ? sums : db : nullptr, mg > 1 ? 1.f : drop.factor, first);
    });
    HIP_TRY(c, e);
  }
  const ColumnSums cs{sums, mg, N, drop.factor, db && mg > 1 ? db : nullptr};
  const uint8_t *gp = store ? reinterpret_cast<const uint8_t *>(g) : static_cast<const uint8_t *>(dy->p);
  NtArgs a{}, b{};
  DenseOut ao{}, bo{};
  if (dx) {
    a.A = NtOperand{gp, nullptr, (int32_t)blocks_of(M, 16), 0, pitch * 2, M};
    a.B = NtOperand{static_cast<const uint8_t *>(w->p), nullptr, (int32_t)blocks_of(K, 16), 0, w->ld * 2, K};
    a.chunks = (int32_t)nch;
    a.cols = (int32_t)N;
    ao = DenseOut{mat_ref(dx), MatRef{}, mat_ref(add), nullptr, M, K, VCR_ACT_NONE, drop.factor, none};
  }
  if (dw) {
    b.A = NtOperand{gp, nullptr, (int32_t)blocks_of(N, 16), 0, pitch * 2, N};
    b.B = NtOperand{static_cast<const uint8_t *>(x->p), nullptr, (int32_t)blocks_of(K, 16), 0, x->ld * 2, K};
    b.chunks = (int32_t)mch;
    b.cols = (int32_t)M;
    bo = DenseOut{mat_ref(dw), MatRef{}, MatRef{}, nullptr, N, K, VCR_ACT_NONE, drop.factor, none};
  }
  if (dx && dw && pair_pays<1, NT_RT, NT_TT>(ao, nch, bo, mch)) {
    HIP_TRY(c, (launch_pair<1, NT_RT, NT_TT>(a, ao, b, bo, cs, s)));
    return op_end(c);
  }
  if (cs.out) {
    hipLaunchKernelGGL(k_dense_sums, dim3((unsigned)blocks_of(N, 64)), dim3(256), 0, s, cs);
    HIP_TRY(c, hipGetLastError());
  }
  if (dx) HIP_TRY(c, (nt_product<1, 1, NT_RT, 32>(a, ao, part, s)));
  if (dw) HIP_TRY(c, (nt_product<1, 1, NT_TT, 32>(b, bo, part, s)));
  return op_end(c);
}

extern "C" {

vcr_status vcr_linear(vcr_ctx *c, const vcr_mat *x, const vcr_mat *w, const vcr_linear_opts *opts, const vcr_mat *y) {
  if (!c) return VCR_ERR_ARG;
  const vcr_linear_opts o = opts ? *opts : vcr_linear_opts{};
  TRY(check_mat(c, x, "x"));
  TRY(check_mat(c, w, "w"));
  if (x->type != w->type) return fail(c, VCR_ERR_ARG, "x and w differ in type");
  if (w->rows == 0) return fail(c, VCR_ERR_SHAPE, "w has no rows");
  if (x->cols != w->cols) return fail(c, VCR_ERR_SHAPE, "x and w differ in columns");
  TRY(check_like(c, y, x->rows, w->rows, "y"));
  TRY(check_opts(c, &o));
  if ((reinterpret_cast<uintptr_t>(o.bias) & 3) != 0) return fail(c, VCR_ERR_ARG, "bias: pointer not aligned to its type");
  if (o.residual) TRY(check_like(c, o.residual, x->rows, w->rows, "residual"));
  if (o.z) TRY(check_like(c, o.z, x->rows, w->rows, "z"));
  TRY(check_rows(c, x->rows));
  TRY(check_rows(c, w->rows));
  TRY(check_contraction(c, x->cols));
  TRY(op_begin(c));
  const int64_t M = x->rows, N = w->rows, K = x->cols;
  if (M == 0) return VCR_OK;
  const bool bf16 = x->type == VCR_BF16;
  const int P = bf16 ? 1 : 3;
  const DenseOut out{mat_ref(y), mat_ref(o.z), mat_ref(o.residual), o.bias, M, N, o.act, 1.f, drop_dev(o.drop)};
  const bool as_stored = bf16 && rows_product(x, w);
  // (few bf16 rows on narrow layers: by the plan a product in parts and their sum; us by rows and by tiles: 1 x 4096 x 2048 8.3 and 11.0, 16 x 4096 x 2048
  // 10.1 and 10.9, 8 x 8192 x 2048 14.5 and 11.6, 1 x 4096 x 4096 9.1 and 8.2)
  if (as_stored ? M <= 16 && N * K <= (int64_t)1 << 23 : M <= 64) {
    const DenseRows p = dense_rows(bf16, M, N, K);
    Workspace *ws = nullptr;
    TRY(op_space(c, p.part_bytes, &ws));
    float *part = reinterpret_cast<float *>(ws->base);
    if (bf16) HIP_TRY(c, launch_dense_rows<true>(dev(x), dev(w), p, out, part, c->stream));
    else HIP_TRY(c, launch_dense_rows<false>(dev(x), dev(w), p, out, part, c->stream));
    return op_end(c);
  }
  const int64_t chunks = blocks_of(K, 32), mb = blocks_of(M, 16), nb = blocks_of(N, 16);
  if (as_stored) {
    NtArgs g{};
    g.A = NtOperand{static_cast<const uint8_t *>(x->p), nullptr, (int32_t)mb, 0, x->ld * 2, M};
    g.B = NtOperand{static_cast<const uint8_t *>(w->p), nullptr, (int32_t)nb, 0, w->ld * 2, N};
    g.chunks = (int32_t)chunks;
    g.cols = (int32_t)K;
    if (skinny(M, N, K)) {
      HIP_TRY(c, skinny_product(g, out, c->stream));
      return op_end(c);
    }
    Workspace *ws = nullptr;
    TRY(op_space(c, part_bytes<1, 1, NT_ROWS, 32>(M, N, chunks), &ws));
    HIP_TRY(c, (nt_product<1, 1, NT_ROWS, 32>(g, out, reinterpret_cast<float *>(ws->base), c->stream)));
    return op_end(c);
  }
  const size_t xb = (size_t)mb * chunks * P * FRAG, wb = (size_t)nb * chunks * P * FRAG, pb = room(bf16, M, N, chunks);
  Workspace *ws = nullptr;
  TRY(op_space(c, al(xb) + al(wb) + al(pb) + 256, &ws));
  uint8_t *xp = take<uint8_t>(*ws, xb), *wp = take<uint8_t>(*ws, wb);
  float *part = take<float>(*ws, pb / 4);
  PlanesArgs xl{}, wl{};
  xl.x = dev(x);
  xl.rows = xp;
  xl.row_blocks = mb;
  wl.x = dev(w);
  wl.rows = wp;
  wl.row_blocks = nb;
  xl.row_chunks = wl.row_chunks = chunks;
  HIP_TRY(c, launch_dense_planes(nullptr, &xl, &wl, GradSource{}, bf16, c->stream));
  NtArgs g{};
  g.A = NtOperand{xp, nullptr, (int32_t)mb, 0};
  g.B = NtOperand{wp, nullptr, (int32_t)nb, 0};
  g.chunks = (int32_t)chunks;
  HIP_TRY(c, product(bf16, g, out, part, c->stream));
  return op_end(c);
}

vcr_status vcr_linear_grad(vcr_ctx *c, const vcr_mat *dy, const vcr_mat *x, const vcr_mat *w, const vcr_linear_opts *opts, const vcr_mat *add,
                           const vcr_mat *dx, const vcr_mat *dw, float *db) {
  if (!c) return VCR_ERR_ARG;
  const vcr_linear_opts o = opts ? *opts : vcr_linear_opts{};
  TRY(check_mat(c, dy, "dy"));
  const int64_t M = dy->rows, N = dy->cols;
  TRY(check_opts(c, &o));
  if (o.act != VCR_ACT_NONE) {
    if (!o.z) return fail(c, VCR_ERR_ARG, "the gradient of an activation needs z");
    TRY(check_like(c, o.z, M, N, "z"));
  }
  if (dw && !x) return fail(c, VCR_ERR_ARG, "dw needs x");
  if (dx && !w) return fail(c, VCR_ERR_ARG, "dx needs w");
  if (x) {
    TRY(check_mat(c, x, "x"));
    if (x->rows != M) return fail(c, VCR_ERR_SHAPE, "x and dy differ in rows");
    if (x->type != dy->type) return fail(c, VCR_ERR_ARG, "x and dy differ in type");
  }
  if (w) {
    TRY(check_mat(c, w, "w"));
    if (w->rows != N) return fail(c, VCR_ERR_SHAPE, "w has %lld rows, dy %lld columns", (long long)w->rows, (long long)N);
    if (w->type != dy->type) return fail(c, VCR_ERR_ARG, "w and dy differ in type");
  }
  if (x && w && x->cols != w->cols) return fail(c, VCR_ERR_SHAPE, "x and w differ in columns");
  if (dx) TRY(check_like(c, dx, M, w->cols, "dx"));
  if (dx && add) TRY(check_like(c, add, M, w->cols, "add"));
  if (dw) TRY(check_like(c, dw, N, x->cols, "dw"));
  if ((reinterpret_cast<uintptr_t>(db) & 3) != 0) return fail(c, VCR_ERR_ARG, "db: pointer not aligned to its type");
  TRY(check_rows(c, M));
  TRY(check_rows(c, N));
  if (dx || dw) TRY(check_rows(c, dx ? w->cols : x->cols));
  if (dx) TRY(check_contraction(c, N));
  if (dw) TRY(check_contraction(c, M));
  TRY(op_begin(c));
  const bool bf16 = dy->type == VCR_BF16, has_dx = dx && M > 0;
  if (!has_dx && !dw && !db) return VCR_OK;
  // (g's rows, where they are written out, have offsets of the tiles' 32 bits up to 2^22 columns, as rows_operand asks of the others)
  if (bf16 && M > 0 && N < (int64_t)1 << 22 && (!dx || rows_operand(w)) && (!dw || rows_operand(x))) return grad_of_rows(c, dy, x, w, o, add, dx, dw, db);
  const int P = bf16 ? 1 : 3;
  const hipStream_t s = c->stream;
  const int64_t K = has_dx ? w->cols : dw ? x->cols : 1;
  const int64_t nch = blocks_of(N, 32), mch = blocks_of(std::max<int64_t>(M, 1), 32), mb = blocks_of(M, 16), nb = blocks_of(N, 16),
                kb = blocks_of(K, 16), mg = blocks_of(M, 64);
  const bool few = !bf16 && has_dx && few_pays(M, N, K);
  // (few_dx takes whole groups of row blocks)
  const int64_t gmb = few ? M <= 16 ? 1 : M <= 32 ? 2 : 4 : mb;
  const size_t b_g = has_dx ? (size_t)gmb * nch * P * FRAG : 0, b_wt = has_dx && !few ? (size_t)kb * nch * P * FRAG : 0;
  const size_t b_gt = dw ? (size_t)nb * mch * P * FRAG : 0, b_xt = dw ? (size_t)kb * mch * P * FRAG : 0;
  const size_t b_sums = db ? (size_t)mg * N * 4 : 0;
  const size_t b_part = std::max(has_dx ? room(bf16, M, K, nch) : 0, dw ? room(bf16, N, K, mch) : 0);
  Workspace *ws = nullptr;
  TRY(op_space(c, al(b_g) + al(b_wt) + al(b_gt) + al(b_xt) + al(b_sums) + al(b_part) + 6 * 256, &ws));
  uint8_t *gp = take<uint8_t>(*ws, b_g), *wt = take<uint8_t>(*ws, b_wt), *gt = take<uint8_t>(*ws, b_gt), *xt = take<uint8_t>(*ws, b_xt);
  float *sums = take<float>(*ws, b_sums / 4), *part = take<float>(*ws, b_part / 4);
  const DropDev drop = drop_dev(o.drop);
  PlanesArgs gl{}, xl{}, wl{};
  gl.x = dev(dy);
  if (has_dx) {
    gl.rows = gp;
    gl.row_blocks = gmb;
    gl.row_chunks = nch;
    wl.x = dev(w);
    wl.cols = wt;
    wl.col_blocks = kb;
    wl.col_chunks = nch;
  }
  if (dw) {
    gl.cols = gt;
    gl.col_blocks = nb;
    xl.x = dev(x);
    xl.cols = xt;
    xl.col_blocks = kb;
    gl.col_chunks = xl.col_chunks = mch;
  }
  gl.sums = db && M > 0 ? sums : nullptr;
  HIP_TRY(c, launch_dense_planes(&gl, dw ? &xl : nullptr, has_dx && !few ? &wl : nullptr, GradSource{mat_ref(o.act != VCR_ACT_NONE ? o.z : nullptr), o.act, drop},
                                 bf16, s));
  const ColumnSums cs{sums, mg, N, drop.factor, db};
  const DropDev none = drop_dev(nullptr);
  NtArgs a{}, b{};
  DenseOut ao{}, bo{};
  if (has_dx) {
    a.A = NtOperand{gp, nullptr, (int32_t)mb, 0};
    a.B = NtOperand{wt, nullptr, (int32_t)kb, 0};
    a.chunks = (int32_t)nch;
    ao = DenseOut{mat_ref(dx), MatRef{}, mat_ref(add), nullptr, M, K, VCR_ACT_NONE, drop.factor, none};
  }
  if (dw) {
    b.A = NtOperand{gt, nullptr, (int32_t)nb, 0};
    b.B = NtOperand{xt, nullptr, (int32_t)kb, 0};
    b.chunks = (int32_t)mch;
    bo = DenseOut{mat_ref(dw), MatRef{}, MatRef{}, nullptr, N, K, VCR_ACT_NONE, drop.factor, none};
  }
  if (few) {
    // dw's tiles go along where they are few, or where dx alone leaves compute units idle (32 columns of w a workgroup); else its own plan has
    // larger ones (us along and apart: 64 x 1024 x 1024 17.1 and 22.6, 64 x 8192 x 256 18.7 and 19.2, 64 x 4096 x 4096 72 and 86, 64 x 5120 x 5120 104 and 115,
    // 64 x 6144 x 8192 192 and 195; 64 x 7000 x 2048 68.4 and 66.0, 64 x 16384 x 1024 78 and 74, 64 x 8192 x 8192 249 and 229)
    const int64_t nb = dw ? nt_tiles(N, K, FewTile::BM, FewTile::BN, false) : 0;
    const bool along = nb <= 512 || (K <= 6144 && nb <= 1 << 20);   // (a launch takes less than 2^32 threads)
    HIP_TRY(c, launch_few(gp, nch, dev(w), ao, b, bo, along ? nb : 0, cs, s));
    if (!along) HIP_TRY(c, product(bf16, b, bo, part, s));
    return op_end(c);
  }
  if (has_dx && dw && (bf16 ? pair_pays<1, NT_BF16, NT_BF16>(ao, nch, bo, mch) : pair_pays<3, NT_BF16_DENSE, NT_BF16_DENSE>(ao, nch, bo, mch))) {
    HIP_TRY(c, bf16 ? (launch_pair<1, NT_BF16, NT_BF16>(a, ao, b, bo, cs, s)) : (launch_pair<3, NT_BF16_DENSE, NT_BF16_DENSE>(a, ao, b, bo, cs, s)));
    return op_end(c);
  }
  if (cs.out) {
    hipLaunchKernelGGL(k_dense_sums, dim3((unsigned)blocks_of(N, 64)), dim3(256), 0, s, cs);
    HIP_TRY(c, hipGetLastError());
  }
  if (has_dx) HIP_TRY(c, product(bf16, a, ao, part, s));
  if (dw) HIP_TRY(c, product(bf16, b, bo, part, s));
  return op_end(c);
}

}  // extern "C"
