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
#include <new>

#include "ctx.h"
#include "layers.h"
#include "planes.h"

namespace vcr {

// ---- 4-bit values ---------------------------------------------------------------------------
__host__ __device__ inline int64_t mx_groups(int64_t cols) { return (cols + 127) / 128; }

struct MxDev {
  const uint8_t *codes, *scales;
  int64_t rows, cols;
};
__device__ __forceinline__ int64_t mx_scale_at(int64_t rb, int64_t group, int64_t groups, int lane) {
  return ((rb * ((groups + 3) >> 2) + (group >> 2)) * 64 + lane) * 4 + (group & 3);
}

// Quantisation.  A workgroup takes 16 rows by 512 columns: a wave reads a row's 512 at once, a thread 8 of
// them, four threads a block; the codes go through LDS into the storage order.  Bound by memory: 8192 x 8192
// float32, 304 MB, in 55 us, 5.5 TB/s, the rate of a large copy (67 to 78 us where the memory is still taking in the 268 MB
// that a call before wrote: read back and quantised in turn, both take 124).
template <bool BF>
__global__ __launch_bounds__(256) void k_mx_quantize(DevMat x, int vec, uint8_t *codes, uint8_t *scales, int64_t first) {
  __shared__ uint32_t cs[4][4][16][4];   // [group][block][row][words]
  __shared__ uint8_t sb[16][16];         // [block of the 512 columns][row]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t groups = mx_groups(x.cols), n4 = (groups + 3) >> 2;
  const int64_t at = first + blockIdx.x, rb = at / n4, c4 = at - rb * n4;
  const int64_t row0 = rb * 16 + wave * 4, col = c4 * 512 + lane * 8;
  float v[4][8];
  if (vec && row0 + 4 <= x.rows && c4 * 512 + 512 <= x.cols) {   // uniform: all loads at once
#pragma unroll
    for (int i = 0; i < 4; ++i) mat_row8<BF>(x, 0, row0 + i, col, true, v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) mat_row8<BF>(x, 0, row0 + i, col, vec, v[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) top = max(top, __builtin_bit_cast(uint32_t, v[i][q]) & 0x7fffffffu);
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0xb1, 15, 15, true));
    top = max(top, (uint32_t)__builtin_amdgcn_mov_dpp((int)top, 0x4e, 15, 15, true));
    const uint32_t e = top >> 23, byte = e == 255 ? 255 : e > 2 ? e - 2 : 0;
    const float s = mx_scale(byte == 255 ? 127 : byte);
    uint32_t u = 0;
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[i][0], v[i][1], s, 0);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[i][2], v[i][3], s, 1);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[i][4], v[i][5], s, 2);
    u = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, v[i][6], v[i][7], s, 3);
    cs[lane >> 4][(lane >> 2) & 3][wave * 4 + i][lane & 3] = u;
    if ((lane & 3) == 0) sb[lane >> 2][wave * 4 + i] = (uint8_t)byte;
  }
  __syncthreads();
  // thread: group `wave`, slot `lane` (block lane / 16, row lane % 16)
  const int64_t grp = c4 * 4 + wave;
  if (grp < groups)
    *reinterpret_cast<uint4 *>(codes + ((rb * groups + grp) * 64 + lane) * 16) = *reinterpret_cast<uint4 *>(cs[wave][lane >> 4][lane & 15]);
  if (wave == 0) {
    const int g = lane >> 4, r = lane & 15;
    *reinterpret_cast<uint32_t *>(scales + (rb * n4 + c4) * 256 + lane * 4) =
        sb[g][r] | (uint32_t)sb[4 + g][r] << 8 | (uint32_t)sb[8 + g][r] << 16 | (uint32_t)sb[12 + g][r] << 24;
  }
}

// The values of a lane's block: 32 consecutive ones of a row
__device__ __forceinline__ void mx_block(const MxDev &w, int64_t rb, int64_t grp, int64_t groups, int lane, uint4 &q,
                                         float &s) {
  q = *reinterpret_cast<const uint4 *>(w.codes + ((rb * groups + grp) * 64 + lane) * 16);
  s = mx_scale(w.scales[mx_scale_at(rb, grp, groups, lane)]);
}
// The reverse, with the same division of work: 8192 x 8192 to float32 in 55 to 60 us, 5.1 to 5.5 TB/s (a thread per block, writing 32
// values in 16-byte pieces of as many lines: 244 us).
template <bool BF>
__global__ __launch_bounds__(256) void k_mx_dequantize(MxDev w, void *y, int64_t ld, int vec, int64_t first) {
  __shared__ uint32_t cs[4][4][16][4];
  __shared__ float ss[16][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t groups = mx_groups(w.cols), n4 = (groups + 3) >> 2;
  const int64_t at = first + blockIdx.x, rb = at / n4, c4 = at - rb * n4, grp = c4 * 4 + wave;
  if (grp < groups) {
    uint4 q;
    float s;
    mx_block(w, rb, grp, groups, lane, q, s);
    *reinterpret_cast<uint4 *>(cs[wave][lane >> 4][lane & 15]) = q;
    ss[wave * 4 + (lane >> 4)][lane & 15] = s;
  }
  __syncthreads();
  const int64_t col = c4 * 512 + lane * 8;
  if (col >= w.cols) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = wave * 4 + i;
    const uint4 b = mx_to_bf16(cs[lane >> 4][(lane >> 2) & 3][r][lane & 3], ss[lane >> 2][r]);
    if (BF && vec == 2 && rb * 16 + r < w.rows && col + 8 <= w.cols) {
      *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(y) + (rb * 16 + r) * ld + col) = b;
      continue;
    }
    const uint32_t h[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const f32v4 v = {__builtin_bit_cast(float, h[2 * k] << 16), __builtin_bit_cast(float, h[2 * k] & 0xffff0000u),
                       __builtin_bit_cast(float, h[2 * k + 1] << 16), __builtin_bit_cast(float, h[2 * k + 1] & 0xffff0000u)};
      store_row4(y, BF, ld, w.rows, w.cols, vec, rb * 16 + r, col + 4 * k, v);
    }
  }
}

// ---- operands of the bf16 products ------------------------------------------------------------
// (a workgroup goes through the column tiles of 64 rows in the grid's order; the first g_tiles workgroups take g, the others,
// if there are any, h)
template <int P, bool BF>
__global__ __launch_bounds__(256) void k_planes(PlanesArgs g, int64_t g_cols, int64_t g_tiles, PlanesArgs h, int64_t h_cols,
                                               int64_t first) {
  __shared__ float tile[64][65];
  const int64_t id = first + blockIdx.x;
  const bool is_g = id < g_tiles;   // uniform
  const int64_t at = is_g ? id : id - g_tiles, ct = is_g ? g_cols : h_cols, tr = at / ct;
  planes_tile<P, BF>(is_g ? g : h, 0, tr, at - tr * ct, PlanesScale{{1.f, 1.f}, 1.f}, tile);
}

// out[c] = the sum of a column over the groups of 64 rows: a workgroup takes 64 columns, a wave every fourth group
__global__ __launch_bounds__(256) void k_column_sums(const float *sums, int64_t groups, int64_t cols, float *out, int64_t first) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = (first + blockIdx.x) * 64 + lane;
  float s = 0.f;
#pragma unroll 8
  for (int64_t p = wave; p < groups; p += 4) s += c < cols ? sums[p * cols + c] : 0.f;
  part[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && c < cols) out[c] = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
}

// The transposed weights as a bf16 operand (exact), rows k and contraction n: a workgroup takes 32 n by 512 k through LDS,
// so that codes are read and fragments written whole.  Bound by what it writes: 8192 x 8192, 163 MB, in 33 us, 4.9 TB/s (with the eight n
// of a slot gathered in one thread's registers, whose stores are 16 bytes apart by rows, 64 us).
__global__ __launch_bounds__(256) void k_mx_planes_t(MxDev w, int64_t chunks, int64_t row_blocks, uint8_t *out) {
  constexpr int PITCH = 512 + 8;
  __shared__ __attribute__((aligned(16))) uint16_t t[32 * PITCH];   // [n][k]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
  const int64_t groups = mx_groups(w.cols), n4 = (groups + 3) >> 2;
  const int64_t ch = blockIdx.x / n4, c4 = blockIdx.x - ch * n4, grp = c4 * 4 + wave;
#pragma unroll
  for (int h = 0; h < 2; ++h) {   // row blocks 2 ch, 2 ch + 1
    uint4 q = make_uint4(0, 0, 0, 0);
    float s = 1.f;
    if (grp < groups && (ch * 2 + h) * 16 + r < w.rows) mx_block(w, ch * 2 + h, grp, groups, lane, q, s);
    uint16_t *d = t + (h * 16 + r) * PITCH + wave * 128 + g * 32;
    *reinterpret_cast<uint4 *>(d) = mx_to_bf16(q.x, s);
    *reinterpret_cast<uint4 *>(d + 8) = mx_to_bf16(q.y, s);
    *reinterpret_cast<uint4 *>(d + 16) = mx_to_bf16(q.z, s);
    *reinterpret_cast<uint4 *>(d + 24) = mx_to_bf16(q.w, s);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {   // row blocks of 16 k; lane: k = r, n = 8 g ..
    const int kb = i * 4 + wave;
    const int64_t rb = c4 * 32 + kb;
    if (rb >= row_blocks) continue;
    const uint16_t *s = t + g * 8 * PITCH + kb * 16 + r;
    uint32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = s[2 * j * PITCH] | (uint32_t)s[(2 * j + 1) * PITCH] << 16;
    *reinterpret_cast<uint4 *>(out + (rb * chunks + ch) * FRAG + lane * 16) = make_uint4(v[0], v[1], v[2], v[3]);
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

// ---- products by tiles ------------------------------------------------------------------------
// (nt.h; in 4 bits 4096 x 8192 x 8192 in 156 us, 3.5 PFLOP/s; bf16 rows with 4-bit weights 256 x 8192 x 8192 in 38 us; the gradients
// of 4096 x 8192 x 8192 in bf16 at 1.4 to 1.5 PFLOP/s, where a library product of that size reaches 1.35 to 1.55.)
template <int PA, int PB, int KIND>
static size_t part_bytes(int64_t M, int64_t N, int64_t chunks) {
  const int parts = nt_parts<NtTiles<PA, PB, KIND>>(M, N, chunks);
  return parts > 1 ? (size_t)parts * M * blocks_of(N, 4) * 16 : 0;
}
// D = A B^T into o; part: room for part_bytes
template <int PA, int PB, int KIND>
static hipError_t nt_product(const NtArgs &g, const OutMat &o, float *part, hipStream_t s) {
  typedef NtTiles<PA, PB, KIND> TS;
  const int parts = nt_parts<TS>(o.rows, o.cols, g.chunks);
  if (parts == 1) return launch_nt_plan<TS>(g, o.rows, o.cols, 1, o.bf16 ? 2.f : 4.f, EpiOut{o}, s);
  const int64_t ld = blocks_of(o.cols, 4) * 4;
  const NtShape &x = TS::shapes[nt_shapes<TS> - 1];
  const hipError_t e = launch_nt<typename TS::T4>(g, o.rows, o.cols, x.bm, x.bn, 0, nt_tiles(o.rows, o.cols, x.bm, x.bn, false), parts,
                                                  EpiPart{part, o.rows, ld}, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_join, dim3((unsigned)blocks_of(o.rows * (ld / 4), 256)), dim3(256), 0, s, part, parts, o.rows, ld, o);
  return hipGetLastError();
}

// ---- few rows ---------------------------------------------------------------------------------
// y = act(x w^T + bias) for few rows x: bound by reading the weights once.  A workgroup takes RB row blocks of weights;
// its 8 waves go through their groups of 128 columns in turn, each with the next ones' loads in flight, and the partial
// sums are added in LDS in wave order.  The matrix instruction has 16 rows whether they are used or not: a bf16 row
// takes one, a float32 row three, one for each of its parts, which are added at the end (1 x 4096 x 262144 in 126 us, 4.5 TB/s;
// with an instruction for each part 172 us, and with the loads alone 101).  What is left over the loads is expanding the
// weights: 16 conversions a lane for every 1 KB, in the way of the matrix instructions that need them.
// The rows are laid out once per workgroup in LDS, [chunk of 32][8 columns][row]; lanes of unused rows read the last one,
// and their results are not stored.  The weights are expanded in registers: a lane has 32 columns of its row, of which
// instruction s takes the s-th eight.  A 4-bit x (X4) is read as it is, 1 KB a group, shared by the RB blocks.
// Columns that do not fit LDS together are taken in slices of `slice` groups.
enum RowsKind : int { X4 = 0, XBF = 1, XF32 = 3 };   // the rows of the instruction that a row takes

template <int X>
__device__ __forceinline__ void rows_stage(const DevMat &x, int vec, int M, int64_t g0, int n, uint8_t *lds) {
  const int rows = M * X;
  for (int it = threadIdx.x; it < n * 16 * M; it += 512) {
    const int m = it / (n * 16), o = it - m * (n * 16);
    float v[8];
    mat_row8<X == XBF>(x, 0, m, g0 * 128 + o * 8, vec, v);
    uint32_t w[4][X];
#pragma unroll
    for (int i = 0; i < 4; ++i) parts_of<X>(v[2 * i], v[2 * i + 1], w[i]);
#pragma unroll
    for (int p = 0; p < X; ++p)
      *reinterpret_cast<uint4 *>(lds + (o * rows + m * X + p) * 16) = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
  }
}

template <int X, int RB>
__global__ __launch_bounds__(512, 2) void k_rows(DevMat x, int vec, MxDev a, MxDev w, int M, int slice, int z_groups, OutMat o, float *part) {
  constexpr int U = RB == 4 ? 2 : 4;   // groups of a wave's batch
  extern __shared__ __attribute__((aligned(16))) uint8_t rows_lds[];
  f32v4 *red = reinterpret_cast<f32v4 *>(rows_lds);   // [RB][8 waves][64]
  uint8_t *lds = rows_lds + RB * 8 * 64 * 16;
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t groups = mx_groups(w.cols), n4 = (groups + 3) >> 2, blocks = (w.rows + 15) >> 4;
  const int64_t g0 = (int64_t)blockIdx.y * z_groups, g1 = min(groups, g0 + z_groups);
  const int rows = M * X, mr = min(r, rows - 1);
  const bool whole = g1 - g0 <= slice;
  const int64_t stride = (int64_t)gridDim.x * RB;
  bool staged = false;
  i32x4 q[2][U][RB], qa[2][X == X4 ? U : 1];
  uint32_t sc[2][U][RB], sa[2][X == X4 ? U : 1];
  f32v4 acc[RB];
  auto load = [&](int64_t b0, int64_t s0, int n, int gi, int buf) {   // groups gi, gi + 8, .. of the n from s0 on
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t gr = s0 + min(gi + 8 * u, n - 1);
      if constexpr (X == X4) {
        qa[buf][u] = *reinterpret_cast<const i32x4 *>(a.codes + (gr * 64 + lane) * 16);
        sa[buf][u] = *reinterpret_cast<const uint32_t *>(a.scales + ((gr >> 2) * 64 + lane) * 4);
      }
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const int64_t rb = min(b0 + b, blocks - 1);
        q[buf][u][b] = *reinterpret_cast<const i32x4 *>(w.codes + ((rb * groups + gr) * 64 + lane) * 16);
        sc[buf][u][b] = *reinterpret_cast<const uint32_t *>(w.scales + ((rb * n4 + (gr >> 2)) * 64 + lane) * 4);
      }
    }
  };
  auto first = [&](int64_t b0, int64_t s0, int n) {
    load(b0, s0, n, wave, 0);
    if (wave + 8 * U < n) load(b0, s0, n, wave + 8 * U, 1);
  };
  auto multiply = [&](int64_t s0, int n, int gi, int buf) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (gi + 8 * u >= n) break;   // wave-uniform
      const int sh = 8 * (int)((s0 + gi + 8 * u) & 3);
      if constexpr (X == X4) {
        const i32x4 av = qa[buf][u];
        const i32x8 aw = {av[0], av[1], av[2], av[3], 0, 0, 0, 0};
#pragma unroll
        for (int b = 0; b < RB; ++b) {
          const i32x4 bv = q[buf][u][b];
          const i32x8 bw = {bv[0], bv[1], bv[2], bv[3], 0, 0, 0, 0};
          acc[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bw, aw, acc[b], 4, 4, 0, (int)(sc[buf][u][b] >> sh), 0,
                                                                    (int)(sa[buf][u] >> sh));
        }
      } else {
        float s[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) s[b] = mx_scale((sc[buf][u][b] >> sh) & 255);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bf16x8 av = *reinterpret_cast<const bf16x8 *>(lds + ((((gi + 8 * u) * 4 + g) * 4 + i) * rows + mr) * 16);
#pragma unroll
          for (int b = 0; b < RB; ++b)
            acc[b] = mfma_bf16(__builtin_bit_cast(bf16x8, mx_to_bf16((uint32_t)q[buf][u][b][i], s[b])), av, acc[b]);
        }
      }
    }
  };
  for (int64_t b0 = (int64_t)blockIdx.x * RB; b0 < blocks; b0 += stride) {
    const bool begun = whole && b0 >= stride;   // its first loads were issued before the last blocks' results
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[b] = f32v4{0.f, 0.f, 0.f, 0.f};
    for (int64_t s0 = g0; s0 < g1; s0 += slice) {
      const int n = (int)min((int64_t)slice, g1 - s0);
      if (!begun) first(b0, s0, n);   // ahead of the rows' staging
      if constexpr (X != X4) {
        if (!staged) {
          if (s0 > g0 || b0 >= stride) __syncthreads();   // the last slice has been read
          rows_stage<X>(x, vec, M, s0, n, lds);
          __syncthreads();
          staged = whole;
        }
      }
      for (int gi = wave; gi < n; gi += 16 * U) {
        multiply(s0, n, gi, 0);
        if (gi + 16 * U < n) load(b0, s0, n, gi + 16 * U, 0);
        if (gi + 8 * U < n) {
          multiply(s0, n, gi + 8 * U, 1);
          if (gi + 24 * U < n) load(b0, s0, n, gi + 24 * U, 1);
        }
      }
    }
    if (whole && b0 + stride < blocks) first(b0 + stride, g0, (int)(g1 - g0));
#pragma unroll
    for (int b = 0; b < RB; ++b) red[(b * 8 + wave) * 64 + lane] = acc[b];
    __syncthreads();
    for (int b = wave; b < RB; b += 8) {
      auto sum = [&](int row) {
        const f32v4 *d = red + b * 512 + g * 16 + row;
        f32v4 v = d[0];
        for (int k = 1; k < 8; ++k) v += d[k * 64];
        return v;
      };
      if (r < M && b0 + b < blocks) {
        f32v4 v = sum(X == XF32 ? 3 * r : r);
        if constexpr (X == XF32) {   // the parts, small ones first; an infinite or NaN large one is the result (nt.h)
          const f32v4 l = sum(3 * r + 2) + sum(3 * r + 1);
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = fabsf(v[i]) < __builtin_huge_valf() ? v[i] + l[i] : v[i];
        }
        const int64_t n = (b0 + b) * 16 + 4 * g;
        if (part) *reinterpret_cast<f32v4 *>(part + ((int64_t)blockIdx.y * M + r) * (blocks * 16) + n) = v;
        else o.put(r, n, v);
      }
    }
    __syncthreads();
  }
}

struct RowsPlan {
  int rb, parts, slice;
  int64_t wgs, z_groups;
  size_t lds, part_bytes;
};
// Up to 16 rows in 4 bits, 8 of bf16 and 5 of float32: laying out more of the others in every workgroup takes longer than
// their operand made once for the products by tiles (8192 x 8192,
// bf16: 16.4 us for 8 rows here, 19.1 for 9 and 19.7 for 17 by tiles, where 16 rows took 27.8 here).
inline bool few_rows(int X, int64_t M) { return M <= (X == X4 ? 16 : X == XBF ? 8 : 5); }
// A workgroup of 8 waves per compute unit or more; the contraction is divided among workgroups only where there are too
// few row blocks for that and every wave keeps 4 groups.  More row blocks a workgroup share the rows' staging and reads, fewer
// leave more workgroups.  One, two and four, us a call at 8192 columns of x, the weights not in the caches:
//   row blocks          256               512              1024              4096            16384
//   bf16, 1 row     8.4 10.6 13.1    14.9 12.7 17.6   27.4 23.0 22.5   66.6 68.3 66.3    218 204 196
//   bf16, 8 rows   14.1 13.6 15.4    25.9 18.6 20.4   48.7 34.6 28.4    179  128 96.6    674 496 349
//   float32, 1 row  9.6 11.0 13.7    16.8 13.6 18.2   31.0 24.6 23.4   71.8 72.2 69.5    232 210 199
//   4 bits, 1 row   6.9  8.8 10.8    11.6  9.5 15.2   20.7 16.5 19.3   60.0 52.8 60.4    222 182 190
// The two borders are for all of them together, and for counts that fill the compute units: 4-bit rows of 4096 and more row blocks would be
// 5 to 15% faster with two, 8 rows of 1024 20% faster with four, and 384 row blocks (one bf16 row, 13.8) 20% with two.
static RowsPlan rows_plan(int X, int64_t M, int64_t N, int64_t groups) {
  RowsPlan p{};
  const int64_t blocks = blocks_of(N, 16);
  p.rb = blocks >= 4096 ? 4 : blocks >= 512 ? 2 : 1;
  p.wgs = std::min<int64_t>(blocks_of(blocks, p.rb), 1024);
  const int64_t z = std::max<int64_t>(1, std::min<int64_t>(256 / p.wgs, groups / 32));
  p.z_groups = blocks_of(groups, z);
  p.parts = (int)blocks_of(groups, p.z_groups);
  const size_t per = (size_t)M * 256 * X;   // bytes of a group's rows
  const size_t room = 112 << 10;   // (registers let one workgroup on a compute unit)
  p.slice = X == X4 ? (int)p.z_groups : (int)std::min<int64_t>(p.z_groups, std::max<int64_t>(8, room / per / 8 * 8));
  p.lds = (size_t)p.rb * 8 * 64 * 16 + per * (X == X4 ? 0 : p.slice);
  p.part_bytes = p.parts > 1 ? (size_t)p.parts * M * blocks * 64 : 0;
  return p;
}
template <int X>
static hipError_t launch_rows(const DevMat &x, const MxDev &a, const MxDev &w, const RowsPlan &p, const OutMat &o, float *part, hipStream_t s) {
  const int vec = x.p && rows_aligned(x.p, x.ld, X == XBF ? 2 : 4), M = (int)o.rows;
  const dim3 grid((unsigned)p.wgs, (unsigned)p.parts);
  if (p.parts == 1) part = nullptr;
  auto go = [&](auto kernel) {
    if (p.lds > 64 << 10) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)p.lds);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, grid, dim3(512), p.lds, s, x, vec, a, w, M, p.slice, (int)p.z_groups, o, part);
    return hipGetLastError();
  };
  hipError_t e = p.rb == 4 ? go(k_rows<X, 4>) : p.rb == 2 ? go(k_rows<X, 2>) : go(k_rows<X, 1>);
  if (e != hipSuccess || !part) return e;
  const int64_t ld = blocks_of(o.cols, 16) * 16;
  hipLaunchKernelGGL(k_join, dim3((unsigned)blocks_of(o.rows * (ld / 4), 256)), dim3(256), 0, s, part, p.parts, o.rows, ld, o);
  return hipGetLastError();
}

// h: another matrix of the same type, in the same launch (x.p null: none)
static hipError_t launch_planes(PlanesArgs g, PlanesArgs h, hipStream_t s) {
  const int bytes = g.x.bf16 ? 2 : 4;
  int64_t cols[2] = {1, 1}, tiles[2] = {0, 0};
  PlanesArgs *each[2] = {&g, &h};
  for (int i = 0; i < 2; ++i) {
    PlanesArgs &p = *each[i];
    if (i == 1 && !p.rows && !p.cols) break;
    p.vec = rows_aligned(p.x.p, p.x.ld, bytes) && (!p.y.p || rows_aligned(p.y.p, p.y.ld, bytes));
    // tiles of 64 rows and columns, those of the padding among them
    cols[i] = std::max(blocks_of(p.x.cols, 64), p.rows ? blocks_of(p.row_chunks, 2) : 0);
    tiles[i] = std::max(blocks_of(p.x.rows, 64), p.cols ? blocks_of(p.col_chunks, 2) : 0) * cols[i];
  }
  // (none of them: no rows, and no padding of columns to write)
  return launch_stretches(tiles[0] + tiles[1], [&](int64_t first, dim3 grid) {
    if (g.x.bf16) hipLaunchKernelGGL((k_planes<1, true>), grid, dim3(256), 0, s, g, cols[0], tiles[0], h, cols[1], first);
    else hipLaunchKernelGGL((k_planes<3, false>), grid, dim3(256), 0, s, g, cols[0], tiles[0], h, cols[1], first);
  });
}

}  // namespace vcr

using namespace vcr;

// ---- the context's room for these calls -------------------------------------------------------
vcr_status op_space(vcr_ctx *c, size_t bytes, Workspace **out) {
  vcr_internal::OpSpace *sp = nullptr;
  for (auto &o : c->op_spaces)
    if (o.stream == c->stream) sp = &o;
  try {   // (room for what is kept below too: no exception crosses the ABI)
    if (!sp) {
      c->op_spaces.emplace_back();
      sp = &c->op_spaces.back();
      sp->stream = c->stream;
    }
    c->op_retired.reserve(c->op_retired.size() + 1);
  } catch (const std::bad_alloc &) {
    return VCR_ERR_OOM;
  }
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(c->stream, &cap) != hipSuccess) (void)hipGetLastError();
  const bool capturing = cap != hipStreamCaptureStatusNone;
  sp->w.used = 0;
  *out = &sp->w;
  if (sp->w.cap < bytes) {
    // the cap is of all these rooms together: those that no recorded graph uses give way
    uint64_t kept = 0, idle = 0;
    for (auto &w : c->op_retired) kept += w.cap;
    for (auto &o : c->op_spaces) {
      if (o.held) kept += o.w.cap;
      else if (&o != sp) idle += o.w.cap;   // (this stream's own is replaced)
    }
    if (c->ws_cap > 0 && bytes + kept > c->ws_cap)
      return fail(c, VCR_ERR_OOM, "the call needs %llu bytes of workspace beside %llu that recorded graphs use, the cap is %llu",
                  (unsigned long long)bytes, (unsigned long long)kept, (unsigned long long)c->ws_cap);
    if (capturing)
      return fail(c, VCR_ERR_STATE, "no workspace can be made while the stream is recorded: make the call once before");
    if (c->ws_cap > 0 && bytes + kept + idle > c->ws_cap) {
      HIP_TRY(c, hipDeviceSynchronize());   // (not by stream: the caller may have destroyed some)
      for (auto &o : c->op_spaces)
        if (&o != sp && !o.held && o.w.base) {
          (void)hipFree(o.w.base);
          o.w = Workspace{};
        }
    }
    if (sp->w.base) {
      if (sp->held) {
        c->op_retired.push_back(sp->w);   // a recorded graph uses it
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
    c->peak_ws = std::max(c->peak_ws, held_workspace(c));
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
vcr_status check_contraction(vcr_ctx *c, int64_t k) {
  if (k > VCR_MAX_CONTRACTION)
    return fail(c, VCR_ERR_UNSUPPORTED, "a contraction of %lld exceeds the limit of %lld", (long long)k, (long long)VCR_MAX_CONTRACTION);
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
  const hipError_t launched = launch_stretches(wg, [&](int64_t first, dim3 grid) {
    if (d.bf16) hipLaunchKernelGGL((k_mx_quantize<true>), grid, dim3(256), 0, c->stream, d, vec, q->codes, q->scales, first);
    else hipLaunchKernelGGL((k_mx_quantize<false>), grid, dim3(256), 0, c->stream, d, vec, q->codes, q->scales, first);
  });
  HIP_TRY(c, launched);
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
  const int64_t wg = blocks_of(y->rows, 16) * blocks_of(mx_groups(y->cols), 4);
  const int vec = o.bf16 && rows_aligned(y->p, y->ld, 2) ? 2 : o.vec;   // 16-byte rows of bf16: 8 columns a store
  const hipError_t launched = launch_stretches(wg, [&](int64_t first, dim3 grid) {
    if (o.bf16) hipLaunchKernelGGL((k_mx_dequantize<true>), grid, dim3(256), 0, c->stream, dev(q), y->p, y->ld, vec, first);
    else hipLaunchKernelGGL((k_mx_dequantize<false>), grid, dim3(256), 0, c->stream, dev(q), y->p, y->ld, o.vec, first);
  });
  HIP_TRY(c, launched);
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
  TRY(check_contraction(c, a->cols));
  TRY(op_begin(c));
  if (y->rows == 0) return VCR_OK;
  if (few_rows(X4, y->rows)) {
    const RowsPlan p = rows_plan(X4, y->rows, y->cols, mx_groups(a->cols));
    Workspace *ws = nullptr;
    TRY(op_space(c, p.part_bytes, &ws));
    HIP_TRY(c, (launch_rows<X4>(DevMat{}, dev(a), dev(w), p, out_mat(y, bias, relu != 0), reinterpret_cast<float *>(ws->base), c->stream)));
    return op_end(c);
  }
  NtArgs g{};
  g.A = NtOperand{a->codes, a->scales, (int32_t)blocks_of(a->rows, 16), 0};
  g.B = NtOperand{w->codes, w->scales, (int32_t)blocks_of(w->rows, 16), 0};
  g.chunks = (int32_t)mx_groups(a->cols);
  Workspace *ws = nullptr;
  const size_t room = part_bytes<1, 1, NT_FP4>(y->rows, y->cols, g.chunks);
  TRY(op_space(c, room, &ws));
  HIP_TRY(c, (nt_product<1, 1, NT_FP4>(g, out_mat(y, bias, relu != 0), reinterpret_cast<float *>(ws->base), c->stream)));
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
  TRY(check_contraction(c, x->cols));
  TRY(op_begin(c));
  if (y->rows == 0) return VCR_OK;
  const DevMat d = dev(x);
  const int P = d.bf16 ? 1 : 3;
  if (few_rows(P, y->rows)) {
    const RowsPlan p = rows_plan(P, y->rows, y->cols, mx_groups(x->cols));
    Workspace *ws = nullptr;
    TRY(op_space(c, p.part_bytes, &ws));
    float *part = reinterpret_cast<float *>(ws->base);
    if (d.bf16) HIP_TRY(c, (launch_rows<XBF>(d, MxDev{}, dev(w), p, out_mat(y, bias, relu != 0), part, c->stream)));
    else HIP_TRY(c, (launch_rows<XF32>(d, MxDev{}, dev(w), p, out_mat(y, bias, relu != 0), part, c->stream)));
    return op_end(c);
  }
  const int64_t chunks = 4 * mx_groups(x->cols), rb = blocks_of(x->rows, 16);
  const size_t room = d.bf16 ? part_bytes<1, 1, NT_MIXED>(y->rows, y->cols, chunks) : part_bytes<3, 1, NT_MIXED>(y->rows, y->cols, chunks);
  const size_t xb = (size_t)rb * chunks * P * FRAG;
  Workspace *ws = nullptr;
  TRY(op_space(c, al(xb) + al(room), &ws));
  uint8_t *xp = take<uint8_t>(*ws, xb);
  float *part = reinterpret_cast<float *>(ws->base + ws->used);
  PlanesArgs pl{};
  pl.x = d;
  pl.rows = xp;
  pl.row_blocks = rb;
  pl.row_chunks = chunks;
  pl.grouped = 1;
  HIP_TRY(c, launch_planes(pl, PlanesArgs{}, c->stream));
  NtArgs g{};
  g.A = NtOperand{xp, nullptr, (int32_t)rb, 0};
  g.B = NtOperand{w->codes, w->scales, (int32_t)blocks_of(w->rows, 16), 0};
  g.chunks = (int32_t)chunks;
  const OutMat o = out_mat(y, bias, relu != 0);
  if (d.bf16) HIP_TRY(c, (nt_product<1, 1, NT_MIXED>(g, o, part, c->stream)));
  else HIP_TRY(c, (nt_product<3, 1, NT_MIXED>(g, o, part, c->stream)));
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
  if (dx && dw && x->cols != w->cols) return fail(c, VCR_ERR_SHAPE, "x and w differ in columns");
  if (dw && x->type != dy->type) return fail(c, VCR_ERR_ARG, "x and dy differ in type");
  if (dx) TRY(check_contraction(c, N));
  if (dw) TRY(check_contraction(c, M));
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
    b_part = P == 1 ? part_bytes<1, 1, NT_BF16>(M, kx, nch) : part_bytes<3, 1, NT_BF16>(M, kx, nch);
  }
  if (dw) {
    b_gt = (size_t)nb * mch * P * FRAG;
    b_xt = (size_t)kwb * mch * P * FRAG;
    b_part = std::max(b_part, P == 1 ? part_bytes<1, 1, NT_BF16>(N, kw, mch) : part_bytes<3, 3, NT_BF16>(N, kw, mch));
  }
  const int64_t mg = blocks_of(std::max<int64_t>(M, 1), 64);
  if (db) b_sums = (size_t)mg * N * 4;
  Workspace *ws = nullptr;
  TRY(op_space(c, al(b_g) + al(b_wt) + al(b_gt) + al(b_xt) + al(b_sums) + al(b_part) + 6 * 256, &ws));
  uint8_t *gp = take<uint8_t>(*ws, b_g), *wt = take<uint8_t>(*ws, b_wt), *gt = take<uint8_t>(*ws, b_gt), *xt = take<uint8_t>(*ws, b_xt);
  float *sums = take<float>(*ws, b_sums / 4), *part = take<float>(*ws, b_part / 4);
  if (has_dx || dw || db) {   // g's rows, its columns and their sums in one pass, and x's columns
    PlanesArgs pl{};
    pl.x = g;
    pl.y = mask;
    if (has_dx) {
      pl.rows = gp;
      pl.row_blocks = mb;
      pl.row_chunks = nch;
    }
    if (dw) {
      pl.cols = gt;
      pl.col_blocks = nb;
      pl.col_chunks = mch;
    }
    pl.sums = db ? sums : nullptr;
    PlanesArgs xl{};
    if (dw) {
      xl.x = dev(x);
      xl.cols = xt;
      xl.col_blocks = kwb;
      xl.col_chunks = mch;
    }
    HIP_TRY(c, launch_planes(pl, xl, s));
  }
  if (db) {
    const hipError_t launched = launch_stretches(blocks_of(N, 64), [&](int64_t first, dim3 grid) {
      hipLaunchKernelGGL(k_column_sums, grid, dim3(256), 0, s, sums, M > 0 ? mg : 0, N, db, first);
    });
    HIP_TRY(c, launched);
  }
  if (has_dx) {
    hipLaunchKernelGGL(k_mx_planes_t, dim3((unsigned)(nch * blocks_of(mx_groups(kx), 4))), dim3(256), 0, s, dev(w), nch, kxb, wt);
    HIP_TRY(c, hipGetLastError());
    NtArgs a{};
    a.A = NtOperand{gp, nullptr, (int32_t)mb, 0};
    a.B = NtOperand{wt, nullptr, (int32_t)kxb, 0};
    a.chunks = (int32_t)nch;
    const OutMat o = out_mat(dx, nullptr, 0);
    if (P == 1) HIP_TRY(c, (nt_product<1, 1, NT_BF16>(a, o, part, s)));
    else HIP_TRY(c, (nt_product<3, 1, NT_BF16>(a, o, part, s)));
  }
  if (dw) {
    NtArgs a{};
    a.A = NtOperand{gt, nullptr, (int32_t)nb, 0};
    a.B = NtOperand{xt, nullptr, (int32_t)kwb, 0};
    a.chunks = (int32_t)mch;
    const OutMat o = out_mat(dw, nullptr, 0);
    if (P == 1) HIP_TRY(c, (nt_product<1, 1, NT_BF16>(a, o, part, s)));
    else HIP_TRY(c, (nt_product<3, 3, NT_BF16>(a, o, part, s)));
  }
  return op_end(c);
}

}  // extern "C"
