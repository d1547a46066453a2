// Products of two operands whose contraction axis is the contiguous one, D[m][n] = sum_k A[m][k] B[n][k],
// on the matrix cores of gfx950, from operands kept in the order the instructions read.
//
// Operands.  A row block is 16 rows; a chunk is what 16 rows hold in 64 bytes each: 32 bf16 or 128
// 4-bit values.  One (row block, chunk) of one part is a fragment of 1 KB in lane order: lane 16 g + r has
// the 16 bytes g of row r (8 bf16 or 32 4-bit values).  An operand is [row blocks][chunks][parts]
// fragments, so that a fragment goes from memory to LDS by one wave-wide load of 1 KB and from LDS to
// registers by one conflict-free 16-byte read a lane, with no swizzle and no edge: padding rows and
// columns are in memory, and hold zeros.
//
// Parts.  float32 values are three bf16 parts h + m + l (split_bf16.h); P parts keep 8 P bits.  Products of
// (A parts, B parts), in order of their size:
//   (1, 1)  h h
//   (3, 1)  l h, m h | h h        B is exact in one part (4-bit values times powers of two)
//   (2, 2)  h m, m h, h h         16 bits of both
//   (3, 3)  h l, l h, m m, h m, m h | h h      float32's products (2^-24)
// Where a bar stands, the small products have an accumulator of their own, added at the end: summed into
// the large one they are cut off at its precision, always downwards (split_bf16.h).
//
// A workgroup owns BM x BN outputs, WM x WN waves of MB x NB blocks of 16 x 16.  A stage holds KS
// chunks of its rows; two stages are in LDS, the next one's loads run while one is multiplied, and the
// one barrier of a stage both publishes it and frees the other.  The 16 x 16 x 32 (x 128 for 4-bit)
// instruction takes 16 cycles of its SIMD and 1 KB of each operand; MB x NB of them share MB + NB reads
// of LDS, which at 128 bytes a cycle is what bounds small wave tiles.
#pragma once

#include "lds_dma.h"
#include "split_bf16.h"

namespace vcr {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int FRAG = 1024;   // bytes of a fragment

// [row blocks][chunks][parts] fragments; 4-bit operands have scales [row blocks][(chunks + 3) / 4][64 lanes][4 chunks]
struct NtOperand {
  const uint8_t *p;
  const uint8_t *scales;
  int32_t row_blocks;
  int64_t stride;   // bytes from one matrix of a batch to the next
};
struct NtArgs {
  NtOperand A, B;
  int32_t chunks;      // of the contraction
  int32_t n_mt, n_nt;  // tiles
  int32_t tri;         // only the tiles that hold a block on or below the diagonal
  int32_t z_chunks;    // chunks of one part of the contraction (a multiple of KS; grid z parts)
};

template <int MB_, int NB_, int WM_, int WN_, int PA_, int PB_, int KS_, bool FP4_ = false>
struct NtTile {
  static constexpr int MB = MB_, NB = NB_, WM = WM_, WN = WN_, PA = PA_, PB = PB_, KS = KS_;
  static constexpr bool FP4 = FP4_;
  static constexpr int NW = WM * WN, T = 64 * NW;
  static constexpr int BM = 16 * MB * WM, BN = 16 * NB * WN;
  static constexpr bool TWO = PA == 3;   // an accumulator for the small products
  static constexpr int FA = BM / 16 * KS * PA, FB = BN / 16 * KS * PB;   // fragments of a stage
  static constexpr int SA = FP4 ? BM / 16 : 0, SB = FP4 ? BN / 16 : 0;   // scale loads (256 bytes) of a stage
  static constexpr int STAGE = (FA + FB) * FRAG + (SA + SB) * 256;
  static_assert(FA % NW == 0 && FB % NW == 0 && SA % NW == 0 && SB % NW == 0, "loads spread evenly over the waves");
  static_assert(!FP4 || (4 % KS == 0), "a stage's scales are in one group of four chunks");
};

// 4 bytes a lane from a wave-uniform base into LDS (dma16's form)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void nt_dma(const void *base, uint32_t off, uint32_t lds, bool wide) {
  const uint64_t b = (uint64_t)(uintptr_t)base;
  const uint64_t ub = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)b) |
                      (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(b >> 32)) << 32;
  const uint32_t l = __builtin_amdgcn_readfirstlane(lds);
  if (wide)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(l), "v"(off), "s"(ub) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(l), "v"(off), "s"(ub) : "memory", "m0");
}
#pragma clang diagnostic pop

// The four lanes r, r ^ 1, r ^ 2, r ^ 3 hold a 4 x 4 block (lane, element); afterwards its transpose.
template <int CTRL>   // quad permutation: 0xb1 the neighbour r ^ 1, 0x4e r ^ 2
__device__ __forceinline__ float quad_swap(float a) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, a), CTRL, 15, 15, true));
}
__device__ __forceinline__ f32v4 quad_transpose(f32v4 v, int lane) {
  const bool b0 = lane & 1, b1 = lane & 2;
  float s = quad_swap<0xb1>(b0 ? v[0] : v[1]), t = quad_swap<0xb1>(b0 ? v[2] : v[3]);
  if (b0) v[0] = s, v[2] = t;
  else v[1] = s, v[3] = t;
  s = quad_swap<0x4e>(b1 ? v[0] : v[2]);
  t = quad_swap<0x4e>(b1 ? v[1] : v[3]);
  if (b1) v[0] = s, v[1] = t;
  else v[2] = s, v[3] = t;
  return v;
}

// The tile of a workgroup.  Workgroup ids go round the 8 XCDs; each XCD gets a contiguous range of
// tiles in an order in which 4 rows of tiles sweep the columns together, so that its L2 serves them.
template <class T>
__device__ __forceinline__ void nt_tile(const NtArgs &g, int id, int total, int &mt, int &nt) {
  const int x = id & 7, t = id >> 3, q = total >> 3, rem = total & 7;
  const int at = x * q + min(x, rem) + t;
  if (!g.tri) {
    const int per = 4 * g.n_nt, first = at / per * 4, rows = min(4, g.n_mt - first), i = at - first * g.n_nt;
    mt = first + i % rows;
    nt = i / rows;
    return;
  }
  // row mt has the tiles nt whose first column is within or left of its last row
  int left = at;
  mt = 0;
  for (;;) {
    const int n = min(g.n_nt, ((mt + 1) * T::BM + T::BN - 1) / T::BN);
    if (left < n || mt + 1 == g.n_mt) break;
    left -= n;
    ++mt;
  }
  nt = left;
}
template <class T>
int nt_tiles(int n_mt, int n_nt, bool tri) {
  if (!tri) return n_mt * n_nt;
  int s = 0;
  for (int mt = 0; mt < n_mt; ++mt) {
    const int n = ((mt + 1) * T::BM + T::BN - 1) / T::BN;
    s += n < n_nt ? n : n_nt;
  }
  return s;
}

// EPI: a struct with store(batch, part of the contraction, m, n, values of n .. n + 3, lane): called by
// whole waves for every block, with the lane's row m and first column n; the other lanes of a block hold
// its other rows and columns.
template <class T, class EPI>
__global__ __launch_bounds__(T::T, 2) void k_nt(const NtArgs g, const EPI epi) {
  constexpr int MB = T::MB, NB = T::NB, NW = T::NW, KS = T::KS, PA = T::PA, PB = T::PB;
  __shared__ __attribute__((aligned(16))) uint8_t lds[2 * T::STAGE];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM;
  int mt, nt;
  nt_tile<T>(g, blockIdx.x, gridDim.x, mt, nt);
  const int rb0 = mt * (T::BM / 16), cb0 = nt * (T::BN / 16);
  const uint8_t *Ap = g.A.p + (int64_t)blockIdx.y * g.A.stride;
  const uint8_t *Bp = g.B.p + (int64_t)blockIdx.y * g.B.stride;
  const int kc0 = blockIdx.z * g.z_chunks, kc1 = min(g.chunks, kc0 + g.z_chunks);
  const int KT = (kc1 - kc0 + KS - 1) / KS;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t *)lds;

  auto issue = [&](int kt, int buf) {
    const uint32_t st = lds0 + buf * T::STAGE;
#pragma unroll
    for (int q = 0; q < T::FA / NW; ++q) {
      const int f = q * NW + wave, i = f / (KS * PA), kp = f - i * (KS * PA), kc = kp / PA;
      const int64_t at = (int64_t)min(rb0 + i, g.A.row_blocks - 1) * g.chunks + min(kc0 + kt * KS + kc, kc1 - 1);
      nt_dma(Ap + (at * PA + (kp - kc * PA)) * FRAG, lane * 16, st + f * FRAG, true);
    }
#pragma unroll
    for (int q = 0; q < T::FB / NW; ++q) {
      const int f = q * NW + wave, i = f / (KS * PB), kp = f - i * (KS * PB), kc = kp / PB;
      const int64_t at = (int64_t)min(cb0 + i, g.B.row_blocks - 1) * g.chunks + min(kc0 + kt * KS + kc, kc1 - 1);
      nt_dma(Bp + (at * PB + (kp - kc * PB)) * FRAG, lane * 16, st + (T::FA + f) * FRAG, true);
    }
    if constexpr (T::FP4) {
      const int c4 = (g.chunks + 3) / 4, at4 = (kc0 + kt * KS) / 4;
#pragma unroll
      for (int q = 0; q < T::SA / NW; ++q) {
        const int i = q * NW + wave;
        nt_dma(g.A.scales + ((int64_t)min(rb0 + i, g.A.row_blocks - 1) * c4 + at4) * 256, lane * 4,
               st + (T::FA + T::FB) * FRAG + i * 256, false);
      }
#pragma unroll
      for (int q = 0; q < T::SB / NW; ++q) {
        const int i = q * NW + wave;
        nt_dma(g.B.scales + ((int64_t)min(cb0 + i, g.B.row_blocks - 1) * c4 + at4) * 256, lane * 4,
               st + (T::FA + T::FB) * FRAG + (T::SA + i) * 256, false);
      }
    }
  };

  f32v4 hi[MB][NB], lo[T::TWO ? MB : 1][T::TWO ? NB : 1];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      hi[i][j] = f32v4{0.f, 0.f, 0.f, 0.f};
      if constexpr (T::TWO) lo[i][j] = f32v4{0.f, 0.f, 0.f, 0.f};
    }

  auto multiply = [&](int kt, const uint8_t *st, int kc) {
    const uint8_t *a = st + ((wm * MB * KS + kc) * PA) * FRAG + lane * 16;
    const uint8_t *b = st + T::FA * FRAG + ((wn * NB * KS + kc) * PB) * FRAG + lane * 16;
    if constexpr (T::FP4) {
      const uint32_t *s = reinterpret_cast<const uint32_t *>(st + (T::FA + T::FB) * FRAG) + lane;
      const int sh = 8 * ((kc0 + kt * KS + kc) & 3);
      i32x4 bv[NB];
      int bs[NB];
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        bv[j] = *reinterpret_cast<const i32x4 *>(b + j * KS * FRAG);
        bs[j] = (int)(s[(T::SA + wn * NB + j) * 64] >> sh);
      }
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        const i32x4 av = *reinterpret_cast<const i32x4 *>(a + i * KS * FRAG);
        const int as = (int)(s[(wm * MB + i) * 64] >> sh);
        const i32x8 aw = {av[0], av[1], av[2], av[3], 0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < NB; ++j) {
          const i32x8 bw = {bv[j][0], bv[j][1], bv[j][2], bv[j][3], 0, 0, 0, 0};
          hi[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bw, aw, hi[i][j], 4, 4, 0, bs[j], 0, as);
        }
      }
    } else {
      bf16x8 bv[NB][PB];
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int p = 0; p < PB; ++p) bv[j][p] = *reinterpret_cast<const bf16x8 *>(b + (j * KS * PB + p) * FRAG);
#pragma unroll
      for (int i = 0; i < MB; ++i) {
        bf16x8 av[PA];
#pragma unroll
        for (int p = 0; p < PA; ++p) av[p] = *reinterpret_cast<const bf16x8 *>(a + (i * KS * PA + p) * FRAG);
        auto each = [&](int pa, int pb, f32v4 (&acc)[NB]) {
#pragma unroll
          for (int j = 0; j < NB; ++j) acc[j] = mfma_bf16(bv[j][pb], av[pa], acc[j]);
        };
        if constexpr (PA == 3 && PB == 3) {
          each(0, 2, lo[i]);
          each(2, 0, lo[i]);
          each(1, 1, lo[i]);
          each(0, 1, lo[i]);
          each(1, 0, lo[i]);
          each(0, 0, hi[i]);
        } else if constexpr (PA == 3) {
          each(2, 0, lo[i]);
          each(1, 0, lo[i]);
          each(0, 0, hi[i]);
        } else if constexpr (PA == 2) {
          each(0, 1, hi[i]);
          each(1, 0, hi[i]);
          each(0, 0, hi[i]);
        } else {
          each(0, 0, hi[i]);
        }
      }
    }
  };

  if (KT > 0) issue(0, 0);
  int cur = 0;
  for (int kt = 0; kt < KT; ++kt) {
    wait_vmcnt<0>();   // this wave's loads of the stage have landed
    barrier_only();    // every wave's have, and the other stage has been read
    if (kt + 1 < KT) issue(kt + 1, cur ^ 1);
    const uint8_t *st = lds + cur * T::STAGE;
    const int left = kc1 - kc0 - kt * KS;
#pragma unroll
    for (int kc = 0; kc < KS; ++kc)
      if (kc < left) multiply(kt, st, kc);   // wave-uniform
    cur ^= 1;
  }

  const int r16 = lane & 15, g4 = lane >> 4;
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      f32v4 v = hi[i][j];
      if constexpr (T::TWO) {
        // (an infinite or NaN large product is the result: the small ones of such operands are NaN)
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = fabsf(v[q]) < __builtin_huge_valf() ? v[q] + lo[i][j][q] : v[q];
      }
      epi.store(blockIdx.y, blockIdx.z, 16 * (rb0 + wm * MB + i) + r16, 16 * (cb0 + wn * NB + j) + 4 * g4, v, lane);
    }
}

template <class T, class EPI>
hipError_t launch_nt(NtArgs g, int64_t M, int64_t N, int batch, int zs, const EPI &epi, hipStream_t s) {
  const int64_t mt = (M + T::BM - 1) / T::BM, nt = (N + T::BN - 1) / T::BN;
  if (mt <= 0 || nt <= 0 || g.chunks <= 0 || mt * nt > 0x7fffffff || batch <= 0 || batch > 65535 || zs <= 0 || zs > 65535)
    return hipErrorInvalidValue;
  g.n_mt = (int32_t)mt;
  g.n_nt = (int32_t)nt;
  const int kt = (g.chunks + T::KS - 1) / T::KS;
  g.z_chunks = (kt + zs - 1) / zs * T::KS;
  const dim3 grid((unsigned)nt_tiles<T>(g.n_mt, g.n_nt, g.tri), (unsigned)batch, (unsigned)zs);
  hipLaunchKernelGGL((k_nt<T, EPI>), grid, dim3(T::T), 0, s, g, epi);
  return hipGetLastError();
}

}  // namespace vcr
