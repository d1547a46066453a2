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
// A bf16 operand may meet a 4-bit one as it is stored (NT_MIXED): the four chunks of a group of 128 are then, for both, the
// first to fourth eight columns of each of its blocks of 32, so that the 16 bytes a lane has of a 4-bit fragment
// are its columns of four instructions in turn; they become bf16 in registers, exactly, where they are multiplied.
//
// Parts.  float32 values are three bf16 parts h + m + l (split_bf16.h); P parts keep 8 P bits.  Products of
// (A parts, B parts), in order of their size:
//   (1, 1)  h h
//   (3, 1)  l h, m h | h h        B is exact in one part (4-bit values times powers of two)
//   (3, 3)  h l, l h, m m, h m, m h | h h      float32's products (2^-24)
// Where a bar stands, the small products have an accumulator of their own, added at the end: summed into
// the large one they are cut off at its precision, always downwards (split_bf16.h).
//
// A workgroup owns BM x BN outputs: WM x WN x WK waves of MB x NB blocks of 16 x 16, of which WK share a
// block and take every WK-th chunk (their sums are added in LDS, in order).  A stage holds KS chunks of
// its rows; NS stages are in LDS, the later ones' loads run while one is multiplied, and the one barrier
// of a stage both publishes it and frees the one before.  A stage's operands are read into registers
// while the stage before is multiplied, and those reads and the loads of a later stage are spread between the
// matrix instructions: a wave issues in order and would stand still until LDS and the memory pipe had taken them
// all.  (256 x 256 tiles of one part over 96 chunks: 1220 TFLOP/s with them in one piece, 1520 spread; 64 x 64 of
// three parts 760 and 1240.)  The 16 x 16 x 32 (x 128 for 4-bit)
// instruction takes 16 cycles of its SIMD and 1 KB of each operand; MB x NB of them share MB + NB reads
// of LDS, at 128 bytes a cycle.
//
// What bounds it: for large tiles the matrix rate that the card's power allows (2.0 PFLOP/s of bf16 with random operands
// in registers; 1.8 with a stage read from LDS over and over, 1.5 with its loads); for small ones the loads from L2 into
// LDS, of which a compute unit takes 40 to 48 bytes a cycle where all hit, and 27 to 35 in these loops.
#pragma once

#include <algorithm>
#include <type_traits>

#include "lds_dma.h"
#include "mx_bits.h"
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
  int32_t chunks;       // of the contraction
  int32_t tri;          // only the tiles that hold a block on or below the diagonal
  int32_t z_chunks;     // chunks of one part of the contraction (a multiple of KS; grid y parts)
  // Tiles are counted in a shape of bm x bn, n_mt x n_nt of them and `tiles` in use per matrix of a batch.  A
  // launch takes those from `first` on, each as sub_m x sub_n of its own.
  int32_t bm, bn, n_mt, n_nt, tiles, first, sub_m, sub_n;
};

enum NtKind : int { NT_BF16 = 0, NT_FP4 = 1, NT_MIXED = 2 };   // both bf16, both 4-bit, A bf16 (grouped) and B 4-bit

template <int KIND_, int MB_, int NB_, int WM_, int WN_, int WK_, int PA_, int PB_, int KS_, int NS_>
struct NtTile {
  static constexpr int MB = MB_, NB = NB_, WM = WM_, WN = WN_, WK = WK_, PA = PA_, PB = PB_, KS = KS_, NS = NS_;
  static constexpr bool FP4 = KIND_ == NT_FP4, MIXED = KIND_ == NT_MIXED;
  static constexpr int PRODUCTS = PA == 3 ? (PB == 3 ? 6 : 3) : 1;
  static constexpr int KW = KS / WK;   // chunks of a stage that a wave multiplies
  static constexpr int NW = WM * WN * WK, T = 64 * NW;
  static constexpr int BM = 16 * MB * WM, BN = 16 * NB * WN;
  static constexpr bool TWO = PA == 3;   // an accumulator for the small products
  static constexpr int BF = MIXED ? KS / 4 : KS * PB;              // fragments of a stage of 16 columns
  static constexpr int FA = BM / 16 * KS * PA, FB = BN / 16 * BF;   // fragments of a stage
  static constexpr int SA = FP4 ? BM / 16 : 0, SB = FP4 || MIXED ? BN / 16 : 0;   // scale loads (256 bytes) of a stage
  static constexpr int FQ = (FA + FB + NW - 1) / NW, SQ = (SA + SB + NW - 1) / NW;
  static constexpr int LOADS = FQ + SQ;   // of a wave (the last of them may be the same for several)
  static constexpr int STAGE = (FA + FB) * FRAG + (SA + SB) * 256;
  static constexpr int LDS = NS * STAGE;
  static_assert(!FP4 || 4 % KS == 0, "a stage's scales are in one group of four chunks");
  static_assert(!MIXED || (KS == 4 && PB == 1), "a stage is a group");
  static_assert(KS % WK == 0 && (WK == 1 || NW * MB * NB * 1024 <= LDS), "waves that share a block");
  static_assert(KW == 1 || KW % 2 == 0, "register sets alternate");
};

// 16 (wide) or 4 bytes a lane, at a 32-bit offset from a wave-uniform base, into LDS at lane times that many (dma16's form)
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

// Columns of tiles in use of row mt of tiles: with tri, those up to its last row's diagonal
__host__ __device__ inline int nt_row_tiles(int mt, int bm, int bn, int n_nt, bool tri) {
  const int n = (int)(((int64_t)(mt + 1) * bm + bn - 1) / bn);
  return tri && n < n_nt ? n : n_nt;
}
// The tile of a workgroup.  Workgroup ids go round the 8 XCDs; each XCD gets a contiguous range of
// tiles in an order in which 4 rows of tiles sweep the columns together, so that its L2 serves them.
__device__ __forceinline__ void nt_tile(const NtArgs &g, int id, int total, int &batch, int &mt, int &nt) {
  const int x = id & 7, t = id >> 3, q = total >> 3, rem = total & 7;
  const int at = x * q + min(x, rem) + t, subs = g.sub_m * g.sub_n, par = g.first + at / subs, sub = at % subs;
  batch = par / g.tiles;
  int left = par - batch * g.tiles;
  if (!g.tri) {
    const int per = 4 * g.n_nt, first = left / per * 4, rows = min(4, g.n_mt - first), i = left - first * g.n_nt;
    mt = first + i % rows;
    nt = i / rows;
  } else {
    mt = 0;
    for (;;) {
      const int n = nt_row_tiles(mt, g.bm, g.bn, g.n_nt, true);
      if (left < n || mt + 1 == g.n_mt) break;
      left -= n;
      ++mt;
    }
    nt = left;
  }
  mt = mt * g.sub_m + sub % g.sub_m;
  nt = nt * g.sub_n + sub / g.sub_m;
}

// EPI: a struct with store(batch, part of the contraction, m, n, values of n .. n + 3, lane): called by
// whole waves for every block, with the lane's row m and first column n; the other lanes of a block hold
// its other rows and columns.
template <class T, class EPI>
__global__ __launch_bounds__(T::T, T::NW == 4 && 2 * T::LDS > 160 * 1024 ? 1 : 2) void k_nt(const NtArgs g, const EPI epi) {
  constexpr int MB = T::MB, NB = T::NB, NW = T::NW, KS = T::KS, NS = T::NS, PA = T::PA, PB = T::PB;
  __shared__ __attribute__((aligned(16))) uint8_t lds[T::LDS];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM % T::WN, wk = wave / (T::WM * T::WN);
  int batch, mt, nt;
  nt_tile(g, blockIdx.x, gridDim.x, batch, mt, nt);
  const int rb0 = mt * (T::BM / 16), cb0 = nt * (T::BN / 16);
  // (parts of a larger tile may lie outside)
  if (rb0 >= g.A.row_blocks || cb0 >= g.B.row_blocks || (g.tri && cb0 >= rb0 + T::BM / 16)) return;
  const int kc0 = blockIdx.y * g.z_chunks, kc1 = min(g.chunks, kc0 + g.z_chunks);
  const int KT = (kc1 - kc0 + KS - 1) / KS;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t *)lds;

  // Loads: a wave-uniform address of the tile's first row block and the stage, and each load's own offset from it,
  // formed once (32 bits: launch_nt).  Row blocks beyond the last one read that.  (Forming the addresses anew for every
  // load cost a wave that has its SIMD to itself as much time as its products.)
  const int b_chunks = T::MIXED ? g.chunks / 4 : g.chunks, bk0 = T::MIXED ? kc0 / 4 : kc0;   // B's fragments of a row block
  const uint8_t *a_base = g.A.p + batch * g.A.stride + ((int64_t)rb0 * g.chunks + kc0) * PA * FRAG;
  const uint8_t *b_base = g.B.p + batch * g.B.stride + ((int64_t)cb0 * b_chunks + bk0) * PB * FRAG;
  uint32_t f_off[T::FQ];
#pragma unroll
  for (int q = 0; q < T::FQ; ++q) {
    const int f = min(q * NW + wave, T::FA + T::FB - 1);
    if (f < T::FA) {   // wave-uniform
      const int i = f / (KS * PA);
      f_off[q] = ((uint32_t)min(i, g.A.row_blocks - 1 - rb0) * g.chunks * PA + (f - i * (KS * PA))) * FRAG + lane * 16;
    } else {
      const int i = (f - T::FA) / T::BF;
      f_off[q] = ((uint32_t)min(i, g.B.row_blocks - 1 - cb0) * b_chunks * PB + (f - T::FA - i * T::BF)) * FRAG + lane * 16;
    }
  }
  // scales: of four fragments together
  constexpr bool SCALES = T::SQ > 0;
  const int c4 = (b_chunks + 3) / 4;
  const uint8_t *s_base[SCALES ? T::SQ : 1];
  if constexpr (SCALES) {
#pragma unroll
    for (int q = 0; q < T::SQ; ++q) {
      const int i = min(q * NW + wave, T::SA + T::SB - 1);
      s_base[q] = i < T::SA ? g.A.scales + (int64_t)min(rb0 + i, g.A.row_blocks - 1) * c4 * 256
                            : g.B.scales + (int64_t)min(cb0 + i - T::SA, g.B.row_blocks - 1) * c4 * 256;
    }
  }

  struct Stage {   // wave-uniform addresses of a stage's loads
    const uint8_t *a, *b;
    uint32_t lds;
    int at4, over;   // over: chunks of the stage beyond the contraction
  };
  auto stage = [&](int kt, int buf) {
    return Stage{a_base + (int64_t)kt * (KS * PA * FRAG), b_base + (int64_t)kt * (T::BF * FRAG), lds0 + buf * T::STAGE,
                 (T::MIXED ? bk0 + kt : kc0 + kt * KS) / 4 * 256, KS - (kc1 - kc0 - kt * KS)};
  };
  auto load = [&](const Stage &s, int q, auto last) {   // load q < LOADS of this wave
    if (q < T::FQ) {
      const int f = min(q * NW + wave, T::FA + T::FB - 1);
      const bool is_a = (q + 1) * NW <= T::FA || (q * NW < T::FA && f < T::FA);
      uint32_t off = f_off[q];
      if constexpr (decltype(last)::value) {   // the contraction's last chunk is read in the place of those beyond it
        const int P = is_a ? PA : PB, kc = (is_a ? f : f - T::FA) % (KS * P) / P;
        off -= max(0, kc - (KS - s.over - 1)) * (P * FRAG);
      }
      nt_dma(is_a ? s.a : s.b, off, s.lds + f * FRAG, true);
    } else if constexpr (SCALES) {
      const int i = min((q - T::FQ) * NW + wave, T::SA + T::SB - 1);
      nt_dma(s_base[q - T::FQ] + s.at4, lane * 4, s.lds + (T::FA + T::FB) * FRAG + i * 256, false);
    }
  };
  auto issue = [&](int kt, int buf) {
    const Stage s = stage(kt, buf);
    if (KS == 1 || T::MIXED || s.over <= 0) {
#pragma unroll
      for (int q = 0; q < T::LOADS; ++q) load(s, q, std::false_type{});
    } else {
#pragma unroll
      for (int q = 0; q < T::LOADS; ++q) load(s, q, std::true_type{});
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

  // operands of a wave's chunk in registers; of a 4-bit B, the stage's
  struct Chunk {
    bf16x8 b[T::MIXED ? 1 : NB][PB], a[MB][PA];
    int bs[T::FP4 ? NB : 1], as[T::FP4 ? MB : 1];
  };
  constexpr int CW = T::WK == 1 ? 4 : T::KW;   // words of a 4-bit fragment that a wave multiplies
  struct Codes {
    uint32_t w[NB][CW], s[NB];
  };
  auto read_a = [&](Chunk &c, int kt, const uint8_t *st, int kc, int i, int p) {
    c.a[i][p] = *reinterpret_cast<const bf16x8 *>(st + (((wm * MB + i) * KS + kc) * PA + p) * FRAG + lane * 16);
    if constexpr (T::FP4) {
      const uint32_t *s = reinterpret_cast<const uint32_t *>(st + (T::FA + T::FB) * FRAG) + lane;
      c.as[i] = (int)(s[(wm * MB + i) * 64] >> 8 * ((kc0 + kt * KS + kc) & 3));
    }
  };
  auto read_b = [&](Chunk &c, int kt, const uint8_t *st, int kc, int j, int p) {
    c.b[j][p] = *reinterpret_cast<const bf16x8 *>(st + (T::FA + ((wn * NB + j) * KS + kc) * PB + p) * FRAG + lane * 16);
    if constexpr (T::FP4) {
      const uint32_t *s = reinterpret_cast<const uint32_t *>(st + (T::FA + T::FB) * FRAG) + lane;
      c.bs[j] = (int)(s[(T::SA + wn * NB + j) * 64] >> 8 * ((kc0 + kt * KS + kc) & 3));
    }
  };
  auto read_codes = [&](Codes &c, int kt, const uint8_t *st, int j) {
    const uint8_t *f = st + (T::FA + wn * NB + j) * FRAG + lane * 16;
    if constexpr (T::WK == 1) {
      const i32x4 q = *reinterpret_cast<const i32x4 *>(f);
#pragma unroll
      for (int k = 0; k < 4; ++k) c.w[j][k] = (uint32_t)q[k];
    } else {
#pragma unroll
      for (int k = 0; k < CW; ++k) c.w[j][k] = *reinterpret_cast<const uint32_t *>(f + (k * T::WK + wk) * 4);
    }
    c.s[j] = *reinterpret_cast<const uint32_t *>(st + (T::FA + T::FB) * FRAG + (wn * NB + j) * 256 + lane * 4) >> 8 * ((bk0 + kt) & 3);
  };
  auto multiply = [&](const Chunk &c, const bf16x8 (&mixed)[T::MIXED ? NB : 1], int i, int p) {   // product p of row block i with the wave's columns
    if constexpr (T::FP4) {
      auto wide = [](bf16x8 v) {
        const i32x4 q = __builtin_bit_cast(i32x4, v);
        return i32x8{q[0], q[1], q[2], q[3], 0, 0, 0, 0};
      };
#pragma unroll
      for (int j = 0; j < NB; ++j)
        hi[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(c.b[j][0]), wide(c.a[i][0]), hi[i][j], 4, 4, 0, c.bs[j], 0, c.as[i]);
    } else {
      // (A part, B part) and accumulator of product p
      constexpr int pa33[6] = {0, 2, 1, 0, 1, 0}, pb33[6] = {2, 0, 1, 1, 0, 0}, pa31[3] = {2, 1, 0};
      const int pa = T::PRODUCTS == 6 ? pa33[p] : PA == 3 ? pa31[p] : 0;
      const int pb = T::PRODUCTS == 6 ? pb33[p] : 0;
      const bool small = T::TWO && p + 1 < T::PRODUCTS;
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        f32v4 &acc = small ? lo[T::TWO ? i : 0][T::TWO ? j : 0] : hi[i][j];
        if constexpr (T::MIXED) acc = mfma_bf16(mixed[j], c.a[i][pa], acc);
        else acc = mfma_bf16(c.b[j][pb], c.a[i][pa], acc);
      }
    }
  };
  auto landed = [&](int kt, int later) {   // this wave's loads of stage kt, with `later` stages issued after it
    if (later > 1 && kt + later < KT) wait_vmcnt<2 * T::LOADS>();
    else if (later > 0 && kt + 1 < KT) wait_vmcnt<T::LOADS>();
    else wait_vmcnt<0>();
  };

  static_assert(NS >= 2 && NS <= 4, "at most two stages in flight behind the one waited for");
  // A wave's chunks in turn: chunk k of stage kt is multiplied while the operands of the next one are read.  With the last
  // chunk of a stage, stage kt + 1 has landed; the barrier publishes it and frees stage kt, whose operands every wave has
  // in registers, for stage kt + NS.  (Two register sets, and the loop takes two stages at a time, so that none is copied.)
  constexpr int KW = T::KW, AREADS = MB * PA, BREADS = T::MIXED ? 0 : NB * PB, GROUPS = MB * T::PRODUCTS;
  Chunk set[2];
  Codes codes[T::MIXED ? 2 : 1];
  auto read = [&](Chunk &c, Codes &q, int kt, int k, int n) {   // read n of chunk k of stage kt, and of a stage's codes with its first
    const uint8_t *st = lds + kt % NS * T::STAGE;
    if (n < BREADS) read_b(c, kt, st, k * T::WK + wk, n / PB, n % PB);
    else if (n < BREADS + AREADS) read_a(c, kt, st, k * T::WK + wk, (n - BREADS) / PA, (n - BREADS) % PA);
    else if constexpr (T::MIXED) read_codes(q, kt, st, n - BREADS - AREADS);
  };
  auto reads = [](int k) { return BREADS + AREADS + (T::MIXED && k == 0 ? NB : 0); };
  // 4-bit columns as bf16: those of a stage's first chunk ahead of its products, the later ones' between the products before
  bf16x8 mixed[2][T::MIXED ? NB : 1];
  float m_scale[T::MIXED ? NB : 1];
  auto expand = [&](const Codes &q, int k, int j) {
    if constexpr (T::MIXED) {
      if (k == 0) m_scale[j] = mx_scale(q.s[j] & 255);
      mixed[k & 1][j] = __builtin_bit_cast(bf16x8, mx_to_bf16(q.w[j][k], m_scale[j]));
    }
  };
  // `now` is in registers: told to the compiler before the reads of the next set, whose end it would otherwise wait for before
  // the products of `now`
  auto arrived = [] { __builtin_amdgcn_s_waitcnt(0xc07f); };   // lgkmcnt(0)
  auto steady = [&](int kt, auto sp) {   // stage kt (sp: its parity), kt + NS + 1 < KT
    constexpr int SP = decltype(sp)::value;
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      const Chunk &now = set[(SP * KW + k) & 1];
      Chunk &next = set[(SP * KW + k + 1) & 1];
      const int nk = k + 1 < KW ? k + 1 : 0, nkt = k + 1 < KW ? kt : kt + 1;
      Codes &ncodes = codes[T::MIXED ? SP ^ 1 : 0];   // (read with a stage's first chunk)
      arrived();
      Stage ns{};
      if (k + 1 == KW) {
        wait_vmcnt<(NS - 2) * T::LOADS>();
        barrier_only();
        ns = stage(kt + NS, kt % NS);
      }
      if (T::MIXED && k == 0) {
#pragma unroll
        for (int j = 0; j < NB; ++j) expand(codes[T::MIXED ? SP : 0], 0, j);
      }
      // Loads and reads are spread between the groups: a wave issues in order, and would stand still until LDS and the
      // memory pipe have taken all of them.
#pragma unroll
      for (int n = 0; n < GROUPS; ++n) {
        if (k + 1 == KW) {
#pragma unroll
          for (int q = n * T::LOADS / GROUPS; q < (n + 1) * T::LOADS / GROUPS; ++q) load(ns, q, std::false_type{});
        }
#pragma unroll
        for (int q = n * reads(nk) / GROUPS; q < (n + 1) * reads(nk) / GROUPS; ++q) read(next, ncodes, nkt, nk, q);
        if (T::MIXED && k + 1 < KW) {
#pragma unroll
          for (int j = n * NB / GROUPS; j < (n + 1) * NB / GROUPS; ++j) expand(codes[T::MIXED ? SP : 0], k + 1, j);
        }
        multiply(now, mixed[k & 1], n / T::PRODUCTS, n % T::PRODUCTS);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  auto last = [&](int kt, auto sp) {   // the same, of the last stages
    constexpr int SP = decltype(sp)::value;
    const int left = kc1 - kc0 - kt * KS;
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      const Chunk &now = set[(SP * KW + k) & 1];
      Chunk &next = set[(SP * KW + k + 1) & 1];
      const int nk = k + 1 < KW ? k + 1 : 0, nkt = k + 1 < KW ? kt : kt + 1;
      arrived();
      if (k + 1 == KW && nkt < KT) {
        landed(nkt, NS - 2);
        barrier_only();
        if (kt + NS < KT) issue(kt + NS, kt % NS);
      }
      if (nkt < KT) {
#pragma unroll
        for (int n = 0; n < reads(nk); ++n) read(next, codes[T::MIXED ? SP ^ 1 : 0], nkt, nk, n);
      }
      if (k * T::WK + wk < left) {   // wave-uniform
        if constexpr (T::MIXED) {
#pragma unroll
          for (int j = 0; j < NB; ++j) expand(codes[T::MIXED ? SP : 0], k, j);
        }
#pragma unroll
        for (int n = 0; n < GROUPS; ++n) multiply(now, mixed[k & 1], n / T::PRODUCTS, n % T::PRODUCTS);
      }
    }
  };
  typedef std::integral_constant<int, 0> Even;
  typedef std::integral_constant<int, 1> Odd;
  if (KT > 0) {
#pragma unroll
    for (int t = 0; t < NS; ++t)
      if (t < KT) issue(t, t);
    // stage 0, with up to NS - 1 behind it
    if (NS > 3 && KT > 3) wait_vmcnt<3 * T::LOADS>();
    else if (NS > 2 && KT > 2) wait_vmcnt<2 * T::LOADS>();
    else if (KT > 1) wait_vmcnt<T::LOADS>();
    else wait_vmcnt<0>();
    barrier_only();
#pragma unroll
    for (int n = 0; n < reads(0); ++n) read(set[0], codes[0], 0, 0, n);
  }
  int kt = 0;
  for (; kt + NS + 2 < KT; kt += 2) {
    steady(kt, Even{});
    steady(kt + 1, Odd{});
  }
#pragma unroll 1
  for (; kt < KT; kt += 2) {
    last(kt, Even{});
    if (kt + 1 < KT) last(kt + 1, Odd{});
  }

  const int r16 = lane & 15, g4 = lane >> 4;
  auto joined = [&](int i, int j) {
    f32v4 v = hi[i][j];
    if constexpr (T::TWO) {
      // (an infinite or NaN large product is the result: the small ones of such operands are NaN)
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = fabsf(v[q]) < __builtin_huge_valf() ? v[q] + lo[i][j][q] : v[q];
    }
    return v;
  };
  auto put = [&](int i, int j, f32v4 v) {
    epi.store(batch, blockIdx.y, 16 * (rb0 + wm * MB + i) + r16, 16 * (cb0 + wn * NB + j) + 4 * g4, v, lane);
  };
  if constexpr (T::WK == 1) {
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) put(i, j, joined(i, j));
  } else {
    f32v4 *red = reinterpret_cast<f32v4 *>(lds) + (wm + T::WM * wn) * T::WK * MB * NB * 64 + lane;
    barrier_only();   // the last stage has been read
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j) red[(wk * MB * NB + i * NB + j) * 64] = joined(i, j);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NB; ++j)
        if ((i * NB + j) % T::WK == wk) {
          f32v4 v = red[(i * NB + j) * 64];
#pragma unroll
          for (int q = 1; q < T::WK; ++q) v += red[(q * MB * NB + i * NB + j) * 64];
          put(i, j, v);
        }
  }
}

// ---- which tiles -------------------------------------------------------------------------------
// The shapes of one class of products, largest first; a tile of one is whole tiles of every later one.  A large shape
// spends less per output, a small one wastes less of the chip's last round, and where two workgroups fit a compute unit
// each hides the other's start and end.  So a product's time is estimated for each from what was measured (us1, us2),
// and the whole rounds may go to one shape and what is left of the last to another, in a launch of its own.
struct NtShape {
  int bm, bn;
  float us1, us2;   // us of a chunk of a workgroup alone on its compute unit, of two together (0: only one fits)
};
constexpr int NT_CUS = 256;
// of a launch, of a workgroup's start and end, and a compute unit's share of the memory's rate
constexpr float NT_LAUNCH_US = 4.f, NT_ROUND_US = 2.f, NT_WRITE_BYTES_US = 20e3f;
struct NtPlan {
  int main = 0, rest = -1;   // shapes
  int64_t main_tiles = 0, rest_tiles = 0;   // counted in main's shape, over the batch
  float us = 0.f;
};
inline int64_t nt_tiles(int64_t M, int64_t N, int bm, int bn, bool tri) {
  const int64_t mt = (M + bm - 1) / bm, nt = (N + bn - 1) / bn;
  if (!tri) return mt * nt;
  int64_t s = 0;
  for (int64_t i = 0; i < mt; ++i) s += nt_row_tiles((int)i, bm, bn, (int)nt, true);
  return s;
}
// out_bytes: what the epilogue writes per output; of a workgroup alone on its compute unit nothing hides it
inline float nt_us(const NtShape &s, int64_t tiles, int64_t chunks, float out_bytes) {
  const int64_t n = (tiles + NT_CUS - 1) / NT_CUS;
  const float end = NT_ROUND_US + (s.us2 > 0.f ? .3f : 1.f) * (float)(s.bm * s.bn) * out_bytes / NT_WRITE_BYTES_US;
  const float one = s.us1 * (float)chunks + end, two = s.us2 * (float)chunks + end;
  return NT_LAUNCH_US + (s.us2 > 0.f ? (float)(n / 2) * two + (float)(n % 2) * one : (float)n * one);
}
// (TS: a class of products, with its `shapes`)
template <class TS>
constexpr int nt_shapes = sizeof(TS::shapes) / sizeof(NtShape);
template <class TS>
NtPlan nt_plan(int64_t M, int64_t N, int64_t chunks, int64_t batch, bool tri, float out_bytes) {
  constexpr const NtShape *sh = TS::shapes;
  NtPlan best;
  for (int a = 0; a < nt_shapes<TS>; ++a) {
    const int64_t t = nt_tiles(M, N, sh[a].bm, sh[a].bn, tri) * batch;
    const float all = nt_us(sh[a], t, chunks, out_bytes);
    if (a == 0 || all < best.us) {
      best.main = a;
      best.rest = -1;
      best.main_tiles = t;
      best.rest_tiles = 0;
      best.us = all;
    }
    const int64_t round = sh[a].us2 > 0.f ? 2 * NT_CUS : NT_CUS, full = t / round * round;
    if (full == 0 || full == t) continue;
    for (int b = a + 1; b < nt_shapes<TS>; ++b) {
      const int64_t subs = (int64_t)(sh[a].bm / sh[b].bm) * (sh[a].bn / sh[b].bn);
      const float us = nt_us(sh[a], full, chunks, out_bytes) + nt_us(sh[b], (t - full) * subs, chunks, out_bytes);
      if (us < best.us) {
        best.main = a;
        best.rest = b;
        best.main_tiles = full;
        best.rest_tiles = t - full;
        best.us = us;
      }
    }
  }
  return best;
}
// Parts of the contraction: few tiles over a long contraction leave compute units idle.  Parts of 16 chunks and more are
// then summed by their own workgroups (the smallest shape) and joined in order, where that pays for the second launch.
template <class TS>
int nt_parts(int64_t M, int64_t N, int64_t chunks) {
  const NtShape &x = TS::shapes[nt_shapes<TS> - 1];
  const int64_t t = nt_tiles(M, N, x.bm, x.bn, false), parts = std::min<int64_t>(NT_CUS / t, chunks / 16);
  if (parts < 2) return 1;
  return nt_us(x, t * parts, (chunks + parts - 1) / parts, 4.f) + NT_LAUNCH_US < nt_plan<TS>(M, N, chunks, 1, false, 4.f).us ? (int)parts : 1;
}

// `count` tiles of shape (bm, bn) from `first` on, by kernels of shape T
template <class T, class EPI>
hipError_t launch_nt(NtArgs g, int64_t M, int64_t N, int bm, int bn, int64_t first, int64_t count, int parts, const EPI &epi, hipStream_t s) {
  const int64_t mt = (M + bm - 1) / bm, nt = (N + bn - 1) / bn;
  g.bm = bm;
  g.bn = bn;
  g.n_mt = (int32_t)mt;
  g.n_nt = (int32_t)nt;
  const int64_t tiles = nt_tiles(M, N, bm, bn, g.tri);
  g.tiles = (int32_t)tiles;
  g.first = (int32_t)first;
  g.sub_m = bm / T::BM;
  g.sub_n = bn / T::BN;
  const int64_t grid = count * g.sub_m * g.sub_n;
  // (a tile's row blocks are reached by 32-bit offsets)
  if ((int64_t)g.chunks * 3 * FRAG * (std::max(T::BM, T::BN) / 16) > 0xffffffffll) return hipErrorInvalidValue;
  if (mt <= 0 || nt <= 0 || g.chunks <= 0 || tiles > 0x7fffffff || grid <= 0 || grid > 0x7fffffff || first + count > 0x7fffffff ||
      g.sub_m * T::BM != bm || g.sub_n * T::BN != bn || parts <= 0 || parts > 65535)
    return hipErrorInvalidValue;
  const int kt = (g.chunks + T::KS - 1) / T::KS;
  g.z_chunks = (kt + parts - 1) / parts * T::KS;
  hipLaunchKernelGGL((k_nt<T, EPI>), dim3((unsigned)grid, (unsigned)parts), dim3(T::T), 0, s, g, epi);
  return hipGetLastError();
}
// A product by the shapes of TS (T0 .. T4 and their `shapes`)
template <class TS, class EPI>
hipError_t launch_nt_plan(const NtArgs &g, int64_t M, int64_t N, int64_t batch, float out_bytes, const EPI &epi, hipStream_t s) {
  const NtPlan p = nt_plan<TS>(M, N, g.chunks, batch, g.tri, out_bytes);
  auto go = [&](int shape, int64_t first, int64_t count) {
    const int bm = TS::shapes[p.main].bm, bn = TS::shapes[p.main].bn;
    switch (shape) {
      case 0: return launch_nt<typename TS::T0>(g, M, N, bm, bn, first, count, 1, epi, s);
      case 1: return launch_nt<typename TS::T1>(g, M, N, bm, bn, first, count, 1, epi, s);
      case 2: return launch_nt<typename TS::T2>(g, M, N, bm, bn, first, count, 1, epi, s);
      case 3: return launch_nt<typename TS::T3>(g, M, N, bm, bn, first, count, 1, epi, s);
      default: return launch_nt<typename TS::T4>(g, M, N, bm, bn, first, count, 1, epi, s);
    }
  };
  const hipError_t e = go(p.main, 0, p.main_tiles);
  return e != hipSuccess || p.rest < 0 ? e : go(p.rest, p.main_tiles, p.rest_tiles);
}

// The shapes of products of PA and PB parts; their times were measured over 24 and 72 chunks of 256 and 512 tiles.  T0 .. T3 and
// T4, the last and smallest one again where a class has fewer.
template <int PA, int PB, int KIND>
struct NtTiles;
template <>
struct NtTiles<1, 1, NT_FP4> {
  typedef NtTile<NT_FP4, 8, 4, 2, 4, 1, 1, 1, 1, 4> T0;
  typedef NtTile<NT_FP4, 4, 4, 2, 2, 1, 1, 1, 1, 4> T1;
  typedef NtTile<NT_FP4, 2, 2, 2, 4, 1, 1, 1, 2, 4> T2;
  typedef NtTile<NT_FP4, 2, 2, 2, 2, 2, 1, 1, 4, 3> T3;
  typedef NtTile<NT_FP4, 2, 4, 1, 1, 4, 1, 1, 4, 3> T4;
  static constexpr NtShape shapes[] = {{256, 256, .98f, 0.f}, {128, 128, .406f, .562f}, {64, 128, .235f, 0.f}, {64, 64, .113f, 0.f}, {32, 64, .084f, .167f}};
};
template <>
struct NtTiles<1, 1, NT_BF16> {
  typedef NtTile<NT_BF16, 8, 4, 2, 4, 1, 1, 1, 1, 4> T0;
  typedef NtTile<NT_BF16, 4, 4, 2, 2, 1, 1, 1, 1, 4> T1;
  typedef NtTile<NT_BF16, 2, 2, 2, 4, 1, 1, 1, 2, 4> T2;
  typedef NtTile<NT_BF16, 2, 2, 2, 2, 1, 1, 1, 2, 4> T3;
  typedef NtTile<NT_BF16, 2, 4, 1, 1, 4, 1, 1, 4, 3> T4;
  static constexpr NtShape shapes[] = {{256, 256, .68f, 0.f}, {128, 128, .242f, .41f}, {64, 128, .147f, 0.f}, {64, 64, .087f, .182f}, {32, 64, .058f, .143f}};
};
template <>
struct NtTiles<3, 1, NT_BF16> {
  // (128 x 128 takes .568 us where two of 64 x 128 on a compute unit take .532)
  typedef NtTile<NT_BF16, 2, 4, 2, 2, 1, 3, 1, 1, 4> T0;
  typedef NtTile<NT_BF16, 2, 2, 2, 2, 1, 3, 1, 1, 4> T1;
  typedef NtTile<NT_BF16, 2, 2, 1, 2, 2, 3, 1, 2, 4> T2;
  typedef NtTile<NT_BF16, 2, 1, 1, 2, 2, 3, 1, 2, 4> T3;
  typedef T3 T4;
  static constexpr NtShape shapes[] = {{64, 128, .316f, .532f}, {64, 64, .197f, .366f}, {32, 64, .114f, .221f}, {32, 32, .078f, .157f}};
};
template <>
struct NtTiles<3, 3, NT_BF16> {
  typedef NtTile<NT_BF16, 4, 2, 2, 4, 1, 3, 3, 1, 3> T0;
  typedef NtTile<NT_BF16, 2, 2, 2, 4, 1, 3, 3, 2, 2> T1;
  typedef NtTile<NT_BF16, 2, 2, 2, 2, 1, 3, 3, 1, 3> T2;
  typedef NtTile<NT_BF16, 2, 1, 1, 4, 1, 3, 3, 1, 4> T3;
  typedef NtTile<NT_BF16, 2, 2, 1, 1, 4, 3, 3, 4, 3> T4;
  static constexpr NtShape shapes[] = {{128, 128, 1.f, 0.f}, {64, 128, .546f, 0.f}, {64, 64, .342f, .595f}, {32, 64, .214f, .413f}, {32, 32, .138f, 0.f}};
};
template <>
struct NtTiles<1, 1, NT_MIXED> {
  typedef NtTile<NT_MIXED, 8, 2, 1, 8, 1, 1, 1, 4, 3> T0;
  typedef NtTile<NT_MIXED, 4, 2, 1, 4, 2, 1, 1, 4, 4> T1;
  typedef NtTile<NT_MIXED, 4, 2, 1, 4, 1, 1, 1, 4, 3> T2;
  typedef NtTile<NT_MIXED, 4, 1, 1, 4, 1, 1, 1, 4, 3> T3;
  typedef NtTile<NT_MIXED, 2, 1, 1, 4, 1, 1, 1, 4, 4> T4;
  static constexpr NtShape shapes[] = {{128, 256, .366f, 0.f}, {64, 128, .126f, 0.f}, {64, 128, .148f, .234f}, {64, 64, .101f, .149f}, {32, 64, .078f, .107f}};
};
template <>
struct NtTiles<3, 1, NT_MIXED> {
  typedef NtTile<NT_MIXED, 2, 4, 2, 4, 1, 3, 1, 4, 2> T0;
  typedef NtTile<NT_MIXED, 2, 2, 2, 4, 1, 3, 1, 4, 2> T1;
  typedef NtTile<NT_MIXED, 2, 2, 1, 4, 1, 3, 1, 4, 2> T2;
  typedef NtTile<NT_MIXED, 2, 4, 1, 1, 4, 3, 1, 4, 2> T3;
  typedef NtTile<NT_MIXED, 2, 2, 1, 1, 4, 3, 1, 4, 3> T4;
  static constexpr NtShape shapes[] = {{64, 256, .49f, 0.f}, {64, 128, .291f, 0.f}, {32, 128, .18f, .305f}, {32, 64, .115f, .174f}, {32, 32, .093f, .147f}};
};

}  // namespace vcr
