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
// bf16 operands may also be as a program has them: rows of a pitch, 16-byte aligned and of a multiple of 8 columns, or of padding
// that may be read up to one.
//   Rows whose columns are contracted (NT_ROWS, and A of NT_RT).  A wave-wide load takes 16 / KS rows' 64 KS bytes, whole lines from two chunks a
//   stage on, into LDS rows of 64 KS bytes, whose 16-byte pieces change places within their row by the row's number, so that the 16 lanes
//   that LDS serves together read from all banks.
//   Rows that are contracted (NT_TT, and B of NT_RT): operand row i is column i of the matrix.  A chunk is 32 rows' 2 BM or 2 BN bytes; a lane's
//   eight values are two of LDS's transposing reads, each of 4 rows by 16 columns for 16 lanes, whose 32-byte pieces change places by the row's number, so
//   that those of the 8 rows that 32 lanes read lie in different banks.
// In both the permutation is applied to the addresses that are read from memory (a load to LDS has no other).  What lies beyond the matrix
// is read in the place of the nearest that does not, and zeroed in LDS where it would be contracted.
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
  int64_t pitch, rows;   // as a program has them: bytes from one row of the matrix to the next, rows of the operand
};
struct NtArgs {
  NtOperand A, B;
  int32_t chunks;       // of the contraction
  int32_t tri;          // only the tiles that hold a block on or below the diagonal
  int32_t z_chunks;     // chunks of one part of the contraction (a multiple of KS; grid y parts)
  // Tiles are counted in a shape of bm x bn, n_mt x n_nt of them and `tiles` in use per matrix of a batch.  A
  // launch takes those from `first` on, each as sub_m x sub_n of its own.
  int32_t bm, bn, n_mt, n_nt, tiles, first, sub_m, sub_n;
  int32_t cols;         // as a program has them: length of the contraction
};

// both bf16, both 4-bit, A bf16 (grouped) and B 4-bit; bf16 as a program has them: both with contracted columns, B or both with contracted rows
enum NtKind : int { NT_BF16 = 0, NT_FP4 = 1, NT_MIXED = 2, NT_ROWS = 3, NT_RT = 4, NT_TT = 5 };
enum : int { NT_BF16_DENSE = 16 };   // classes of NtTiles alone: NT_BF16 with other shapes

template <int KIND_, int MB_, int NB_, int WM_, int WN_, int WK_, int PA_, int PB_, int KS_, int NS_>
struct NtTile {
  static constexpr int MB = MB_, NB = NB_, WM = WM_, WN = WN_, WK = WK_, PA = PA_, PB = PB_, KS = KS_, NS = NS_;
  static constexpr bool FP4 = KIND_ == NT_FP4, MIXED = KIND_ == NT_MIXED, ROWS = KIND_ >= NT_ROWS;
  static constexpr bool AT = KIND_ == NT_TT, BT = KIND_ >= NT_RT;   // contracted rows
  static constexpr int PIECES = 4 * KS_;   // 16-byte pieces of a stage's row with contracted columns
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
  static_assert(!ROWS || (PA == 1 && PB == 1 && (KS & (KS - 1)) == 0 && KS <= 4 && (MB & (MB - 1)) == 0 && (NB & (NB - 1)) == 0), "rows of one part");
  // contracted columns: where piece p of row r (of 16) lies in its row
  static __device__ __forceinline__ int place(int r, int p) { return p ^ (r / (4 / KS) & (PIECES - 1)); }
  // contracted rows: by what the 32-byte pieces of row n of `rows` operand rows change places
  static __device__ __forceinline__ int turn(int rows, int n) {
    return rows >= 128 ? (n & 3) | (n >> 3 & 1) << 2 : rows == 64 ? (n >> 1 & 1) | (n >> 3 & 1) << 1 : rows == 32 ? n >> 3 & 1 : 0;
  }
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
// One with STAGED is given eight columns of a row instead: the tile goes through LDS, so that a wave has whole stretches of rows
// (an epilogue that reads other matrices, or writes two, then moves whole lines, and its code is there once and not for every
// block of a wave).  Col col(n): what it takes of columns n .. n + 7, asked for once; store8(m, n, values, col).
template <class EPI, class = void>
struct nt_staged : std::false_type {};
template <class EPI>
struct nt_staged<EPI, std::enable_if_t<EPI::STAGED>> : std::true_type {};
// Row blocks of a wave that go through LDS together (rows of BN + 4 floats)
template <class T>
constexpr int nt_stage_blocks() {
  int n = T::MB;
  while (n > 1 && (n * T::WM * 16 * (T::BN + 4) * 4 > T::LDS || T::MB % n)) --n;
  return n;
}
// The tile of workgroup `id` of `total`, over part `z` of the contraction; lds: T::LDS bytes
template <class T, class EPI>
__device__ __forceinline__ void nt_run(const NtArgs &g, const EPI &epi, uint8_t *lds, int id, int total, int z) {
  constexpr int MB = T::MB, NB = T::NB, NW = T::NW, KS = T::KS, NS = T::NS, PA = T::PA, PB = T::PB;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave % T::WM, wn = wave / T::WM % T::WN, wk = wave / (T::WM * T::WN);
  int batch, mt, nt;
  nt_tile(g, id, total, batch, mt, nt);
  const int rb0 = mt * (T::BM / 16), cb0 = nt * (T::BN / 16);
  // (parts of a larger tile may lie outside)
  if (rb0 >= g.A.row_blocks || cb0 >= g.B.row_blocks || (g.tri && cb0 >= rb0 + T::BM / 16)) return;
  const int kc0 = z * g.z_chunks, kc1 = min(g.chunks, kc0 + g.z_chunks);
  const int KT = (kc1 - kc0 + KS - 1) / KS;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t *)lds;

  // Loads: a wave-uniform address of the tile's first row block and the stage, and each load's own offset from it,
  // formed once (32 bits: launch_nt).  Row blocks beyond the last one read that.  (Forming the addresses anew for every
  // load cost a wave that has its SIMD to itself as much time as its products.)
  const int b_chunks = T::MIXED ? g.chunks / 4 : g.chunks, bk0 = T::MIXED ? kc0 / 4 : kc0;   // B's fragments of a row block
  const uint8_t *a_base = g.A.p + (T::AT ? 32 * kc0 * g.A.pitch + (int64_t)rb0 * 32 : T::ROWS ? 16 * rb0 * g.A.pitch + (int64_t)kc0 * 64 : batch * g.A.stride + ((int64_t)rb0 * g.chunks + kc0) * PA * FRAG);
  const uint8_t *b_base = g.B.p + (T::BT ? 32 * kc0 * g.B.pitch + (int64_t)cb0 * 32 : T::ROWS ? 16 * cb0 * g.B.pitch + (int64_t)kc0 * 64 : batch * g.B.stride + ((int64_t)cb0 * b_chunks + bk0) * PB * FRAG);
  uint32_t f_off[T::FQ];
  // contracted rows: the row of load l of br operand rows; a wave's loads of a stage are NW apart, which is a multiple of 16 rows, so that all have the
  // lane's offset of the first, and a step apart
  auto t_row = [&](int l, int br) { return l * (FRAG / 2 / br) + lane / (br / 8); };
  auto t_offset = [&](const NtOperand &o, int br, int rb) {
    const int n = t_row(wave, br), p = lane % (br / 8) ^ 2 * T::turn(br, n);
    return (uint32_t)(n * o.pitch) + (uint32_t)min((int64_t)p, (o.rows - 1 - 16 * (int64_t)rb) / 8) * 16;
  };
  static_assert(!T::ROWS || (T::FA % NW == 0 && T::FB % NW == 0 && NW * (FRAG / 2 / T::BM) % 16 == 0 && NW * (FRAG / 2 / T::BN) % 16 == 0), "loads in step");
  const uint32_t ta_off = T::AT ? t_offset(g.A, T::BM, rb0) : 0, tb_off = T::BT ? t_offset(g.B, T::BN, cb0) : 0;
  const int64_t ta_step = T::AT ? NW * (FRAG / 2 / T::BM) * g.A.pitch : 0, tb_step = T::BT ? NW * (FRAG / 2 / T::BN) * g.B.pitch : 0;
#pragma unroll
  for (int q = 0; q < T::FQ; ++q) {
    const int f = min(q * NW + wave, T::FA + T::FB - 1);
    if constexpr (T::ROWS) {
      const bool is_a = q * NW < T::FA;
      if (is_a ? T::AT : T::BT) {
        f_off[q] = 0;   // (t_off)
      } else {
        const int l = is_a ? f : f - T::FA, r = l % KS * (16 / KS) + lane / T::PIECES, row = l / KS * 16 + r;
        const NtOperand &o = is_a ? g.A : g.B;
        const int64_t first = 16 * (int64_t)(is_a ? rb0 : cb0);
        f_off[q] = (uint32_t)((min(first + row, o.rows - 1) - first) * o.pitch) + T::place(r, lane % T::PIECES) * 16;
      }
    } else if (f < T::FA) {   // wave-uniform
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
    int first;       // as a program has them: its first place in the contraction
  };
  auto stage = [&](int kt, uint32_t at) {   // at: its place in LDS
    return Stage{a_base + kt * (T::AT ? 32 * KS * g.A.pitch : (int64_t)(T::ROWS ? KS * 64 : KS * PA * FRAG)),
                 b_base + kt * (T::BT ? 32 * KS * g.B.pitch : (int64_t)(T::ROWS ? KS * 64 : T::BF * FRAG)), lds0 + at,
                 (T::MIXED ? bk0 + kt : kc0 + kt * KS) / 4 * 256, KS - (kc1 - kc0 - kt * KS), (kc0 + kt * KS) * 32};
  };
  auto load = [&](const Stage &s, int q, auto last) {   // load q < LOADS of this wave
    if (q < T::FQ) {
      const int f = min(q * NW + wave, T::FA + T::FB - 1);
      const bool is_a = (q + 1) * NW <= T::FA || (q * NW < T::FA && f < T::FA);
      const bool rows = is_a ? T::AT : T::BT;   // contracted ones (then is_a is known for the whole q)
      const int qi = is_a ? q : q - T::FA / NW;
      uint32_t off = rows ? is_a ? ta_off : tb_off : f_off[q];
      const uint8_t *base = is_a ? s.a : s.b;
      if (T::ROWS && rows) base += qi * (is_a ? ta_step : tb_step);
      if constexpr (decltype(last)::value) {   // the contraction's last chunk is read in the place of those beyond it
        if constexpr (T::ROWS) {   // (the last row or piece of columns)
          const int l = is_a ? f : f - T::FA;
          if (rows) {   // (from the stage's first row on: the lane's own may lie beyond the last)
            const int br = is_a ? T::BM : T::BN;
            off += (uint32_t)((min(t_row(l, br), g.cols - 1 - s.first) - t_row(wave, br)) * (is_a ? g.A.pitch : g.B.pitch));
            base -= qi * (is_a ? ta_step : tb_step);
          } else {
            const int r = l % KS * (16 / KS) + lane / T::PIECES;
            off -= max(0, s.first / 8 + T::place(r, lane % T::PIECES) - (g.cols - 1) / 8) * 16;
          }
        } else {
          const int P = is_a ? PA : PB, kc = (is_a ? f : f - T::FA) % (KS * P) / P;
          off -= max(0, kc - (KS - s.over - 1)) * (P * FRAG);
        }
      }
      nt_dma(base, off, s.lds + f * FRAG, true);
    } else if constexpr (SCALES) {
      const int i = min((q - T::FQ) * NW + wave, T::SA + T::SB - 1);
      nt_dma(s_base[q - T::FQ] + s.at4, lane * 4, s.lds + (T::FA + T::FB) * FRAG + i * 256, false);
    }
  };
  auto issue = [&](int kt, int buf) {
    const Stage s = stage(kt, buf * T::STAGE);
    if (!T::ROWS && (KS == 1 || T::MIXED || s.over <= 0)) {
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
  auto row_at = [&](int blk, int kc) { return blk * (KS * FRAG) + (lane & 15) * (KS * 64) + T::place(lane & 15, kc * 4 + (lane >> 4)) * 16; };
  // contracted rows of br columns: where this lane's values of the wave's first block begin (t_base; a power of two of blocks, so that
  // block i's are at that with i's bits turned), and chunk kc of block i
  auto t_base = [&](int br, int blk) {
    const int n = 8 * (lane >> 4) + (lane >> 2 & 3);   // and n + 4, which turns as n
    return (uint32_t)(n * (2 * br) + (blk ^ T::turn(br, n)) * 32 + (lane & 3) * 8);
  };
  uint32_t ta = T::AT ? t_base(T::BM, wm * MB) : 0, tb = T::BT ? t_base(T::BN, wn * NB) : 0;
  auto transposed = [&](const uint8_t *st, uint32_t base, int br, int i, int kc) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef const __attribute__((address_space(3))) uint8_t *Lds;
    const Lds at = (Lds)st + (base ^ i * 32) + kc * (64 * br);
    s16x4 v[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) v[t] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(at + t * (8 * br)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto turned_anew = [&] {   // (the blocks' addresses are formed where they are used: kept over the loop, they would not fit the registers)
    if constexpr (T::AT) asm volatile("" : "+v"(ta));
    if constexpr (T::BT) asm volatile("" : "+v"(tb));
  };
  auto read_a = [&](Chunk &c, int kt, const uint8_t *st, int kc, int i, int p) {
    if constexpr (T::AT) {
      c.a[i][p] = transposed(st, ta, T::BM, i, kc);
      return;
    }
    if constexpr (T::ROWS) {
      c.a[i][p] = *reinterpret_cast<const bf16x8 *>(st + row_at(wm * MB + i, kc));
      return;
    }
    c.a[i][p] = *reinterpret_cast<const bf16x8 *>(st + (((wm * MB + i) * KS + kc) * PA + p) * FRAG + lane * 16);
    if constexpr (T::FP4) {
      const uint32_t *s = reinterpret_cast<const uint32_t *>(st + (T::FA + T::FB) * FRAG) + lane;
      c.as[i] = (int)(s[(wm * MB + i) * 64] >> 8 * ((kc0 + kt * KS + kc) & 3));
    }
  };
  auto read_b = [&](Chunk &c, int kt, const uint8_t *st, int kc, int j, int p) {
    if constexpr (T::BT) {
      c.b[j][p] = transposed(st + T::FA * FRAG, tb, T::BN, j, kc);
      return;
    }
    if constexpr (T::ROWS) {
      c.b[j][p] = *reinterpret_cast<const bf16x8 *>(st + T::FA * FRAG + row_at(wn * NB + j, kc));
      return;
    }
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
    if (NS > 5 && later > 3 && kt + 4 < KT) wait_vmcnt<4 * T::LOADS>();
    else if (NS > 4 && later > 2 && kt + 3 < KT) wait_vmcnt<3 * T::LOADS>();
    else if (later > 1 && kt + 2 < KT) wait_vmcnt<2 * T::LOADS>();
    else if (later > 0 && kt + 1 < KT) wait_vmcnt<T::LOADS>();
    else wait_vmcnt<0>();
  };

  static_assert(NS >= 2 && NS <= 6, "at most four stages in flight behind the one waited for");
  // A wave's chunks in turn: chunk k of stage kt is multiplied while the operands of the next one are read.  With the last
  // chunk of a stage, stage kt + 1 has landed; the barrier publishes it and frees stage kt, whose operands every wave has
  // in registers, for stage kt + NS.  (Two register sets, and the loop takes two stages at a time, so that none is copied.)
  constexpr int KW = T::KW, AREADS = MB * PA, BREADS = T::MIXED ? 0 : NB * PB, GROUPS = MB * T::PRODUCTS;
  Chunk set[2];
  Codes codes[T::MIXED ? 2 : 1];
  // Where stage kt lies in LDS, as one number: taken apart by the compiler, every address of a loop of two stages has a sum of its own (five
  // updates of 1024 x 1024, whose tiles have three stages, 733 us and 720; of two stages the loop knows the places, and keeps them).
  auto stage_at = [&](int kt) {
    uint32_t at = kt % NS * T::STAGE;
    if constexpr (NS > 2) asm("" : "+s"(at));
    return at;
  };
  auto read = [&](Chunk &c, Codes &q, int kt, const uint8_t *st, int k, int n) {   // read n of chunk k of stage kt (at st), and of a stage's codes with its first
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
  // as a program has them: what lies beyond the contraction in its last stage (which may be anything, in both operands) is zeroed in LDS, and the
  // stage multiplied as the others
  const bool whole = kc1 < g.chunks || g.cols % (32 * KS) == 0;
  auto zero_beyond = [&](int kt) {
    uint8_t *st = lds + kt % NS * T::STAGE;
    const int valid = g.cols - (kc0 + kt * KS) * 32;
    auto operand = [&](uint8_t *at, int br, bool rows) {
      for (int it = threadIdx.x; it < br * 4 * KS; it += T::T) {   // 16-byte pieces
        if (rows) {
          if (it / (br / 8) >= valid) *reinterpret_cast<uint4 *>(at + it * 16) = make_uint4(0, 0, 0, 0);
        } else {
          const int row = it / T::PIECES, p = it % T::PIECES, left = valid - 8 * p;
          if (left >= 8) continue;
          uint4 *d = reinterpret_cast<uint4 *>(at + row / 16 * (KS * FRAG) + row % 16 * (KS * 64) + T::place(row % 16, p) * 16);
          uint4 v = *d;
          uint32_t *w = reinterpret_cast<uint32_t *>(&v);
#pragma unroll
          for (int q = 0; q < 4; ++q) w[q] &= left > 2 * q + 1 ? 0xffffffffu : left == 2 * q + 1 ? 0xffffu : 0u;
          *d = v;
        }
      }
    };
    operand(st, T::BM, T::AT);
    operand(st + T::FA * FRAG, T::BN, T::BT);
    barrier_only();
  };
  // stage kt (sp: its parity), kt + NS + 1 < KT.  LOAD: stage kt + NS is loaded, and is not the last one in part; else it is loaded if there is one.  NEXT:
  // there is a stage after this one
  auto steady_of = [&](int kt, auto sp, auto loads, auto next_one) {
    constexpr int SP = decltype(sp)::value;
    constexpr bool LOAD = decltype(loads)::value, NEXT = decltype(next_one)::value;
#pragma unroll
    for (int k = 0; k < KW; ++k) {
      const Chunk &now = set[(SP * KW + k) & 1];
      Chunk &next = set[(SP * KW + k + 1) & 1];
      const int nk = k + 1 < KW ? k + 1 : 0, nkt = k + 1 < KW ? kt : kt + 1;
      Codes &ncodes = codes[T::MIXED ? SP ^ 1 : 0];   // (read with a stage's first chunk)
      const uint8_t *nst = lds + stage_at(nkt);
      arrived();
      turned_anew();
      Stage ns{};
      if (k + 1 == KW && NEXT) {
        if constexpr (LOAD) wait_vmcnt<(NS - 2) * T::LOADS>();
        else landed(nkt, NS - 2);
        barrier_only();
        if constexpr (LOAD) {
          ns = stage(kt + NS, stage_at(kt));
        } else {
          if (kt + NS < KT) issue(kt + NS, kt % NS);
          if (nkt + 1 == KT && !whole) zero_beyond(nkt);
        }
      }
      if (T::MIXED && k == 0) {
#pragma unroll
        for (int j = 0; j < NB; ++j) expand(codes[T::MIXED ? SP : 0], 0, j);
      }
      // Loads and reads are spread between the groups: a wave issues in order, and would stand still until LDS and the
      // memory pipe have taken all of them.
#pragma unroll
      for (int n = 0; n < GROUPS; ++n) {
        if (k + 1 == KW && LOAD) {
#pragma unroll
          for (int q = n * T::LOADS / GROUPS; q < (n + 1) * T::LOADS / GROUPS; ++q) load(ns, q, std::false_type{});
        }
        if (k + 1 < KW || NEXT) {
#pragma unroll
          for (int q = n * reads(nk) / GROUPS; q < (n + 1) * reads(nk) / GROUPS; ++q) read(next, ncodes, nkt, nst, nk, q);
        }
        if (T::MIXED && k + 1 < KW) {
#pragma unroll
          for (int j = n * NB / GROUPS; j < (n + 1) * NB / GROUPS; ++j) expand(codes[T::MIXED ? SP : 0], k + 1, j);
        }
        multiply(now, mixed[k & 1], n / T::PRODUCTS, n % T::PRODUCTS);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };
  auto steady = [&](int kt, auto sp) { steady_of(kt, sp, std::true_type{}, std::true_type{}); };
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
        for (int n = 0; n < reads(nk); ++n) read(next, codes[T::MIXED ? SP ^ 1 : 0], nkt, lds + nkt % NS * T::STAGE, nk, n);
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
    if (NS > 5 && KT > 5) wait_vmcnt<5 * T::LOADS>();
    else if (NS > 4 && KT > 4) wait_vmcnt<4 * T::LOADS>();
    else if (NS > 3 && KT > 3) wait_vmcnt<3 * T::LOADS>();
    else if (NS > 2 && KT > 2) wait_vmcnt<2 * T::LOADS>();
    else if (KT > 1) wait_vmcnt<T::LOADS>();
    else wait_vmcnt<0>();
    barrier_only();
    if constexpr (T::ROWS) {
      if (KT == 1 && !whole) zero_beyond(0);
    }
#pragma unroll
    for (int n = 0; n < reads(0); ++n) read(set[0], codes[0], 0, lds, 0, n);
  }
  int kt = 0;
  if constexpr (T::ROWS) {
    const int full = KT - (whole ? 0 : 1);
    auto loaded = [&](int t, auto sp) { steady_of(t, sp, std::false_type{}, std::true_type{}); };
    auto final = [&](int t, auto sp) { steady_of(t, sp, std::false_type{}, std::false_type{}); };
    if constexpr (KW % 2 == 0) {   // every stage begins with the first register set
      for (; kt + NS + 1 < full; kt += 2) {
        steady(kt, Even{});
        steady(kt + 1, Even{});
      }
#pragma unroll 1
      for (; kt + 1 < KT; ++kt) loaded(kt, Even{});
      if (KT > 0) final(kt, Even{});
    } else {
      for (; kt + NS + 1 < full; kt += 2) {
        steady(kt, Even{});
        steady(kt + 1, Odd{});
      }
#pragma unroll 1
      for (; kt + 2 < KT; kt += 2) {
        loaded(kt, Even{});
        loaded(kt + 1, Odd{});
      }
      if (kt + 1 < KT) {
        loaded(kt, Even{});
        final(kt + 1, Odd{});
      } else if (KT > 0) {
        final(kt, Even{});
      }
    }
  } else {
    for (; kt + NS + 2 < KT; kt += 2) {
      steady(kt, Even{});
      steady(kt + 1, Odd{});
    }
#pragma unroll 1
    for (; kt < KT; kt += 2) {
      last(kt, Even{});
      if (kt + 1 < KT) last(kt + 1, Odd{});
    }
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
    if constexpr (!nt_staged<EPI>::value) epi.store(batch, z, 16 * (rb0 + wm * MB + i) + r16, 16 * (cb0 + wn * NB + j) + 4 * g4, v, lane);
  };
  if constexpr (nt_staged<EPI>::value) {
    constexpr int PITCH = T::BN + 4, IB = T::WK == 1 ? nt_stage_blocks<T>() : MB;   // row blocks of a wave in a pass
    constexpr int OCTS = T::BN / 8, STEP = T::T / OCTS, HELD = T::WM * IB * 16, ITEMS = (HELD + STEP - 1) / STEP;
    static_assert(T::T % OCTS == 0 && (HELD % STEP == 0 || ITEMS == 1), "whole rows for every thread");
    float *tile = reinterpret_cast<float *>(lds);
    const int oct = threadIdx.x % OCTS, row0 = threadIdx.x / OCTS, n_at = 16 * cb0 + oct * 8;
    auto row_of = [&](int pass, int it) {   // of a thread's item: its row in the tile as it lies in LDS, and in the result
      const int q = row0 + it * STEP, w = q / (16 * IB);
      return 16 * (rb0 + w * MB + pass * IB) + q - w * (16 * IB);
    };
    const typename EPI::Col col = epi.col(n_at);
    auto rows_out = [&](int pass) {
      barrier_only();
      if (HELD % STEP != 0 && row0 >= HELD) return;
      // (rolled: with the items' copies of its code an epilogue outgrows the instruction cache, 9 us a tile of 256 x 256)
#pragma unroll 1
      for (int it = 0; it < ITEMS; ++it) {
        const float *s = tile + (row0 + it * STEP) * PITCH + oct * 8;
        const f32v4 a = *reinterpret_cast<const f32v4 *>(s), b = *reinterpret_cast<const f32v4 *>(s + 4);
        float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        epi.store8(row_of(pass, it), n_at, v, col);
      }
    };
    if constexpr (T::WK == 1) {
      static_assert(IB * T::WM * 16 * PITCH * 4 <= T::LDS, "rows of a tile in LDS");
#pragma unroll
      for (int p = 0; p < MB / IB; ++p) {
        barrier_only();   // what LDS held has been read
#pragma unroll
        for (int i = 0; i < IB; ++i)
#pragma unroll
          for (int j = 0; j < NB; ++j)
            *reinterpret_cast<f32v4 *>(tile + ((wm * IB + i) * 16 + r16) * PITCH + (wn * NB + j) * 16 + 4 * g4) = joined(p * IB + i, j);
        rows_out(p);
      }
    } else {
      constexpr int B = MB * NB, PER = (B + T::WK - 1) / T::WK;
      static_assert(T::BM * PITCH * 4 <= T::LDS, "the tile in LDS");
      f32v4 *red = reinterpret_cast<f32v4 *>(lds) + (wm + T::WM * wn) * T::WK * B * 64 + lane;
      barrier_only();   // the last stage has been read
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) red[(wk * B + i * NB + j) * 64] = joined(i, j);
      __syncthreads();
      f32v4 sum[PER];   // of blocks wk, wk + WK, ..
#pragma unroll
      for (int n = 0; n < PER; ++n) {
        const int blk = min(n * T::WK + wk, B - 1);
        sum[n] = red[blk * 64];
#pragma unroll
        for (int q = 1; q < T::WK; ++q) sum[n] += red[(q * B + blk) * 64];
      }
      __syncthreads();
#pragma unroll
      for (int n = 0; n < PER; ++n) {
        const int blk = n * T::WK + wk, i = blk / NB, j = blk - i * NB;
        if (blk < B) *reinterpret_cast<f32v4 *>(tile + ((wm * MB + i) * 16 + r16) * PITCH + (wn * NB + j) * 16 + 4 * g4) = sum[n];
      }
      rows_out(0);
    }
  } else if constexpr (T::WK == 1) {
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

constexpr int nt_min_blocks(int waves, int lds) { return waves == 4 && 2 * lds > 160 * 1024 ? 1 : 2; }
template <class T, class EPI>
__global__ __launch_bounds__(T::T, nt_min_blocks(T::NW, T::LDS)) void k_nt(const NtArgs g, const EPI epi) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[T::LDS];
  nt_run<T>(g, epi, lds, blockIdx.x, gridDim.x, blockIdx.y);
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
      if (sh[a].bm % sh[b].bm || sh[a].bn % sh[b].bn) continue;   // (not whole tiles of it)
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

// g for `count` tiles of shape (bm, bn) from `first` on, by kernels of shape T
template <class T>
hipError_t nt_args(NtArgs &g, int64_t M, int64_t N, int bm, int bn, int64_t first, int64_t count, int parts) {
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
  if (T::ROWS ? std::max(g.A.pitch, g.B.pitch) * std::max({T::BM, T::BN, 32 * T::KS}) > 0xffffffffll
              : (int64_t)g.chunks * 3 * FRAG * (std::max(T::BM, T::BN) / 16) > 0xffffffffll)
    return hipErrorInvalidValue;
  if (mt <= 0 || nt <= 0 || g.chunks <= 0 || tiles > 0x7fffffff || grid <= 0 || grid > 0x7fffffff || first + count > 0x7fffffff ||
      g.sub_m * T::BM != bm || g.sub_n * T::BN != bn || parts <= 0 || parts > 65535)
    return hipErrorInvalidValue;
  const int kt = (g.chunks + T::KS - 1) / T::KS;
  g.z_chunks = (kt + parts - 1) / parts * T::KS;
  return hipSuccess;
}
// (in launches of what each can count, 32 bits of threads)
template <class T, class EPI>
hipError_t launch_nt(NtArgs g, int64_t M, int64_t N, int bm, int bn, int64_t first, int64_t count, int parts, const EPI &epi, hipStream_t s) {
  const int64_t subs = (int64_t)(bm / T::BM) * (bn / T::BN), most = std::max<int64_t>(1, 0xffffffffll / T::T / std::max<int64_t>(1, subs));
  for (int64_t at = first; at < first + count || at == first; at += most) {
    const int64_t n = std::min(most, first + count - at);
    hipError_t e = nt_args<T>(g, M, N, bm, bn, at, n, parts);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_nt<T, EPI>), dim3((unsigned)(n * subs), (unsigned)parts), dim3(T::T), 0, s, g, epi);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
// The smallest shape
template <class TS, class = void>
struct nt_last {
  typedef typename TS::T4 T;
};
template <class TS>
struct nt_last<TS, std::void_t<typename TS::T5>> {
  typedef typename TS::T5 T;
};
// A product by the shapes of TS (T0 .. T4, or to T5, and their `shapes`)
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
      case 5:
        if constexpr (nt_shapes<TS> > 5) return launch_nt<typename TS::T5>(g, M, N, bm, bn, first, count, 1, epi, s);
        [[fallthrough]];
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
// Operands as a program has them: two chunks a stage, so that wave-wide loads read whole lines of 128 bytes, and two stages for the large tiles (128 KB of
// LDS; four of one chunk read half lines).  4096 x 8192 x 8192: NT_ROWS 364 us (1.51 PFLOP/s), NT_RT 371, NT_TT 399 with the writes of 8192 x 8192 results.
template <int KIND>
struct NtTilesOfRows {
  typedef NtTile<KIND, 8, 4, 2, 4, 1, 1, 1, 2, 2> T0;
  typedef NtTile<KIND, 4, 4, 2, 2, 1, 1, 1, 2, 2> T1;
  typedef NtTile<KIND, 2, 2, 2, 4, 1, 1, 1, 2, 4> T2;
  typedef NtTile<KIND, 2, 2, 2, 2, 1, 1, 1, 2, 4> T3;
  typedef NtTile<KIND, 2, 4, 1, 1, 4, 1, 1, 4, 3> T4;
  static constexpr NtShape shapes[] = {{256, 256, .68f, 0.f}, {128, 128, .242f, .41f}, {64, 128, .147f, 0.f}, {64, 64, .087f, .182f}, {32, 64, .058f, .143f}};
};
template <>
struct NtTiles<1, 1, NT_ROWS> : NtTilesOfRows<NT_ROWS> {};
template <>
struct NtTiles<1, 1, NT_RT> : NtTilesOfRows<NT_RT> {};
template <>
struct NtTiles<1, 1, NT_TT> : NtTilesOfRows<NT_TT> {};
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
// (with 96 x 128: 2001 x 1500 outputs are 252 of them, one round, where of 128 x 128 a quarter of the compute units has none and of 64 x 128 it
// takes one and a half: 43 us, 47 without)
template <>
struct NtTiles<3, 3, NT_BF16_DENSE> {
  typedef NtTile<NT_BF16, 4, 2, 2, 4, 1, 3, 3, 1, 3> T0;
  typedef NtTile<NT_BF16, 3, 2, 2, 4, 1, 3, 3, 1, 3> T1;
  typedef NtTile<NT_BF16, 2, 2, 2, 4, 1, 3, 3, 2, 2> T2;
  typedef NtTile<NT_BF16, 2, 2, 2, 2, 1, 3, 3, 1, 3> T3;
  typedef NtTile<NT_BF16, 2, 1, 1, 4, 1, 3, 3, 1, 4> T4;
  typedef NtTile<NT_BF16, 2, 2, 1, 1, 4, 3, 3, 4, 3> T5;
  static constexpr NtShape shapes[] = {{128, 128, 1.f, 0.f}, {96, 128, .77f, 0.f}, {64, 128, .546f, 0.f}, {64, 64, .342f, .595f}, {32, 64, .214f, .413f}, {32, 32, .138f, 0.f}};
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
