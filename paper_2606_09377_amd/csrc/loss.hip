// Cross entropy with its gradient: vcr_cross_entropy of vcrown.h.
//
// With m = max x, S = sum exp(x - m), e = m + log S, a row's loss is (m - (1 - s) x_t - s mean x) + log S + c e^2 and its gradient
// a multiple of exp(x - m) less a constant, and less another at the label.  exp(x - m) is 2^((x - m) L), L = log2 e, or where that is safe
// 2^(x L - m L), an instruction less (ExpLess).  The exponent is rounded to float32, by up to 2^-24 of |x - m| L, as x - m is in a plain form; L itself is
// rounded too, which makes it 2^-26 of that too small.  So exp(x - m) is off by about 2^-24 |x - m| of itself: 2e-7 at random where |x - m| is 2 to 8, 4e-7 at 16 to 40 (a
// plain form 1.5e-7 and 6e-7 on float32 logits; nothing on those of few bits, whose differences are exact).  A second word of L would correct the 2^-26 alone, at
// an instruction more for every value; half a unit of the sum's last place is what it amounts to.
#include "training.h"

namespace vcr {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int SELF_COUNT = 1024;   // rows up to which every group of threads counts the labels itself

struct LossArgs {
  MatRef x, d;
  int64_t rows, cols;
  const int64_t *label;
  float smoothing, lse2, scale;
  int32_t mean;
  const float *inv;   // 1 / N, or null: counted here, with `mean`
  float *loss;        // or null
};

// Maximum, sum of exp(x - maximum) and mean's share of some of a row's values.  `top` -infinity: nothing but -infinity so far
// (sum 0); +infinity and NaN make the sum NaN.
struct RowSum {
  float top, sum, mean;
};
// what is subtracted under a maximum
__device__ __forceinline__ float base_of(float top) { return top == -__builtin_huge_valf() ? 0.f : top; }
__device__ __forceinline__ float exp_less(float x, float base) { return __builtin_amdgcn_exp2f((x - base) * LOG2E); }
__device__ __forceinline__ RowSum joined(const RowSum &a, const RowSum &b) {
  const float top = fmaxf(a.top, b.top), base = base_of(top);
  return RowSum{top, a.sum * exp_less(a.top, base) + b.sum * exp_less(b.top, base), a.mean + b.mean};
}
// Of many values: 2^(x L - base L), a multiply-add less than exp_less, and what base L was rounded by as a factor of them all.  That is half a
// unit of base L's last place: below 2^24 the factor lies between 1/2 and 2 (at 2^30 it may be 2^64, from 1.5e9 on infinite or 0, and NaN with the values'
// opposite).  Beyond, or where base is infinite or NaN: exp_less.  (A thread's base is the maximum of its own values so far, which may all be masked.)
struct ExpLess {
  float base, scaled, factor;
  bool fast;
  __device__ __forceinline__ explicit ExpLess(float b) : base(b), scaled(b * LOG2E), factor(1.f), fast(fabsf(b) < 0x1p24f) {
    if (fast) factor = __builtin_amdgcn_exp2f(-fmaf(b, LOG2E, -scaled));
  }
  template <bool FAST>
  __device__ __forceinline__ float of(float x) const {
    if constexpr (FAST) return __builtin_amdgcn_exp2f(fmaf(x, LOG2E, -scaled));
    else return exp_less(x, base);
  }
};
// the largest of three (a NaN among them may be left out: its exponential says so)
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
template <int W>   // over W lanes side by side
__device__ __forceinline__ RowSum lanes_joined(RowSum s) {
#pragma unroll
  for (int d = W / 2; d; d >>= 1) s = joined(s, RowSum{__shfl_xor(s.top, d), __shfl_xor(s.sum, d), __shfl_xor(s.mean, d)});
  return s;
}

// ---- rows in pieces of 16 bytes ---------------------------------------------------------------
// A row is `head` columns up to a 16-byte border, `whole` aligned pieces of E columns and `tail` columns, whatever the pitch: a
// group's first thread takes the head and its second the tail, column by column.  Where dlogits' rows lie otherwise to that border their pieces are
// written unaligned.
template <bool BF, bool DBF>   // types of the logits and of dlogits
struct Row {
  static constexpr int E = BF ? 8 : 4;
  const uint8_t *x;    // the first whole piece
  uint8_t *d;          // dlogits' column there, or null
  int head, whole, cols;
  __device__ __forceinline__ Row(const LossArgs &a, int64_t r) {
    constexpr int B = 16 / E;
    const uint8_t *at = static_cast<const uint8_t *>(a.x.p) + r * a.x.ld * B;
    cols = (int)a.cols;
    head = min(cols, (int)(-(uintptr_t)at & 15) / B);
    whole = (cols - head) / E;
    x = at + head * B;
    d = a.d.p ? static_cast<uint8_t *>(a.d.p) + (r * a.d.ld + head) * (DBF ? 2 : 4) : nullptr;
  }
  __device__ __forceinline__ uint4 load(int j0, unsigned t) const {   // piece j0 + t (j0 uniform)
    return *reinterpret_cast<const uint4 *>(x + (int64_t)j0 * 16 + t * 16u);
  }
  __device__ __forceinline__ float at(int64_t c) const {   // column head + c
    if constexpr (BF) return bf16_value(reinterpret_cast<const uint16_t *>(x)[c]);
    else return reinterpret_cast<const float *>(x)[c];
  }
  static __device__ __forceinline__ void values(const uint4 &q, float (&v)[E]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF) {
        v[2 * i] = __builtin_bit_cast(float, w[i] << 16);
        v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
      } else {
        v[i] = __builtin_bit_cast(float, w[i]);
      }
    }
  }
  __device__ __forceinline__ void put(int64_t c, float v) const {   // column head + c
    if constexpr (DBF) reinterpret_cast<uint16_t *>(d)[c] = bf16_round(v);
    else reinterpret_cast<float *>(d)[c] = v;
  }
  __device__ __forceinline__ void store(int j0, unsigned t, const float (&v)[E]) const {
    uint8_t *to = d + (int64_t)j0 * (E * (DBF ? 2 : 4)) + t * (unsigned)(E * (DBF ? 2 : 4));
    if constexpr (DBF) {
      uint32_t w[E / 2];
#pragma unroll
      for (int i = 0; i < E / 2; ++i) w[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
      __builtin_memcpy(__builtin_assume_aligned(to, 2), w, sizeof(w));
    } else {
#pragma unroll
      for (int i = 0; i < E; i += 4) {
        const f32v4 w = {v[i], v[i + 1], v[i + 2], v[i + 3]};
        __builtin_memcpy(__builtin_assume_aligned(to + i * 4, 4), &w, 16);
      }
    }
  }
  // f(c) for the columns head + c outside the whole pieces that are thread t's
  template <class F>
  __device__ __forceinline__ void edges(int t, F &&f) const {
    const int c0 = t == 0 ? -head : whole * E, c1 = t == 0 ? 0 : cols - head;
    if (t > 1) return;
#pragma unroll 1
    for (int c = c0; c < c1; ++c) f(c);
  }
};

// H pieces join s
template <class ROW, int H>
__device__ __forceinline__ void add_pieces(RowSum &s, uint4 (&q)[H], int n, bool smooth, float inv_n) {   // n of them
  constexpr int E = ROW::E;
  float v[E], top = s.top;
#pragma unroll
  for (int h = 0; h < H; ++h)
    if (h < n) {
      ROW::values(q[h], v);
#pragma unroll
      for (int i = 0; i < E; i += 2) top = max3(top, v[i], v[i + 1]);
      // (unpacked anew where they are used next: the registers hold pieces)
      asm volatile("" : "+v"(q[h].x), "+v"(q[h].y), "+v"(q[h].z), "+v"(q[h].w));
      __builtin_amdgcn_sched_barrier(0);
    }
  const ExpLess exp(base_of(top));
  auto sums = [&](auto fast) {
    float sum = 0.f;
#pragma unroll
    for (int h = 0; h < H; ++h)
      if (h < n) {
        ROW::values(q[h], v);
#pragma unroll
        for (int i = 0; i < E; ++i) sum += exp.of<decltype(fast)::value>(v[i]);
        if (smooth) {   // uniform
#pragma unroll
          for (int i = 0; i < E; ++i) s.mean = fmaf(v[i], inv_n, s.mean);
        }
        asm volatile("" : "+v"(q[h].x), "+v"(q[h].y), "+v"(q[h].z), "+v"(q[h].w));
        __builtin_amdgcn_sched_barrier(0);
      }
    return sum;
  };
  const float sum = exp.fast ? sums(std::true_type{}) : sums(std::false_type{});
  s.sum = fmaf(sum, exp.factor, s.sum * exp_less(s.top, exp.base));
  s.top = top;
}
template <class ROW>
__device__ __forceinline__ void add_edges(RowSum &s, const ROW &row, int t, float inv_n) {
  row.edges(t, [&](int c) {
    const float v = row.at(c);
    s = joined(s, RowSum{v, 1.f, v * inv_n});
  });
}

// What a row's gradient takes: exp(x - base) times `factor`, less `each`, less `hit` at the label
struct RowGrad {
  ExpLess exp;
  float factor, each, hit;
};
__device__ __forceinline__ float row_loss(const LossArgs &a, const RowSum &s, float xt) {
  const float logs = logf(s.sum), e = s.top + logs;
  float l = s.top - (a.smoothing < 1.f ? (1.f - a.smoothing) * xt : 0.f);
  if (a.smoothing > 0.f) l -= a.smoothing * s.mean;
  l += logs;
  if (a.lse2 > 0.f) l += a.lse2 * e * e;
  return l;
}
__device__ __forceinline__ RowGrad row_grad(const LossArgs &a, const RowSum &s, float inv) {
  const float f = a.scale * inv, e = a.lse2 > 0.f ? s.top + logf(s.sum) : 0.f;
  const ExpLess exp(base_of(s.top));
  return RowGrad{exp, exp.factor * (f * (1.f + 2.f * a.lse2 * e) / s.sum), f * a.smoothing / (float)a.cols, f * (1.f - a.smoothing)};
}
template <class ROW, bool FAST>
__device__ __forceinline__ void grad_piece(const ROW &row, const RowGrad &g, int j0, unsigned t, int at, const uint4 &q) {   // head + at: the label's column
  constexpr int E = ROW::E;
  float v[E];
  ROW::values(q, v);
#pragma unroll
  for (int i = 0; i < E; ++i) v[i] = fmaf(g.exp.of<FAST>(v[i]), g.factor, -g.each);
  const int hit = at - (j0 + (int)t) * E;
  if ((unsigned)hit < (unsigned)E) {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = hit == i ? v[i] - g.hit : v[i];
  }
  row.store(j0, t, v);
}
template <class ROW>
__device__ __forceinline__ void grad_edges(const ROW &row, const RowGrad &g, int t, int at) {
  row.edges(t, [&](int c) {
    const float v = fmaf(exp_less(row.at(c), g.exp.base), g.factor / g.exp.factor, -g.each);
    row.put(c, c == at ? v - g.hit : v);
  });
}
template <class ROW>
__device__ __forceinline__ void fill_pieces(const ROW &row, float f, int t, int j0, int lane, int j1, int step) {   // pieces j0 + lane .. below j1
  float v[ROW::E];
#pragma unroll
  for (int i = 0; i < ROW::E; ++i) v[i] = f;
  for (; j0 + lane < j1; j0 += step) row.store(j0, lane, v);
  row.edges(t, [&](int c) { row.put(c, f); });
}

// 1 / N by the W threads of a group, thread `t`: labels counted by each, then over lanes (and LDS by the caller)
template <int W>
__device__ __forceinline__ int labels_counted(const LossArgs &a, int t) {
  int n = 0;
  for (int64_t i = t; i < a.rows; i += W) n += a.label[i] >= 0;
#pragma unroll
  for (int d = W < 64 ? W / 2 : 32; d; d >>= 1) n += __shfl_xor(n, d);
  return n;
}

// N: labels of 0 or more
__global__ __launch_bounds__(1024) void k_loss_count(const int64_t *label, int64_t rows, float *inv) {
  __shared__ int64_t part[16];
  int64_t n = 0;
  for (int64_t i = threadIdx.x; i < rows; i += 1024) n += label[i] >= 0;
#pragma unroll
  for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) n += part[i];
    *inv = 1.f / (float)(n > 0 ? n : 1);
  }
}

// The sum of a value of each of 1024 threads, in thread 0
__device__ __forceinline__ float block_sum(float s, float (&part)[16]) {
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int i = 1; i < 16; ++i) s += part[i];
  return s;
}
// total = sum of the rows' losses over N
__global__ __launch_bounds__(1024) void k_loss_total(const LossArgs a, float *total) {
  __shared__ float part[16];
  __shared__ int count[16];
  float s = 0.f;
  for (int64_t i = threadIdx.x; i < a.rows; i += 1024) s += a.loss[i];
  const bool self = a.mean && !a.inv;
  if (self) {
    const int n = labels_counted<1024>(a, threadIdx.x);
    if ((threadIdx.x & 63) == 0) count[threadIdx.x >> 6] = n;
  }
  s = block_sum(s, part);   // (a barrier)
  if (threadIdx.x == 0) {
    if (self) {
      int n = 0;
      for (int i = 0; i < 16; ++i) n += count[i];
      s *= 1.f / (float)max(n, 1);
    } else if (a.mean) {
      s *= *a.inv;
    }
    *total = s;
  }
}

// ---- rows held in registers -------------------------------------------------------------------
// A row is read once: its T threads (a wave, or a workgroup) hold up to H pieces each while the maximum and the sum are joined; what is beyond
// H T pieces is read again (MORE: the largest register file's worth, half of a bf16 row of 262144, which the last-level cache
// still has).  Bound by memory: bf16 2048 x 262144 in 490 to 500 us, 4.3 TB/s, where a large copy on that card ran at 4.9; 8192 x 32768 in 224, 4.8 TB/s;
// float32 8192 x 32768 in 390, 5.5 TB/s (twice read by workgroups of 256, 718 us for the first).  Two workgroups of 512 on a compute unit, of which
// one reads while the other writes, where a row fits one's registers: bf16 4096 x 65536 in 229 us, by one of 1024 305.  Left out: the next row's
// pieces loaded into the places of those just used, whose addresses spilled registers (590 us and more).
template <class ROW, int T, int H, bool MORE>
__device__ __forceinline__ void loss_row(const LossArgs &a, int64_t r, int t, float inv, RowSum *part, float *loss_out) {
  const int64_t label = a.label[r];
  const ROW row(a, r);
  if (label < 0 || label >= a.cols) {   // uniform in the group
    const float fill = label < 0 ? 0.f : __builtin_nanf("");
    if (t == 0) *loss_out = fill;
    if (row.d) fill_pieces(row, fill, t, 0, t, row.whole, T);
    return;
  }
  uint4 q[H];
#pragma unroll
  for (int h = 0; h < H; ++h)
    if (t + h * T < row.whole) q[h] = row.load(h * T, t);
  const int at = (int)label - row.head, held = row.whole <= t ? 0 : (row.whole - t + T - 1) / T;
  const float xt = t == 0 ? row.at(at) : 0.f;
  const bool smooth = a.smoothing > 0.f;
  const float inv_n = 1.f / (float)a.cols;
  RowSum s{-__builtin_huge_valf(), 0.f, 0.f};
  add_pieces<ROW, H>(s, q, held, smooth, inv_n);
  if constexpr (MORE) {
    for (int j = H * T; j + t < row.whole; j += 4 * T) {
      uint4 m[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (j + i * T + t < row.whole) m[i] = row.load(j + i * T, t);
      add_pieces<ROW, 4>(s, m, (row.whole - j - t + T - 1) / T, smooth, inv_n);
    }
  }
  add_edges(s, row, t, inv_n);
  s = lanes_joined<T < 64 ? T : 64>(s);
  if constexpr (T > 64) {
    if ((t & 63) == 0) part[t >> 6] = s;
    if (t == 0) part[T / 64].top = xt;   // (the label's logit is in a register before any of the row is written over)
    __syncthreads();
    s = lanes_joined<T / 64>(part[t & (T / 64 - 1)]);
    __syncthreads();   // before the next row's
  }
  if (t == 0) *loss_out = row_loss(a, s, xt);
  if (!row.d) return;
  const RowGrad g = row_grad(a, s, inv);
  auto grads = [&](auto fast) {
    constexpr bool FAST = decltype(fast)::value;
#pragma unroll
    for (int h = 0; h < H; ++h)
      if (h < held) grad_piece<ROW, FAST>(row, g, h * T, t, at, q[h]);
    if constexpr (MORE) {
      for (int j = H * T; j + t < row.whole; j += 4 * T) {
        uint4 m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (j + i * T + t < row.whole) m[i] = row.load(j + i * T, t);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (j + i * T + t < row.whole) grad_piece<ROW, FAST>(row, g, j + i * T, t, at, m[i]);
      }
    }
  };
  if (g.exp.fast) grads(std::true_type{});
  else grads(std::false_type{});
  grad_edges(row, g, t, at);
}
// T threads a row, several rows a workgroup of 256 where T is a wave
template <class ROW, int T, int H, bool MORE>
__global__ __launch_bounds__(T < 256 ? 256 : T) void k_loss_rows(const LossArgs a) {
  constexpr int B = T < 256 ? 256 : T, PER = B / T;
  __shared__ RowSum part[T > 64 ? T / 64 + 1 : 1];
  __shared__ int count[B / 64];
  __shared__ float sink;
  float inv = 1.f;
  if (a.mean && a.inv) {
    inv = *a.inv;
  } else if (a.mean) {
    const int n = labels_counted<B>(a, threadIdx.x);
    if ((threadIdx.x & 63) == 0) count[threadIdx.x >> 6] = n;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int i = 0; i < B / 64; ++i) all += count[i];
    inv = 1.f / (float)max(all, 1);
  }
  for (int64_t r = (int64_t)blockIdx.x * PER + (PER > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / T) : 0); r < a.rows; r += (int64_t)gridDim.x * PER)
    loss_row<ROW, T, H, MORE>(a, r, threadIdx.x % T, inv, part, a.loss ? a.loss + r : &sink);
}

// Few rows of few classes, their count and total among them, by one workgroup: T threads a row (less than a wave, or one).
template <class ROW, int T, int H>
__global__ __launch_bounds__(1024) void k_loss_small(const LossArgs a, float *total) {
  __shared__ float part[16];
  __shared__ int count[16];
  __shared__ float loss[SELF_COUNT];
  if (a.mean) {
    const int n = labels_counted<1024>(a, threadIdx.x);
    if ((threadIdx.x & 63) == 0) count[threadIdx.x >> 6] = n;
  }
  __syncthreads();
  float inv = 1.f;
  if (a.mean) {
    int all = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) all += count[i];
    inv = 1.f / (float)max(all, 1);
  }
  for (int r = threadIdx.x / T; r < (int)a.rows; r += 1024 / T) loss_row<ROW, T, H, false>(a, r, threadIdx.x % T, inv, nullptr, loss + r);
  __syncthreads();
  float s = 0.f;
  for (int r = threadIdx.x; r < (int)a.rows; r += 1024) {
    s += loss[r];
    if (a.loss) a.loss[r] = loss[r];
  }
  s = block_sum(s, part);
  if (threadIdx.x == 0 && total) *total = s * inv;
}

// ---- few long rows ----------------------------------------------------------------------------
// The row's pieces are divided among `parts` workgroups: one launch for the parts' maxima and sums (and the labels' logits), one that joins them, by
// each workgroup for itself, and writes the gradient; a workgroup of its own writes the losses and their sum.
template <class ROW>
__global__ __launch_bounds__(256) void k_loss_parts(const LossArgs a, int per, RowSum *sums, float *label_x) {
  __shared__ RowSum part[4];
  const int64_t r = blockIdx.y, label = a.label[r];
  if (label < 0 || label >= a.cols) return;
  const ROW row(a, r);
  const int j0 = blockIdx.x * per, j1 = min(j0 + per, row.whole);
  const bool smooth = a.smoothing > 0.f;
  const float inv_n = 1.f / (float)a.cols;
  RowSum s{-__builtin_huge_valf(), 0.f, 0.f};
  for (int j = j0; j + (int)threadIdx.x < j1; j += 1024) {
    uint4 m[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (j + i * 256 + (int)threadIdx.x < j1) m[i] = row.load(j + i * 256, threadIdx.x);
    add_pieces<ROW, 4>(s, m, (j1 - j - (int)threadIdx.x + 255) / 256, smooth, inv_n);
  }
  if (blockIdx.x == 0) {
    add_edges(s, row, threadIdx.x, inv_n);
    if (threadIdx.x == 0) label_x[r] = row.at(label - row.head);
  }
  s = lanes_joined<64>(s);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) sums[r * gridDim.x + blockIdx.x] = joined(joined(part[0], part[1]), joined(part[2], part[3]));
}
// A row's parts, by a wave
__device__ __forceinline__ RowSum parts_joined(const RowSum *sums, int64_t r, int parts, int lane) {
  RowSum s{-__builtin_huge_valf(), 0.f, 0.f};
  for (int i = lane; i < parts; i += 64) s = joined(s, sums[r * parts + i]);
  return lanes_joined<64>(s);
}
// (grid y: one for the losses, which takes longest, and then the rows, if there is a gradient)
template <class ROW>
__global__ __launch_bounds__(256) void k_loss_split(const LossArgs a, int per, int parts, const RowSum *sums, const float *label_x, float *total) {
  const int lane = threadIdx.x & 63;
  float inv = 1.f;
  if (a.mean) inv = 1.f / (float)max(labels_counted<64>(a, lane), 1);   // (64 rows at most)
  if (blockIdx.y == 0) {
    if (blockIdx.x > 0) return;
    __shared__ float loss[64];
    for (int r = threadIdx.x >> 6; r < (int)a.rows; r += 4) {
      const int64_t label = a.label[r];
      float l = label < 0 ? 0.f : __builtin_nanf("");
      if (label >= 0 && label < a.cols) l = row_loss(a, parts_joined(sums, r, parts, lane), label_x[r]);   // wave-uniform
      if (lane == 0) loss[r] = l;
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    float s = lane < (int)a.rows ? loss[lane] : 0.f;
    if (a.loss && lane < (int)a.rows) a.loss[lane] = s;
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if (total && lane == 0) *total = s * inv;
    return;
  }
  const int64_t r = blockIdx.y - 1, label = a.label[r];
  const ROW row(a, r);
  const int j0 = blockIdx.x * per, j1 = min(j0 + per, row.whole), t = blockIdx.x == 0 ? threadIdx.x : 2;   // t: who takes the edges
  if (label < 0 || label >= a.cols) {
    fill_pieces(row, label < 0 ? 0.f : __builtin_nanf(""), t, j0, threadIdx.x, j1, 256);
    return;
  }
  const RowGrad g = row_grad(a, parts_joined(sums, r, parts, lane), inv);
  const int at = (int)label - row.head;
  auto grads = [&](auto fast) {
#pragma unroll 4
    for (int j = j0; j + (int)threadIdx.x < j1; j += 256) grad_piece<ROW, decltype(fast)::value>(row, g, j, threadIdx.x, at, row.load(j, threadIdx.x));
  };
  if (g.exp.fast) grads(std::true_type{});
  else grads(std::false_type{});
  grad_edges(row, g, t, at);
}

// One workgroup for everything saves a launch where it has few rows a group (us a call, this way and by rows: 64 x 10 10.0 and 13;
// 256 x 60 11.0 and 13.5, 512 x 60 17 and 13; 32 x 1000 11.1 and 13.6, 48 x 1000 13.4 and 13.6).  Rows are divided where there are too few of them for the
// chip and each takes long (this way and by rows: 1 x 30000 bf16 16 and 14, 5 x 100001 13.4 and 19, 64 x 100000 19 and 20, float32 64 x
// 50000 18 and 14, bf16 64 x 262144 28 and 38, 128 x 262144 48 and 45).
struct LossPlan {
  bool small;
  int parts;   // of a row, 0: rows are not divided
};
static LossPlan loss_plan(bool bf16, int64_t rows, int64_t cols) {
  const int64_t pieces = blocks_of(cols, bf16 ? 8 : 4);
  LossPlan p{};
  p.small = rows > 0 && ((pieces <= 8 && rows <= 256) || (pieces <= 256 && rows <= 32));
  if (rows > 0 && ((pieces > 12288 && rows <= 32) || (pieces > 24576 && rows <= 64))) p.parts = (int)std::min<int64_t>(blocks_of(pieces, 512), 2048 / rows);
  return p;
}

template <class ROW>
static hipError_t launch_loss(LossArgs a, const LossPlan &p, float *total, float *inv, RowSum *sums, hipStream_t s) {
  const int pieces = (int)blocks_of(a.cols, ROW::E);
  if (p.small) {
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(1), dim3(1024), 0, s, a, total); };
    if (pieces <= 8) go(k_loss_small<ROW, 8, 1>);
    else if (pieces <= 64) go(k_loss_small<ROW, 64, 1>);
    else go(k_loss_small<ROW, 64, 4>);
    return hipGetLastError();
  }
  if (p.parts) {
    const int per = (int)blocks_of(pieces, p.parts);
    float *label_x = reinterpret_cast<float *>(sums + p.parts * a.rows);
    hipLaunchKernelGGL((k_loss_parts<ROW>), dim3((unsigned)p.parts, (unsigned)a.rows), dim3(256), 0, s, a, per, sums, label_x);
    const dim3 grid = a.d.p ? dim3((unsigned)p.parts, (unsigned)a.rows + 1) : dim3(1, 1);
    hipLaunchKernelGGL((k_loss_split<ROW>), grid, dim3(256), 0, s, a, per, p.parts, sums, label_x, total);
    return hipGetLastError();
  }
  if (a.mean && a.rows > SELF_COUNT) {
    hipLaunchKernelGGL(k_loss_count, dim3(1), dim3(1024), 0, s, a.label, a.rows, inv);
    a.inv = inv;
  }
  if (a.rows > 0) {
    auto go = [&](auto kernel, int threads, int per) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)std::min<int64_t>(blocks_of(a.rows, per), 1 << 20)), dim3(threads), 0, s, a);
    };
    if (pieces <= 64) go(k_loss_rows<ROW, 64, 1, false>, 256, 4);
    else if (pieces <= 256) go(k_loss_rows<ROW, 64, 4, false>, 256, 4);
    else if (pieces <= 1024) go(k_loss_rows<ROW, 256, 4, false>, 256, 1);
    else if (pieces <= 2048) go(k_loss_rows<ROW, 256, 8, false>, 256, 1);
    else if (pieces <= 4096) go(k_loss_rows<ROW, 512, 8, false>, 512, 1);
    else if (pieces <= 8192) go(k_loss_rows<ROW, 512, 16, false>, 512, 1);
    else go(k_loss_rows<ROW, 1024, 16, true>, 1024, 1);
  }
  if (total) hipLaunchKernelGGL(k_loss_total, dim3(1), dim3(1024), 0, s, a, total);
  return hipGetLastError();
}

}  // namespace vcr

using namespace vcr;
#define TRY(expr)                       \
  do {                                  \
    const vcr_status st_ = (expr);      \
    if (st_ != VCR_OK) return st_;      \
  } while (0)

extern "C" vcr_status vcr_cross_entropy(vcr_ctx *c, const vcr_mat *logits, const int64_t *label, const vcr_loss_opts *opts, float *loss,
                                        float *total, const vcr_mat *dlogits) {
  if (!c) return VCR_ERR_ARG;
  TRY(check_mat(c, logits, "logits"));
  if (!opts) return fail(c, VCR_ERR_ARG, "opts: null");
  if (!(opts->smoothing >= 0.f && opts->smoothing <= 1.f)) return fail(c, VCR_ERR_ARG, "smoothing %g is not in [0, 1]", (double)opts->smoothing);
  if (!(opts->lse2 >= 0.f && std::isfinite(opts->lse2))) return fail(c, VCR_ERR_ARG, "lse2 %g is not a finite number of 0 or more", (double)opts->lse2);
  if (!std::isfinite(opts->scale)) return fail(c, VCR_ERR_ARG, "scale is not finite");
  const int64_t rows = logits->rows;
  if (rows > 0 && !label) return fail(c, VCR_ERR_ARG, "label: null pointer");
  if ((reinterpret_cast<uintptr_t>(label) & 7) != 0) return fail(c, VCR_ERR_ARG, "label: pointer not aligned to its type");
  if (((reinterpret_cast<uintptr_t>(loss) | reinterpret_cast<uintptr_t>(total)) & 3) != 0)
    return fail(c, VCR_ERR_ARG, "loss, total: pointer not aligned to its type");
  if (dlogits) {
    TRY(check_mat(c, dlogits, "dlogits"));
    if (dlogits->rows != rows || dlogits->cols != logits->cols) return fail(c, VCR_ERR_SHAPE, "logits and dlogits differ in shape");
  }
  TRY(op_begin(c));
  if (!loss && !total && !dlogits) return VCR_OK;
  const bool bf16 = logits->type == VCR_BF16;
  const LossPlan p = loss_plan(bf16, rows, logits->cols);
  const bool own = total && !loss && !p.small && !p.parts && rows > 0;   // the rows' losses have no other place
  Workspace *ws = nullptr;
  TRY(op_space(c, 256 + al(own ? (size_t)rows * 4 : 0) + al(p.parts ? (size_t)p.parts * rows * sizeof(RowSum) + rows * 4 : 0) + 256, &ws));
  float *inv = take<float>(*ws, 1);
  if (own) loss = take<float>(*ws, rows);
  RowSum *sums = p.parts ? reinterpret_cast<RowSum *>(take<uint8_t>(*ws, (size_t)p.parts * rows * sizeof(RowSum) + rows * 4)) : nullptr;
  const LossArgs a{mat_ref(logits), mat_ref(dlogits), rows, logits->cols, label, opts->smoothing, opts->lse2, opts->scale, opts->mean != 0, nullptr, loss};
  auto go = [&](auto x, auto d) {
    return launch_loss<Row<decltype(x)::value, decltype(d)::value>>(a, p, total, inv, sums, c->stream);
  };
  const bool d_bf16 = dlogits ? dlogits->type == VCR_BF16 : bf16;
  const std::true_type yes{};
  const std::false_type no{};
  HIP_TRY(c, bf16 ? (d_bf16 ? go(yes, yes) : go(yes, no)) : (d_bf16 ? go(no, yes) : go(no, no)));
  return op_end(c);
}
