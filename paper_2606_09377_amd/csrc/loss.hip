// Cross entropy with its gradient: vcr_cross_entropy of vcrown.h.
//
// With m = max x, S = sum exp(x - m), e = m + log S, a row's loss is (m - (1 - s) x_t - s mean x) + log S + c e^2 and its gradient
// a multiple of exp(x - m) less a constant, and less another at the label.  exp(x - m) is 2^((x - m) L), L = log2 e.  (2^(x L - m L)
// would take one instruction less, but m L overflows where all that a mask left is the type's lowest value.)
#include "training.h"

namespace vcr {

constexpr float LOG2E = 1.4426950408889634f;

struct LossArgs {
  MatRef x, d;
  int64_t rows, cols;
  const int64_t *label;
  float smoothing, lse2, scale;
  const float *inv;   // 1 / N, or null
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
__device__ __forceinline__ RowSum wave_joined(RowSum s) {
#pragma unroll
  for (int d = 32; d; d >>= 1) s = joined(s, RowSum{__shfl_xor(s.top, d), __shfl_xor(s.sum, d), __shfl_xor(s.mean, d)});
  return s;
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

// total = sum of the rows' losses over N
__global__ __launch_bounds__(1024) void k_loss_total(const float *loss, int64_t rows, const float *inv, float *total) {
  __shared__ float part[16];
  float s = 0.f;
  for (int64_t i = threadIdx.x; i < rows; i += 1024) s += loss[i];
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; ++i) s += part[i];
    *total = inv ? s * *inv : s;
  }
}

// What a row's gradient takes: exp(x - base) times `factor`, less `each`, less `hit` at the label
struct RowGrad {
  float base, factor, each, hit;
};
__device__ __forceinline__ RowGrad row_grad(const LossArgs &a, const RowSum &s, float xt, float *loss) {
  const float logs = logf(s.sum), e = s.top + logs;
  float l = s.top - (a.smoothing < 1.f ? (1.f - a.smoothing) * xt : 0.f);
  if (a.smoothing > 0.f) l -= a.smoothing * s.mean;
  l += logs;
  if (a.lse2 > 0.f) l += a.lse2 * e * e;
  *loss = l;
  const float f = a.inv ? a.scale * *a.inv : a.scale;
  return RowGrad{base_of(s.top), f * (1.f + 2.f * a.lse2 * e) / s.sum, f * a.smoothing / (float)a.cols, f * (1.f - a.smoothing)};
}
__device__ __forceinline__ void grad8(const RowGrad &g, int64_t c, int64_t t, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float y = fmaf(exp_less(v[i], g.base), g.factor, -g.each);
    v[i] = c + i == t ? y - g.hit : y;
  }
}

// A workgroup per row, which it reads twice
__global__ __launch_bounds__(256) void k_loss_rows(const LossArgs a) {
  __shared__ RowSum part[4];
  __shared__ float label_x;
  const float inv_n = 1.f / (float)a.cols;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const int64_t t = a.label[r];
    if (t < 0 || t >= a.cols) {
      const float fill = t < 0 ? 0.f : __builtin_nanf("");
      if (threadIdx.x == 0 && a.loss) a.loss[r] = fill;
      if (a.d.p) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fill;
        for (int64_t c = threadIdx.x * 8; c < a.cols; c += 2048) save8(a.d, r, c, a.cols, v);
      }
      continue;   // uniform
    }
    RowSum s{-__builtin_huge_valf(), 0.f, 0.f};
    for (int64_t c = threadIdx.x * 8; c < a.cols; c += 2048) {
      float v[8];
      load8(a.x, r, c, a.cols, v);
      RowSum q{-__builtin_huge_valf(), 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const bool in = c + i < a.cols;
        if (in) q.top = fmaxf(q.top, v[i]), q.mean = fmaf(v[i], inv_n, q.mean);
        if (c + i == t) label_x = v[i];
      }
      const float base = base_of(q.top);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < a.cols) q.sum += exp_less(v[i], base);
      s = joined(s, q);
    }
    s = wave_joined(s);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    s = joined(joined(part[0], part[1]), joined(part[2], part[3]));
    float loss;
    const RowGrad g = row_grad(a, s, label_x, &loss);
    __syncthreads();   // read by all before the next row's
    if (threadIdx.x == 0 && a.loss) a.loss[r] = loss;
    if (a.d.p)
      for (int64_t c = threadIdx.x * 8; c < a.cols; c += 2048) {
        float v[8];
        load8(a.x, r, c, a.cols, v);
        grad8(g, c, t, v);
        save8(a.d, r, c, a.cols, v);
      }
  }
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
  const bool sums = total && !loss && rows > 0;
  Workspace *ws = nullptr;
  TRY(op_space(c, 256 + (sums ? al((size_t)rows * 4) : 0), &ws));
  float *inv = opts->mean ? take<float>(*ws, 1) : nullptr;
  if (sums) loss = take<float>(*ws, rows);
  LossArgs a{mat_ref(logits), mat_ref(dlogits), rows, logits->cols, label, opts->smoothing, opts->lse2, opts->scale, inv, loss};
  if (inv) hipLaunchKernelGGL(k_loss_count, dim3(1), dim3(1024), 0, c->stream, label, rows, inv);
  if (rows > 0) hipLaunchKernelGGL(k_loss_rows, dim3((unsigned)std::min<int64_t>(rows, 1 << 20)), dim3(256), 0, c->stream, a);
  if (total) hipLaunchKernelGGL(k_loss_total, dim3(1), dim3(1024), 0, c->stream, loss, rows, inv, total);
  HIP_TRY(c, hipGetLastError());
  return op_end(c);
}
