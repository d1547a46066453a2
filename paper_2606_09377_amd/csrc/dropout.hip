// Dropout on its own: vcr_dropout of vcrown.h (training.h has its random bits).
#include "training.h"

namespace vcr {

// Eight columns a thread, one Philox output for them, whose ten rounds hide behind the loads.  Bound by memory: bf16 4096 x 8192 onto a residual, 201 MB,
// 37.7 us (5.3 TB/s, a large copy 4.9).  Rows that are not 16-byte aligned go by single elements: 4096 x 8191 117 us, float32 777 x 1001 6.8.
__global__ __launch_bounds__(256) void k_dropout(MatRef x, MatRef res, MatRef y, int64_t cols, int64_t per, int64_t total, DropDev d) {
  const uint64_t offset = drop_offset(d);
  for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += (int64_t)gridDim.x * 256) {
    const int64_t r = id / per, c = (id - r * per) * 8;
    float v[8];
    load8(x, r, c, cols, v);
    if (d.k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= d.factor;
      drop8(d, offset, r, c, v);
    }
    if (res.p) {
      float a[8];
      load8(res, r, c, cols, a);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += a[i];
    }
    save8(y, r, c, cols, v);
  }
}

}  // namespace vcr

using namespace vcr;
#define TRY(expr)                       \
  do {                                  \
    const vcr_status st_ = (expr);      \
    if (st_ != VCR_OK) return st_;      \
  } while (0)

extern "C" vcr_status vcr_dropout(vcr_ctx *c, const vcr_mat *x, const vcr_drop *drop, const vcr_mat *residual, const vcr_mat *y) {
  if (!c) return VCR_ERR_ARG;
  TRY(check_mat(c, x, "x"));
  if (!drop) return fail(c, VCR_ERR_ARG, "drop: null");
  TRY(check_drop(c, drop));
  if (residual) TRY(check_mat(c, residual, "residual"));
  TRY(check_mat(c, y, "y"));
  if (y->rows != x->rows || y->cols != x->cols) return fail(c, VCR_ERR_SHAPE, "x and y differ in shape");
  if (residual && (residual->rows != x->rows || residual->cols != x->cols)) return fail(c, VCR_ERR_SHAPE, "x and residual differ in shape");
  TRY(op_begin(c));
  if (x->rows == 0) return VCR_OK;
  const int64_t per = blocks_of(x->cols, 8), total = x->rows * per;
  const int64_t wgs = std::min<int64_t>(blocks_of(total, 256), 1 << 20);
  hipLaunchKernelGGL(k_dropout, dim3((unsigned)wgs), dim3(256), 0, c->stream, mat_ref(x), mat_ref(residual), mat_ref(y), x->cols, per, total,
                     drop_dev(drop));
  HIP_TRY(c, hipGetLastError());
  return op_end(c);
}
