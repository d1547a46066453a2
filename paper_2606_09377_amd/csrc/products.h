// Products by the tiles of nt.h into a matrix, the contraction divided where that pays.  Part of layers.hip and dense.hip.
//
// OUT: where results go.  rows, cols, bytes() that an output takes, and put(m, n, values of n .. n + 3), or with STAGED
// col and store8 of eight columns (nt.h).
#pragma once

#include "planes.h"

namespace vcr {

template <class OUT, class = void>
struct EpiOut {
  OUT o;
  __device__ __forceinline__ void store(int, int, int m, int n, f32v4 v, int) const { o.put(m, n, v); }
};
template <class OUT>
struct EpiOut<OUT, std::enable_if_t<OUT::STAGED>> {
  static constexpr bool STAGED = true;
  typedef typename OUT::Col Col;
  OUT o;
  __device__ __forceinline__ Col col(int n) const { return o.col(n); }
  __device__ __forceinline__ void store8(int m, int n, float (&v)[8], const Col &c) const { o.store8(m, n, v, c); }
};
// sums over one part of the contraction, [parts][rows][ld]
struct EpiPart {
  float *p;
  int64_t rows, ld;
  __device__ __forceinline__ void store(int, int z, int m, int n, f32v4 v, int) const {
    if (m < rows && n < ld) *reinterpret_cast<f32v4 *>(p + (z * rows + m) * ld + n) = v;
  }
};
template <class OUT>
static __global__ __launch_bounds__(256) void k_join(const float *p, int parts, int64_t rows, int64_t ld, OUT o) {
  constexpr int W = nt_staged<OUT>::value ? 2 : 1;   // quads a thread
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, per = (ld / 4 + W - 1) / W, m = id / per, n = (id - m * per) * 4 * W;
  if (m >= rows) return;
  f32v4 v[W];
#pragma unroll
  for (int q = 0; q < W; ++q) {
    v[q] = f32v4{0.f, 0.f, 0.f, 0.f};
    if (q == 0 || n + 4 * q < ld)
#pragma unroll 4
      for (int z = 0; z < parts; ++z) v[q] += *reinterpret_cast<const f32v4 *>(p + (z * rows + m) * ld + n + 4 * q);
  }
  if constexpr (W == 1) {
    o.put(m, n, v[0]);
  } else {
    float x[8] = {v[0][0], v[0][1], v[0][2], v[0][3], v[1][0], v[1][1], v[1][2], v[1][3]};
    o.store8(m, n, x, o.col(n));
  }
}

// MOST: parts of the contraction
template <int PA, int PB, int KIND, int MOST = NT_CUS>
static size_t part_bytes(int64_t M, int64_t N, int64_t chunks) {
  const int parts = std::min(MOST, nt_parts<NtTiles<PA, PB, KIND>>(M, N, chunks));
  return parts > 1 ? (size_t)parts * M * blocks_of(N, 4) * 16 : 0;
}
// What nt_product is estimated to take, us
template <int PA, int PB, int KIND, int MOST = NT_CUS>
static float product_us(int64_t M, int64_t N, int64_t chunks, float out_bytes) {
  typedef NtTiles<PA, PB, KIND> TS;
  const int parts = std::min(MOST, nt_parts<TS>(M, N, chunks));
  if (parts == 1) return nt_plan<TS>(M, N, chunks, 1, false, out_bytes).us;
  const NtShape &x = TS::shapes[nt_shapes<TS> - 1];
  return nt_us(x, nt_tiles(M, N, x.bm, x.bn, false) * parts, blocks_of(chunks, parts), 4.f) + NT_LAUNCH_US;
}
// D = A B^T into o; part: room for part_bytes
template <int PA, int PB, int KIND, int MOST = NT_CUS, class OUT>
static hipError_t nt_product(const NtArgs &g, const OUT &o, float *part, hipStream_t s) {
  typedef NtTiles<PA, PB, KIND> TS;
  const int parts = std::min(MOST, nt_parts<TS>(o.rows, o.cols, g.chunks));
  if (parts == 1) return launch_nt_plan<TS>(g, o.rows, o.cols, 1, o.bytes(), EpiOut<OUT>{o}, s);
  const int64_t ld = blocks_of(o.cols, 4) * 4;
  const NtShape &x = TS::shapes[nt_shapes<TS> - 1];
  const hipError_t e = launch_nt<typename nt_last<TS>::T>(g, o.rows, o.cols, x.bm, x.bn, 0, nt_tiles(o.rows, o.cols, x.bm, x.bn, false), parts,
                                                  EpiPart{part, o.rows, ld}, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_join<OUT>), dim3((unsigned)blocks_of(o.rows * (ld / 4), 256)), dim3(256), 0, s, part, parts, o.rows, ld, o);
  return hipGetLastError();
}

}  // namespace vcr
