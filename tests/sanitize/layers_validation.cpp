// Drives a validation-only context through the entry points on layers' weights with seeded random descriptors: valid ones,
// null ones, and sizes at and beyond every limit.  Each call ends in a status; none reaches the device.
#include <cstdio>
#include <cstdlib>
#include <random>

#include "vcrown.h"

int main(int argc, char **argv) {
  const int rounds = argc > 1 ? atoi(argv[1]) : 1000;
  vcr_ctx *c = nullptr;
  if (vcr_create(-1, &c) != VCR_OK) return 1;
  alignas(64) static unsigned char buf[4096];
  std::mt19937_64 rng(7);
  const int64_t sizes[] = {-9223372036854775807ll - 1, -1, 0, 1, 2, 15, 16, 17, 40, 127, 128, 129, 1 << 20, 1 << 21, (1 << 21) + 1,
                           1ll << 30, (1ll << 30) + 1, 1ll << 32, 1ll << 40, 9223372036854775807ll};
  auto size = [&] { return rng() % 3 ? (int64_t)(rng() % 64) : sizes[rng() % (sizeof(sizes) / sizeof(*sizes))]; };
  auto mat = [&](int64_t r, int64_t k) {
    vcr_mat m{};
    m.p = rng() % 16 ? buf + (rng() % 8 ? 0 : rng() % 8) : nullptr;
    m.type = rng() % 16 ? (int32_t)(rng() % 2) : (int32_t)rng();
    m.rows = rng() % 8 ? r : size();
    m.cols = rng() % 8 ? k : size();
    m.ld = rng() % 4 ? m.cols : size();
    return m;
  };
  auto mx = [&](int64_t r, int64_t k) {
    vcr_mx m{};
    m.codes = rng() % 16 ? buf : nullptr;
    m.scales = rng() % 16 ? buf + (rng() % 8 ? 64 : rng() % 16) : nullptr;
    m.rows = rng() % 8 ? r : size();
    m.cols = rng() % 8 ? k : size();
    return m;
  };
  auto maybe = [&](auto *p) { return rng() % 8 ? p : nullptr; };
  long seen[8] = {};
  for (int i = 0; i < rounds; ++i) {
    const int64_t m = size(), k = size(), n = size();
    vcr_mat x = mat(m, k), y = mat(m, n), dy = mat(m, n), dx = mat(m, k), dw = mat(n, k), b = mat(m, k), o = mat(m, k);
    vcr_mx w = mx(n, k), q = mx(m, k);
    x.type = y.type = dy.type = rng() % 2;
    float *bias = reinterpret_cast<float *>(buf + (rng() % 8 ? 0 : rng() % 8));
    vcr_ns_opts op{(int32_t)(rng() % 16 ? 5 : rng()), 3.4f, -4.7f, 2.f, rng() % 16 ? 1e-7f : -1.f, 1.f, 1.f};
    uint64_t s0, s1;
    vcr_ctx *ctx = rng() % 64 ? c : nullptr;
    const vcr_status got[] = {
        vcr_mx_bytes(m, k, rng() % 16 ? &s0 : nullptr, &s1),
        vcr_mx_quantize(ctx, maybe(&x), maybe(&q)),
        vcr_mx_dequantize(ctx, maybe(&q), maybe(&o)),
        vcr_mx_product(ctx, maybe(&q), maybe(&w), bias, (int32_t)rng(), maybe(&y)),
        vcr_mx_linear(ctx, maybe(&x), maybe(&w), bias, (int32_t)rng(), maybe(&y)),
        vcr_mx_linear_grad(ctx, maybe(&dy), maybe(&y), maybe(&x), maybe(&w), maybe(&dx), maybe(&dw), bias),
        vcr_orthogonalize(ctx, maybe(&x), (int32_t)(rng() % 4 ? 1 : rng()), size(), maybe(&op), maybe(&b), size(), maybe(&o), size()),
    };
    for (const vcr_status st : got) {
      if (st < 0 || st > VCR_ERR_UNSUPPORTED || st == VCR_ERR_DEVICE) {
        printf("round %d: status %d: %s\n", i, (int)st, vcr_last_error(c));
        return 1;
      }
      ++seen[st];
    }
  }
  vcr_destroy(c);
  printf("statuses:");
  for (long v : seen) printf(" %ld", v);
  printf("\nall checks passed\n");
  return seen[VCR_ERR_ARG] && seen[VCR_ERR_SHAPE] && seen[VCR_ERR_STATE] ? 0 : 1;
}
