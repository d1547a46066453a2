// Drives a validation-only context through the entry points on float layers, dropout and the loss with seeded random descriptors: valid
// ones, null ones, and sizes at and beyond every limit.  Each call ends in a status; none reaches the device.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "vcrown.h"

int main(int argc, char **argv) {
  const int rounds = argc > 1 ? atoi(argv[1]) : 1000;
  vcr_ctx *c = nullptr;
  if (vcr_create(-1, &c) != VCR_OK) return 1;
  alignas(64) static unsigned char buf[4096];
  std::mt19937_64 rng(11);
  const int64_t sizes[] = {-9223372036854775807ll - 1, -1, 0, 1, 7, 8, 9, 64, 65, 1 << 20, 1 << 21, (1 << 21) + 1, 1 << 24, (1 << 24) + 1,
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
  const float odd[] = {-1.f, 2.f, INFINITY, -INFINITY, NAN, 1.f, 0x1.fffffep-1f, 0x1p-149f};
  auto number = [&] { return rng() % 4 ? (float)(rng() % 1000) / 1000.f : odd[rng() % 8]; };
  auto maybe = [&](auto *p) { return rng() % 8 ? p : nullptr; };
  long seen[8] = {};
  for (int i = 0; i < rounds; ++i) {
    const int64_t m = size(), k = size(), n = size();
    vcr_mat x = mat(m, k), w = mat(n, k), y = mat(m, n), r = mat(m, n), z = mat(m, n), dy = mat(m, n), dx = mat(m, k), add = mat(m, k), dw = mat(n, k),
            d = mat(m, k), e = mat(m, k);
    if (rng() % 4) x.type = w.type = dy.type = rng() % 2;
    float *f = reinterpret_cast<float *>(buf + (rng() % 8 ? 0 : rng() % 8));
    vcr_drop drop{number(), rng(), rng(), reinterpret_cast<uint64_t *>(rng() % 4 ? nullptr : buf + rng() % 16)};
    vcr_linear_opts o{maybe(f), (int32_t)(rng() % 8 ? rng() % 4 : rng()), maybe(&drop), maybe(&r), maybe(&z)};
    vcr_loss_opts lo{number(), number(), (int32_t)rng(), number()};
    vcr_ctx *ctx = rng() % 64 ? c : nullptr;
    const vcr_status got[] = {
        vcr_dropout(ctx, maybe(&x), maybe(&drop), maybe(&d), maybe(&e)),
        vcr_linear(ctx, maybe(&x), maybe(&w), maybe(&o), maybe(&y)),
        vcr_linear_grad(ctx, maybe(&dy), maybe(&x), maybe(&w), maybe(&o), maybe(&add), maybe(&dx), maybe(&dw), maybe(f)),
        vcr_cross_entropy(ctx, maybe(&x), reinterpret_cast<int64_t *>(rng() % 8 ? buf + (rng() % 8 ? 0 : rng() % 16) : nullptr), maybe(&lo), maybe(f),
                          maybe(f), maybe(&d)),
    };
    for (const vcr_status st : got) {
      if (st < 0 || st > VCR_ERR_UNSUPPORTED || st == VCR_ERR_DEVICE || st == VCR_OK) {
        printf("round %d: status %d: %s\n", i, (int)st, vcr_last_error(c));
        return 1;
      }
      ++seen[st];
    }
  }
  for (unsigned char b : buf)
    if (b) return 1;
  vcr_destroy(c);
  // every refusal has been met
  for (const int st : {VCR_ERR_ARG, VCR_ERR_SHAPE, VCR_ERR_STATE, VCR_ERR_UNSUPPORTED})
    if (!seen[st]) {
      printf("status %d never seen\n", st);
      return 1;
    }
  printf("all checks passed\n");
  return 0;
}
