// Which tiles the products of nt.h take: reads lines "class rows columns chunks batch tri out_bytes parts" (parts: 1 where
// the contraction may be divided), prints for each the number of parts and per launch the shape, its stages over
// the contraction and the stages in LDS.  "shapes" prints every class and its number of shapes.
#include <cstdio>
#include <cstring>

#include "nt.h"

using namespace vcr;

template <class TS, class T>
static void launch(int shape, int64_t chunks) {
  printf(" %d:%d:%d", shape, (int)((chunks + T::KS - 1) / T::KS), T::NS);
}
template <class TS>
static void one(int shape, int64_t chunks) {
  switch (shape) {
    case 0: return launch<TS, typename TS::T0>(0, chunks);
    case 1: return launch<TS, typename TS::T1>(1, chunks);
    case 2: return launch<TS, typename TS::T2>(2, chunks);
    case 3: return launch<TS, typename TS::T3>(3, chunks);
    default: return launch<TS, typename TS::T4>(4, chunks);
  }
}
template <class TS>
static void plan(int64_t M, int64_t N, int64_t chunks, int64_t batch, int tri, float out_bytes, int divide) {
  const int parts = divide ? nt_parts<TS>(M, N, chunks) : 1;
  printf("%d", parts);
  if (parts > 1) {
    one<TS>(nt_shapes<TS> - 1, (chunks + parts - 1) / parts);
  } else {
    const NtPlan p = nt_plan<TS>(M, N, chunks, batch, tri != 0, out_bytes);
    one<TS>(p.main, chunks);
    if (p.rest >= 0) one<TS>(p.rest, chunks);
  }
  printf("\n");
}
#define CLASSES(F)                    \
  F("4x4", NtTiles<1, 1, NT_FP4>)     \
  F("1x1", NtTiles<1, 1, NT_BF16>)    \
  F("3x1", NtTiles<3, 1, NT_BF16>)    \
  F("3x3", NtTiles<3, 3, NT_BF16>)    \
  F("1x4", NtTiles<1, 1, NT_MIXED>)   \
  F("3x4", NtTiles<3, 1, NT_MIXED>)

int main(int argc, char **) {
  if (argc > 1) {
#define SHAPES(name, ...) printf("%s %d\n", name, nt_shapes<__VA_ARGS__>);
    CLASSES(SHAPES)
    return 0;
  }
  char cls[8];
  long long M, N, chunks, batch;
  int tri, divide;
  float out_bytes;
  while (scanf("%7s %lld %lld %lld %lld %d %f %d", cls, &M, &N, &chunks, &batch, &tri, &out_bytes, &divide) == 8) {
#define PLAN(name, ...) \
  if (!strcmp(cls, name)) plan<__VA_ARGS__>(M, N, chunks, batch, tri, out_bytes, divide);
    CLASSES(PLAN)
  }
  return 0;
}
