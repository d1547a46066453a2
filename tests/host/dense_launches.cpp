// What vcr_linear, vcr_linear_grad, vcr_dropout and vcr_cross_entropy launch for given sizes, without a GPU: the entry points' own host code is
// compiled here with launches recorded instead of made; matrices and workspaces are addresses alone.  (Compiled for the host only, with -fuse-cuid=none.)
//
// Every recorded launch is checked: its grid is one that the device takes, its tiles cover the results, its parts the contraction, and what its
// arguments say is written lies inside the call's workspace, no two buffers over each other.
//
//   dense_launches            reads calls, one a line, and prints each one's launches
//     linear rows k n bf16 pitch act drop residual z other     grad rows k n bf16 pitch act drop need (1 dx, 2 dw, 4 db) other     loss rows n bf16 pitch other
//     other: results (y, dw, dlogits) of the other type
//   dense_launches random N   makes N calls of legal sizes, the smallest and the largest among them
#include <cxxabi.h>
#include <dlfcn.h>

#include <cinttypes>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <string>
#include <type_traits>
#include <vector>

#include <hip/hip_runtime.h>

namespace launches {
template <class K, class... A>
void record(K kernel, dim3 grid, dim3 block, const A &...args);
}
// the runtime's calls of these sources
#define hipSetDevice(d) hipSuccess
#define hipDeviceSynchronize() hipSuccess
#define hipStreamSynchronize(s) hipSuccess
#define hipStreamIsCapturing(s, p) (*(p) = hipStreamCaptureStatusNone, hipSuccess)
#define hipFree(p) hipSuccess
#undef hipLaunchKernelGGL
#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) launches::record(&*(kernel), grid, block, __VA_ARGS__)
#define hipGetLastError() hipSuccess

#define dev layers_dev   // (a name of both)
#include "layers.hip"
#undef dev
#include "dense.hip"
#include "dropout.hip"
#include "loss.hip"

char *const WORKSPACE = reinterpret_cast<char *>(0x200000000000ull);
hipError_t device_alloc(vcr_ctx *, void **p, size_t) {
  *p = WORKSPACE;
  return hipSuccess;
}
// No device code stands beside this program, and none is registered.
extern "C" {
char __hip_fatbin[1];
void **__hipRegisterFatBinary(const void *) {
  static void *none;
  return &none;
}
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
void __hipUnregisterFatBinary(void **) {}
}

namespace launches {
static vcr_ctx *ctx;
static std::string call, text;
struct Span {
  uint64_t at, bytes;
};
static std::vector<Span> spans;   // of the call's workspace
static int64_t tiles_left;        // of a product whose results are not covered yet

[[noreturn]] static void wrong(const char *what) {
  printf("%s: %s\n%s\n", call.c_str(), what, text.c_str());
  exit(1);
}
static void span(const void *p, uint64_t bytes) {
  const uint64_t at = (uint64_t)p, base = (uint64_t)WORKSPACE;
  if (!p || bytes == 0 || at < base) return;   // a matrix of the caller's
  if (ctx->op_spaces.empty()) wrong("no workspace");
  const Workspace &w = ctx->op_spaces[0].w;
  if (at < base || at - base > w.cap || bytes > w.cap - (at - base)) wrong("beyond the workspace");
  for (const Span &s : spans) {
    if (s.at == at) {
      continue;   // the same buffer
    }
    if (at < s.at + s.bytes && s.at < at + bytes) wrong("buffers over each other");
  }
  spans.push_back({at, bytes});
}
static std::string name_of(const void *f) {
  Dl_info d{};
  if (!dladdr(f, &d) || !d.dli_sname) return "(static)";
  int st = 0;
  char *s = abi::__cxa_demangle(d.dli_sname, nullptr, nullptr, &st);
  std::string r = s ? s : d.dli_sname;
  free(s);
  for (const char *cut : {"void ", "vcr::", "__device_stub__"})
    for (size_t at; (at = r.find(cut)) != std::string::npos;) r.erase(at, strlen(cut));
  size_t depth = 0, end = 0;   // up to the parameters
  for (; end < r.size() && (depth || r[end] != '('); ++end) depth += r[end] == '<' ? 1 : r[end] == '>' ? -1 : 0;
  r.resize(end);
  std::string t;
  for (char ch : r)
    if (ch != ' ') t += ch;
  return t;
}
// what arguments say
static void operand(const NtOperand &o, int chunks, int parts) {
  if (o.pitch == 0) span(o.p, (uint64_t)o.row_blocks * chunks * parts * FRAG);
}
static std::string notes;
static void note(const vcr::NtArgs &g, dim3 grid, int parts) {
  if (g.chunks <= 0) return;   // a product that does not go along
  operand(g.A, g.chunks, parts);
  operand(g.B, g.chunks, parts);
  if ((int64_t)g.z_chunks * grid.y < g.chunks) wrong("parts do not cover the contraction");
  notes += (int64_t)g.z_chunks * (grid.y - 1) >= g.chunks ? " empty" : "";   // (a part without a share: its sums are zeros)
  notes += " chunks=" + std::to_string(g.chunks) + " z=" + std::to_string(g.z_chunks) + " cols=" + std::to_string(g.cols) + " first=" + std::to_string(g.first);
}
static void epilogue(const vcr::EpiPart &e, dim3 grid) { span(e.p, (uint64_t)grid.y * e.rows * e.ld * 4); }
static void epilogue(const vcr::EpiOut<DenseOut> &, dim3) {}
static void planes(const vcr::PlanesOf &o, int parts) {
  if (o.tiles == 0) return;
  span(o.p.rows, (uint64_t)o.p.row_blocks * o.p.row_chunks * parts * FRAG);
  span(o.p.cols, (uint64_t)o.p.col_blocks * o.p.col_chunks * parts * FRAG);
  span(o.p.sums, (uint64_t)blocks_of(o.p.x.rows, 64) * o.p.x.cols * 4);
}
static int64_t next_first;
// by kernel
template <class EPI>
static auto seen(const std::string &n, dim3 grid, const vcr::NtArgs &g, const EPI &e) -> decltype(epilogue(e, grid)) {   // k_nt
  if (g.first == 0) next_first = 0;
  if (g.first != next_first) wrong("tiles left out");
  const int64_t per = (int64_t)g.sub_m * g.sub_n;
  if (grid.x % per) wrong("a tile in part");
  next_first = g.first + grid.x / per;
  tiles_left = g.tiles - next_first;
  if (tiles_left < 0) wrong("more tiles than there are");
  note(g, grid, n.find("Tile<0,") == std::string::npos ? 0 : n.find(",3,3,") != std::string::npos ? 3 : 1);
  epilogue(e, grid);
}
static void seen(const std::string &, dim3 grid, const float *p, int parts, int64_t rows, int64_t ld, const DenseOut &o) {   // k_join
  span(p, (uint64_t)parts * rows * ld * 4);
  const int64_t per = (ld / 4 + 1) / 2;
  if ((int64_t)grid.x * 256 < rows * per) wrong("results not joined");
  if (ld < o.cols) wrong("rows of parts too short");
}
static void seen(const std::string &, dim3 grid, const vcr::DevMat &x, const vcr::DevMat &w, const DenseOut &, float *part, int z_groups) {   // k_dense_rows
  span(part, (uint64_t)grid.y * x.rows * blocks_of(w.rows, 16) * 64);
  if (z_groups <= 0) wrong("no groups");
  if (!part && grid.y != 1) wrong("parts without a place");
  notes += part ? " parts" : "";
}
static void seen(const std::string &, dim3 grid, const vcr::NtArgs &ga, const vcr::EpiOut<DenseOut> &, int na, const vcr::NtArgs &gb, const vcr::EpiOut<DenseOut> &, int nb,
                 const vcr::ColumnSums &s) {   // k_dense_pair
  note(ga, dim3(1), 1);
  note(gb, dim3(1), 1);
  if (ga.first || gb.first || ga.tiles != na || gb.tiles != nb) wrong("tiles left out");
  if ((int64_t)grid.x != na + nb + (s.out ? blocks_of(s.cols, 64) : 0)) wrong("workgroups of two products and the sums");
  span(s.out ? s.sums : nullptr, (uint64_t)s.groups * s.cols * 4);
  notes += s.out ? " sums" : "";
}
static void seen(const std::string &n, dim3 grid, const uint8_t *gp, int nch, const vcr::DevMat &w, const DenseOut &o, int na, const vcr::NtArgs &g,
                 const vcr::EpiOut<DenseOut> &, int nb, const vcr::ColumnSums &s) {   // k_dense_few
  const int mt = atoi(n.c_str() + n.find('<') + 1);
  if (mt * 16 < o.rows || (int64_t)na * 32 < w.cols) wrong("results left out");
  span(gp, (uint64_t)mt * nch * 3 * FRAG);
  if (nb) note(g, dim3(1), 3);
  if (nb && (g.first || g.tiles != nb)) wrong("tiles left out");
  if ((int64_t)grid.x != na + nb + (s.out ? blocks_of(s.cols, 64) : 0)) wrong("workgroups of two products and the sums");
  span(s.out ? s.sums : nullptr, (uint64_t)s.groups * s.cols * 4);
  notes += s.out ? " sums" : "";
  notes += nb ? " along" : "";
}
static int64_t stretch;
static void stretches(dim3 grid, int64_t first, int64_t all) {
  if (first == 0) stretch = 0;
  if (first != stretch) wrong("a stretch left out");
  stretch += grid.x;
  if (stretch > all) wrong("more than there is");
  tiles_left = all - stretch;
}
static void seen(const std::string &n, dim3 grid, const vcr::PlanesOf &a, const vcr::PlanesOf &b, const vcr::PlanesOf &c, const vcr::GradSource &, int64_t first) {   // k_dense_planes
  const int parts = n.find("<1,") != std::string::npos ? 1 : 3;
  planes(a, parts);
  planes(b, parts);
  planes(c, parts);
  stretches(grid, first, a.tiles + b.tiles + c.tiles);
}
static void seen(const std::string &, dim3 grid, const vcr::DevMat &dy, int, const vcr::GradSource &, uint16_t *out, int64_t pitch, float *sums, float, int64_t first) {   // k_grad_rows
  const int64_t mg = blocks_of(dy.rows, 64);
  span(out, (uint64_t)dy.rows * pitch * 2);
  if (sums && mg > 1) span(sums, (uint64_t)mg * dy.cols * 4);
  if (out && pitch < blocks_of(dy.cols, 8) * 8) wrong("rows of g too short");
  stretches(grid, first, mg * blocks_of(dy.cols, 64));
  notes += out ? " stored" : "";
  notes += sums ? " sums" : "";
}
static void seen(const std::string &, dim3 grid, const vcr::ColumnSums &s) {   // k_dense_sums
  if ((int64_t)grid.x * 64 < s.cols) wrong("columns left out");
  if (s.groups) span(s.sums, (uint64_t)s.groups * s.cols * 4);
}
static void seen(const std::string &, dim3 grid, const vcr::MatRef &, const vcr::MatRef &, const vcr::MatRef &, int64_t, int64_t, int64_t, const vcr::DropDev &) {   // k_dropout
  if (grid.x == 0) wrong("no workgroups");
}
static void losses(const vcr::LossArgs &a) {
  if ((uint64_t)a.loss >= (uint64_t)WORKSPACE) span(a.loss, (uint64_t)a.rows * 4);
  if (a.inv) span(a.inv, 4);
}
static void seen(const std::string &, dim3, const vcr::LossArgs &a) { losses(a); }                   // k_loss_rows
static void seen(const std::string &, dim3, const vcr::LossArgs &a, float *) { losses(a); }          // k_loss_small, k_loss_total
static void seen(const std::string &, dim3, const int64_t *, int64_t, float *inv) { span(inv, 4); }  // k_loss_count
static void divided(const vcr::LossArgs &a, int per, int parts, const vcr::RowSum *sums, const float *label_x) {
  losses(a);
  span(sums, (uint64_t)parts * a.rows * sizeof(vcr::RowSum));
  span(label_x, (uint64_t)a.rows * 4);
  if (a.rows > 64) wrong("more rows than a wave has lanes");
  if ((int64_t)per * parts < blocks_of(a.cols, 8)) wrong("pieces left out");
}
static void seen(const std::string &, dim3 grid, const vcr::LossArgs &a, int per, vcr::RowSum *sums, float *label_x) {   // k_loss_parts
  divided(a, per, grid.x, sums, label_x);
}
static void seen(const std::string &, dim3, const vcr::LossArgs &a, int per, int parts, const vcr::RowSum *sums, const float *label_x, float *) {   // k_loss_split
  divided(a, per, parts, sums, label_x);
}

template <class... A>
static auto known(int, const std::string &n, dim3 grid, const A &...args) -> decltype(seen(n, grid, args...)) {
  seen(n, grid, args...);
}
template <class... A>
static void known(long, const std::string &, dim3, const A &...) {   // (those of the other calls of layers.hip)
  wrong("a kernel of arguments that are not known here");
}
template <class K, class... A>
void record(K kernel, dim3 grid, dim3 block, const A &...args) {
  const std::string n = name_of(reinterpret_cast<const void *>(kernel));
  text += "  " + n + " " + std::to_string(grid.x) + "x" + std::to_string(grid.y);
  if (grid.x == 0 || grid.y == 0 || grid.z != 1) wrong("an empty grid");
  if ((uint64_t)grid.x * block.x > 0xffffffffull || grid.x > 0x7fffffffu || grid.y > 65535u || block.x > 1024u || block.y != 1 || block.z != 1) wrong("too large a launch");
  notes.clear();
  known(0, n, grid, args...);
  text += notes;
}

struct Call {
  std::string kind;
  int64_t m = 1, k = 1, n = 1, pitch = 0;
  int bf16 = 0, act = 0, drop = 0, residual = 0, z = 0, need = 7, other = 0;
};
static vcr_mat mat(int where, int64_t rows, int64_t cols, const Call &c, int bf16 = -1) {
  vcr_mat m{};
  m.p = reinterpret_cast<void *>(0x100000000000ull + ((uint64_t)where << 40));   // (16 of them, below the workspace)
  m.type = bf16 < 0 ? c.bf16 : bf16;
  m.rows = rows;
  m.cols = cols;
  m.ld = cols + c.pitch;
  return m;
}
static vcr_status make(const Call &c) {
  spans.clear();
  text.clear();
  tiles_left = 0;
  next_first = 0;
  call = c.kind + " " + std::to_string(c.m) + " " + std::to_string(c.k) + " " + std::to_string(c.n) + " bf16 " + std::to_string(c.bf16) + " pitch " + std::to_string(c.pitch) +
         " act " + std::to_string(c.act) + " drop " + std::to_string(c.drop) + " residual " + std::to_string(c.residual) + " z " + std::to_string(c.z) + " need " +
         std::to_string(c.need) + " other " + std::to_string(c.other);
  const vcr_drop drop{.25f, 1, 2, nullptr};
  float *vec = reinterpret_cast<float *>(0x10000);
  vcr_status st;
  if (c.kind == "linear") {
    const vcr_mat x = mat(0, c.m, c.k, c), w = mat(1, c.n, c.k, c), y = mat(2, c.m, c.n, c, c.bf16 ^ c.other), z = mat(4, c.m, c.n, c);
    const vcr_linear_opts o{vec, c.act, c.drop ? &drop : nullptr, c.residual ? &y : nullptr, c.z ? &z : nullptr};
    st = vcr_linear(ctx, &x, &w, &o, &y);
  } else if (c.kind == "grad") {
    const vcr_mat dy = mat(0, c.m, c.n, c), x = mat(1, c.m, c.k, c), w = mat(2, c.n, c.k, c), z = mat(3, c.m, c.n, c), dx = mat(4, c.m, c.k, c), dw = mat(5, c.n, c.k, c, c.bf16 ^ c.other);
    const vcr_linear_opts o{nullptr, c.act, c.drop ? &drop : nullptr, nullptr, &z};
    st = vcr_linear_grad(ctx, &dy, c.need & 2 ? &x : nullptr, c.need & 1 ? &w : nullptr, &o, nullptr, c.need & 1 ? &dx : nullptr, c.need & 2 ? &dw : nullptr,
                         c.need & 4 ? vec : nullptr);
  } else if (c.kind == "dropout") {
    const vcr_mat x = mat(0, c.m, c.n, c), r = mat(1, c.m, c.n, c), y = mat(2, c.m, c.n, c);
    st = vcr_dropout(ctx, &x, &drop, c.residual ? &r : nullptr, &y);
  } else {   // need: 1 dlogits, 2 losses, 4 total
    const vcr_mat x = mat(0, c.m, c.n, c), d = mat(1, c.m, c.n, c, c.bf16 ^ c.other);
    const vcr_loss_opts o{.1f, 0.f, 1, 1.f};
    st = vcr_cross_entropy(ctx, &x, reinterpret_cast<int64_t *>(vec), &o, c.need & 2 ? vec : nullptr, c.need & 4 ? vec : nullptr, c.need & 1 ? &d : nullptr);
  }
  if (st == VCR_OK && tiles_left) wrong("tiles left out at the end");
  for (const auto &o : ctx->op_spaces)
    if (o.w.used > o.w.cap) wrong("more taken than asked for");
  return st;
}
}  // namespace launches

using namespace launches;

int main(int argc, char **argv) {
  vcr_ctx c;
  c.device = 0;
  ctx = &c;
  if (argc > 2) {
    std::mt19937_64 rng(17);
    const int rounds = atoi(argv[2]);
    auto size = [&](int64_t most) {   // between 1 and `most`, over the logarithm; often one of the ends or a border's neighbour
      const int64_t at[] = {1, 2, 7, 8, 9, 16, 17, 64, 65, most - 1, most};
      if (rng() % 5 == 0) return std::min(most, at[rng() % 11]);
      return std::max<int64_t>(1, (int64_t)std::exp2(std::log2((double)most) * (double)(rng() >> 11) * 0x1p-53));
    };
    long ok = 0, refused = 0;
    for (int i = 0; i < rounds; ++i) {
      Call q;
      q.kind = (const char *[]){"linear", "grad", "loss", "dropout"}[rng() % 4];
      q.bf16 = rng() % 2;
      q.pitch = (int64_t[]){0, 0, 0, 8, 8, 3, 31, 1 << 22}[rng() % 8];
      q.act = rng() % 4, q.drop = rng() % 2, q.residual = rng() % 2, q.z = rng() % 2, q.need = rng() % 8, q.other = rng() % 2;
      if (q.kind == "linear") q.m = size(VCR_MAX_LINEAR_ROWS), q.k = size(VCR_MAX_CONTRACTION), q.n = size(VCR_MAX_LINEAR_ROWS);
      else if (q.kind == "grad") q.m = size(VCR_MAX_CONTRACTION), q.k = size(VCR_MAX_LINEAR_ROWS), q.n = size(VCR_MAX_CONTRACTION);
      else q.m = size(VCR_MAX_NODE_ELEMENTS), q.n = size(VCR_MAX_NODE_ELEMENTS);
      if (rng() % 64 == 0) q.m = 0;
      // what fits the card's memory
      const double t = q.bf16 ? 2 : 4, u = q.bf16 ^ q.other ? 2 : 4, m = (double)q.m, n = (double)q.n, k = (double)q.k;
      if ((q.kind == "grad" ? t * (m * n + m * k) + u * n * k : q.kind == "linear" ? t * (m * k + n * k + q.z * m * n) + u * m * n : t * m * n) > 280e9) continue;
      const vcr_status st = make(q);
      if (st != VCR_OK && st != VCR_ERR_UNSUPPORTED) {
        printf("%s: status %d: %s\n%s\n", call.c_str(), (int)st, c.err.c_str(), text.c_str());
        return 1;
      }
      (st == VCR_OK ? ok : refused)++;
    }
    printf("%ld calls, %ld refused: all checks passed\n", ok, refused);
    return ok > rounds / 8 ? 0 : 1;
  }
  char kind[16];
  while (scanf("%15s", kind) == 1) {
    Call q;
    q.kind = kind;
    bool good;
    if (q.kind == "linear") good = scanf("%" SCNd64 " %" SCNd64 " %" SCNd64 " %d %" SCNd64 " %d %d %d %d %d", &q.m, &q.k, &q.n, &q.bf16, &q.pitch, &q.act, &q.drop, &q.residual, &q.z, &q.other) == 10;
    else if (q.kind == "grad") good = scanf("%" SCNd64 " %" SCNd64 " %" SCNd64 " %d %" SCNd64 " %d %d %d %d", &q.m, &q.k, &q.n, &q.bf16, &q.pitch, &q.act, &q.drop, &q.need, &q.other) == 9;
    else good = scanf("%" SCNd64 " %" SCNd64 " %d %" SCNd64 " %d", &q.m, &q.n, &q.bf16, &q.pitch, &q.other) == 5;
    if (!good) return 2;
    const vcr_status st = make(q);
    printf("%d%s\n", (int)st, text.c_str());
  }
  return 0;
}
