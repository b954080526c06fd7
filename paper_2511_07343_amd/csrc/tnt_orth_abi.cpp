// C ABI of the orthogonalised update: validation, workspace layout, launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/tnt.h"
#include "tnt_kernels.h"
#include "tnt_orth.h"

using namespace tnt;

namespace {

inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
constexpr float DEFAULT_COEF[3] = {3.4445f, -4.7750f, 2.0315f};
constexpr int MAX_SIDE = 1 << 15;

tnt_status validate(const tnt_orth_config* c) {
  if (!c) return TNT_ERR_NULL;
  if (c->dtype < 0 || c->dtype > 1) return TNT_ERR_ARG;
  if (c->n < 0 || c->rows <= 0 || c->cols <= 0 || c->steps < 1) return TNT_ERR_SHAPE;
  if (c->steps > ORTH_MAX_STEPS || c->rows > MAX_SIDE || c->cols > MAX_SIDE) return TNT_ERR_UNSUPPORTED;
  if (!(c->eps >= 0.f) || !std::isfinite(c->eps) || !std::isfinite(c->scale)) return TNT_ERR_ARG;
  if (c->g_row < 0 || c->g_batch < 0 || c->out_row < 0 || c->out_batch < 0) return TNT_ERR_ARG;
  // outputs that overlap: rows within a matrix, and matrices neither one after the other nor
  // with their rows side by side
  if (c->out_row && c->out_row < c->cols) return TNT_ERR_ARG;
  const int64_t orow = c->out_row ? c->out_row : c->cols;
  if (c->out_batch && c->n > 1 && c->out_batch < (int64_t)(c->rows - 1) * orow + c->cols &&
      (c->out_batch < c->cols || orow < (int64_t)(c->n - 1) * c->out_batch + c->cols))
    return TNT_ERR_ARG;
  return TNT_OK;
}

// The largest |a x + b x^3 + c x^5| and |b y + c y^2| that singular values up to s can
// reach (y = x^2): at the ends and at the stationary points.
void bounds(double a, double b, double c, double s, double* next, double* mid) {
  auto p = [&](double x) { return std::fabs(x * (a + x * x * (b + c * x * x))); };
  auto r = [&](double y) { return std::fabs(y * (b + c * y)); };
  double best = p(s), other = r(s * s);
  if (c != 0.) {
    const double disc = 9. * b * b - 20. * a * c;
    if (disc >= 0.)
      for (int i = -1; i <= 1; i += 2) {
        const double y = (-3. * b + i * std::sqrt(disc)) / (10. * c);
        if (y > 0. && y < s * s) best = std::max(best, p(std::sqrt(y)));
      }
    const double y = -b / (2. * c);
    if (y > 0. && y < s * s) other = std::max(other, r(y));
  } else if (b != 0.) {
    const double y = -a / (3. * b);
    if (y > 0. && y < s * s) best = std::max(best, p(std::sqrt(y)));
  }
  *next = best;
  *mid = other;
}

struct Lay {
  bool small;
  int m, k, mp, kp, lm, lk;
  size_t part, X, XT, XT2, A, B, bytes;
};

Lay lay_of(const tnt_orth_config* c) {
  Lay l{};
  l.m = std::min(c->rows, c->cols);
  l.k = std::max(c->rows, c->cols);
  // (whose elements are addressed by 32-bit offsets from the matrix)
  const int64_t apart = std::max(std::max(c->g_row, c->out_row), (int64_t)c->cols);
  l.small = orth_small(c->n, l.m, l.k) && apart < INT32_MAX / 1024;
  if (l.small) return l;
  l.mp = (l.m + ORTH_TILE - 1) / ORTH_TILE * ORTH_TILE;
  l.kp = (l.k + ORTH_TILE - 1) / ORTH_TILE * ORTH_TILE;
  l.lm = l.mp + 64;
  l.lk = l.kp + 64;
  const size_t x = up256((size_t)c->n * 2 * l.mp * l.lk * 2), xt = up256((size_t)c->n * 2 * l.kp * l.lm * 2),
               a = up256((size_t)c->n * 2 * l.mp * l.lm * 2);
  l.part = 0;
  l.X = up256((size_t)c->n * ORTH_PART * sizeof(double));
  l.XT = l.X + x;
  l.XT2 = l.XT + xt;
  l.A = l.XT2 + xt;
  l.B = l.A + a;
  l.bytes = l.B + a;
  return l;
}

bool misaligned(const void* p, size_t to) { return (uintptr_t)p % to != 0; }

}  // namespace

extern "C" {

size_t tnt_orth_workspace_size(const tnt_orth_config* cfg) {
  if (validate(cfg) != TNT_OK) return 0;
  const Lay l = lay_of(cfg);
  return l.bytes ? l.bytes : 16;
}

tnt_status tnt_orth_update(const tnt_orth_config* cfg, const float* coef, const void* G, void* out,
                           void* workspace, size_t ws_bytes, void* stream) {
  const tnt_status s = validate(cfg);
  if (s != TNT_OK) return s;
  OrthArgs a{};
  double sv = 1.;  // X's singular values are at most its Frobenius norm
  for (int i = 0; i < cfg->steps; ++i) {
    for (int j = 0; j < 3; ++j) {
      a.coef[3 * i + j] = coef ? coef[3 * i + j] : DEFAULT_COEF[j];
      if (!std::isfinite(a.coef[3 * i + j])) return TNT_ERR_ARG;
    }
    double mid;
    bounds(a.coef[3 * i], a.coef[3 * i + 1], a.coef[3 * i + 2], sv, &sv, &mid);
    if (!(sv <= 4.) || !(mid <= 64.) || std::fabs(a.coef[3 * i]) > 64.) return TNT_ERR_ARG;
  }
  if (cfg->n == 0) return TNT_OK;
  if (!G || !out) return TNT_ERR_NULL;
  const Lay l = lay_of(cfg);
  if (l.bytes && !workspace) return TNT_ERR_NULL;
  const size_t elem = cfg->dtype == TNT_BF16 ? 2 : 4;
  if (misaligned(G, elem) || misaligned(out, elem) || misaligned(workspace, 16)) return TNT_ERR_ALIGN;
  if (ws_bytes < l.bytes) return TNT_ERR_WORKSPACE;
  if (!l.small && (int64_t)cfg->n * (l.kp / 64) * (l.mp / 64) > INT32_MAX / 256) return TNT_ERR_UNSUPPORTED;
  if (cfg->n > 65535) return TNT_ERR_UNSUPPORTED;
  a.G = G; a.out = out;
  a.n = cfg->n; a.rows = cfg->rows; a.cols = cfg->cols;
  a.m = l.m; a.k = l.k; a.mp = l.mp; a.kp = l.kp; a.lm = l.lm; a.lk = l.lk;
  a.flip = cfg->rows > cfg->cols;
  a.bf16 = cfg->dtype == TNT_BF16;
  a.gr = cfg->g_row ? cfg->g_row : cfg->cols;
  a.gb = cfg->g_batch ? cfg->g_batch : (int64_t)cfg->rows * a.gr;
  a.orow = cfg->out_row ? cfg->out_row : cfg->cols;
  a.ob = cfg->out_batch ? cfg->out_batch : (int64_t)cfg->rows * a.orow;
  a.steps = cfg->steps; a.eps = cfg->eps; a.scale = cfg->scale;
  char* ws = (char*)workspace;
  a.part = (double*)(ws + l.part);
  // 16 times 256 elements a part: one round of a workgroup's loads
  a.parts = (int)std::min<int64_t>(ORTH_PART, ((int64_t)cfg->rows * ((cfg->cols + 255) / 256) + 15) / 16);
  a.X = (_Float16*)(ws + l.X);
  a.XT = (_Float16*)(ws + l.XT);
  a.XT2 = (_Float16*)(ws + l.XT2);
  a.A = (_Float16*)(ws + l.A);
  a.B = (_Float16*)(ws + l.B);
  hipStream_t st = (hipStream_t)stream;
  const int t = section_begin("orth_update", st);
  const hipError_t e = l.small ? launch_orth_small(a, st) : launch_orth_large(a, st);
  section_end(t, st);
  return e == hipSuccess ? TNT_OK : TNT_ERR_HIP;
}

}  // extern "C"
