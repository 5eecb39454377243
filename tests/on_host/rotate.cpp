// rotate T HEADS KV_HEADS D ROTATED INTERLEAVED bf16|f16|f32 NORM PAD INPLACE
// Norm and rotation of random heads against sums in double.  PAD elements lie between tokens (odd ones take away the
// alignment); every buffer ends with its last element.
#include "more_on_host.h"
#include "festina.h"
#include <random>
#include <string>
static void *take(size_t n) { void *p = nullptr; if (posix_memalign(&p, 256, n ? n : 1)) abort(); return p; }
int main(int argc, char **v) {
  std::mt19937 g(11);
  std::normal_distribution<float> N(0, 1);
  const int T = atoi(v[1]), heads[2] = {atoi(v[2]), atoi(v[3])}, D = atoi(v[4]), rot = atoi(v[5]), inter = atoi(v[6]);
  const std::string type = v[7];
  const int norm = atoi(v[8]), pad = atoi(v[9]), inplace = atoi(v[10]), size = type == "f32" ? 4 : 2;
  const auto get = [&](const void *p, size_t i) {
    if (type == "f32") return (double)((const float *)p)[i];
    const uint16_t u = ((const uint16_t *)p)[i];
    if (type == "f16") { _Float16 y; memcpy(&y, &u, 2); return (double)(float)y; }
    return (double)__builtin_bit_cast(float, (unsigned)u << 16);
  };
  const auto put = [&](void *p, size_t i, float x) {
    if (type == "f32") { ((float *)p)[i] = x; return; }
    if (type == "f16") { _Float16 y = (_Float16)x; memcpy((uint16_t *)p + i, &y, 2); return; }
    __bf16 y = (__bf16)x;
    memcpy((uint16_t *)p + i, &y, 2);
  };
  void *x[2], *y[2];
  float *w[2];
  int64_t token[2];
  std::vector<double> in[2];
  for (int k = 0; k < 2; ++k) {
    token[k] = (int64_t)heads[k] * D + pad;
    const size_t n = T && heads[k] ? (T - 1) * token[k] + (size_t)heads[k] * D : 0;
    x[k] = take(n * size);
    y[k] = inplace ? x[k] : take(n * size);
    for (size_t i = 0; i < n; ++i) { put(x[k], i, N(g)); }
    for (size_t i = 0; i < n; ++i) in[k].push_back(get(x[k], i));
    w[k] = (float *)take(4 * D);
    for (int i = 0; i < D; ++i) w[k][i] = 1 + 0.2f * N(g);
  }
  uint64_t *turn = (uint64_t *)take(8 * (rot / 2));
  int *position = (int *)take(4 * T);
  for (int i = 0; i < rot / 2; ++i) turn[i] = (uint64_t)ldexp(pow(1e4, -2. * i / rot) / (2 * M_PI), 64);
  for (int t = 0; t < T; ++t) position[t] = t % 3 == 0 ? (int)g() : t;
  festina_rotary q{D, rot, inter, 1e-6f, turn, norm ? w[0] : nullptr, norm ? w[1] : nullptr};
  festina_heads a{T, heads[0], heads[1], type == "f32" ? FESTINA_F32 : type == "f16" ? FESTINA_F16 : FESTINA_BF16, position, x[0], x[1],
                  token[0], D, token[1], D, y[0], y[1], token[0], D, token[1], D};
  const int st = festina_rotate_heads(&q, &a, nullptr);
  if (st) { printf("status %d\n", st); return 2; }
  double worst = 0;
  for (int k = 0; k < 2; ++k) for (int t = 0; t < T; ++t) for (int h = 0; h < heads[k]; ++h) {
    const size_t at = t * token[k] + (size_t)h * D;
    std::vector<double> z(in[k].begin() + at, in[k].begin() + at + D);
    double s = 0;
    for (double e : z) s += e * e;
    if (norm) for (int i = 0; i < D; ++i) z[i] *= w[k][i] / sqrt(s / D + 1e-6);
    std::vector<double> o = z;
    for (int i = 0; i < rot / 2; ++i) {
      const int e = inter ? 2 * i : i, f = inter ? 2 * i + 1 : i + rot / 2;
      const double part = ldexp((double)(int64_t)((uint64_t)(int64_t)position[t] * turn[i]), -64) * 2 * M_PI, c = cos(part), n = sin(part);
      o[e] = z[e] * c - z[f] * n;
      o[f] = z[f] * c + z[e] * n;
    }
    for (int i = 0; i < D; ++i) {
      const double e = fabs(get(y[k], at + i) - o[i]) / (1 + fabs(o[i]));
      if (!(e <= worst)) worst = e;
    }
  }
  const double bound = type == "f32" ? 2e-6 : type == "f16" ? 0x1p-11 + 2e-6 : 0x1p-8 + 2e-6;
  printf("T %d heads %d %d D %d rotated %d %s: off by at most %.3g (%.3g)\n", T, heads[0], heads[1], D, rot, v[7], worst, bound);
  return !(worst <= bound);
}
