// cache T H D BT TYPE(0 bf16, 1 f16, 2 f32) LONGEST_RUN
// One store of ragged runs into a cache of random codes against the definition.  Every buffer has the size that the caller owes.
#include "hip_on_host.h"
#include "festina.h"
#include <random>
static void *take(size_t n) { void *p = nullptr; if (posix_memalign(&p, 256, n ? n : 1)) abort(); return p; }
int main(int argc, char **v) {
  std::mt19937 g(5);
  std::normal_distribution<float> N(0, 1);
  const int T = atoi(v[1]), H = atoi(v[2]), D = atoi(v[3]), bt = atoi(v[4]), ty = atoi(v[5]), most = atoi(v[6]);
  int *slot = (int *)take(4ull * T);
  int nb = 0, t = 0;
  std::vector<std::array<int, 3>> runs;
  while (t < T) {
    int off = g() % bt, n = std::min(T - t, (int)(1 + g() % most));
    while (n) { int m = std::min(n, bt - off); runs.push_back({t, nb * bt + off, m}); for (int i = 0; i < m; ++i) slot[t++] = nb * bt + off + i; n -= m; off = 0; ++nb; }
  }
  const int NB = nb + 1, sz = ty == 2 ? 4 : 2;
  // shuffled blocks
  std::vector<int> perm(NB); for (int i = 0; i < NB; ++i) perm[i] = i; std::shuffle(perm.begin(), perm.end(), g);
  for (int i = 0; i < T; ++i) slot[i] = perm[slot[i] / bt] * bt + slot[i] % bt;
  for (auto &r : runs) r[1] = perm[r[1] / bt] * bt + r[1] % bt;
  const size_t C = (size_t)NB * H * bt * D;
  uint8_t *k = (uint8_t *)take(C), *w = (uint8_t *)take(C);
  float *ks = (float *)take(4ull * NB * H), *vs = (float *)take(4ull * NB * H);
  for (size_t i = 0; i < C; ++i) k[i] = g() % 256, w[i] = g() % 256;
  for (int i = 0; i < NB * H; ++i) ks[i] = exp2f(-9 + (int)(g() % 5)), vs[i] = exp2f(-9 + (int)(g() % 5));
  const size_t n = (size_t)T * H * D;
  char *xk = (char *)take(n * sz), *xv = (char *)take(n * sz);
  std::vector<float> fk(n), fv(n);
  for (size_t i = 0; i < n; ++i) for (int a = 0; a < 2; ++a) {
    float x = N(g); if (g() % 5000 == 0) x = g() % 2 ? INFINITY : NAN;
    char *p = (a ? xv : xk) + i * sz;
    if (ty == 0) { __bf16 y = (__bf16)x; memcpy(p, &y, 2); x = (float)y; } else if (ty == 1) { _Float16 y = (_Float16)x; memcpy(p, &y, 2); x = (float)y; } else memcpy(p, &x, 4);
    (a ? fv : fk)[i] = x;
  }
  std::vector<uint8_t> K(k, k + C), V(w, w + C); std::vector<float> KS(ks, ks + NB * H), VS(vs, vs + NB * H);
  for (auto &r : runs) for (int h = 0; h < H; ++h) for (int a = 0; a < 2; ++a) {
    const int b = r[1] / bt, o = r[1] % bt;
    auto &X = a ? fv : fk; auto &Q = a ? V : K; float &s = (a ? VS : KS)[b * H + h];
    auto at = [&](int p, int d) -> uint8_t & { const size_t bh = (size_t)b * H + h; return a ? Q[(bh * D + d) * bt + p] : Q[(bh * bt + p) * D + d]; };
    float m = 0;
    for (int i = 0; i < r[2]; ++i) for (int d = 0; d < D; ++d) { const float x = X[((size_t)(r[0] + i) * H + h) * D + d]; if (std::isfinite(x)) m = std::max(m, fabsf(x)); }
    float now = 0x1p-32f; while (now < 0x1p32f && m > 448 * now) now *= 2;
    if (o) { now = std::max(now, s); if (now > s) for (int p = 0; p < o; ++p) for (int d = 0; d < D; ++d) at(p, d) = emu_enc(emu_e4m3(at(p, d)) * (s / now)); }
    for (int i = 0; i < r[2]; ++i) for (int d = 0; d < D; ++d) { const float x = X[((size_t)(r[0] + i) * H + h) * D + d]; at(o + i, d) = std::isfinite(x) ? emu_enc(std::clamp(x / now, -448.f, 448.f)) : 0x7f; }
    s = now;
  }
  festina_kv_cache c{NB, bt, H, D, k, w, ks, vs};
  festina_kv_tokens tk{T, ty, xk, xv, (int64_t)H * D, D, (int64_t)H * D, D, slot};
  if (int st = festina_store_kv(&c, &tk, nullptr)) { printf("status %d\n", st); return 2; }
  long long bad = 0;
  auto ne = [](uint8_t a, uint8_t b) { return a != b && !((a & 127) == 127 && (b & 127) == 127); };
  for (size_t i = 0; i < C; ++i) bad += ne(k[i], K[i]) + ne(w[i], V[i]);
  for (int i = 0; i < NB * H; ++i) bad += ks[i] != KS[i], bad += vs[i] != VS[i];
  printf("T %d H %d D %d bt %d type %d runs %zu span %d: bad %lld\n", T, H, D, bt, ty, runs.size(), std::min(std::max(T * H / 4096, 1), 64), bad);
  return bad != 0;
}
