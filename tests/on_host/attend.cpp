// attend D H G BT bf16|f16 WINDOW COLUMNS MAX_NEW EXTRA LARGE LENGTH:NEW[xCOUNT] ...
// One attention call over random codes in a shuffled pool against a sum in double.  COLUMNS and MAX_NEW 0: as few as the
// requests need; EXTRA tokens belong to no request; LARGE > 0: value scales over that many powers of two, blocks of large
// ones with one large element.  Every buffer has the size that the caller owes; ON_HOST_SHORT takes a block off the keys.
#include "hip_on_host.h"
#include "festina.h"
#include <random>
#include <string>
static void *take(size_t n) { void *p = nullptr; if (posix_memalign(&p, 256, n ? n : 1)) abort(); return p; }
static int arg(char **v, int i) { return atoi(v[i]); }
int main(int argc, char **v) {
  std::mt19937 g(7);
  std::normal_distribution<float> N(0, 1);
  const int D = arg(v, 1), H = arg(v, 2), G = arg(v, 3), bt = arg(v, 4);
  const bool bf = std::string(v[5]) == "bf16";
  const int window = arg(v, 6);
  int MB = arg(v, 7), max_new = arg(v, 8);
  const int extra = arg(v, 9), spread = arg(v, 10);
  std::vector<int> len, cnt;
  for (int i = 11; i < argc; ++i) { int a, b, rep = 1; if (sscanf(v[i], "%d:%dx%d", &a, &b, &rep) < 2) abort(); while (rep--) len.push_back(a), cnt.push_back(b); }
  const int R = len.size(), base = bf ? -24 : -12;
  int nb = 0, most = 1, nmax = 1;
  for (int i = 0; i < R; ++i) { nb += (len[i] + bt - 1) / bt; most = std::max(most, (len[i] + bt - 1) / bt); nmax = std::max(nmax, cnt[i]); }
  if (!MB) MB = most;
  if (!max_new) max_new = nmax;
  const int NB = nb + 2;
  std::vector<int> ids(NB);
  for (int i = 0; i < NB; ++i) ids[i] = i;
  std::shuffle(ids.begin(), ids.end(), g);
  int *table = (int *)take(4ull * R * MB), *length = (int *)take(4 * R), *first = (int *)take(4 * (R + 1));
  for (int i = 0; i < R * MB; ++i) table[i] = -1;
  int at = 0, T = 0;
  for (int r = 0; r < R; ++r) {
    length[r] = len[r];
    first[r] = T;
    T += cnt[r];
    for (int c = 0; c < (len[r] + bt - 1) / bt; ++c) table[(size_t)r * MB + c] = ids[at++];
  }
  first[R] = T;
  T += extra;
  const size_t codes = (size_t)NB * H * bt * D;
  uint8_t *k = (uint8_t *)take(codes - (getenv("ON_HOST_SHORT") ? (size_t)H * bt * D : 0)), *vv = (uint8_t *)take(codes);
  float *ks = (float *)take(4ull * NB * H), *vs = (float *)take(4ull * NB * H);
  const size_t filled = codes - (getenv("ON_HOST_SHORT") ? (size_t)H * bt * D : 0);
  for (size_t i = 0; i < filled; ++i) k[i] = emu_enc(std::clamp(N(g) * 112, -448.f, 448.f));
  for (size_t i = 0; i < codes; ++i) vv[i] = emu_enc(std::clamp(N(g) * 112, -448.f, 448.f));
  for (int i = 0; i < NB * H; ++i) ks[i] = exp2f(-8 + (int)(g() % 3)), vs[i] = exp2f((spread ? base : -10) + (int)(g() % (spread ? spread : 7)));
  for (int r = 0; r < R; ++r) if (len[r] % bt) {
    const int b = table[(size_t)r * MB + len[r] / bt];
    for (int h = 0; h < H; ++h) for (int o = len[r] % bt; o < bt; ++o) for (int d = 0; d < D; ++d)
      k[(((size_t)b * H + h) * bt + o) * D + d] = 0xff, vv[(((size_t)b * H + h) * D + d) * bt + o] = 0x7f;
  }
  // blocks of large value scales have one large element dim: the other dims' sums are the small blocks'
  if (spread) for (int b = 0; b < NB * H; ++b) if (vs[b] > exp2f(base + 6)) for (int d = 1; d < D; ++d) for (int o = 0; o < bt; ++o) if (vv[((size_t)b * D + d) * bt + o] != 0x7f) vv[((size_t)b * D + d) * bt + o] = 0;
  const int Hq = H * G;
  uint16_t *q = (uint16_t *)take(2ull * T * Hq * D), *out = (uint16_t *)take(2ull * T * Hq * D);
  float *lse = (float *)take(4ull * T * Hq);
  for (size_t i = 0; i < (size_t)T * Hq * D; ++i) { const float x = N(g); if (bf) { __bf16 y = (__bf16)x; memcpy(q + i, &y, 2); } else { _Float16 y = (_Float16)x; memcpy(q + i, &y, 2); } }
  memset(out, 0x55, 2ull * T * Hq * D);
  for (int i = 0; i < T * Hq; ++i) lse[i] = 12345.f;
  const auto val = [&](uint16_t u) { if (bf) { __bf16 y; memcpy(&y, &u, 2); return (double)(float)y; } _Float16 y; memcpy(&y, &u, 2); return (double)(float)y; };
  festina_kv_cache c{NB, bt, H, D, k, vv, ks, vs};
  festina_attention a{R, MB, T, Hq, max_new, bf ? FESTINA_BF16 : FESTINA_F16, window, 1.f / sqrtf(D), table, length, first, q, (int64_t)Hq * D, D, out, (int64_t)Hq * D, D, lse};
  const size_t n = festina_attend_workspace_bytes(&c, &a);
  void *ws = take(n);
  memset(ws, 0xff, n);
  const int st = festina_attend(&c, &a, ws, n, nullptr);
  if (st) { printf("status %d\n", st); return 2; }
  double worst = 0, worst_l = 0;
  for (int r = 0; r < R; ++r) for (int i = 0; i < cnt[r]; ++i) for (int y = 0; y < Hq; ++y) {
    const int p = len[r] - cnt[r] + i, t = first[r] + i, h = y / G, lo = window ? std::max(0, p - window + 1) : 0;
    std::vector<double> w, o(D, 0), ab(D, 0);
    double top = -INFINITY, sum = 0;
    for (int j = lo; j <= p; ++j) {
      const size_t bh = (size_t)table[(size_t)r * MB + j / bt] * H + h;
      double s = 0;
      for (int d = 0; d < D; ++d) s += (double)emu_e4m3(k[(bh * bt + j % bt) * D + d]) * val(q[((size_t)t * Hq + y) * D + d]);
      w.push_back(s * ks[bh] * a.scale);
      top = std::max(top, w.back());
    }
    for (double &x : w) sum += x = exp(x - top);
    for (int j = lo; j <= p; ++j) {
      const size_t bh = (size_t)table[(size_t)r * MB + j / bt] * H + h;
      for (int d = 0; d < D; ++d) { const double z = w[j - lo] / sum * vs[bh] * emu_e4m3(vv[(bh * D + d) * bt + j % bt]); o[d] += z; ab[d] += fabs(z); }
    }
    for (int d = 0; d < D; ++d) { const double e = fabs(val(out[((size_t)t * Hq + y) * D + d]) - o[d]) / (ab[d] + 1e-30); if (!(e <= worst)) worst = e; }
    const double want = sum > 0 ? top + log(sum) : -INFINITY, got = lse[(size_t)t * Hq + y];
    const double e = want == got ? 0 : fabs(want - got);
    if (!(e <= worst_l)) worst_l = e;
  }
  bool kept = true;
  for (size_t i = (size_t)(T - extra) * Hq * D; i < (size_t)T * Hq * D; ++i) kept &= out[i] == 0x5555;
  printf("D %d H %d G %d bt %d %s R %d T %d MB %d: scratch %.1f MiB, out %.2g of sum|wv| lse %.2g rows of none %s\n", D, H, G, bt, v[5], R, T, MB, n / 1048576., worst, worst_l, kept ? "kept" : "WRITTEN");
  free(table), free(length), free(first), free(k), free(vv), free(ks), free(vs), free(q), free(out), free(lse), free(ws);
  return !(worst < (bf ? 0.01 : 0.002) && worst_l < 1e-3 && kept);
}
