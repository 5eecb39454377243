// attend_drafts D H G BT bf16|f16 WINDOW COLUMNS MAX_NEW EXTRA TREE LENGTH:NEW[xCOUNT] ...
// One attention call over drafted tokens against a sum in double: random trees (TREE 1), chains (2), or random words that are no
// trees (3), random codes in a shuffled pool; every buffer has the size that the caller owes.  Keys that a tree leaves out
// hold a NaN here and there.
#include "more_on_host.h"
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
  const int extra = arg(v, 9), kind = arg(v, 10);
  std::vector<int> len, cnt;
  for (int i = 11; i < argc; ++i) { int a, b, rep = 1; if (sscanf(v[i], "%d:%dx%d", &a, &b, &rep) < 2) abort(); while (rep--) len.push_back(a), cnt.push_back(b); }
  const int R = len.size();
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
  uint64_t *seen = (uint64_t *)take(8ull * T);
  for (int r = 0; r < R; ++r) for (int i = 0; i < cnt[r]; ++i) {
    uint64_t w = i < 64 ? 1ull << i : 0;
    if (i && i < 64) w |= seen[first[r] + (kind == 2 ? i - 1 : i - 1 - (int)(g() % (unsigned)std::min(i, 4)))];
    if (kind == 3) w = (uint64_t)g() << 32 | g();
    if (kind == 3 && g() % 5 == 0) w = 0;
    seen[first[r] + i] = w;
  }
  const size_t codes = (size_t)NB * H * bt * D;
  uint8_t *k = (uint8_t *)take(codes), *vv = (uint8_t *)take(codes);
  float *ks = (float *)take(4ull * NB * H), *vs = (float *)take(4ull * NB * H);
  for (size_t i = 0; i < codes; ++i) k[i] = emu_enc(std::clamp(N(g) * 112, -448.f, 448.f));
  for (size_t i = 0; i < codes; ++i) vv[i] = emu_enc(std::clamp(N(g) * 112, -448.f, 448.f));
  for (int i = 0; i < NB * H; ++i) ks[i] = exp2f(-8 + (int)(g() % 3)), vs[i] = exp2f(-10 + (int)(g() % 7));
  for (int r = 0; r < R; ++r) if (len[r] % bt) {
    const int b = table[(size_t)r * MB + len[r] / bt];
    for (int h = 0; h < H; ++h) for (int o = len[r] % bt; o < bt; ++o) for (int d = 0; d < D; ++d)
      k[(((size_t)b * H + h) * bt + o) * D + d] = 0xff, vv[(((size_t)b * H + h) * D + d) * bt + o] = 0x7f;
  }
  // NaN at the last node of every tree: rows that do not see it are as if it were not there
  for (int r = 0; r < R; ++r) if (cnt[r] > 1 && cnt[r] <= 64 && len[r] >= cnt[r]) {
    const int p = len[r] - 1, b = table[(size_t)r * MB + p / bt];
    for (int h = 0; h < H; ++h) k[(((size_t)b * H + h) * bt + p % bt) * D + 3] = 0x7f, vv[(((size_t)b * H + h) * D + 5) * bt + p % bt] = 0xff;
  }
  const int Hq = H * G;
  uint16_t *q = (uint16_t *)take(2ull * T * Hq * D), *out = (uint16_t *)take(2ull * T * Hq * D);
  float *lse = (float *)take(4ull * T * Hq);
  for (size_t i = 0; i < (size_t)T * Hq * D; ++i) { const float x = N(g); if (bf) { __bf16 y = (__bf16)x; memcpy(q + i, &y, 2); } else { _Float16 y = (_Float16)x; memcpy(q + i, &y, 2); } }
  memset(out, 0x55, 2ull * T * Hq * D);
  for (int i = 0; i < T * Hq; ++i) lse[i] = 12345.f;
  const auto val = [&](uint16_t u) { if (bf) return (double)__builtin_bit_cast(float, (unsigned)u << 16); _Float16 y; memcpy(&y, &u, 2); return (double)(float)y; };
  festina_kv_cache c{NB, bt, H, D, k, vv, ks, vs};
  festina_attention a{R, MB, T, Hq, max_new, bf ? FESTINA_BF16 : FESTINA_F16, window, 1.f / sqrtf(D), table, length, first, q, (int64_t)Hq * D, D, out, (int64_t)Hq * D, D, lse};
  const size_t n = festina_attend_drafts_workspace_bytes(&c, &a);
  void *ws = take(n);
  memset(ws, 0xff, n);
  const int st = festina_attend_drafts(&c, &a, seen, ws, n, nullptr);
  if (st) { printf("status %d\n", st); return 2; }
  double worst = 0, worst_l = 0;
  int nans = 0;
  for (int r = 0; r < R; ++r) for (int i = 0; i < cnt[r]; ++i) for (int y = 0; y < Hq; ++y) {
    const int before = len[r] - cnt[r], t = first[r] + i, h = y / G;
    const bool run = cnt[r] > 64;
    std::vector<int> nodes;
    for (int j = 0; j < cnt[r] && !run; ++j) if (seen[t] >> j & 1) nodes.push_back(j);
    const int p = run ? before + i : before + std::max((int)nodes.size() - 1, 0);
    std::vector<int> keys;
    for (int j = 0; j <= (run ? p : before - 1); ++j) if (!window || j > p - window) keys.push_back(j);
    for (size_t z = window && (int)nodes.size() > window ? nodes.size() - window : 0; z < nodes.size(); ++z) if (before + nodes[z] >= 0) keys.push_back(before + nodes[z]);
    std::vector<double> w, o(D, 0), ab(D, 0);
    double top = -INFINITY, sum = 0;
    bool bad = false;
    for (int j : keys) {
      const size_t bh = (size_t)table[(size_t)r * MB + j / bt] * H + h;
      double s = 0;
      for (int d = 0; d < D; ++d) s += (double)emu_e4m3(k[(bh * bt + j % bt) * D + d]) * val(q[((size_t)t * Hq + y) * D + d]);
      bad |= s != s;
      w.push_back(s * ks[bh] * a.scale);
      top = std::max(top, w.back());
    }
    const double got = lse[(size_t)t * Hq + y];
    if (bad) {                                         // a NaN key that the row sees: its results are NaN
      ++nans;
      bool all = got != got;
      for (int d = 0; d < D; ++d) all &= std::isnan(val(out[((size_t)t * Hq + y) * D + d]));
      if (!all) worst_l = INFINITY;
      continue;
    }
    for (double &x : w) sum += x = exp(x - top);
    for (size_t z = 0; z < keys.size(); ++z) {
      const int j = keys[z];
      const size_t bh = (size_t)table[(size_t)r * MB + j / bt] * H + h;
      for (int d = 0; d < D; ++d) { const double e = w[z] / sum * vs[bh] * emu_e4m3(vv[(bh * D + d) * bt + j % bt]); o[d] += e; ab[d] += fabs(e); }
    }
    for (int d = 0; d < D; ++d) { const double e = fabs(val(out[((size_t)t * Hq + y) * D + d]) - o[d]) / (ab[d] + 1e-30); if (!(e <= worst)) worst = e; }
    const double want = sum > 0 ? top + log(sum) : -INFINITY;
    const double e = want == got ? 0 : fabs(want - got);
    if (!(e <= worst_l)) worst_l = e;
  }
  bool kept = true;
  for (size_t i = (size_t)(T - extra) * Hq * D; i < (size_t)T * Hq * D; ++i) kept &= out[i] == 0x5555;
  printf("D %d H %d G %d bt %d %s R %d T %d MB %d: scratch %.1f MiB, out %.2g of sum|wv| lse %.2g, %d NaN rows, rows of none %s\n", D, H, G, bt, v[5], R, T, MB, n / 1048576., worst, worst_l, nans, kept ? "kept" : "WRITTEN");
  return !(worst < (bf ? 0.01 : 0.002) && worst_l < 1e-3 && kept);
}
