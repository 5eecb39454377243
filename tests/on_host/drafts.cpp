// drafts R NODES D H BT LAYERS SEED ODD
// One step's plan, acceptance and moves over random trees of at most NODES tokens (some requests bring runs of more than 64)
// against loops.  ODD: parents, paths, counts, lengths and block ids that no caller should bring.  Every buffer has the size
// that the caller owes.
#include "more_on_host.h"
#include "festina.h"
#include <random>
static void *take(size_t n) { void *p = nullptr; if (posix_memalign(&p, 256, n ? n : 1)) abort(); return p; }
static uint8_t moved(uint8_t c, float f) {
  const float x = emu_e4m3(c) * f;
  return (uint8_t)emu_enc(x);
}
static bool same(uint8_t a, uint8_t b) { return a == b || ((a & 0x7f) == 0x7f && (b & 0x7f) == 0x7f); }
int main(int argc, char **v) {
  const int R = atoi(v[1]), nodes = atoi(v[2]), D = atoi(v[3]), H = atoi(v[4]), bt = atoi(v[5]), L = atoi(v[6]), odd = atoi(v[8]);
  std::mt19937 g(atoi(v[7]));
  const auto below = [&](int n) { return (int)(g() % (unsigned)std::max(n, 1)); };
  std::vector<int> len(R), cnt(R);
  int nb = 0, MB = 1;
  for (int r = 0; r < R; ++r) {
    cnt[r] = below(9) == 0 ? 65 + below(40) : below(nodes + 1);
    len[r] = cnt[r] + below(3 * bt);
    if (odd && below(5) == 0 && cnt[r]) len[r] = below(cnt[r]);           // fewer than the new ones
    nb += (len[r] + bt - 1) / bt;
    MB = std::max(MB, (len[r] + bt - 1) / bt);
  }
  const int NB = nb + 2;
  std::vector<int> ids(NB);
  for (int i = 0; i < NB; ++i) ids[i] = i;
  std::shuffle(ids.begin(), ids.end(), g);
  int *table = (int *)take(4ull * R * MB), *length = (int *)take(4 * R), *first = (int *)take(4 * (R + 1));
  int at = 0, T = 0;
  for (int r = 0; r < R; ++r) {
    first[r] = T;
    length[r] = len[r];
    T += cnt[r];
    for (int c = 0; c < MB; ++c) table[(size_t)r * MB + c] = c < (len[r] + bt - 1) / bt ? ids[at++] : -1;
    if (odd && below(4) == 0) table[(size_t)r * MB + below(MB)] = below(2) ? -7 : NB + below(9);
    if (odd && below(7) == 0) length[r] = MB * bt + 1 + below(100);       // more than the table holds
  }
  first[R] = T;
  const int extra = 5, N = T + extra;                  // tokens that no request has
  int *parent = (int *)take(4 * N), *token = (int *)take(4 * N), *choice = (int *)take(4 * N);
  for (int t = 0; t < N; ++t) parent[t] = -1, token[t] = below(3), choice[t] = below(3);
  for (int r = 0; r < R; ++r) for (int i = 0; i < cnt[r]; ++i) {
    parent[first[r] + i] = i ? i - 1 - below(std::min(i, 1 + below(5))) : -1;
    if (odd && below(6) == 0) parent[first[r] + i] = below(3) ? i + below(70) : -5;
  }
  uint64_t *seen = (uint64_t *)take(8 * N);
  int *position = (int *)take(4 * N), *path = (int *)take(4 * N), *kept = (int *)take(4 * R), *next = (int *)take(4 * R), *left = (int *)take(4 * R);
  for (int t = 0; t < N; ++t) seen[t] = 77, position[t] = 77, path[t] = 77;
  festina_drafts d{R, N, first, length, parent};
  festina_accepted acc{path, kept, next, left};
  if (festina_plan_drafts(&d, seen, position, nullptr) || festina_accept_drafts(&d, token, choice, &acc, nullptr)) return 2;
  bool good = true;
  const auto want = [&](bool ok, const char *what, int r, int i) { if (!ok && good) printf("%s of request %d, %d is wrong\n", what, r, i); good &= ok; };
  for (int r = 0; r < R; ++r) {
    const int n = cnt[r], before = length[r] - n, f = first[r];
    std::vector<uint64_t> w(n, 0);
    std::vector<int> up(n, -1);
    for (int i = 0; i < n; ++i) {
      const bool run = n > 64;
      if (!run) {
        up[i] = parent[f + i] >= 0 && parent[f + i] < i ? parent[f + i] : -1;
        w[i] = (up[i] >= 0 ? w[up[i]] : 0) | 1ull << i;
      }
      want(seen[f + i] == w[i], "seen", r, i);
      want(position[f + i] == before + (run ? i : __builtin_popcountll(w[i]) - 1), "position", r, i);
    }
    std::vector<int> p;
    if (n > 64) for (int i = 0; i < n; ++i) p.push_back(i);
    else for (int node = n ? 0 : -1; node >= 0;) {
      p.push_back(node);
      int then = -1;
      for (int c = n - 1; c > 0; --c) if (up[c] == node && token[f + c] == choice[f + node]) then = c;
      node = then;
    }
    want(kept[r] == (int)p.size(), "kept", r, kept[r]);
    want(left[r] == before + (int)p.size(), "length", r, left[r]);
    want(next[r] == (n ? choice[f + p.back()] : -1), "next", r, next[r]);
    for (int i = 0; i < n; ++i) want(path[f + i] == (i < (int)p.size() ? p[i] : -1), "path", r, i);
  }
  for (int t = T; t < N; ++t) want(seen[t] == 77 && position[t] == 77 && path[t] == 77, "token of no request", -1, t);
  // moves: paths as accepted, or (more moves) drawn anew
  for (int r = 0; r < R; ++r) if (cnt[r] && cnt[r] <= 64 && below(2)) {
    int k = 0;
    for (int i = 0; i < cnt[r]; ++i) if (below(3) == 0) path[first[r] + k++] = i;
    kept[r] = k;
    for (int i = k; i < cnt[r]; ++i) path[first[r] + i] = -1;
    if (odd && below(3) == 0) kept[r] = below(2) ? cnt[r] + 3 : -2;
    if (odd && below(3) == 0) path[first[r] + below(cnt[r])] = below(2) ? cnt[r] : 0;
  }
  const size_t codes = (size_t)NB * H * bt * D;
  std::vector<festina_kv_cache> caches;
  std::vector<std::vector<uint8_t>> kc(L), vc(L);
  std::vector<std::vector<float>> ks(L), vs(L);
  for (int l = 0; l < L; ++l) {
    festina_kv_cache c{NB, bt, H, D, (uint8_t *)take(codes), (uint8_t *)take(codes), (float *)take(4ull * NB * H), (float *)take(4ull * NB * H)};
    for (size_t i = 0; i < codes; ++i) c.k[i] = (uint8_t)g(), c.v[i] = (uint8_t)g();
    for (int i = 0; i < NB * H; ++i) c.k_scale[i] = exp2f(-8 + below(5)), c.v_scale[i] = exp2f(-6 + below(6)) * (below(20) ? 1.f : 0.f);
    kc[l].assign(c.k, c.k + codes), vc[l].assign(c.v, c.v + codes), ks[l].assign(c.k_scale, c.k_scale + NB * H), vs[l].assign(c.v_scale, c.v_scale + NB * H);
    caches.push_back(c);
  }
  festina_kept q{R, MB, N, table, length, first, path, kept};
  if (festina_keep_tokens(caches.data(), L, &q, nullptr)) return 2;
  int moves = 0;
  for (int r = 0; r < R; ++r) {
    const int n = cnt[r], before = length[r] - n, k = std::min(kept[r], n);
    bool sound = n <= 64 && k > 0 && before >= 0 && length[r] <= MB * bt;
    for (int i = 0; sound && i < k; ++i) { const int p = path[first[r] + i]; sound = p >= 0 && p < n && (i == 0 || p > path[first[r] + i - 1]); }
    for (int c = before / bt; sound && c <= (length[r] - 1) / bt; ++c) sound = table[(size_t)r * MB + c] >= 0 && table[(size_t)r * MB + c] < NB;
    if (!sound) continue;
    const auto block = [&](int p) { return table[(size_t)r * MB + p / bt]; };
    for (int l = 0; l < L; ++l) for (int h = 0; h < H; ++h) for (int x = 0; x < 2; ++x) {
      auto &code = x ? vc[l] : kc[l];
      auto &scale = x ? vs[l] : ks[l];
      const auto was = code;
      const auto had = scale;
      const auto idx = [&](int b, int o, int dd) { return x ? (((size_t)b * H + h) * D + dd) * bt + o : (((size_t)b * H + h) * bt + o) * D + dd; };
      for (int c = before / bt; c <= (before + k - 1) / bt; ++c) {
        const int lo = std::max(before, c * bt), hi = std::min(before + k, (c + 1) * bt), b = block(lo);
        float now = 0;
        if (lo > c * bt) now = had[b * H + h];
        for (int p = lo; p < hi; ++p) now = std::max(now, had[block(before + path[first[r] + p - before]) * H + h]);
        scale[b * H + h] = now;
        for (int o = c * bt; o < hi; ++o) {
          const int from = o < lo ? o : before + path[first[r] + o - before];
          moves += from != o;
          const float f = now > 0 ? had[block(from) * H + h] / now : 1.f;
          if (from != o || f != 1.f) for (int dd = 0; dd < D; ++dd) code[idx(b, o % bt, dd)] = moved(was[idx(block(from), from % bt, dd)], f);
        }
      }
    }
  }
  for (int l = 0; l < L; ++l) {
    for (size_t i = 0; i < codes; ++i) want(same(caches[l].k[i], kc[l][i]), "key code", l, (int)i), want(same(caches[l].v[i], vc[l][i]), "value code", l, (int)i);
    for (int i = 0; i < NB * H; ++i) want(caches[l].k_scale[i] == ks[l][i], "key scale", l, i), want(caches[l].v_scale[i] == vs[l][i], "value scale", l, i);
  }
  printf("R %d T %d MB %d NB %d: %d moves, %s\n", R, T, MB, NB, moves, good ? "equal" : "WRONG");
  return !good;
}
