// blocks R BT LONGEST DECODING% BUDGET(0 all, 1 blocks, 2 tokens) IN_PLACE BUSY
// One extend and one release against the requests one after the other; every BUSY-th request adds tokens, three are
// invalid.  Every buffer has the size that the caller owes.
#include "hip_on_host.h"
#include "festina.h"
#include <random>
static void *take(size_t n) { void *p = nullptr; if (posix_memalign(&p, 256, n ? n : 1)) abort(); return p; }
int main(int argc, char **v) {
  std::mt19937 g(5);
  const int R = atoi(v[1]), bt = atoi(v[2]), longest = atoi(v[3]), dec = atoi(v[4]), budget = atoi(v[5]), alias = atoi(v[6]), every = atoi(v[7]);
  std::vector<int> held(R), add(R);
  int MB = 1; long long have = 0, need = 0, tokens = 0;
  for (int r = 0; r < R; ++r) {
    held[r] = (int)(g() % 100) < dec ? g() % (longest + 1) : 0;
    add[r] = held[r] ? g() % 3 : g() % (longest + 1);
    if (every > 1 && r % every) add[r] = 0;
    if (r == 5) held[r] = -3;
    if (r == 9) add[r] = -1;
    if (r == 11) held[r] = add[r] = 2147483647;
    if (r == 5 || r == 9 || r == 11) continue;
    MB = std::max(MB, (held[r] + add[r] + bt - 1) / bt);
    have += (held[r] + bt - 1) / bt;
    need += (held[r] + add[r] + bt - 1) / bt - (held[r] + bt - 1) / bt;
    tokens += add[r];
  }
  const int NB = (int)(have + need + 3);
  int *table = (int *)take(4ull * R * MB), *free_ids = (int *)take(4ull * NB), *nf = (int *)take(4), *H = (int *)take(4 * R), *A = (int *)take(4 * R);
  std::vector<int> ids(NB);
  for (int i = 0; i < NB; ++i) ids[i] = i;
  std::shuffle(ids.begin(), ids.end(), g);
  long long at = 0;
  for (int r = 0; r < R; ++r) for (int c = 0; c < MB; ++c) table[(size_t)r * MB + c] = held[r] > 0 && held[r] < 1 << 30 && c < (held[r] + bt - 1) / bt ? ids[at++] : -1;
  int n_free = NB - (int)at;
  for (int i = 0; i < NB; ++i) free_ids[i] = i < n_free ? ids[at + i] : -5;
  if (budget == 1) n_free = n_free * 2 / 3;
  int mt = (int)(budget == 2 ? tokens * 2 / 3 : tokens + 13);
  *nf = n_free;
  for (int r = 0; r < R; ++r) H[r] = held[r], A[r] = add[r];
  // sequential
  std::vector<int> T(table, table + (size_t)R * MB), S(mt, -1), F(R + 1), L(held), SV(R);
  long long b = 0, t = 0; int used = 0, filled = 0;
  for (int r = 0; r < R; ++r) {
    F[r] = filled;
    if (held[r] < 0 || add[r] < 0 || (long long)held[r] + add[r] > (long long)MB * bt) continue;
    const int h = (held[r] + bt - 1) / bt, n = (held[r] + add[r] + bt - 1) / bt;
    b += n - h, t += add[r];
    if (b > n_free || t > mt) continue;
    for (int c = h; c < n; ++c) T[(size_t)r * MB + c] = free_ids[n_free - 1 - used++];
    for (int p = held[r]; p < held[r] + add[r]; ++p) { const int k = T[(size_t)r * MB + p / bt]; if (k >= 0 && k < NB) S[filled] = k * bt + p % bt; ++filled; }
    L[r] = held[r] + add[r], SV[r] = 1;
  }
  F[R] = filled;
  int *first = (int *)take(4 * (R + 1)), *slot = (int *)take(4ull * mt), *len = alias ? H : (int *)take(4 * R), *nfo = alias ? nf : (int *)take(4);
  uint8_t *served = (uint8_t *)take(R), *done = (uint8_t *)take(R);
  const size_t n = festina_blocks_workspace_bytes(R, mt);
  void *ws = take(n);
  memset(ws, 0xff, n);
  festina_kv_requests q{R, MB, bt, NB, H, A, table, free_ids, nf};
  festina_kv_step o{mt, first, slot, len, served, nfo};
  if (int st = festina_extend_blocks(&q, &o, ws, n, nullptr)) { printf("status %d\n", st); return 2; }
  int bad = 0;
  bad |= memcmp(table, T.data(), 4ull * R * MB) ? 1 : 0;
  bad |= memcmp(slot, S.data(), 4ull * mt) ? 2 : 0;
  bad |= memcmp(first, F.data(), 4ull * (R + 1)) ? 4 : 0;
  bad |= memcmp(len, L.data(), 4ull * R) ? 8 : 0;
  for (int r = 0; r < R; ++r) bad |= served[r] != SV[r] ? 16 : 0;
  bad |= *nfo != n_free - used ? 32 : 0;
  // release
  std::vector<int> FI(free_ids, free_ids + NB);
  int c2 = *nfo;
  for (int r = 0; r < R; ++r) {
    done[r] = g() % 5 < 2;
    if (!done[r]) continue;
    if (len[r] >= 0 && len[r] <= MB * bt) for (int c = 0; c < (len[r] + bt - 1) / bt; ++c) if (c2 < NB) FI[c2++] = table[(size_t)r * MB + c];
    L[r] = 0;
  }
  int *len2 = alias ? len : (int *)take(4 * R), *nf2 = alias ? nfo : (int *)take(4);
  festina_kv_requests q2{R, MB, bt, NB, len, nullptr, table, free_ids, nfo};
  festina_kv_step o2{0, nullptr, nullptr, len2, nullptr, nf2};
  memset(ws, 0xff, n);
  const size_t n2 = festina_blocks_workspace_bytes(R, 0);
  void *ws2 = take(n2);
  if (int st = festina_release_blocks(&q2, done, &o2, ws2, n2, nullptr)) { printf("status %d\n", st); return 2; }
  bad |= memcmp(free_ids, FI.data(), 4ull * NB) ? 64 : 0;
  bad |= memcmp(len2, L.data(), 4ull * R) ? 128 : 0;
  bad |= *nf2 != c2 ? 256 : 0;
  printf("R %d bt %d longest %d tokens %d budget %d alias %d: bad %d\n", R, bt, longest, mt, budget, alias, bad);
  return bad != 0;
}
