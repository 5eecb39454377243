// attend.hip -- MI355X (gfx950) kernels and C-ABI host dispatch of attention over the 8-bit key/value cache.
//
// With codes kc, vc and scales ks, vs of a key's block, the logit in base 2 is
//   x_j = (scale log2 e) ks <q, kc_j>,
// and one pass over the keys keeps, for each query row, the running maximum m of y_j = x_j + log2 vs_j, the sum
// l = sum 2^(y_j - m) / vs_j and the vector o = sum 2^(y_j - m) vc_j; then out = o / l and
// lse = (m + log2 l) ln 2.  Folding vs into the exponent costs nothing (the scaling of the logit
// is a fused multiply-add either way), leaves weights of bounded size for the second product, and lets the codes
// be its other operand as they are.
//
// Both products run on the matrix cores, keys (and values' dims) as rows and queries as columns: S' = K Q' and
// O' = V' P'.  A column then stays in the same lanes through both, so P goes from the first product's
// result straight into the second's operand: the keys of a tile are dealt to the first product's rows in the
// order in which the second wants them, and no value crosses lanes but the maximum and the sum.  Codes are
// converted exactly (e4m3 fits bfloat16 and half); q keeps its own type, the weights and the value
// codes are taken in half precision, whose 11 bits leave less error than the outputs' rounding; sums are
// float32.
//
// k_rows    up to 64 query rows (16 to 64, as registers allow) a request and key head (single tokens, short runs): 16 NT rows against 64 keys
//   per wave and step, operands loaded from the cache into the lanes that use them.  Bound by the cache's bytes.
//   All requests' keys form one line of 64-key units, cut into equal pieces, one a wave, so that
//   ragged lengths leave no wave behind; a row tile that a cut falls into is joined by k_rows_join.
//   64 requests up to 32,768 tokens, 8 heads of 128: 2.15 GB in 413 us, 5.2 TB/s (a large copy: 4.96).
// k_rows_whole   the same for short tables: a workgroup a row tile, joined in LDS, one launch.  One request of 403 tokens: 7 us,
//   a launch and a few round trips to memory.
// k_tiles   prompts: 128 query rows a workgroup, tiles of 64 keys converted once into LDS (two buffers, the next
//   tile's loads in flight meanwhile) and read by four waves of 32 rows.  Bound by the matrix cores and the exponentials.
//   Few tiles over a long cache are split over the keys (how far, the kernel decides, which knows how many there are) and
//   joined by k_tiles_join.
//   8,192 tokens, 32 heads over 8 of 128: 550 GFLOP in 558 us (985 TFLOP/s; a large library product 1,189), matrix cores
//   41% of the cycles, VALU issue 39%.  9,012 tokens of 16 heads of 64: 170 us, 27% and 52%: half the products an exponential.
// k_plan    running sums of the requests' units and tiles, for many requests.
#include <hip/hip_runtime.h>

#include <climits>
#include <cstddef>
#include <cstdint>

#include "festina.h"
#include "kv.h"

namespace {

using namespace festina_kv;

typedef __bf16 bf16;
typedef _Float16 f16;
typedef bf16 bf2 __attribute__((ext_vector_type(2)));
typedef bf16 bf8 __attribute__((ext_vector_type(8)));
typedef f16 h2 __attribute__((ext_vector_type(2)));
typedef f16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned u2 __attribute__((ext_vector_type(2)));

constexpr int kUnit = 64;            // keys of a step
constexpr int kWaves = 4;
constexpr int kBlock = 64 * kWaves;
// Waves of k_rows on a SIMD, and the pieces that it cuts the keys into: one for each wave of 256 compute units.  (Three
// waves of 128 dims and one row tile, 168 registers each, were slower: 64 requests up to 32,768 tokens 473 us against 440.)
constexpr int waves_of(int D, int NT) { return D > 128 || NT > 2 ? 1 : 2; }
constexpr int workers_of(int D, int NT) { return 1024 * waves_of(D, NT); }
constexpr int kGroups = 512;         // workgroups of k_tiles that fill the chip: two a compute unit
constexpr int kJoins = 2048;         // and of its join: eight
constexpr int kListed = 512;         // requests whose running sums a workgroup forms by itself
constexpr int kMaxRequests = 1 << 20;
constexpr long long kThreadsMost = UINT_MAX;     // along one axis of a grid
constexpr float kLn2 = 0.6931471805599453f;

template <typename T> struct Vec8;
template <> struct Vec8<bf16> { typedef bf8 type; };
template <> struct Vec8<f16> { typedef h8 type; };

struct AttArgs {
  int32_t R, MB, T, Hq, H, G, shift, NB, window;
  int32_t rows_max;                  // requests of at most so many rows are k_rows' (the others k_tiles')
  int32_t tiles_each;                // k_rows without cuts: row tiles a request
  int32_t workers;
  int32_t tiles_most, splits_most;   // k_tiles: bounds of all row tiles and of the parts of one's keys
  int32_t tile_rows;                 // query rows a workgroup of k_tiles
  float scale;                       // times log2 e
  const int32_t *table, *length, *first;
  const void *q;
  int64_t q_token, q_head;
  void *out;
  int64_t out_token, out_head;
  float *lse;
  const uint8_t *k, *v;
  const float *ks, *vs;
  const long long *plan;             // [2][R + 1] running sums of units and of tiles, or NULL
  float *part_o, *part_ml;           // pieces: unnormalised rows; (m, l)
  struct Cut *cuts;                  // [workers]
  int4 *joins;                       // what k_tiles_join needs: (groups, splits), then for each row tile the request's
                                     // first token, the tile's first row, the request's rows
};

// What k_rows_join needs of the row tile that begins a join at a piece's start; n = 0: none.
struct Cut {
  int32_t n;                         // pieces
  int32_t second;                    // the first of them is its piece's second part
  int32_t row0, rows;                // first row of the tile, rows of the request
  int32_t first, head;               // the request's first token, the key head's first query head
  int32_t unused[2];
};

struct Request {
  int first, n, length;
};

__device__ __forceinline__ Request request(const AttArgs &a, int r) {
  Request q;
  q.first = min(max(a.first[r], 0), a.T);
  q.n = min(max(a.first[r + 1], q.first), a.T) - q.first;
  q.length = min(max(a.length[r], 0), a.MB << a.shift);
  return q;
}

__device__ __forceinline__ int cdiv(int x, int y) { return (x + y - 1) / y; }

// First 64-key unit that any of the request's rows sees, and how many from there on (at least one, so that rows
// without keys are written too).
__device__ __forceinline__ int first_unit(const AttArgs &a, const Request &q) {
  return a.window > 0 ? max(q.length - q.n - a.window + 1, 0) / kUnit : 0;
}
__device__ __forceinline__ int units(const AttArgs &a, const Request &q) {
  return max(cdiv(q.length, kUnit) - first_unit(a, q), 1);
}

// A value that is the same in all lanes, kept once.
__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long same(long long x) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
  return (long long)((unsigned long long)hi << 32 | lo);
}

template <int ROWS>
__device__ __forceinline__ long long units_of(const AttArgs &a, int r) {
  const Request q = request(a, r);
  const int rows = q.n * a.G;
  return rows > 0 && rows <= a.rows_max ? (long long)units(a, q) * cdiv(rows, ROWS) * a.H : 0;
}

__device__ __forceinline__ long long tiles_of(const AttArgs &a, int r) {
  const int rows = request(a, r).n * a.G;
  return rows > a.rows_max ? cdiv(rows, a.tile_rows) : 0;
}

// Running sums over a workgroup of N threads: returns the exclusive sum and the whole.
template <int N>
__device__ __forceinline__ long long scan(long long x, long long *lds, long long *whole) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  long long s = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long y = __shfl_up(s, d);
    if (lane >= d) s += y;
  }
  if (lane == 63) lds[wave] = s;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < N / 64; ++w) {
    const long long y = lds[w];
    before += w < wave ? y : 0;
    all += y;
  }
  __syncthreads();
  *whole = all;
  return s - x + before;
}

// list[0 .. R]: running sums of f(r) over the requests, R <= kListed; every wave of a workgroup forms and writes
// all of them, so no wave waits for another.
template <typename F>
__device__ __forceinline__ void list_sums(const AttArgs &a, F f, long long *list) {
  const int lane = threadIdx.x & 63;
  long long sum = 0;
  for (int r0 = 0; r0 < a.R; r0 += 64) {
    const int r = r0 + lane;
    long long x = r < a.R ? f(r) : 0;
    const long long own = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const long long y = __shfl_up(x, d);
      if (lane >= d) x += y;
    }
    if (r < a.R) list[r] = sum + x - own;
    sum += __shfl(x, 63);
  }
  if (lane == 0) list[a.R] = sum;
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// The r with list[r] <= u < list[r + 1]: a wave compares 64 entries a time.
__device__ __forceinline__ int find(const long long *list, int R, long long u) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = R;
  while (n > 1) {
    const int s = (n + 63) >> 6, i = lo + lane * s;
    const unsigned long long at = __ballot(lane * s < n && list[i < lo + n ? i : lo] <= u);
    const int k = (__builtin_popcountll(at) - 1) * s;
    lo += k;
    n = min(s, n - k);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

template <int ROWS>
__global__ void __launch_bounds__(1024) k_plan(AttArgs a, long long *plan) {
  __shared__ long long lds[16];
  long long u0 = 0, t0 = 0, whole;
  for (int r0 = 0; r0 < a.R; r0 += 1024) {
    const int r = r0 + threadIdx.x;
    const long long u = scan<1024>(r < a.R ? units_of<ROWS>(a, r) : 0, lds, &whole) + u0;
    u0 += whole;
    const long long t = scan<1024>(r < a.R ? tiles_of(a, r) : 0, lds, &whole) + t0;
    t0 += whole;
    if (r < a.R) {
      plan[r] = u;
      plan[a.R + 1 + r] = t;
    }
  }
  if (threadIdx.x == 0) {
    plan[a.R] = u0;
    plan[2 * a.R + 1] = t0;
  }
}

// ------------------------------------------------------------------ operands

__device__ __forceinline__ void decode4(unsigned c, bf16 *x) {
  *reinterpret_cast<bf2 *>(x) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c, 1.f, false);
  *reinterpret_cast<bf2 *>(x + 2) = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)c, 1.f, true);
}
__device__ __forceinline__ void decode4(unsigned c, f16 *x) {
  *reinterpret_cast<h2 *>(x) = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)c, 1.f, false);
  *reinterpret_cast<h2 *>(x + 2) = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)c, 1.f, true);
}
template <typename T>
__device__ __forceinline__ typename Vec8<T>::type decode8(unsigned c0, unsigned c1) {
  union { T x[8]; typename Vec8<T>::type v; } u;
  decode4(c0, u.x);
  decode4(c1, u.x + 4);
  return u.v;
}

__device__ __forceinline__ f4 mfma16(bf8 a, bf8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f4 mfma16(h8 a, h8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f16v mfma32(bf8 a, bf8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f16v mfma32(h8 a, h8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }
__device__ __forceinline__ float kNegInf() { return -__builtin_inff(); }

// Over the lanes that differ by 16 and 32, or by 32 alone.
template <typename F>
__device__ __forceinline__ float across32(float x, F f) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <typename F>
__device__ __forceinline__ float across16(float x, F f) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_(float x, float y) { return fmaxf(x, y); }
__device__ __forceinline__ float add_(float x, float y) { return x + y; }

// The keys a row sees: `count` from `from` on.
struct Span {
  int from, count;
  __device__ __forceinline__ bool has(int key) const { return (unsigned)(key - from) < (unsigned)count; }
};
__device__ __forceinline__ Span span(const AttArgs &a, int pos) {
  const int from = a.window > 0 ? max(pos - a.window + 1, 0) : 0;
  return Span{from, max(pos - from + 1, 0)};
}
// Keeps a rare branch a branch: without it the compiler computes the masks of every step.
__device__ __forceinline__ void rarely() { asm volatile(""); }

// Which bytes of a word of four codes are NaN, as 0xff each.
__device__ __forceinline__ unsigned nan_bytes(unsigned c) {
  const unsigned h = ((c & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
  return (h >> 7) * 0xffu;
}
constexpr unsigned kOnes = 0x38383838u;     // four codes of 1.0

// Bytes of the word of codes 4w .. 4w + 3 that lie below n.
__device__ __forceinline__ unsigned below(int n, int w) {
  const int k = n - 4 * w;
  return k >= 4 ? ~0u : k <= 0 ? 0u : (1u << (8 * k)) - 1;
}

// A row's weights are taken relative to a reference m that follows the keys at hand in strides: logits are formed relative
// to it, and while the largest of a step lies between kLow and kSlack (in base 2) nothing has to be rescaled.  Else the
// reference is placed kHead below that largest.  Half precision keeps 11 bits of weights of up to 2^15 and down to 2^-14 and
// is off by at most 2^-25 below that: 2^-19 of the step's largest weight.  The reference goes down as well as up, so that keys
// beside one of far more weight, or behind a block whose value scale (which weighs in the maximum) is far larger, are
// not lost to the format; the sums, in 32 bits, may then be far larger than what is added to them.  -inf: no key seen
// yet, logits are relative to 0.
constexpr float kHead = 7.f, kSlack = 15.f, kLow = -6.f;
// The same for k_tiles, on the sum of a lane's weights of 16 keys: 2^-6 .. 2^15, as one comparison of its bits.  (A sum of 0
// is looked at too: a tile of which a row sees nothing.)
constexpr unsigned kLeastSum = 0x3c800000, kSums = 0x47000000 - kLeastSum;
// (Both ends cost 1% of a prompt of 8,192 tokens, 2% of units of 64 dims; a kHead of 10, which keeps three bits more, as much
// again, since new maxima then move the reference more often.)
// How far down the reference may go, by a row's sum of weights so far: the sums of values, at most 448 * 2^32 times
// as large, stay below 2^104.
__device__ __forceinline__ float down(float top, float l) { return fminf(fmaxf(top - kHead, log2_(l) - 60.f), 0.f); }
__device__ __forceinline__ bool moves(float top, float m) {
  return m == kNegInf() ? top > kNegInf() : top > kSlack || (top < kLow && top > kNegInf());
}
// Turns `top`, a row's largest logit relative to the reference, into how far the reference moves; scales l (of which each lane
// has a part) and returns the factor for the row's other sums.
__device__ __forceinline__ float move(float &top, float &m, float &l) {
  const bool fresh = m == kNegInf();
  const float all = across32(across16(l, add_), add_);
  if (!moves(top, m)) top = 0.f;
  else top = top < kLow && !fresh ? down(top, all) : top - kHead, m = fresh ? top : m + top;
  const float f = fresh ? 1.f : exp2_(-top);
  l *= f;
  return f;
}

// Weight of a piece with reference m in a row whose largest is M.
__device__ __forceinline__ float weight(float m, float M) { return m == kNegInf() ? 0.f : exp2_(m - M); }

template <typename T>
__device__ __forceinline__ void put4(T *p, const float *x) {
  union { T t[4]; u2 w; } u;
#pragma unroll
  for (int i = 0; i < 4; ++i) u.t[i] = (T)x[i];
  *reinterpret_cast<u2 *>(p) = u.w;
}

// ------------------------------------------------------------------ k_rows

// What one wave keeps of the cache for a step: the raw codes of 64 keys and values.
template <int D>
struct RowsStep {
  u4 k[4][D / 64];
  u2 kr[4][D % 64 ? 1 : 1];
  u4 v[D / 16];
  float ks, vs;
  bool ok;
};

template <typename T, int D, int NT>
struct Rows {
  static constexpr int kRows = 16 * NT, kSteps = D / 32, kPitch = D + 4;

  struct Shared {
    float o[kWaves][16][kPitch];
    float m[kWaves][kRows], l[kWaves][kRows];
  };

  // Row m of the first product's tile u is key 16 (m / 4) + 4 u + m % 4 of the step; a lane holds the values of
  // keys 16 g .. 16 g + 15.  Their blocks:
  static __device__ __forceinline__ int key_of_k(int base) { return base + ((threadIdx.x & 15) >> 2) * 16; }
  static __device__ __forceinline__ int key_of_v(int base) { return base + ((threadIdx.x & 63) >> 4) * 16; }
  static __device__ __forceinline__ int2 blocks(const AttArgs &a, const int32_t *table, int base) {
    return make_int2(table[min(key_of_k(base) >> a.shift, a.MB - 1)], table[min(key_of_v(base) >> a.shift, a.MB - 1)]);
  }

  // (Reads that mark the codes as not to be kept were slower: 64 requests up to 32,768 tokens 479 us against 419.)
  static __device__ __forceinline__ void load(const AttArgs &a, int2 ids, int h, int base, RowsStep<D> &s) {
    const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4, bt = 1 << a.shift;
    const int key_k = key_of_k(base), key_v = key_of_v(base);
    int id_k = ids.x, id_v = ids.y;
    s.ok = (unsigned)id_v < (unsigned)a.NB;
    id_k = (unsigned)id_k < (unsigned)a.NB ? id_k : 0;
    id_v = s.ok ? id_v : 0;
    const size_t bh_k = (size_t)id_k * a.H + h, bh_v = (size_t)id_v * a.H + h;
    const uint8_t *k = a.k + (bh_k * bt + (key_k & (bt - 1)) + (m & 3)) * D;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int j = 0; j < D / 64; ++j) s.k[u][j] = *reinterpret_cast<const u4 *>(k + u * 4 * D + j * 64 + g * 16);
      if constexpr (D % 64 != 0) s.kr[u][0] = *reinterpret_cast<const u2 *>(k + u * 4 * D + D / 64 * 64 + g * 8);
    }
    s.ks = a.ks[bh_v];
    s.vs = a.vs[bh_v];
    const uint8_t *v = a.v + (bh_v * D + m) * bt + (key_v & (bt - 1));
#pragma unroll
    for (int t = 0; t < D / 16; ++t) s.v[t] = *reinterpret_cast<const u4 *>(v + (size_t)t * 16 * bt);
  }

  struct State {
    typename Vec8<T>::type q[NT][kSteps];
    f4 o[NT][D / 16];
    float m[NT], l[NT];
    Span sees[NT];
  };

  static __device__ __forceinline__ void step(const AttArgs &a, const Request &rq, int base, int pos_min, int pos_max,
                                              RowsStep<D> &s, State &st) {
    const int g = (threadIdx.x & 63) >> 4;
    f4 x[NT][4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) x[nt][u] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        typename Vec8<T>::type kf;
        if (i < D / 64 * 2) kf = decode8<T>(s.k[u][i / 2][(i & 1) * 2], s.k[u][i / 2][(i & 1) * 2 + 1]);
        else kf = decode8<T>(s.kr[u][0][0], s.kr[u][0][1]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) x[nt][u] = mfma16(kf, st.q[nt][i], x[nt][u]);
      }
    }
    const float c = a.scale * s.ks, vs = fminf(fmaxf(s.vs, kScaleMin), kScaleMax);
    const float lv = log2_(vs), iv = __builtin_amdgcn_rcpf(vs);
    const bool masked = base + kUnit - 1 > pos_min || (a.window > 0 && base <= pos_max - a.window) || __any(!s.ok);
    h8 w[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float shift = st.m[nt] == kNegInf() ? lv : lv - st.m[nt];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[nt][u][i] = fmaf(x[nt][u][i], c, shift);
      if (masked) {
        rarely();
        const Span sees{st.sees[nt].from - base - 16 * g, s.ok ? st.sees[nt].count : 0};
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) x[nt][u][i] = sees.has(4 * u + i) ? x[nt][u][i] : kNegInf();
      }
      float top = x[nt][0][0];
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, x[nt][u][i]);
      top = across32(across16(top, max_), max_);
      if (__any(moves(top, st.m[nt]))) {
        rarely();
        const float f = move(top, st.m[nt], st.l[nt]);
#pragma unroll
        for (int u = 0; u < 4; ++u) x[nt][u] -= top;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) st.o[nt][t] *= f;
      }
      float sum = 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = exp2_(x[nt][u][i]);
          sum += p;
          w[nt][u >> 1][(u & 1) * 4 + i] = (f16)p;
        }
      st.l[nt] = fmaf(sum, iv, st.l[nt]);
    }
    if (masked) {
      rarely();
      // what lies behind the last token may be anything: no product with it
      const int n = s.ok ? min(max(rq.length - (base + 16 * g), 0), 16) : 0;
      unsigned any = 0;
#pragma unroll
      for (int t = 0; t < D / 16; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s.v[t][i] &= below(n, i);
          any |= nan_bytes(s.v[t][i]);
        }
      if (__any(any != 0)) {
        rarely();
        // a NaN that some rows see and others do not is put into the rows that see it and left out of the product
#pragma unroll
        for (int t = 0; t < D / 16; ++t) {
          unsigned nan[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            nan[i] = nan_bytes(s.v[t][i]);
            s.v[t][i] &= ~nan[i];
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            f4 hits = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              h8 sees;
#pragma unroll
              for (int j = 0; j < 8; ++j)
                sees[j] = s.ok && st.sees[nt].has(base + 16 * g + 8 * i + j) ? (f16)1.f : (f16)0.f;
              hits = mfma16(decode8<f16>(nan[2 * i] & kOnes, nan[2 * i + 1] & kOnes), sees, hits);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) st.o[nt][t][i] = hits[i] > 0.f ? __builtin_nanf("") : st.o[nt][t][i];
          }
          __builtin_amdgcn_sched_barrier(0);           // one tile's operands at a time
        }
      }
    }
#pragma unroll
    for (int t = 0; t < D / 16; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const h8 vf = decode8<f16>(s.v[t][2 * i], s.v[t][2 * i + 1]);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) st.o[nt][t] = mfma16(vf, w[nt][i], st.o[nt][t]);
      }
  }

  // Rows `tile` of request r and key head h: every `stride`th of its units from k0 to k1.
  static __device__ __forceinline__ void scan_keys(const AttArgs &a, int r, const Request &rq, int h, int tile, int k0,
                                                   int k1, int stride, State &st) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    const int rows = rq.n * a.G, row0 = tile * kRows, before = rq.length - rq.n;
    const int pos_min = before + row0 / a.G, pos_max = before + (min(row0 + kRows, rows) - 1) / a.G;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int i = row0 + nt * 16 + c, t = i / a.G;
      const bool in = i < rows;
      st.sees[nt] = span(a, in ? before + t : -1);
      st.m[nt] = kNegInf();
      st.l[nt] = 0.f;
#pragma unroll
      for (int d = 0; d < D / 16; ++d) st.o[nt][d] = f4{0.f, 0.f, 0.f, 0.f};
      const T *q = static_cast<const T *>(a.q) + (int64_t)(rq.first + (in ? t : 0)) * a.q_token +
                   (int64_t)(h * a.G + (in ? i - t * a.G : 0)) * a.q_head;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const int d = s < D / 64 * 2 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : D / 64 * 64 + g * 8;
        u4 raw = *reinterpret_cast<const u4 *>(q + d);
        if (!in) raw = u4{0u, 0u, 0u, 0u};
        st.q[nt][s] = __builtin_bit_cast(typename Vec8<T>::type, raw);
      }
    }
    const int32_t *table = a.table + (size_t)r * a.MB;
    const int u0 = first_unit(a, rq);
    // the next step's blocks are read while this one is worked on (behind the last step: some column's, not used): 64
    // requests up to 32,768 tokens 441 -> 416 us
    int2 ids = blocks(a, table, (u0 + k0) * kUnit);
    for (int u = k0; u < k1; u += stride) {
      RowsStep<D> s;
      load(a, ids, h, (u0 + u) * kUnit, s);
      ids = blocks(a, table, (u0 + u + stride) * kUnit);
      step(a, rq, (u0 + u) * kUnit, pos_min, pos_max, s, st);
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) st.l[nt] = across32(across16(st.l[nt], add_), add_);
  }

  // One wave's keys alone: the rows themselves (part < 0), or the piece's result at its place.
  static __device__ __forceinline__ void piece(const AttArgs &a, int r, const Request &rq, int h, int tile, int k0, int k1,
                                               int part) {
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4;
    State st;
    scan_keys(a, r, rq, h, tile, k0, k1, 1, st);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int i = tile * kRows + nt * 16 + c;
      if (i >= rq.n * a.G) continue;
      if (part < 0) {
        const int t = i / a.G;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) finish(a, rq.first + t, h * a.G + i - t * a.G, d * 16 + g * 4, st.m[nt], st.l[nt], st.o[nt][d]);
      } else {
        const size_t p = (size_t)part * kRows + nt * 16 + c;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) *reinterpret_cast<f4 *>(a.part_o + p * D + d * 16 + g * 4) = st.o[nt][d];
        if (g == 0) {
          a.part_ml[p * 2] = st.m[nt];
          a.part_ml[p * 2 + 1] = st.l[nt];
        }
      }
    }
  }

  // A workgroup's keys: its waves' parts of each row joined in LDS.
  static __device__ __forceinline__ void whole(const AttArgs &a, int r, const Request &rq, int h, int tile, Shared &sh) {
    const int lane = threadIdx.x & 63, wave = same((int)threadIdx.x >> 6), c = lane & 15, g = lane >> 4;
    const int rows = rq.n * a.G, row0 = tile * kRows;
    State st;
    scan_keys(a, r, rq, h, tile, wave, units(a, rq), kWaves, st);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      if (g == 0) {
        sh.m[wave][nt * 16 + c] = st.m[nt];
        sh.l[wave][nt * 16 + c] = st.l[nt];
      }
#pragma unroll
      for (int t = 0; t < D / 16; ++t) *reinterpret_cast<f4 *>(&sh.o[wave][c][t * 16 + g * 4]) = st.o[nt][t];
      __syncthreads();
      for (int e = threadIdx.x; e < 16 * (D / 4); e += kBlock) {
        const int y = e / (D / 4), d = (e % (D / 4)) * 4, i = row0 + nt * 16 + y;
        if (i >= rows) break;
        float M = kNegInf(), L = 0.f;
        f4 O = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, sh.m[w][nt * 16 + y]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = weight(sh.m[w][nt * 16 + y], M);
          L = fmaf(sh.l[w][nt * 16 + y], f, L);
          O += *reinterpret_cast<const f4 *>(&sh.o[w][y][d]) * f;
        }
        const int t = i / a.G;
        finish(a, rq.first + t, h * a.G + i - t * a.G, d, M, L, O);
      }
      __syncthreads();
    }
  }

  static __device__ __forceinline__ void finish(const AttArgs &a, int t, int head, int d, float M, float L, f4 O) {
    const bool none = M == kNegInf() && L == L;     // (NaN logits leave the maximum alone)
    const float f = none ? 0.f : 1.f / L;
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = none ? 0.f : O[i] * f;
    put4(static_cast<T *>(a.out) + (int64_t)t * a.out_token + (int64_t)head * a.out_head + d, x);
    if (d == 0 && a.lse) a.lse[(size_t)t * a.Hq + head] = none ? kNegInf() : (M + log2_(L)) * kLn2;
  }
};

// Pieces of equal length; more rows take longer pieces, since a piece's result is read and written once more.
template <int NT>
__device__ __forceinline__ int pieces(const AttArgs &a, long long all) {
  return (int)min((long long)a.workers, max((all + NT - 1) / NT, 1ll));
}
__device__ __forceinline__ long long piece_start(long long all, int w, int n) { return all * w / n; }

// A workgroup for each row tile and key head, its waves over the keys in turn: few keys, one launch.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(kBlock, (D <= 128 && NT <= 2) ? 2 : 1) k_rows_whole(AttArgs a) {
  typedef Rows<T, D, NT> K;
  __shared__ typename K::Shared sh;
  const int tile = blockIdx.x % a.tiles_each, rest = blockIdx.x / a.tiles_each, h = rest % a.H, r = rest / a.H;
  const Request rq = request(a, r);
  const int rows = rq.n * a.G;
  if (rows > a.rows_max || tile * K::kRows >= rows) return;
  K::whole(a, r, rq, h, tile, sh);
}

// A wave a piece.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(64, waves_of(D, NT)) k_rows(AttArgs a) {
  typedef Rows<T, D, NT> K;
  __shared__ long long list_[kListed + 1];
  const long long *list = a.plan;
  if (!list) {
    list_sums(a, [&](int r) { return units_of<K::kRows>(a, r); }, list_);
    list = list_;
  }
  const long long all = same(list[a.R]);
  const int n = pieces<NT>(a, all), w = blockIdx.x;
  Cut cut{};
  if (w < n) {
    long long u = piece_start(all, w, n);
    const long long start = u, end = piece_start(all, w + 1, n);
    for (int place = 2 * w; u < end; ++place) {
      const int r = find(list, a.R, u);
      const Request rq = request(a, r);
      const long long begin = same(list[r]);
      const int each = units(a, rq), at = (int)((u - begin) / each), tiles = cdiv(rq.n * a.G, K::kRows);
      const long long tile0 = begin + (long long)at * each;
      const int k0 = (int)(u - tile0), k1 = (int)min((long long)each, k0 + (end - u));
      const int h = at / tiles, tile = at % tiles;
      if (u == start && k0 > 0) {
        // this piece's start cuts the tile: the first such cut is where the tile's pieces are joined
        const long long prior = piece_start(all, w - 1, n);
        if (prior <= tile0) {
          const int last = (int)(((tile0 + each) * n - 1) / all);      // piece of the tile's last unit
          cut = Cut{last - w + 2, prior < tile0 ? 1 : 0, tile * K::kRows, rq.n * a.G, rq.first, h * a.G, {0, 0}};
        }
      }
      K::piece(a, r, rq, h, tile, k0, k1, k0 == 0 && k1 == each ? -1 : min(place, 2 * w + 1));
      u += k1 - k0;
    }
  }
  if (threadIdx.x == 0) a.cuts[w] = cut;
}

// Joins one row's n pieces, the first at p0 and the others from p1 on: a wave, as many groups of lanes as a row leaves
// room for each taking every kSides-th piece, eight of them with their loads in flight at a time.
// (32 requests, a token each, up to 8,192 held: 24.1 -> 21.5 us against a piece a time for the whole wave; sixteen in flight 22.2.)
template <typename T, int D>
__device__ __forceinline__ void join_row(const AttArgs &a, size_t p0, size_t p1, size_t stride, int n, int t, int head) {
  constexpr int kAtOnce = 8, kLanes = D <= 64 ? 16 : D <= 128 ? 32 : 64, kSides = 64 / kLanes;
  const int lane = threadIdx.x & 63, side = lane / kLanes, d = lane % kLanes * 4;
  if (d >= D) return;
  float M = kNegInf(), L = 0.f;
  f4 O = f4{0.f, 0.f, 0.f, 0.f};
  for (int i0 = side; i0 < n; i0 += kAtOnce * kSides) {
    f4 o[kAtOnce];
    float2 ml[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = min(i0 + k * kSides, n - 1);
      const size_t at = i == 0 ? p0 : p1 + (size_t)(i - 1) * stride;
      ml[k] = *reinterpret_cast<const float2 *>(a.part_ml + at * 2);
      o[k] = *reinterpret_cast<const f4 *>(a.part_o + at * D + d);
    }
    float now = M;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) now = fmaxf(now, ml[k].x);
    const float f = weight(M, now);
    M = now;
    L *= f;
    O *= f;
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const bool there = i0 + k * kSides < n;
      const float g = there ? weight(ml[k].x, M) : 0.f;
      if (there) {
        L = fmaf(ml[k].y, g, L);
        O += o[k] * g;
      }
    }
  }
  // the sides' sums; one without a piece has M = -inf and adds nothing
#pragma unroll
  for (int x = kLanes; x < 64; x <<= 1) {
    const float other = __shfl_xor(M, x), now = fmaxf(M, other), f = weight(M, now), g = weight(other, now);
    M = now;
    L = fmaf(__shfl_xor(L, x), g, L * f);
#pragma unroll
    for (int i = 0; i < 4; ++i) O[i] = fmaf(__shfl_xor(O[i], x), g, O[i] * f);
  }
  if (side == 0) Rows<T, D, 1>::finish(a, t, head, d, M, L, O);
}

// A wave joins rows of the tile that the cut at piece blockIdx.x + 1 leaves to it: one where the grid has a wave a row.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(kBlock) k_rows_join(AttArgs a) {
  constexpr int kRows = 16 * NT;
  const int w = blockIdx.x + 1;
  const Cut cut = a.cuts[w];
  if (cut.n == 0) return;
  for (int row = blockIdx.y * kWaves + (threadIdx.x >> 6); row < kRows; row += gridDim.y * kWaves) {
    const int i = cut.row0 + row, t = i / a.G;
    if (i >= cut.rows) return;
    join_row<T, D>(a, (size_t)(2 * (w - 1) + cut.second) * kRows + row, (size_t)(2 * w) * kRows + row, 2 * kRows, cut.n,
                   cut.first + t, cut.head + i - t * a.G);
  }
}

// ------------------------------------------------------------------ k_tiles

// A tile of 64 keys in LDS.
template <typename T, int D>
struct KeyTile {
  static constexpr int kPitch = D + 8;
  __attribute__((aligned(16))) T k[kUnit][kPitch];
  float c[4], lv[4], iv[4];          // for 16 keys each: scale, log2 and reciprocal of the values' scale
};

// Its values.
template <int D, int W>
struct ValueTile {
  static constexpr int kPitch = kUnit + 8;
  __attribute__((aligned(16))) f16 v[D][kPitch];
  __attribute__((aligned(16))) int nans[W];          // a wave staged a NaN that not every row sees
  __attribute__((aligned(8))) uint16_t nan[D][4];    // which: a bit a key
};

// What a thread stages of each tile: a 16-byte piece of the keys and one of the values, `kLoads` times.
template <typename T, int D, int W>
struct Stage {
  static constexpr int kThreads = 64 * W, kItems = kUnit * D / 16, kLoads = (kItems + kThreads - 1) / kThreads;

  const uint8_t *k[kLoads], *v[kLoads];              // the pieces in block 0
  unsigned at_k[kLoads], at_v[kLoads], at_s;         // where their blocks stand in a tile's part of the table, in bytes
  int id_k[kLoads], id_v[kLoads], id_s;              // the blocks of the next tile
  u4 raw_k[kLoads], raw_v[kLoads];
  float ks, vs;
  bool ok;

  // keys to the first threads, values to the last, so that all have some where there are fewer pieces than threads
  static __device__ __forceinline__ int key_item(int i) { return threadIdx.x + i * kThreads; }
  static __device__ __forceinline__ int value_item(int i) { return kThreads - 1 - threadIdx.x + i * kThreads; }
  static __device__ __forceinline__ bool has(int item) { return kItems % kThreads == 0 || item < kItems; }
  static __device__ __forceinline__ int key_of(int item) { return item / (D / 16); }
  static __device__ __forceinline__ int key_of_value(int item) { return (item & 3) * 16; }

  __device__ __forceinline__ void begin(const AttArgs &a, int h) {
    const int bt = 1 << a.shift;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int x = key_item(i), y = has(value_item(i)) ? value_item(i) : 0;
      k[i] = a.k + (size_t)h * bt * D + (key_of(x) & (bt - 1)) * D + x % (D / 16) * 16;
      v[i] = a.v + (size_t)h * bt * D + (size_t)(y >> 2) * bt + (key_of_value(y) & (bt - 1));
      at_k[i] = (min(key_of(x), kUnit - 1) >> a.shift) * 4;
      at_v[i] = (key_of_value(y) >> a.shift) * 4;
    }
    at_s = ((threadIdx.x & 3) * 16 >> a.shift) * 4;
  }

  // A tile begins at a multiple of 64 keys, so a key's column is the tile's first one and its own part: offsets of less
  // than 2^29 bytes from the row's start, of which only the tile's part changes.
  __device__ __forceinline__ void blocks(const AttArgs &a, const int32_t *table, int base) {
    const unsigned from = (unsigned)(base >> a.shift) * 4, last = (unsigned)(a.MB - 1) * 4;
    const auto block_at = [&](unsigned at) {
      return *reinterpret_cast<const int32_t *>(reinterpret_cast<const char *>(table) + min(from + at, last));
    };
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      id_k[i] = block_at(at_k[i]);
      id_v[i] = block_at(at_v[i]);
    }
    id_s = block_at(at_s);
  }

  // The codes of the tile at `base`, whose blocks were read.  A block that is not there reads as zeros.
  static __device__ __forceinline__ unsigned block_bytes(const AttArgs &a) { return (unsigned)a.H * D << a.shift; }   // below 2^27
  static __device__ __forceinline__ int within(const AttArgs &a, int base) {   // its place in a block longer than a tile
    return a.shift > 6 ? base & ((1 << a.shift) - 1) : 0;
  }
  __device__ __forceinline__ void load_keys(const AttArgs &a, int h, int base) {
    bool all = true;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool there = (unsigned)id_k[i] < (unsigned)a.NB;
      all &= there;
      raw_k[i] = u4{0u, 0u, 0u, 0u};
      if (has(key_item(i)))
        raw_k[i] = *reinterpret_cast<const u4 *>(k[i] + (size_t)min((unsigned)id_k[i], (unsigned)a.NB - 1) * block_bytes(a) + within(a, base) * D);
    }
    if (__any(!all)) {
      rarely();
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if ((unsigned)id_k[i] >= (unsigned)a.NB) raw_k[i] = u4{0u, 0u, 0u, 0u};
    }
    if (threadIdx.x < 64) {
      ok = (unsigned)id_s < (unsigned)a.NB;
      const size_t at = (size_t)(ok ? id_s : 0) * a.H + h;
      ks = a.ks[at];
      vs = a.vs[at];
    }
  }
  __device__ __forceinline__ void load_values(const AttArgs &a, int base) {
    bool all = true;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool there = (unsigned)id_v[i] < (unsigned)a.NB;
      all &= there;
      raw_v[i] = u4{0u, 0u, 0u, 0u};
      if (has(value_item(i)))
        raw_v[i] = *reinterpret_cast<const u4 *>(v[i] + (size_t)min((unsigned)id_v[i], (unsigned)a.NB - 1) * block_bytes(a) + within(a, base));
    }
    if (__any(!all)) {
      rarely();
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        if ((unsigned)id_v[i] >= (unsigned)a.NB) raw_v[i] = u4{0u, 0u, 0u, 0u};
    }
  }

  __device__ __forceinline__ void put_keys(KeyTile<T, D> &b) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int x = key_item(i), d = x % (D / 16) * 16;
      if (!has(x)) continue;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        *reinterpret_cast<typename Vec8<T>::type *>(&b.k[key_of(x)][d + j * 8]) = decode8<T>(raw_k[i][2 * j], raw_k[i][2 * j + 1]);
    }
  }
  __device__ __forceinline__ void put_scales(const AttArgs &a, KeyTile<T, D> &b) const {
    if (threadIdx.x < 4) {
      // a block that is not there: its codes are zeros and its logits -inf
      const float s = fminf(fmaxf(vs, kScaleMin), kScaleMax);
      b.c[threadIdx.x] = ok ? a.scale * ks : 0.f;
      b.lv[threadIdx.x] = ok ? log2_(s) : kNegInf();
      b.iv[threadIdx.x] = ok ? __builtin_amdgcn_rcpf(s) : 0.f;
    }
  }

  // `n`: keys of the tile that there are.  For tiles of which some row of the workgroup does not see all.
  __device__ __forceinline__ void clean_values(int n, ValueTile<D, W> &b) {
    {
      unsigned any = 0;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int y = value_item(i);
        unsigned bits = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          // what lies behind the last token may be anything; a NaN that some rows see and others do not is left out of
          // the product and put into the rows that see it
          raw_v[i][j] &= below(n - key_of_value(y), j);
          const unsigned x = nan_bytes(raw_v[i][j]);
          raw_v[i][j] &= ~x;
          bits |= ((x & 0x01010101u) * 0x01020408u >> 24) << (4 * j);
        }
        if (has(y)) b.nan[y >> 2][y & 3] = (uint16_t)bits;
        any |= has(y) ? bits : 0u;
      }
      const int nans = __any(any != 0);
      if ((threadIdx.x & 63) == 0) b.nans[threadIdx.x >> 6] = nans;
    }
  }
  __device__ __forceinline__ void put_values(ValueTile<D, W> &b) const {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int y = value_item(i);
      if (!has(y)) continue;
#pragma unroll
      for (int j = 0; j < 2; ++j)
        *reinterpret_cast<h8 *>(&b.v[y >> 2][key_of_value(y) + j * 8]) = decode8<f16>(raw_v[i][2 * j], raw_v[i][2 * j + 1]);
    }
  }
};

// 32 query rows of a wave: columns of the products.
template <typename T, int D>
struct TileRows {
  typedef typename Vec8<T>::type Vec;

  Vec q[D / 16];
  f16v o[D / 32];
  f16v x[2];                         // logits of a tile, 32 keys each
  h8 w[2][2];                        // its weights
  float ref, l;                      // the reference (0 where no key was seen)
  unsigned sums_kept;                // sums of kLeastSum and so many more leave it; 0 where no key was seen
  Span sees;

  // x = K Q': two chains of products side by side, each operand read from LDS a step before it is used
  __device__ __forceinline__ void products(const KeyTile<T, D> &b) {
    const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
    // row c of a first product is key 16 (c / 4 % 2) + 4 (c / 8) + c % 4 of its 32
    const int key_row = ((c >> 2) & 1) * 16 + (c >> 3) * 4 + (c & 3);
    const auto keys = [&](int g, int i) { return *reinterpret_cast<const Vec *>(&b.k[g * 32 + key_row][i * 16 + h * 8]); };
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[g][i] = 0.f;
    Vec kf[2][2];
#pragma unroll
    for (int g = 0; g < 2; ++g) kf[0][g] = keys(g, 0);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      if (i + 1 < D / 16)
#pragma unroll
        for (int g = 0; g < 2; ++g) kf[(i + 1) & 1][g] = keys(g, i + 1);
#pragma unroll
      for (int g = 0; g < 2; ++g) x[g] = mfma32(kf[i & 1][g], q[i], x[g]);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
  }

  // The logits relative to the reference; `masked`: some row does not see all of the tile
  __device__ __forceinline__ void logits(const KeyTile<T, D> &b, int base, bool masked) {
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const float cc = b.c[g * 2 + h], shift = b.lv[g * 2 + h] - ref;
#pragma unroll
      for (int i = 0; i < 16; ++i) x[g][i] = fmaf(x[g][i], cc, shift);
    }
    if (masked) {
      rarely();
      const Span s{sees.from - base - h * 16, sees.count};
#pragma unroll
      for (int g = 0; g < 2; ++g)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[g][i] = s.has(g * 32 + i) ? x[g][i] : kNegInf();
    }
  }

  // w = 2^logits of 32 keys, and their sum
  template <int g>
  __device__ __forceinline__ float powers() {
    float sum[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float p = exp2_(x[g][i]);
      sum[i & 1] = i < 2 ? p : sum[i & 1] + p;
      w[g][i >> 3][i & 7] = (f16)p;
    }
    return sum[0] + sum[1];
  }

  // The weights and their part of l.  Their largest lies between a 16th of their sum and their sum, so while that is
  // neither large nor small the reference holds and the logits' maximum need not be known.
  template <int g>
  __device__ __forceinline__ void weights(const KeyTile<T, D> &b) {
    float sum = powers<g>();
    if (__any(__float_as_uint(sum) - kLeastSum >= sums_kept) && __any(sum > 0.f || sums_kept == 0)) {
      rarely();
      float top = x[g][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, x[g][i]);
      top = across32(top, max_);
      const float all = across32(l, add_);
      const bool fresh = sums_kept != kSums, up = top > (fresh ? kNegInf() : kHead);
      top = up ? top - kHead : !fresh && top < kLow && top > kNegInf() ? down(top, all) : 0.f;
      const float f = fresh ? 1.f : exp2_(-top);
      ref += top;
      sums_kept = up ? kSums : sums_kept;
      l *= f;
#pragma unroll
      for (int y = g; y < 2; ++y) x[y] -= top;
#pragma unroll
      for (int t = 0; t < D / 32; ++t) o[t] *= f;
      sum = powers<g>();
    }
    l = fmaf(sum, b.iv[g * 2 + ((threadIdx.x & 63) >> 5)], l);
  }

  // A NaN among the values goes to the rows that see it; `look` as for Stage::clean_values
  template <int W>
  __device__ __forceinline__ void nans(const ValueTile<D, W> &b, int base, bool look) {
    const int h = (threadIdx.x & 63) >> 5;
    if (look) {
      rarely();
      int nans = 0;
#pragma unroll
      for (int i = 0; i < W; ++i) nans |= b.nans[i];
      if (__any(nans)) {
        unsigned long long seen = 0;
#pragma unroll 1
        for (int key = 0; key < kUnit; ++key) seen |= (unsigned long long)sees.has(base + key) << key;
#pragma unroll
        for (int t = 0; t < D / 32; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int d = t * 32 + (i >> 2) * 8 + h * 4 + (i & 3);
            const unsigned long long nan = *reinterpret_cast<const unsigned long long *>(b.nan[d]);
            o[t][i] = nan & seen ? __builtin_nanf("") : o[t][i];
          }
      }
    }
  }

  // o += V' w over 32 keys: as many chains as there are tiles of 32 dims
  template <int g, int W>
  __device__ __forceinline__ void sums(const ValueTile<D, W> &b) {
    const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
    constexpr int kT = D / 32;
    const auto values = [&](int j, int t) { return *reinterpret_cast<const h8 *>(&b.v[t * 32 + c][(j >> 1) * 32 + h * 16 + (j & 1) * 8]); };
    h8 vf[2][kT];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < kT; ++t) vf[j][t] = values(2 * g + j, t);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < kT; ++t) o[t] = mfma32(vf[j][t], w[g][j], o[t]);
  }
};

// All requests' row tiles, and the parts that the keys of each are cut into: as many as give two workgroups a compute unit,
// at the next whole number (1,900 tokens of 32 heads over 8 of 128 dims, 480 workgroups, on 8,192: one part 260 us, two
// 294), and above it for 64 dims, where a compute unit holds three (1,900 tokens of 16 heads, 240 workgroups: three parts
// 114 us, two 128).  Single tokens have none, so only the sums on the device tell; less than 2 kGroups workgroups have a part.
struct Tiling {
  int tiles, groups, splits;         // groups: tiles of all key heads
};
template <int D>
__device__ __forceinline__ Tiling tiling(const AttArgs &a, const long long *list) {
  Tiling t;
  t.tiles = same((int)min(list[a.R], (long long)a.tiles_most));
  t.groups = t.tiles * a.H;
  t.splits = t.groups > 0 && t.groups < kGroups ? min((kGroups + (D <= 64 ? t.groups - 1 : t.groups / 2)) / t.groups, a.splits_most) : 1;
  return t;
}

// A workgroup's row tile: which request, head and rows, and the tiles of keys that it goes over.
struct TileWork {
  Request rq;
  int at;                            // row tile
  int splits, part;
  int h, r, rows, row0;
  int pos_lo, pos_hi;                // first and last row's positions
  int begin, end;                    // units
  bool none;

  __device__ __forceinline__ bool look(const AttArgs &a, int unit) const {
    return unit * kUnit + kUnit - 1 > pos_lo || (a.window > 0 && unit * kUnit <= pos_hi - a.window);
  }
};

template <int D, int ROWS>
__device__ __forceinline__ TileWork tile_work(const AttArgs &a, long long *list_) {
  TileWork k{};
  const long long *list = a.plan ? a.plan + a.R + 1 : nullptr;
  if (!list) {
    list_sums(a, [&](int r) { return tiles_of(a, r); }, list_);
    list = list_;
  }
  const Tiling all = tiling<D>(a, list);
  k.splits = all.splits;
  if (a.splits_most > 1 && blockIdx.x == 0 && threadIdx.x == 0) a.joins[0] = make_int4(all.groups, all.splits, 0, 0);
  int i = blockIdx.x;
  if (all.splits > 1) {
    k.part = i / all.groups;
    i -= k.part * all.groups;
  }
  // neighbouring workgroups take different key heads, so that (for 8 heads) the workgroups of one XCD share one
  // head's keys in its L2; a request's last rows, which see most keys, come first
  k.h = i % a.H;
  k.at = all.tiles - 1 - i / a.H;
  k.none = k.at < 0 || k.part >= all.splits;
  if (k.none) return k;
  k.r = find(list, a.R, k.at);
  k.rq = request(a, k.r);
  k.rows = k.rq.n * a.G;
  k.row0 = (k.at - (int)same(list[k.r])) * ROWS;
  const int before = k.rq.length - k.rq.n;
  k.pos_lo = before + k.row0 / a.G;
  k.pos_hi = before + (min(k.row0 + ROWS, k.rows) - 1) / a.G;
  if (k.splits > 1 && k.part == 0 && k.h == 0 && threadIdx.x == 0)
    a.joins[1 + k.at] = make_int4(k.rq.first, k.row0, k.rows, 0);
  const int u = a.window > 0 ? max(k.pos_lo - a.window + 1, 0) / kUnit : 0;
  const int n = k.pos_hi < 0 ? 0 : max(cdiv(k.pos_hi + 1, kUnit) - u, 0);
  k.begin = u + (int)((long long)n * k.part / k.splits);
  k.end = u + (int)((long long)n * (k.part + 1) / k.splits);
  return k;
}

// One wave's rows: where they stand, their queries, and where their results go.
template <typename T, int D, int ROWS>
struct TileWave {
  int i, t, pos_min, pos_max;
  bool in, live;

  __device__ __forceinline__ void begin(const AttArgs &a, const TileWork &k, TileRows<T, D> &st) {
    const int lane = threadIdx.x & 63, wave0 = k.row0 + same((int)threadIdx.x >> 6) * 32, before = k.rq.length - k.rq.n;
    i = wave0 + (lane & 31);
    t = i / a.G;
    in = i < k.rows;
    live = wave0 < k.rows;
    pos_min = before + wave0 / a.G;
    pos_max = before + (min(wave0 + 32, k.rows) - 1) / a.G;
    st.sees = span(a, in ? before + t : -1);
    st.ref = st.l = 0.f;
    st.sums_kept = st.sees.count > 0 ? 0u : ~0u;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int y = 0; y < 16; ++y) st.o[d][y] = 0.f;
    const T *q = static_cast<const T *>(a.q) + (int64_t)(k.rq.first + (in ? t : 0)) * a.q_token +
                 (int64_t)(k.h * a.G + (in ? i - t * a.G : 0)) * a.q_head;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      u4 raw = *reinterpret_cast<const u4 *>(q + s * 16 + (lane >> 5) * 8);
      if (!in) raw = u4{0u, 0u, 0u, 0u};
      st.q[s] = __builtin_bit_cast(typename Vec8<T>::type, raw);
    }
  }
  // Some row sees some of the tile; some row does not see all of it.
  __device__ __forceinline__ bool sees(const AttArgs &a, int base) const {
    return live && base <= pos_max && (a.window <= 0 || base + kUnit - 1 > pos_min - a.window);
  }
  __device__ __forceinline__ bool masked(const AttArgs &a, int base) const {
    return base + kUnit - 1 > pos_min || (a.window > 0 && base <= pos_max - a.window);
  }
  __device__ __forceinline__ void end(const AttArgs &a, const TileWork &k, TileRows<T, D> &st) const {
    const int half = (threadIdx.x & 63) >> 5;
    st.l = across32(st.l, add_);
    const float m = st.sums_kept == kSums ? st.ref : kNegInf();
    if (!in) return;
    if (k.splits > 1) {
      const size_t p = ((size_t)(k.at * a.H + k.h) * k.splits + k.part) * ROWS + i - k.row0;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          *reinterpret_cast<f4 *>(a.part_o + p * D + d * 32 + y * 8 + half * 4) =
              f4{st.o[d][y * 4], st.o[d][y * 4 + 1], st.o[d][y * 4 + 2], st.o[d][y * 4 + 3]};
      if (half == 0) {
        a.part_ml[p * 2] = m;
        a.part_ml[p * 2 + 1] = st.l;
      }
      return;
    }
    const int head = k.h * a.G + i - t * a.G;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int y = 0; y < 4; ++y)
        Rows<T, D, 1>::finish(a, k.rq.first + t, head, d * 32 + y * 8 + half * 4, m, st.l,
                              f4{st.o[d][y * 4], st.o[d][y * 4 + 1], st.o[d][y * 4 + 2], st.o[d][y * 4 + 3]});
  }
};

// A barrier for what lies in LDS alone: loads from memory stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Each tile is staged while the one before is worked on.
template <typename T, int D, int W>
__global__ void __launch_bounds__(64 * W, D <= 64 && W == 4 ? 3 : D <= 128 ? 2 : 1) k_tiles(AttArgs a) {
  constexpr int ROWS = 32 * W;
  __shared__ KeyTile<T, D> keys[2];
  __shared__ ValueTile<D, W> values[2];
  __shared__ long long list_[kListed + 1];
  const TileWork k = tile_work<D, ROWS>(a, list_);
  if (k.none) return;
  TileRows<T, D> st;
  TileWave<T, D, ROWS> wave;
  wave.begin(a, k, st);
  const int32_t *table = a.table + (size_t)k.r * a.MB;
  Stage<T, D, W> g;
  const auto blocks = [&](int u) { g.blocks(a, table, u * kUnit); };
  const auto load = [&](int u) {
    g.load_keys(a, k.h, u * kUnit);
    g.load_values(a, u * kUnit);
  };
  const auto store = [&](int u) {
    g.put_keys(keys[u & 1]);
    g.put_scales(a, keys[u & 1]);
    if (k.look(a, u)) {
      rarely();
      g.clean_values(k.rq.length - u * kUnit, values[u & 1]);
    }
    g.put_values(values[u & 1]);
  };
  if (k.begin < k.end) {
    g.begin(a, k.h);
    blocks(k.begin);
    load(k.begin);
    blocks(k.begin + 1);
    store(k.begin);
  }
  lds_barrier();
  for (int u = k.begin; u < k.end; ++u) {
    const int base = u * kUnit;
    if (u + 1 < k.end) {
      load(u + 1);
      blocks(u + 2);
    }
    if (wave.sees(a, base)) {
      st.products(keys[u & 1]);
      st.logits(keys[u & 1], base, wave.masked(a, base));
      st.nans(values[u & 1], base, k.look(a, u));
      st.template weights<0>(keys[u & 1]);
      st.template sums<0>(values[u & 1]);
      st.template weights<1>(keys[u & 1]);
      st.template sums<1>(values[u & 1]);
    }
    if (u + 1 < k.end) store(u + 1);
    lds_barrier();
  }
  wave.end(a, k, st);
}

// A wave a row, in turn; nothing where the keys were not cut.
template <typename T, int D>
__global__ void __launch_bounds__(kBlock) k_tiles_join(AttArgs a) {
  const int4 all = a.joins[0];
  const int groups = all.x, splits = all.y;
  if (splits == 1) return;
  for (int i = blockIdx.x * kWaves + (threadIdx.x >> 6); i < groups * a.tile_rows; i += gridDim.x * kWaves) {
    const int group = i / a.tile_rows, row = i - group * a.tile_rows;
    const int4 tile = a.joins[1 + group / a.H];
    const int y = tile.y + row, t = y / a.G;
    if (y >= tile.z) continue;
    const size_t p = (size_t)group * splits * a.tile_rows + row;
    join_row<T, D>(a, p, p + a.tile_rows, a.tile_rows, splits, tile.x + t, group % a.H * a.G + y - t * a.G);
  }
}

// ------------------------------------------------------------------ host

struct Shape {
  int nt;                            // k_rows' row tiles of 16, 0: k_rows does not run
  int rows_max;
  bool cut, tiles;                   // k_rows with pieces; k_tiles runs
  int tiles_each;
  int tile_rows;
  long long tiles_most;              // bound of the row tiles of all requests
  int splits_most;                   // and of the parts of one's keys
  long long tile_groups, join_groups;   // workgroups of k_tiles, of k_tiles_join
  int join_rows;                     // rows of a row tile that are mostly in use: the join's waves
  size_t plan, cuts, joins, part_ml, part_o, bytes;
};

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

// Row tiles that k_rows keeps in registers, nothing spilled to memory.
constexpr int row_tiles_most(int D) { return D <= 96 ? 4 : D <= 128 ? 2 : 1; }

festina_status shape_of(const festina_kv_cache *c, const festina_attention *t, Shape *s) {
  const festina_status bad = check_cache(c);
  if (bad != FESTINA_OK) return bad;
  if (!t || t->n_requests < 0 || t->max_blocks < 1 || t->n_tokens < 0 || t->n_heads < 1 || t->max_new < 1 || t->window < 0)
    return FESTINA_ERR_INVALID;
  if (t->n_heads % c->n_kv_heads) return FESTINA_ERR_INVALID;
  if (t->dtype != FESTINA_BF16 && t->dtype != FESTINA_F16) return FESTINA_ERR_UNSUPPORTED;
  if ((long long)t->max_blocks * c->block_tokens > INT_MAX / 2 || (long long)t->n_tokens * t->n_heads > INT_MAX / 2 ||
      t->n_requests > kMaxRequests || t->n_heads > 65536)
    return FESTINA_ERR_UNSUPPORTED;
  const int G = t->n_heads / c->n_kv_heads, H = c->n_kv_heads, D = c->head_dim;
  const long long most = (long long)t->max_new * G;                   // rows of one request and key head
  const int nt_most = row_tiles_most(D);
  *s = Shape{};
  s->tiles = most > 16 * nt_most && t->max_new > 1;
  const long long rows = s->tiles ? G : most;                         // with prompts about: the single tokens' rows
  s->nt = rows <= 16 ? 1 : min(rows <= 32 ? 2 : 4, nt_most);
  s->join_rows = (int)min(rows, 16ll * s->nt);
  if (s->tiles && G > 16 * nt_most) s->nt = 0;
  s->rows_max = s->tiles ? 16 * s->nt : INT_MAX;
  const long long keys = (long long)t->max_blocks * c->block_tokens;
  s->tiles_each = (int)((rows + 16 * s->nt - 1) / max(16 * s->nt, 1));
  s->cut = keys > 2 * kWaves * kUnit;
  if (s->nt && !s->cut && (long long)t->n_requests * H * s->tiles_each > kThreadsMost / kBlock)
    return FESTINA_ERR_UNSUPPORTED;
  size_t parts = 0;
  if (s->nt && s->cut) parts = (size_t)2 * workers_of(D, s->nt) * 16 * s->nt;
  if (s->tiles) {
    // 256 rows a workgroup stage each tile half as often for a row, where registers allow and enough workgroups are
    // left: a prompt of 8,192 tokens (32 heads over 8 of 128 dims) 641 us against 662 with 128; 9,012 tokens of 16
    // heads of 64 dims, with three smaller workgroups a compute unit, 183 against 234 the other way
    const long long rows_all = (long long)t->n_tokens * G * H;
    s->tile_rows = (D == 96 || D == 128) && rows_all >= 256ll * kGroups ? 256 : 128;
    // whole row tiles, and one more a request that has more than rows_max rows, of which there are no more than tokens allow
    const long long few = s->rows_max / G, requests = min((long long)t->n_requests, t->n_tokens / (few + 1));
    s->tiles_most = max((long long)t->n_tokens * G / s->tile_rows + requests, 1ll);
    if (s->tiles_most * H > kThreadsMost / (2 * s->tile_rows)) return FESTINA_ERR_UNSUPPORTED;
    // parts of at least 16 steps each; none where, with every request but the prompts' having as many tokens as it may,
    // prompts still fill the chip (tokens of no request would only leave them in one part)
    const long long sure = ((long long)t->n_tokens - t->n_requests * few) * G / s->tile_rows * H;
    s->splits_most = sure >= kGroups ? 1 : (int)max(min(keys / (16 * kUnit), (long long)kGroups), 1ll);
    s->tile_groups = s->tiles_most * H;
    if (s->splits_most > 1) {
      const long long groups = s->tile_groups;
      const size_t pieces = (size_t)min(groups * s->splits_most, kGroups + min(groups, (long long)kGroups));
      s->join_groups = min(min(groups, (long long)kGroups) * s->tile_rows / kWaves, (long long)kJoins);
      s->tile_groups = max(groups, (long long)pieces);
      parts = max(parts, pieces * s->tile_rows);
    }
  }
  s->plan = 0;
  s->cuts = up((size_t)2 * (t->n_requests + 1) * 8);
  s->joins = s->cuts + up((size_t)workers_of(D, max(s->nt, 1)) * sizeof(Cut));
  s->part_ml = s->joins + up((kGroups + 1) * sizeof(int4));
  s->part_o = s->part_ml + up(parts * 8);
  s->bytes = s->part_o + up(parts * D * 4);
  return FESTINA_OK;
}

template <typename T, int D, int NT>
void run_rows(AttArgs a, const Shape &s, hipStream_t st) {
  a.workers = workers_of(D, NT);
  if (!s.cut) {
    k_rows_whole<T, D, NT><<<(unsigned)(a.R * a.H * s.tiles_each), kBlock, 0, st>>>(a);
    return;
  }
  k_rows<T, D, NT><<<a.workers, 64, 0, st>>>(a);
  k_rows_join<T, D, NT><<<dim3(a.workers - 1, (s.join_rows + kWaves - 1) / kWaves), kBlock, 0, st>>>(a);
}

template <typename T, int D>
void run(AttArgs a, const Shape &s, long long *plan, hipStream_t st) {
  if (a.R > kListed) {
    if (s.nt == 1) k_plan<16><<<1, 1024, 0, st>>>(a, plan);
    else if (s.nt == 2) k_plan<32><<<1, 1024, 0, st>>>(a, plan);
    else k_plan<64><<<1, 1024, 0, st>>>(a, plan);
    a.plan = plan;
  }
  if (s.nt == 1) run_rows<T, D, 1>(a, s, st);
  if constexpr (row_tiles_most(D) >= 2)
    if (s.nt == 2) run_rows<T, D, 2>(a, s, st);
  if constexpr (row_tiles_most(D) >= 4)
    if (s.nt == 4) run_rows<T, D, 4>(a, s, st);
  if (s.tiles) {
    const unsigned grid = (unsigned)s.tile_groups;
    if constexpr (D == 96 || D == 128)
      if (s.tile_rows == 256) k_tiles<T, D, 8><<<grid, 512, 0, st>>>(a);
    if (s.tile_rows == 128) k_tiles<T, D, 4><<<grid, kBlock, 0, st>>>(a);
    if (s.splits_most > 1)
      k_tiles_join<T, D><<<(unsigned)s.join_groups, kBlock, 0, st>>>(a);
  }
}

template <typename T>
void run_dim(const AttArgs &a, const Shape &s, int D, long long *plan, hipStream_t st) {
  switch (D) {
    case 64: run<T, 64>(a, s, plan, st); break;
    case 96: run<T, 96>(a, s, plan, st); break;
    case 128: run<T, 128>(a, s, plan, st); break;
    default: run<T, 256>(a, s, plan, st); break;
  }
}

}  // namespace

extern "C" size_t festina_attend_workspace_bytes(const festina_kv_cache *cache, const festina_attention *att) {
  Shape s;
  return shape_of(cache, att, &s) == FESTINA_OK ? s.bytes : 0;
}

extern "C" festina_status festina_attend(const festina_kv_cache *cache, const festina_attention *att, void *workspace,
                                         size_t workspace_bytes, void *stream) {
  Shape s;
  const festina_status bad = shape_of(cache, att, &s);
  if (bad != FESTINA_OK) return bad;
  if (att->n_requests == 0 || att->n_tokens == 0) return FESTINA_OK;
  if (!att->block_table || !att->length || !att->first || !att->q || !att->out) return FESTINA_ERR_INVALID;
  if (att->q_token_stride < 0 || att->q_head_stride < 0 || att->out_token_stride < 0 || att->out_head_stride < 0 ||
      !(att->scale == att->scale))
    return FESTINA_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(att->q) | reinterpret_cast<uintptr_t>(att->out)) & 15) return FESTINA_ERR_INVALID;
  if ((att->q_token_stride | att->q_head_stride | att->out_token_stride | att->out_head_stride) & 7)
    return FESTINA_ERR_INVALID;
  if (!workspace || workspace_bytes < s.bytes || (reinterpret_cast<uintptr_t>(workspace) & 255)) return FESTINA_ERR_INVALID;
  char *w = static_cast<char *>(workspace);
  AttArgs a{};
  a.R = att->n_requests;
  a.MB = att->max_blocks;
  a.T = att->n_tokens;
  a.Hq = att->n_heads;
  a.H = cache->n_kv_heads;
  a.G = a.Hq / a.H;
  a.shift = __builtin_ctz((unsigned)cache->block_tokens);
  a.NB = cache->n_blocks;
  a.window = att->window;
  a.rows_max = s.rows_max;
  a.tiles_each = s.tiles_each;
  a.tiles_most = (int)s.tiles_most;
  a.splits_most = s.splits_most;
  a.tile_rows = s.tile_rows;
  a.scale = att->scale * 1.44269504088896341f;
  a.table = att->block_table;
  a.length = att->length;
  a.first = att->first;
  a.q = att->q;
  a.q_token = att->q_token_stride;
  a.q_head = att->q_head_stride;
  a.out = att->out;
  a.out_token = att->out_token_stride;
  a.out_head = att->out_head_stride;
  a.lse = att->lse;
  a.k = cache->k;
  a.v = cache->v;
  a.ks = cache->k_scale;
  a.vs = cache->v_scale;
  a.cuts = reinterpret_cast<Cut *>(w + s.cuts);
  a.joins = reinterpret_cast<int4 *>(w + s.joins);
  a.part_ml = reinterpret_cast<float *>(w + s.part_ml);
  a.part_o = reinterpret_cast<float *>(w + s.part_o);
  long long *plan = reinterpret_cast<long long *>(w + s.plan);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (att->dtype == FESTINA_BF16) run_dim<bf16>(a, s, cache->head_dim, plan, st);
  else run_dim<f16>(a, s, cache->head_dim, plan, st);
  return hipGetLastError() == hipSuccess ? FESTINA_OK : FESTINA_ERR_DEVICE;
}
