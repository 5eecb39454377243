// cache.hip -- MI355X (gfx950) kernel and C-ABI host dispatch of the write into the 8-bit key/value cache.
//
// k_store  a workgroup takes the runs (stretches of tokens in one block) that begin among its tokens, for one key
//   head and either the keys or the values.  For each run: the largest finite magnitude over the run's
//   elements (which stay in registers), the block's scale from it, where that grew the older codes anew, then
//   the new codes.
//   Keys are stored as they come ([token][dim]); values pass through LDS, 64 slots at a time, and leave with
//   their tokens running fastest, 16 tokens of a row in one 16-byte store.
//
// Scales are powers of two, so x / scale and the change from one scale to another are exact and each code
// is one rounding of its element (v_cvt_pk_fp8_f32: to nearest, ties to even), in whatever portions
// the tokens arrive; a block's scale grows a few times in its life rather than with every new maximum.
// Bound by the bytes it moves on prompts (32 prompts, 41,100 tokens of 8 heads of 128 in bfloat16: 253 MB in 54 us, 4.7 TB/s;
// a large copy 4.96) and by latency on a step of single tokens (32 tokens: 7 us).
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "festina.h"
#include "kv.h"

namespace {

using namespace festina_kv;

// A run has a workgroup of N threads: the fewest, of 64, 128 and 256, whose registers hold a block's rows of one head in at most
// four pieces of eight elements a thread, else 256; slots_of() rows are held, and pass through the values' transpose, at a
// time.  More threads have little to load each and a barrier to wait for, and more pieces leave too few waves on a SIMD.  32 prompts,
// 41,100 tokens of 8 heads of 128, us: blocks of 16 slots 61 (256 threads: 122), of 32 59 (78); 16,900 tokens of 12 heads
// of 64, blocks of 32 27 (40); 16,900 of 12 heads of 256, blocks of 128 136 (161 with eight pieces a thread).  512 threads
// were slower (256 dims, blocks of 64: 137 against 100), and so were reads that mark the elements as
// not to be kept (12 heads of 64: 32 against 28).
constexpr int slots_of(int D, int N) { return N * 32 / D >= 64 ? 64 : N * 32 / D / 16 * 16; }
constexpr int kSpanMost = 64;

typedef float f2 __attribute__((ext_vector_type(2)));

struct StoreArgs {
  int32_t T, H, shift, slots;        // tokens, key heads, log2 of the block's tokens, NB * BT
  int32_t span;                      // tokens a workgroup looks for runs in
  const void *x[2];                  // keys, values
  int64_t token_stride[2], head_stride[2];
  bool vec[2];                       // rows of 8 elements are 16-byte aligned
  const int32_t *slot;
  uint8_t *codes[2];
  float *scale[2];
};

__device__ __forceinline__ bool finite(float x) { return __builtin_fabsf(x) < __builtin_inff(); }

// Four codes; `inv` is the scale's reciprocal, a power of two.  Elements of at most 448 times the scale need nothing
// else (the conversion keeps NaN); `careful` where some may be larger or infinite.
__device__ __forceinline__ unsigned encode4(const float *x, float inv, bool careful) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = x[i] * inv;
  if (careful) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = finite(x[i]) ? fminf(fmaxf(y[i], -448.f), 448.f) : __builtin_nanf("");
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  return (unsigned)w;
}

// Four older codes under a scale that is 1 / ratio times larger (exact products, one rounding).
__device__ __forceinline__ unsigned recode4(unsigned c, float ratio) {
  const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a.x * ratio, a.y * ratio, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(b.x * ratio, b.y * ratio, w, true);
  return (unsigned)w;
}

// The least power of two s with amax <= 448 s = 1.75 * 2^8 s, from amax's bits: a fraction above 1.75 carries
// into the exponent.
__device__ __forceinline__ float scale_of(float amax) {
  const int e = (int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - 8;
  return fminf(fmaxf(__uint_as_float((unsigned)max(e, 1) << 23), kScaleMin), kScaleMax);
}

// Eight elements as they were read.
template <int TYPE>
struct Raw8 {
  uint4 w[TYPE == FESTINA_F32 ? 2 : 1];
};

template <int TYPE>
__device__ __forceinline__ Raw8<TYPE> read8(const void *base, int64_t at, bool vec) {
  Raw8<TYPE> r;
  if constexpr (TYPE == FESTINA_F32) {
    const float *p = static_cast<const float *>(base) + at;
    if (vec) {
      r.w[0] = reinterpret_cast<const uint4 *>(p)[0];
      r.w[1] = reinterpret_cast<const uint4 *>(p)[1];
    } else {
      unsigned u[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(p[i]);
      r.w[0] = make_uint4(u[0], u[1], u[2], u[3]);
      r.w[1] = make_uint4(u[4], u[5], u[6], u[7]);
    }
  } else {
    const uint16_t *p = static_cast<const uint16_t *>(base) + at;
    if (vec) {
      r.w[0] = *reinterpret_cast<const uint4 *>(p);
    } else {
      unsigned u[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = p[2 * i] | (unsigned)p[2 * i + 1] << 16;
      r.w[0] = make_uint4(u[0], u[1], u[2], u[3]);
    }
  }
  return r;
}

template <int TYPE>
__device__ __forceinline__ void values8(const Raw8<TYPE> &r, float (&x)[8]) {
  if constexpr (TYPE == FESTINA_F32) {
    const unsigned u[8] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w, r.w[1].x, r.w[1].y, r.w[1].z, r.w[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(u[i]);
  } else {
    const unsigned u[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (TYPE == FESTINA_BF16) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
      } else {
        x[2 * i] = (float)__builtin_bit_cast(_Float16, (uint16_t)u[i]);
        x[2 * i + 1] = (float)__builtin_bit_cast(_Float16, (uint16_t)(u[i] >> 16));
      }
    }
  }
}

// One run, for keys (WHICH = 0) or values.  The elements of its first kSlots tokens stay in registers between the
// maximum and the codes; a longer run's others are read again.
template <int TYPE, int D, int N, int WHICH>
__device__ __forceinline__ void store_run(const StoreArgs &a, int h, int t, int n, int slot, float *lds_max, uint8_t *tile) {
  constexpr int kSlots = slots_of(D, N), kVecs = D / 8, kPitch = D + 4, kKept = kSlots * kVecs / N;
  const int bt = 1 << a.shift, off = slot & (bt - 1);
  const size_t bh = (size_t)(slot >> a.shift) * a.H + h;
  const int64_t ts = a.token_stride[WHICH], row0 = (int64_t)h * a.head_stride[WHICH] + (int64_t)t * ts;
  const void *x = a.x[WHICH];
  const bool vec = a.vec[WHICH];
  uint8_t *codes = a.codes[WHICH] + bh * D * bt;
  const float old = a.scale[WHICH][bh];
  const auto read = [&](int i) { return read8<TYPE>(x, row0 + (int64_t)(i / kVecs) * ts + (i % kVecs) * 8, vec); };
  Raw8<TYPE> kept[kKept];
  float v[8], amax = 0.f;
#pragma unroll
  for (int j = 0; j < kKept; ++j)
    if ((int)threadIdx.x + j * N < n * kVecs) kept[j] = read(threadIdx.x + j * N);
  const auto join = [&]() {                            // over the workgroup
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) amax = fmaxf(amax, __shfl_xor(amax, d));
    if ((threadIdx.x & 63) == 0) lds_max[threadIdx.x >> 6] = amax;
    __syncthreads();
    amax = lds_max[0];
#pragma unroll
    for (int w = 1; w < N / 64; ++w) amax = fmaxf(amax, lds_max[w]);
  };
  // the maximum leaves NaN out by itself
#pragma unroll
  for (int j = 0; j < kKept; ++j)
    if ((int)threadIdx.x + j * N < n * kVecs) {
      values8<TYPE>(kept[j], v);
#pragma unroll
      for (int k = 0; k < 8; ++k) amax = fmaxf(amax, __builtin_fabsf(v[k]));
    }
  for (int i = threadIdx.x + kKept * N; i < n * kVecs; i += N) {
    values8<TYPE>(read(i), v);
#pragma unroll
    for (int k = 0; k < 8; ++k) amax = fmaxf(amax, __builtin_fabsf(v[k]));
  }
  join();
  bool careful = !finite(amax);
  if (careful) {                                       // infinities: once more without them
    __syncthreads();
    amax = 0.f;
    for (int i = threadIdx.x; i < n * kVecs; i += N) {
      values8<TYPE>(read(i), v);
#pragma unroll
      for (int k = 0; k < 8; ++k) amax = fmaxf(amax, finite(v[k]) ? __builtin_fabsf(v[k]) : 0.f);
    }
    join();
  }
  float scale = scale_of(amax);
  careful |= scale == kScaleMax;
  if (off > 0) scale = fmaxf(scale, old);
  const float inv = 1.f / scale;                       // exact
  if (threadIdx.x == 0) a.scale[WHICH][bh] = scale;
  if (off > 0 && scale > old) {
    const float ratio = old / scale;
    if (WHICH == 0) {
      uint4 *p = reinterpret_cast<uint4 *>(codes);
      for (int i = threadIdx.x; i < off * D / 16; i += N) {
        uint4 c = p[i];
        c.x = recode4(c.x, ratio), c.y = recode4(c.y, ratio), c.z = recode4(c.z, ratio), c.w = recode4(c.w, ratio);
        p[i] = c;
      }
    } else {
      const int words = (off + 3) / 4;
      for (int i = threadIdx.x; i < D * words; i += N) {
        const int d = i / words, o = (i - d * words) * 4;
        uint8_t *p = codes + (size_t)d * bt + o;
        const unsigned c = recode4(*reinterpret_cast<const unsigned *>(p), ratio);
        if (o + 4 <= off) {
          *reinterpret_cast<unsigned *>(p) = c;
        } else {                                       // the run's first slots share this word
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (o + j < off) p[j] = (uint8_t)(c >> (8 * j));
        }
      }
    }
  }
  if (WHICH == 0) {
    const auto put = [&](int i) {
      *reinterpret_cast<uint2 *>(codes + (size_t)off * D + (size_t)i * 8) = make_uint2(encode4(v, inv, careful), encode4(v + 4, inv, careful));
    };
#pragma unroll
    for (int j = 0; j < kKept; ++j)
      if ((int)threadIdx.x + j * N < n * kVecs) {
        values8<TYPE>(kept[j], v);
        put(threadIdx.x + j * N);
      }
    for (int i = threadIdx.x + kKept * N; i < n * kVecs; i += N) {
      values8<TYPE>(read(i), v);
      put(i);
    }
    __syncthreads();                                   // lds_max serves the next run
    return;
  }
  for (int s0 = off & ~(kSlots - 1); s0 < off + n; s0 += kSlots) {     // slots s0 .. s0 + kSlots - 1 of the block
    const int lo = max(off, s0), hi = min(off + n, s0 + kSlots);
    const int i0 = (lo - off) * kVecs, i1 = (hi - off) * kVecs;        // the run's elements among them
    const auto put = [&](int i) {
      unsigned *p = reinterpret_cast<unsigned *>(tile + (off + i / kVecs - s0) * kPitch + (i % kVecs) * 8);
      p[0] = encode4(v, inv, careful);
      p[1] = encode4(v + 4, inv, careful);
    };
#pragma unroll
    for (int j = 0; j < kKept; ++j) {
      const int i = threadIdx.x + j * N;
      if (i >= i0 && i < i1) {
        values8<TYPE>(kept[j], v);
        put(i);
      }
    }
    for (int i = max(i0, kKept * N) + threadIdx.x; i < i1; i += N) {
      values8<TYPE>(read(i), v);
      put(i);
    }
    __syncthreads();
    constexpr int kSixteens = kSlots / 16;
    for (int i = threadIdx.x; i < D / 4 * kSixteens; i += N) {         // groups of four rows x groups of 16 slots
      const int g = i % kSixteens, d = i / kSixteens * 4, s = s0 + g * 16;
      if (s >= hi || s + 16 <= lo) continue;
      unsigned w[4][4];                                                // [row][word of four slots]
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        unsigned c[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) c[q] = *reinterpret_cast<const unsigned *>(tile + (g * 16 + j * 4 + q) * kPitch + d);
        const unsigned x0 = __builtin_amdgcn_perm(c[1], c[0], 0x05010400), x1 = __builtin_amdgcn_perm(c[1], c[0], 0x07030602);
        const unsigned y0 = __builtin_amdgcn_perm(c[3], c[2], 0x05010400), y1 = __builtin_amdgcn_perm(c[3], c[2], 0x07030602);
        w[0][j] = __builtin_amdgcn_perm(y0, x0, 0x05040100);
        w[1][j] = __builtin_amdgcn_perm(y0, x0, 0x07060302);
        w[2][j] = __builtin_amdgcn_perm(y1, x1, 0x05040100);
        w[3][j] = __builtin_amdgcn_perm(y1, x1, 0x07060302);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        uint8_t *p = codes + (size_t)(d + r) * bt + s;
        if (s >= lo && s + 16 <= hi) {
          *reinterpret_cast<uint4 *>(p) = make_uint4(w[r][0], w[r][1], w[r][2], w[r][3]);
        } else {
#pragma unroll
          for (int o = 0; o < 16; ++o)
            if (s + o >= lo && s + o < hi) p[o] = (uint8_t)(w[r][o >> 2] >> (8 * (o & 3)));
        }
      }
    }
    __syncthreads();
  }
}

template <int TYPE, int D, int N>
__global__ void __launch_bounds__(N) k_store(StoreArgs a) {
  __shared__ float lds_max[N / 64];
  __shared__ __attribute__((aligned(16))) uint8_t tile[slots_of(D, N) * (D + 4)];
  // heads vary fastest: a token's heads lie beside each other in what is read
  const int h = blockIdx.x % a.H, which = blockIdx.y, bt = 1 << a.shift, lane = threadIdx.x & 63;
  const int64_t t0 = (int64_t)(blockIdx.x / a.H) * a.span;
  // the first tokens of runs among this workgroup's: every wave finds them all
  const int64_t tl = t0 + lane;
  int mine = -1, prior = -2;
  if (lane < a.span && tl < a.T) {
    mine = a.slot[tl];
    if (tl > 0) prior = a.slot[tl - 1];
  }
  unsigned long long begins =
      __ballot((unsigned)mine < (unsigned)a.slots && ((mine & (bt - 1)) == 0 || prior != mine - 1));
  while (begins) {
    const int b = __builtin_ctzll(begins);
    begins &= begins - 1;
    const int slot = __builtin_amdgcn_readlane(mine, b), t = (int)t0 + b;
    const int most = min(bt - (slot & (bt - 1)), a.T - t);
    int n = 0;
    for (;;) {                                         // the run ends at the first slot that does not follow
      const int k = n + lane;
      const unsigned long long follows = __ballot(k < most && a.slot[min(t + k, a.T - 1)] == slot + k);
      n += follows == ~0ull ? 64 : __builtin_ctzll(~follows);
      if (follows != ~0ull) break;
    }
    if (which == 0) store_run<TYPE, D, N, 0>(a, h, t, n, slot, lds_max, tile);
    else store_run<TYPE, D, N, 1>(a, h, t, n, slot, lds_max, tile);
  }
}

template <int TYPE, int D>
void launch(const StoreArgs &a, dim3 grid, hipStream_t st) {
  constexpr int kLeast = D < 256 ? 64 : 128;           // of threads, for blocks of 16
  const int bt = 1 << a.shift;
  if (bt <= slots_of(D, kLeast)) k_store<TYPE, D, kLeast><<<grid, kLeast, 0, st>>>(a);
  else if (D > 64 && D < 256 && bt <= slots_of(D, 2 * kLeast)) k_store<TYPE, D, 2 * kLeast><<<grid, 2 * kLeast, 0, st>>>(a);
  else k_store<TYPE, D, D == 64 ? 128 : 256><<<grid, D == 64 ? 128 : 256, 0, st>>>(a);
}
template <int TYPE>
void launch(const StoreArgs &a, int D, dim3 grid, hipStream_t st) {
  switch (D) {
    case 64: launch<TYPE, 64>(a, grid, st); break;
    case 96: launch<TYPE, 96>(a, grid, st); break;
    case 128: launch<TYPE, 128>(a, grid, st); break;
    default: launch<TYPE, 256>(a, grid, st); break;
  }
}

}  // namespace

extern "C" festina_status festina_store_kv(const festina_kv_cache *cache, const festina_kv_tokens *tokens,
                                           void *stream) {
  const festina_status bad = check_cache(cache);
  if (bad != FESTINA_OK) return bad;
  if (!tokens || tokens->n_tokens < 0) return FESTINA_ERR_INVALID;
  if (tokens->dtype != FESTINA_BF16 && tokens->dtype != FESTINA_F16 && tokens->dtype != FESTINA_F32)
    return FESTINA_ERR_INVALID;
  if (tokens->k_token_stride < 0 || tokens->k_head_stride < 0 || tokens->v_token_stride < 0 || tokens->v_head_stride < 0)
    return FESTINA_ERR_INVALID;
  if (tokens->n_tokens == 0) return FESTINA_OK;
  if (!tokens->k || !tokens->v || !tokens->slot) return FESTINA_ERR_INVALID;
  const int size = tokens->dtype == FESTINA_F32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(tokens->k) | reinterpret_cast<uintptr_t>(tokens->v)) % size) return FESTINA_ERR_INVALID;
  StoreArgs a;
  a.T = tokens->n_tokens;
  a.H = cache->n_kv_heads;
  a.shift = __builtin_ctz((unsigned)cache->block_tokens);
  a.slots = cache->n_blocks * cache->block_tokens;
  a.x[0] = tokens->k;
  a.x[1] = tokens->v;
  a.token_stride[0] = tokens->k_token_stride;
  a.token_stride[1] = tokens->v_token_stride;
  a.head_stride[0] = tokens->k_head_stride;
  a.head_stride[1] = tokens->v_head_stride;
  for (int i = 0; i < 2; ++i)
    a.vec[i] = ((reinterpret_cast<uintptr_t>(a.x[i]) | (uintptr_t)(a.token_stride[i] * size) |
                 (uintptr_t)(a.head_stride[i] * size)) & 15) == 0;
  a.slot = tokens->slot;
  a.codes[0] = cache->k;
  a.codes[1] = cache->v;
  a.scale[0] = cache->k_scale;
  a.scale[1] = cache->v_scale;
  // few tokens: a workgroup each, so that runs of single tokens are not done one after the other; many: enough that
  // most workgroups have a run to store (they are dispatched at a rate that empty ones take their share of)
  a.span = (int)min(max((long long)a.T * a.H / 4096, 1ll), (long long)kSpanMost);
  const long long groups = ((long long)a.T + a.span - 1) / a.span * a.H;
  if (groups > UINT_MAX / 256) return FESTINA_ERR_UNSUPPORTED;   // threads along one axis of a grid
  const dim3 grid((unsigned)groups, 2);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (tokens->dtype == FESTINA_BF16) launch<FESTINA_BF16>(a, cache->head_dim, grid, st);
  else if (tokens->dtype == FESTINA_F16) launch<FESTINA_F16>(a, cache->head_dim, grid, st);
  else launch<FESTINA_F32>(a, cache->head_dim, grid, st);
  return hipGetLastError() == hipSuccess ? FESTINA_OK : FESTINA_ERR_DEVICE;
}
