// rotate.hip -- MI355X (gfx950) kernel and C-ABI host dispatch of a step's queries and keys between their projections and
// the cache: the norm of each head, and the rotation by the token's position, in one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * weight,   (a, b) -> (a cos - b sin, b cos + a sin) for the pairs of rotated elements.
//
// Angles: a frequency is given in turns per position times 2^64, so position * frequency modulo 2^64 is the part of a turn
// that is left, exactly and however far the position; it is rounded once, to float32, and only then turned into a cosine and
// a sine.  (A product of floats would be off by 2^-24 of all the turns made.)
//
// A wave takes a token: a lane makes a cosine and a sine or two, which all heads share through LDS, then each lane holds
// 16 elements of a head, eight of either half (or pairs of neighbours), so that no element crosses lanes, only the sum
// of squares does; neighbouring lanes hold neighbouring 16 bytes.  Bound by the bytes it moves: 41,100 tokens of 32 and 8 heads of
// 128 in bfloat16, 842 MB in 150 us, 5.6 TB/s (a large copy: 4.9); on a step of 256 tokens by latency: 4.9 us.
// (Stores that mark the outputs as not to be kept: 142 us, and float32 heads 77 us against 57.)
#include <hip/hip_runtime.h>

#include <climits>
#include <cstddef>
#include <cstdint>

#include "festina.h"
#include "kv.h"

namespace {

constexpr int kWaves = 4;
constexpr int kAtOnce = 4;           // groups of heads with their loads in flight together

typedef __bf16 bf16;
typedef _Float16 f16;

struct RotateArgs {
  int32_t T, rotated, interleaved, parts;
  int32_t heads[2];                  // queries, keys
  float eps;
  const int32_t *position;
  const unsigned long long *turn;
  const float *weight[2];
  const void *x[2];
  void *y[2];
  int64_t x_token[2], x_head[2], y_token[2], y_head[2];
  bool vec;                          // eight elements are 16-byte aligned everywhere
};

template <int TYPE> struct Element { typedef float type; };
template <> struct Element<FESTINA_BF16> { typedef bf16 type; };
template <> struct Element<FESTINA_F16> { typedef f16 type; };

typedef unsigned u4 __attribute__((ext_vector_type(4)));

// 16 bytes as they lie: eight elements, or four of float32.
template <typename T>
union Piece {
  T x[16 / sizeof(T)];
  u4 w;
};

template <typename T>
__device__ __forceinline__ Piece<T> read(const T *p, bool vec) {
  Piece<T> e;
  if (vec) {
    e.w = *reinterpret_cast<const u4 *>(p);
  } else {
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(T); ++i) e.x[i] = p[i];
  }
  return e;
}
template <typename T>
__device__ __forceinline__ void write(T *p, const float *y, bool vec) {
  Piece<T> e;
#pragma unroll
  for (int i = 0; i < 16 / (int)sizeof(T); ++i) e.x[i] = (T)y[i];
  if (vec) {
    *reinterpret_cast<u4 *>(p) = e.w;
  } else {
#pragma unroll
    for (int i = 0; i < 16 / (int)sizeof(T); ++i) p[i] = e.x[i];
  }
}

template <int TYPE, int D>
__global__ void __launch_bounds__(64 * kWaves) k_rotate(RotateArgs a) {
  typedef typename Element<TYPE>::type T;
  constexpr int kLanes = D == 96 ? 8 : D / 16, kHeads = 64 / kLanes;   // of a head; heads of a wave
  __shared__ __attribute__((aligned(16))) float cosines[kWaves][D / 2], sines[kWaves][D / 2];
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * kWaves + wave;
  if (t >= a.T) return;
  const int l = lane % kLanes, side = lane / kLanes, pairs = a.rotated / 16;
  const bool rotates = l < pairs, in = l < D / 16;
  // element of piece j of the lane's first half (s = 0) or second: neighbouring lanes have neighbouring pieces
  constexpr int kSize = 16 / (int)sizeof(T), kPieces = 8 / kSize;
  const int apart = rotates ? pairs : D / 16 - pairs, base = rotates ? l : in ? a.rotated / kSize + l - pairs : 0;
  const auto element = [&](int s, int j) { return in ? (base + (s * kPieces + j) * apart) * kSize : 0; };
  const long long position = a.position[t];
  for (int i = lane; i < a.rotated / 2; i += 64) {
    // a signed part of a turn: -1/2 .. 1/2
    const float part = (float)(long long)((unsigned long long)position * a.turn[i]) * 0x1p-64f;
    float s, c;
    sincospif(2.f * part, &s, &c);
    cosines[wave][i] = c;
    sines[wave][i] = s;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    // pair i of the lane: elements 2i and 2i + 1 of its 16, or i and i + 8
    const int e = a.interleaved ? 2 * i : i, of = e % 8, first = element(e / 8, of / kSize) + of % kSize;
    const int at = a.interleaved ? first / 2 : first;
    cs[i] = rotates ? cosines[wave][at] : 1.f;
    sn[i] = rotates ? sines[wave][at] : 0.f;
  }
  const int groups0 = (a.heads[0] + kHeads - 1) / kHeads, groups = groups0 + (a.heads[1] + kHeads - 1) / kHeads;
  const int from = (int)((long long)groups * blockIdx.y / a.parts), to = (int)((long long)groups * (blockIdx.y + 1) / a.parts);
#pragma unroll
  for (int k = 0; k < 2; ++k) {                        // queries, then keys
    const int lo = k ? max(from - groups0, 0) : from, hi = k ? to - groups0 : min(to, groups0);
    const float *weight = a.weight[k];
    const T *x = static_cast<const T *>(a.x[k]) + t * a.x_token[k];
    T *y = static_cast<T *>(a.y[k]) + t * a.y_token[k];
    float w[16];
    if (weight && lo < hi) {
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = weight[element(i / 8, i % 8 / kSize) + i % kSize];
    }
    for (int i0 = lo; i0 < hi; i0 += kAtOnce) {
      Piece<T> raw[kAtOnce][2 * kPieces];
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int head = (i0 + j) * kHeads + side;
        const bool there = i0 + j < hi && head < a.heads[k] && in;
#pragma unroll
        for (int e = 0; e < 2 * kPieces; ++e) {
          raw[j][e].w = u4{0u, 0u, 0u, 0u};
          if (there) raw[j][e] = read<T>(x + head * a.x_head[k] + element(e / kPieces, e % kPieces), a.vec);
        }
      }
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        if (i0 + j >= hi) break;
        const int head = (i0 + j) * kHeads + side;
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = (float)raw[j][i / kSize].x[i % kSize];
        if (weight) {
          float sum = 0.f;
#pragma unroll
          for (int i = 0; i < 16; ++i) sum = fmaf(v[i], v[i], sum);
#pragma unroll
          for (int d = kLanes / 2; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
          const float f = 1.f / sqrtf(sum * (1.f / D) + a.eps);
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = v[i] * f * w[i];
        }
        if (rotates) {
          if (a.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float p = v[2 * i], q = v[2 * i + 1];
              v[2 * i] = p * cs[i] - q * sn[i];
              v[2 * i + 1] = q * cs[i] + p * sn[i];
            }
          } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float p = v[i], q = v[i + 8];
              v[i] = p * cs[i] - q * sn[i];
              v[i + 8] = q * cs[i] + p * sn[i];
            }
          }
        }
        if (head < a.heads[k] && in) {
#pragma unroll
          for (int e = 0; e < 2 * kPieces; ++e)
            write<T>(y + head * a.y_head[k] + element(e / kPieces, e % kPieces), v + e * kSize, a.vec);
        }
      }
    }
  }
}

template <int TYPE>
void launch(const RotateArgs &a, int D, dim3 grid, hipStream_t st) {
  switch (D) {
    case 64: k_rotate<TYPE, 64><<<grid, 64 * kWaves, 0, st>>>(a); break;
    case 96: k_rotate<TYPE, 96><<<grid, 64 * kWaves, 0, st>>>(a); break;
    case 128: k_rotate<TYPE, 128><<<grid, 64 * kWaves, 0, st>>>(a); break;
    default: k_rotate<TYPE, 256><<<grid, 64 * kWaves, 0, st>>>(a); break;
  }
}

}  // namespace

extern "C" festina_status festina_rotate_heads(const festina_rotary *rotary, const festina_heads *heads, void *stream) {
  if (!rotary || !heads) return FESTINA_ERR_INVALID;
  const int D = rotary->head_dim, rotated = rotary->rotated;
  if (D < 1 || rotated < 0 || rotated > D || !(rotary->eps >= 0.f)) return FESTINA_ERR_INVALID;
  if ((D != 64 && D != 96 && D != 128 && D != 256) || rotated % 16) return FESTINA_ERR_UNSUPPORTED;
  if (rotated > 0 && (!rotary->turn || (reinterpret_cast<uintptr_t>(rotary->turn) & 7))) return FESTINA_ERR_INVALID;
  if (heads->n_tokens < 0 || heads->n_heads < 0 || heads->n_kv_heads < 0) return FESTINA_ERR_INVALID;
  if (heads->n_heads > 65536 || heads->n_kv_heads > 65536) return FESTINA_ERR_UNSUPPORTED;
  if (heads->dtype != FESTINA_BF16 && heads->dtype != FESTINA_F16 && heads->dtype != FESTINA_F32) return FESTINA_ERR_INVALID;
  if (heads->n_tokens == 0 || heads->n_heads + heads->n_kv_heads == 0) return FESTINA_OK;
  if (!heads->position) return FESTINA_ERR_INVALID;
  if (heads->n_heads > 0 && (!heads->q || !heads->q_out)) return FESTINA_ERR_INVALID;
  if (heads->n_kv_heads > 0 && (!heads->k || !heads->k_out)) return FESTINA_ERR_INVALID;
  RotateArgs a;
  a.T = heads->n_tokens;
  a.rotated = rotated;
  a.interleaved = rotary->interleaved != 0;
  a.eps = rotary->eps;
  a.position = heads->position;
  a.turn = reinterpret_cast<const unsigned long long *>(rotary->turn);
  const int64_t strides[2][4] = {
      {heads->q_token_stride, heads->q_head_stride, heads->q_out_token_stride, heads->q_out_head_stride},
      {heads->k_token_stride, heads->k_head_stride, heads->k_out_token_stride, heads->k_out_head_stride}};
  const int size = heads->dtype == FESTINA_F32 ? 4 : 2;
  uintptr_t at = 0;
  for (int k = 0; k < 2; ++k) {
    a.heads[k] = k ? heads->n_kv_heads : heads->n_heads;
    a.weight[k] = k ? rotary->k_weight : rotary->q_weight;
    a.x[k] = k ? heads->k : heads->q;
    a.y[k] = k ? heads->k_out : heads->q_out;
    a.x_token[k] = strides[k][0], a.x_head[k] = strides[k][1], a.y_token[k] = strides[k][2], a.y_head[k] = strides[k][3];
    if (a.heads[k] == 0) continue;
    for (int i = 0; i < 4; ++i) {
      if (strides[k][i] < 0) return FESTINA_ERR_INVALID;
      at |= (uintptr_t)(strides[k][i] * size);
    }
    at |= reinterpret_cast<uintptr_t>(a.x[k]) | reinterpret_cast<uintptr_t>(a.y[k]);
  }
  if (at % size) return FESTINA_ERR_INVALID;
  a.vec = (at & 15) == 0;
  const int each = 64 / (D == 96 ? 8 : D / 16);
  const int groups = (a.heads[0] + each - 1) / each + (a.heads[1] + each - 1) / each;
  // few tokens: the heads of each over several waves, so that none makes two round trips to memory; each of them makes the token's
  // cosines anew.  One wave a token and one a group of heads, us: 32 and 8 heads of 128 in bfloat16, 256 tokens 7.3 and 4.8, 1,024: 8.5
  // and 8.2, 2,048: 11.6 and 12.9, 4,096: 16.3 and 21.0; 14 and 2 heads of 64 in half, 1,024: 5.5 and 4.9, 2,048: 6.1 and 6.1, 4,096:
  // 8.3 and 9.5; 16 and 16 heads of 96 in float32, 512: 9.3 and 6.6, 1,024: 10.1 and 10.5, 2,048: 14.2 and 18.9
  a.parts = a.T <= 2048 ? groups : 1;
  const long long blocks = ((long long)a.T + kWaves - 1) / kWaves;
  if (blocks > UINT_MAX / (64 * kWaves)) return FESTINA_ERR_UNSUPPORTED;   // threads along one axis of a grid
  const dim3 grid((unsigned)blocks, (unsigned)a.parts);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (heads->dtype == FESTINA_BF16) launch<FESTINA_BF16>(a, D, grid, st);
  else if (heads->dtype == FESTINA_F16) launch<FESTINA_F16>(a, D, grid, st);
  else launch<FESTINA_F32>(a, D, grid, st);
  return hipGetLastError() == hipSuccess ? FESTINA_OK : FESTINA_ERR_DEVICE;
}
