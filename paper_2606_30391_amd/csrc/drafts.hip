// drafts.hip -- MI355X (gfx950) kernels and C-ABI host dispatch of a step of drafted tokens: what the nodes of a
// request's draft tree see and where they stand, which of them the model accepts, and the move of the accepted ones'
// keys and values to where a cache without the others would hold them.
//
// A tree has at most 64 nodes, so a wave holds one, a lane a node, and a node's ancestors are a word of 64 bits.
//
// k_plan_drafts    seen(i) = bit i | seen(parent(i)), by doubling: after s steps a lane has the 2^s nearest of its path and
//   the node behind them, so six steps do, whatever the depth.
// k_accept_drafts  from node 0 on, the first child whose token the model chose there: one comparison of all
//   nodes with their parents' choices, then a ballot a node of the path.
// k_keep_tokens    a wave for a request, key head, layer, and keys or values.  Kept token i comes from path[i] >= i, in ascending
//   order, so that a token's new slot never lies behind the slots still to be read: some tokens at a time are read, then
//   written.  The first codes are on their way together with the scales, whose largest each block waits for (7.1 us for
//   32 trees of 8 in four layers without that, 6.6 with it).  A block's scale afterwards is the largest among the blocks
//   that its tokens came from; scales are powers of two, so codes are multiplied exactly and rounded once (only where they
//   become subnormal).  All layers are one launch: a launch a layer costs the host 5 us each.
//
// All three are bound by latency, a launch and a chain of three to six dependent reads: 2.5 and 3.0 us for the plan and
// the acceptance of 32 trees of 8, 3.8 each of 4,096 trees of up to 64; 6.6 us for the kept tokens of 32 trees in four layers,
// 14 for those of 160 trees of up to 63, 17 MB, where 10,240 waves take turns and values move a byte a lane.  (Values by
// 16 columns of a row a lane, which change places in LDS: 8.7 and 15.3 us, since few of a tree's nodes are kept.)
#include <hip/hip_runtime.h>

#include <climits>
#include <cstddef>
#include <cstdint>

#include "festina.h"
#include "kv.h"

namespace {

using namespace festina_kv;

constexpr int kNodes = 64;           // nodes of a tree: a request with more new tokens is a run
constexpr int kWaves = 4;
constexpr int kMaxRequests = 1 << 20;

struct DraftArgs {
  int32_t R, T;
  const int32_t *first, *length, *parent;
  unsigned long long *seen;
  int32_t *position;
  const int32_t *token, *choice;
  int32_t *path, *kept, *next, *left;
};

// A value that is the same in all lanes, kept once.
__device__ __forceinline__ int same(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Request r's first token and how many it has.
__device__ __forceinline__ int2 tokens_of(const int32_t *first, int T, int r) {
  const int f = min(max(same(first[r]), 0), T);
  return make_int2(f, min(max(same(first[r + 1]), f), T) - f);
}
// The parent of node i (a lane each), -1 for none.
__device__ __forceinline__ int parent_of(const DraftArgs &a, int2 q, int i) {
  int p = i - 1;
  if (a.parent && i < q.y) p = a.parent[q.x + i];
  return (unsigned)p < (unsigned)i ? p : -1;
}

__global__ void __launch_bounds__(64 * kWaves) k_plan_drafts(DraftArgs a) {
  const int r = blockIdx.x * kWaves + same((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= a.R) return;
  const int2 q = tokens_of(a.first, a.T, r);
  const int before = same(a.length[r]) - q.y;
  if (q.y > kNodes) {
    for (int i = lane; i < q.y; i += 64) {
      if (a.position) a.position[q.x + i] = before + i;
      if (a.seen) a.seen[q.x + i] = 0ull;
    }
    return;
  }
  int up = parent_of(a, q, lane);
  unsigned long long word = 1ull << lane;
#pragma unroll
  for (int s = 0; s < 6; ++s) {
    const unsigned long long w = __shfl(word, max(up, 0));
    const int u = __shfl(up, max(up, 0));
    word |= up >= 0 ? w : 0ull;
    up = up >= 0 ? u : -1;
  }
  if (lane < q.y) {
    if (a.seen) a.seen[q.x + lane] = word;
    if (a.position) a.position[q.x + lane] = before + __builtin_popcountll(word) - 1;
  }
}

__global__ void __launch_bounds__(64 * kWaves) k_accept_drafts(DraftArgs a) {
  const int r = blockIdx.x * kWaves + same((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (r >= a.R) return;
  const int2 q = tokens_of(a.first, a.T, r);
  const int before = same(a.length[r]) - q.y;
  int kept = q.y, next = -1;
  if (q.y > kNodes) {
    for (int i = lane; i < q.y; i += 64) a.path[q.x + i] = i;
    next = a.choice[q.x + q.y - 1];
  } else if (q.y > 0) {
    const bool there = lane < q.y;
    const int up = parent_of(a, q, lane);
    const int token = there ? a.token[q.x + lane] : 0, choice = there ? a.choice[q.x + lane] : 0;
    const bool right = __shfl(choice, max(up, 0)) == token && there && up >= 0;
    int node = 0, mine = -1;
    kept = 0;
    for (;;) {                                         // children come after their parents: at most 64 nodes
      mine = lane == kept ? node : mine;
      ++kept;
      const unsigned long long m = __ballot(right && up == node);
      if (m == 0) break;
      node = __builtin_ctzll(m);
    }
    next = __builtin_amdgcn_readlane(choice, node);
    if (there) a.path[q.x + lane] = mine;
  }
  if (lane == 0) {
    a.kept[r] = kept;
    a.next[r] = next;
    a.left[r] = before + kept;
  }
}

// ------------------------------------------------------------------ the accepted tokens' keys and values

// Caches of a launch.  Their addresses are arguments, 2 KiB of them for 64 caches, which the host takes 0.2 us longer to hand over
// (32 trees of 8 in four layers, a call: 6.2 us with room for 8, 6.4 for 64; the kernel takes 6.8 with either).  More layers, us:
// 8: 10.4, 16: 15.9, 32: 26.4, 64: 45.7; 160 trees of up to 63 over blocks of 16: 20, 31, 52 and 118.
constexpr int kFewLayers = 8, kLayers = 64;

struct Layer {
  uint8_t *codes[2];
  float *scale[2];
};
template <int LAYERS>
struct KeepArgs {
  int32_t R, MB, T, H, shift, NB;
  const int32_t *table, *length, *first, *path, *kept;
  Layer layer[LAYERS];
};

typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef float f2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ unsigned recode4(unsigned c, float ratio) {
  const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a.x * ratio, a.y * ratio, 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(b.x * ratio, b.y * ratio, w, true);
  return (unsigned)w;
}

// Everything read so far has arrived: what is written next may lie where it was.
__device__ __forceinline__ void all_read() { __builtin_amdgcn_s_waitcnt(0); }

template <int LAYERS, int D>
__global__ void __launch_bounds__(64) k_keep_tokens(KeepArgs<LAYERS> a) {
  constexpr int kBlocks = kNodes / 16 + 1;             // that 64 tokens lie in
  __shared__ unsigned most[kBlocks];                   // the new scale of each block from the first changed one on
  __shared__ int2 from_[kNodes], to_[kNodes];          // of each moved token: block and slot where it was, and where it goes
  __shared__ float factor_[kNodes];                    // of its codes
  const int lane = threadIdx.x, which = blockIdx.y & 1, bt = 1 << a.shift;
  const Layer &layer = a.layer[blockIdx.y >> 1];
  const int h = blockIdx.x % a.H, r = blockIdx.x / a.H;
  const int length = a.length[r], some = a.kept[r];
  const int2 q = tokens_of(a.first, a.T, r);
  const int before = same(length) - q.y, kept = min(same(some), q.y);
  if (q.y > kNodes || kept < 1 || before < 0 || before + q.y > a.MB << a.shift) return;
  const int c_base = before >> a.shift, cols = ((before + q.y - 1) >> a.shift) - c_base + 1;    // the new tokens' columns
  const int at_col = lane < cols ? a.table[(size_t)r * a.MB + c_base + lane] : 0;
  const int mine = lane < kept ? a.path[q.x + lane] : INT_MAX;
  const int prior = __shfl_up(mine, 1);
  // ascending and of its own tokens, which makes path[i] >= i; and blocks that there are
  const bool bad = lane < kept && ((unsigned)mine >= (unsigned)q.y || (lane > 0 && prior >= mine));
  const unsigned long long moves = __ballot(lane < kept && mine != lane);
  if (__any(bad || (unsigned)at_col >= (unsigned)a.NB) || moves == 0) return;
  const int m = __builtin_ctzll(moves), n = kept - m;  // the first token that moves, and how many
  const int c0 = (before + m) >> a.shift, stay = (before + m) & (bt - 1);
  uint8_t *codes = layer.codes[which];
  float *scales = layer.scale[which];
  const size_t head = (size_t)D << a.shift;          // codes of a block and head
  const auto block_of = [&](int b) { return codes + ((size_t)b * a.H + h) * head; };
  const int last = before + q.y - 1, to = min(before + lane, last), since = before + min(mine, q.y - 1);
  const bool moved = lane >= m && lane < kept;
  const int b_to = __shfl(at_col, (to >> a.shift) - c_base), b_from = __shfl(at_col, (since >> a.shift) - c_base);
  const int b_first = __shfl(at_col, c0 - c_base);
  if (moved) {
    from_[lane - m] = make_int2(b_from, since & (bt - 1));
    to_[lane - m] = make_int2(b_to, to & (bt - 1));
  }
  if (lane < kBlocks) most[lane] = 0u;
  __syncthreads();

  // keys: 16 codes of a token a lane and load; values: one, whose neighbours are other rows'
  constexpr int kKeys = 4, kValues = 8;
  const int groups = D / 16, keys = n * groups, values = n * D;
  u4 k[kKeys];
  unsigned v[kValues];
  const auto key_at = [&](int i, const int2 *place) {
    const int t = i / groups;
    return reinterpret_cast<u4 *>(block_of(place[t].x) + (size_t)place[t].y * D + (i - t * groups) * 16);
  };
  const auto value_at = [&](int i, const int2 *place) {
    const int t = i / D;
    return block_of(place[t].x) + (size_t)(i - t * D) * bt + place[t].y;
  };
  const auto read_keys = [&](int i0) {
#pragma unroll
    for (int y = 0; y < kKeys; ++y)
      if (i0 + y * 64 + lane < keys) k[y] = *key_at(i0 + y * 64 + lane, from_);
  };
  const auto read_values = [&](int i0) {
#pragma unroll
    for (int y = 0; y < kValues; ++y)
      if (i0 + y * 64 + lane < values) v[y] = *value_at(i0 + y * 64 + lane, from_);
  };
  if (which == 0) read_keys(0);
  else read_values(0);
  const float s_from = moved ? scales[(size_t)b_from * a.H + h] : 0.f;
  const float s_stay = stay ? scales[(size_t)b_first * a.H + h] : 0.f;     // tokens of the first changed block that stay
  if (moved) atomicMax(&most[(to >> a.shift) - c0], __float_as_uint(s_from));
  if (lane == 0 && stay) atomicMax(&most[0], __float_as_uint(s_stay));
  all_read();
  __syncthreads();
  const float s_first = __uint_as_float(most[0]);
  if (moved) {
    const float s_to = __uint_as_float(most[(to >> a.shift) - c0]);
    factor_[lane - m] = s_to > 0.f ? s_from / s_to : 1.f;
    if (lane == m || (to & (bt - 1)) == 0) scales[(size_t)b_to * a.H + h] = s_to;
  }
  __syncthreads();
  if (stay && s_first > s_stay) {                      // the tokens that stay, anew, before others come beside them
    const float ratio = s_stay / s_first;
    uint8_t *c = block_of(b_first);
    if (which == 0) {
      for (int i = lane; i < stay * D / 4; i += 64) {
        unsigned *p = reinterpret_cast<unsigned *>(c) + i;
        *p = recode4(*p, ratio);
      }
    } else {
      const int words = (stay + 3) / 4;
      for (int i = lane; i < D * words; i += 64) {
        const int d = i / words, o = (i - d * words) * 4;
        uint8_t *p = c + (size_t)d * bt + o;
        const unsigned w = *reinterpret_cast<const unsigned *>(p), x = recode4(w, ratio);
        const unsigned mask = o + 4 <= stay ? ~0u : (1u << (8 * (stay - o))) - 1;
        *reinterpret_cast<unsigned *>(p) = (x & mask) | (w & ~mask);
      }
    }
    all_read();
  }
  if (which == 0) {
    for (int i0 = 0; i0 < keys; i0 += 64 * kKeys) {
      if (i0 > 0) {
        read_keys(i0);
        all_read();
      }
#pragma unroll
      for (int y = 0; y < kKeys; ++y) {
        const int i = i0 + y * 64 + lane;
        if (i >= keys) continue;
        const float f = factor_[i / groups];
        *key_at(i, to_) = u4{recode4(k[y][0], f), recode4(k[y][1], f), recode4(k[y][2], f), recode4(k[y][3], f)};
      }
      all_read();
    }
  } else {
    for (int i0 = 0; i0 < values; i0 += 64 * kValues) {
      if (i0 > 0) {
        read_values(i0);
        all_read();
      }
#pragma unroll
      for (int y = 0; y < kValues; ++y) {
        const int i = i0 + y * 64 + lane;
        if (i < values) *value_at(i, to_) = (uint8_t)recode4(v[y], factor_[i / D]);
      }
      all_read();
    }
  }
}

template <int LAYERS>
void keep(const festina_kv_cache *caches, int n, const festina_kept &kept, hipStream_t st) {
  KeepArgs<LAYERS> a;
  a.R = kept.n_requests;
  a.MB = kept.max_blocks;
  a.T = kept.n_tokens;
  a.H = caches[0].n_kv_heads;
  a.shift = __builtin_ctz((unsigned)caches[0].block_tokens);
  a.NB = caches[0].n_blocks;
  a.table = kept.block_table;
  a.length = kept.length;
  a.first = kept.first;
  a.path = kept.path;
  a.kept = kept.kept;
  for (int i = 0; i < n; ++i) a.layer[i] = Layer{{caches[i].k, caches[i].v}, {caches[i].k_scale, caches[i].v_scale}};
  const dim3 grid((unsigned)((long long)a.R * a.H), (unsigned)(2 * n));
  switch (caches[0].head_dim) {
    case 64: k_keep_tokens<LAYERS, 64><<<grid, 64, 0, st>>>(a); break;
    case 96: k_keep_tokens<LAYERS, 96><<<grid, 64, 0, st>>>(a); break;
    case 128: k_keep_tokens<LAYERS, 128><<<grid, 64, 0, st>>>(a); break;
    default: k_keep_tokens<LAYERS, 256><<<grid, 64, 0, st>>>(a); break;
  }
}

// What both calls over the trees share.
festina_status check_drafts(const festina_drafts *d) {
  if (!d || d->n_requests < 0 || d->n_tokens < 0) return FESTINA_ERR_INVALID;
  if (d->n_requests > kMaxRequests) return FESTINA_ERR_UNSUPPORTED;
  if (d->n_requests > 0 && (!d->first || !d->length)) return FESTINA_ERR_INVALID;
  return FESTINA_OK;
}
DraftArgs arguments(const festina_drafts *d) {
  DraftArgs a{};
  a.R = d->n_requests;
  a.T = d->n_tokens;
  a.first = d->first;
  a.length = d->length;
  a.parent = d->parent;
  return a;
}

}  // namespace

extern "C" festina_status festina_plan_drafts(const festina_drafts *drafts, uint64_t *seen, int32_t *position, void *stream) {
  const festina_status bad = check_drafts(drafts);
  if (bad != FESTINA_OK) return bad;
  if ((reinterpret_cast<uintptr_t>(seen) & 7) || (drafts->n_tokens > 0 && !seen && !position)) return FESTINA_ERR_INVALID;
  if (drafts->n_requests == 0 || drafts->n_tokens == 0) return FESTINA_OK;
  DraftArgs a = arguments(drafts);
  a.seen = reinterpret_cast<unsigned long long *>(seen);
  a.position = position;
  hipStream_t st = static_cast<hipStream_t>(stream);
  k_plan_drafts<<<(unsigned)((a.R + kWaves - 1) / kWaves), 64 * kWaves, 0, st>>>(a);
  return hipGetLastError() == hipSuccess ? FESTINA_OK : FESTINA_ERR_DEVICE;
}

extern "C" festina_status festina_accept_drafts(const festina_drafts *drafts, const int32_t *token, const int32_t *choice,
                                                festina_accepted *out, void *stream) {
  const festina_status bad = check_drafts(drafts);
  if (bad != FESTINA_OK) return bad;
  if (!out) return FESTINA_ERR_INVALID;
  if (drafts->n_requests == 0) return FESTINA_OK;
  if (!out->kept || !out->next || !out->length) return FESTINA_ERR_INVALID;
  if (drafts->n_tokens > 0 && (!token || !choice || !out->path)) return FESTINA_ERR_INVALID;
  DraftArgs a = arguments(drafts);
  a.token = token;
  a.choice = choice;
  a.path = out->path;
  a.kept = out->kept;
  a.next = out->next;
  a.left = out->length;
  hipStream_t st = static_cast<hipStream_t>(stream);
  k_accept_drafts<<<(unsigned)((a.R + kWaves - 1) / kWaves), 64 * kWaves, 0, st>>>(a);
  return hipGetLastError() == hipSuccess ? FESTINA_OK : FESTINA_ERR_DEVICE;
}

extern "C" festina_status festina_keep_tokens(const festina_kv_cache *caches, int32_t n_caches, const festina_kept *kept,
                                              void *stream) {
  if (n_caches < 0 || (n_caches > 0 && !caches) || !kept) return FESTINA_ERR_INVALID;
  if (kept->n_requests < 0 || kept->max_blocks < 1 || kept->n_tokens < 0) return FESTINA_ERR_INVALID;
  for (int i = 0; i < n_caches; ++i) {
    const festina_status bad = check_cache(caches + i);
    if (bad != FESTINA_OK) return bad;
    const festina_kv_cache &c = caches[i], &d = caches[0];
    if (c.n_blocks != d.n_blocks || c.block_tokens != d.block_tokens || c.n_kv_heads != d.n_kv_heads || c.head_dim != d.head_dim)
      return FESTINA_ERR_INVALID;
  }
  if (kept->n_requests > kMaxRequests) return FESTINA_ERR_UNSUPPORTED;
  if (n_caches == 0 || kept->n_requests == 0 || kept->n_tokens == 0) return FESTINA_OK;
  if ((long long)kept->max_blocks * caches[0].block_tokens > INT_MAX) return FESTINA_ERR_UNSUPPORTED;
  if (!kept->block_table || !kept->length || !kept->first || !kept->path || !kept->kept) return FESTINA_ERR_INVALID;
  if ((long long)kept->n_requests * caches[0].n_kv_heads > UINT_MAX / 64) return FESTINA_ERR_UNSUPPORTED;      // threads along one axis of a grid
  hipStream_t st = static_cast<hipStream_t>(stream);
  for (int i = 0; i < n_caches; i += kLayers) {
    const int n = n_caches - i < kLayers ? n_caches - i : kLayers;
    if (n <= kFewLayers) keep<kFewLayers>(caches + i, n, *kept, st);
    else keep<kLayers>(caches + i, n, *kept, st);
  }
  return hipGetLastError() == hipSuccess ? FESTINA_OK : FESTINA_ERR_DEVICE;
}
