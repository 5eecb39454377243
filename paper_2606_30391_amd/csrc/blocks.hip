// blocks.hip -- MI355X (gfx950) kernels and C-ABI host dispatch of a serving step's cache blocks:
// block tables and slot maps from request lengths, and the release of finished requests' blocks.
//
// Request r holds held[r] tokens and adds add[r]; it needs
//   need[r] = ceil((held + add) / BT) - ceil(held / BT)
// new blocks.  With B and T the running sums of need and add over the requests, r is served iff
// B[r] <= n_free and T[r] <= max_tokens; both sums never fall, so the served requests are the first
// ones, the total of their tokens is the largest T among them, and every request's first token is
// min(T[r] - add[r], total).  Its i-th new block is free_ids[n_free - 1 - (B[r] - need[r] + i)].
//
// k_extend_small   one workgroup: the sums in LDS, then a thread per token (small steps, where launches count).
// k_extend_sums, k_extend_scan, k_extend_fill   the sums of each kChunk requests; each chunk's running sums
//   from those of the chunks before it; then the slots, kFill tokens a workgroup.  The scan leaves for each
//   workgroup of the fill the request that its first token belongs to, so that no search crosses
//   the whole list: a thread searches the few requests of its stretch in LDS.
// k_release_sums, k_release_fill   the same two sums for release, then a thread per returned id.
//
// All arithmetic is on integers; the largest T is taken by an atomic maximum, which does not
// depend on order.  Bound by the bytes of the slot map on large steps, by latency on small ones.
#include <hip/hip_runtime.h>

#include <climits>
#include <cstddef>
#include <cstdint>

#include "festina.h"

namespace {

constexpr int kChunk = 256;          // requests a workgroup of the sums and scans
constexpr int kFill = 2048;          // slots a workgroup of the fill
constexpr int kSmall = 1024;         // threads of the one-workgroup kernel, a request each
constexpr int kSmallTokens = 8192;   // and its slots
constexpr int kMaxRequests = 1 << 20;

struct BlockArgs {
  int32_t R, MB, shift, NB, max_tokens;
  const int32_t *held, *add, *n_free;
  int32_t *table, *free_ids;
  int32_t *first, *slot, *length, *n_free_out;
  uint8_t *served;
  const uint8_t *done;
  // workspace
  long long *sum_blocks, *sum_tokens;   // [chunks]
  int32_t *total;                       // served tokens, last request with any, blocks they take, n_free
  int32_t *before;                      // [R] blocks taken by the requests before r
  int32_t *owner;                       // [fill workgroups] request of a stretch's first token
};

struct Demand {
  int held, add;
  int have;          // blocks held
  int need, takes;   // blocks and tokens taken if served
  bool fits;
};

__device__ __forceinline__ int blocks_of(int tokens, int shift) {
  return (int)(((unsigned)tokens + (1u << shift) - 1) >> shift);
}

__device__ __forceinline__ Demand demand(const BlockArgs &a, int r) {
  Demand d;
  d.held = a.held[r];
  d.add = a.add[r];
  const long long room = (long long)a.MB << a.shift;
  d.fits = d.held >= 0 && d.add >= 0 && (long long)d.held + d.add <= room;
  d.have = d.fits ? blocks_of(d.held, a.shift) : 0;
  d.need = d.fits ? blocks_of(d.held + d.add, a.shift) - d.have : 0;
  d.takes = d.fits ? d.add : 0;
  return d;
}

__device__ __forceinline__ int free_count(const BlockArgs &a) { return min(max(*a.n_free, 0), a.NB); }

// Inclusive sums over a workgroup of N threads; `tot` is the workgroup's sum.
template <int N>
__device__ __forceinline__ long long scan(long long x, long long *lds, long long *tot) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const long long y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < N / 64; ++w) {
    const long long y = lds[w];
    before += w < wave ? y : 0;
    all += y;
  }
  __syncthreads();
  *tot = all;
  return x + before;
}

// Where token t of request r goes; fills the table's new column when the token is its first.
__device__ __forceinline__ int place(const BlockArgs &a, int r, int p, int have, int before, int n_free) {
  const int c = p >> a.shift, o = p & ((1 << a.shift) - 1);
  int id;
  if (c >= have) {
    id = a.free_ids[max(n_free - 1 - (before + c - have), 0)];
    if (o == 0) a.table[(size_t)r * a.MB + c] = id;
  } else {
    id = a.table[(size_t)r * a.MB + c];
  }
  return (unsigned)id < (unsigned)a.NB ? (id << a.shift) + o : -1;
}

__global__ void __launch_bounds__(kSmall) k_extend_small(BlockArgs a) {
  __shared__ long long lds[kSmall / 64];
  __shared__ int first[kSmall + 1], held[kSmall], have[kSmall], before[kSmall];
  __shared__ int total, taken;
  const int r = threadIdx.x;
  const int n_free = free_count(a);
  Demand d{0, 0, 0, 0, 0, false};
  if (r < a.R) d = demand(a, r);
  if (r == 0) total = taken = 0;
  long long unused;
  const long long B = scan<kSmall>(d.need, lds, &unused);
  const long long T = scan<kSmall>(d.takes, lds, &unused);
  const bool served = d.fits && B <= n_free && T <= a.max_tokens;
  if (served) {
    atomicMax(&total, (int)T);
    atomicMax(&taken, (int)B);
  }
  __syncthreads();
  const int end = total;
  if (r < a.R) {
    first[r] = (int)min(T - d.takes, (long long)end);
    held[r] = d.held;
    have[r] = d.have;
    before[r] = (int)min(B - d.need, (long long)INT_MAX);
    a.first[r] = first[r];
    a.length[r] = served ? d.held + d.add : d.held;
    a.served[r] = served;
  }
  if (r == 0) {
    first[a.R] = end;
    a.first[a.R] = end;
    *a.n_free_out = n_free - taken;
  }
  __syncthreads();
  for (int t = threadIdx.x; t < a.max_tokens; t += kSmall) {
    int s = -1;
    if (t < end) {
      int lo = 0, hi = a.R;                        // first[lo] <= t < first[hi]
      while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (first[m] <= t) lo = m; else hi = m;
      }
      s = place(a, lo, held[lo] + t - first[lo], have[lo], before[lo], n_free);
    }
    a.slot[t] = s;
  }
}

__global__ void __launch_bounds__(kChunk) k_extend_sums(BlockArgs a) {
  __shared__ long long lds[kChunk / 64];
  const int r = blockIdx.x * kChunk + threadIdx.x;
  Demand d{0, 0, 0, 0, 0, false};
  if (r < a.R) d = demand(a, r);
  long long B, T;
  scan<kChunk>(d.need, lds, &B);
  scan<kChunk>(d.takes, lds, &T);
  if (threadIdx.x == 0) {
    a.sum_blocks[blockIdx.x] = B;
    a.sum_tokens[blockIdx.x] = T;
    if (blockIdx.x == 0) {
      a.total[0] = a.total[1] = a.total[2] = 0;
      a.total[3] = free_count(a);
    }
  }
}

__global__ void __launch_bounds__(kChunk) k_extend_scan(BlockArgs a) {
  __shared__ long long lds[kChunk / 64];
  const int r = blockIdx.x * kChunk + threadIdx.x;
  long long b = 0, t = 0, B0, T0, unused;
  for (int i = threadIdx.x; i < (int)blockIdx.x; i += kChunk) {
    b += a.sum_blocks[i];
    t += a.sum_tokens[i];
  }
  scan<kChunk>(b, lds, &B0);
  scan<kChunk>(t, lds, &T0);
  Demand d{0, 0, 0, 0, 0, false};
  if (r < a.R) d = demand(a, r);
  const long long B = B0 + scan<kChunk>(d.need, lds, &unused);
  const long long T = T0 + scan<kChunk>(d.takes, lds, &unused);
  const int n_free = a.total[3];
  const bool served = d.fits && B <= n_free && T <= a.max_tokens;
  if (r < a.R) {
    a.first[r] = (int)min(T - d.takes, (long long)a.max_tokens);   // the fill takes the least of this and the total
    a.before[r] = (int)min(B - d.need, (long long)INT_MAX);
    a.length[r] = served ? d.held + d.add : d.held;
    a.served[r] = served;
  }
  if (served && d.takes) {
    const int f = (int)(T - d.takes), e = (int)T;
    for (int w = (f + kFill - 1) / kFill; w * kFill < e; ++w) a.owner[w] = r;
    atomicMax(&a.total[0], e);
    atomicMax(&a.total[1], r);
    atomicMax(&a.total[2], (int)B);
  }
}

__global__ void __launch_bounds__(256) k_extend_fill(BlockArgs a, int32_t fills, int32_t vec) {
  constexpr int kList = kFill + 256;
  __shared__ int first[kList + 1];
  const int end = a.total[0], n_free = a.total[3];
  // the scan's first tokens of requests that are not served lie past the end
  for (int i = blockIdx.x * 256 + threadIdx.x; i <= a.R; i += gridDim.x * 256) {
    if (i == a.R || a.first[i] > end) a.first[i] = end;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.n_free_out = n_free - a.total[2];
  for (int w = blockIdx.x; w < fills; w += gridDim.x) {
    const int t0 = w * kFill;
    int lo0 = 0, n = 0;
    if (t0 < end) {
      lo0 = a.owner[w];
      n = (t0 + kFill < end ? a.owner[w + 1] : a.total[1]) - lo0 + 1;     // requests lo0 .. lo0 + n - 1
    }
    __syncthreads();
    if (n <= kList)
      for (int i = threadIdx.x; i < n; i += 256) first[i] = a.first[lo0 + i];
    __syncthreads();
#pragma unroll
    for (int g = 0; g < kFill / 1024; ++g) {
      const int t = t0 + g * 1024 + threadIdx.x * 4;
      if (t >= a.max_tokens) break;
      int s[4] = {-1, -1, -1, -1};
      if (t < end) {
        int lo = 0, hi = n;
        while (hi - lo > 1) {
          const int m = (lo + hi) >> 1;
          const int f = n <= kList ? first[m] : a.first[lo0 + m];
          if (f <= t) lo = m; else hi = m;
        }
        int r = -1, have = 0, before = 0, shift_p = 0, stop = t;       // stop: where request r's tokens end
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (t + i >= end) break;
          if (t + i >= stop) {
            // the next request with tokens
            int f, add;
            r = r < 0 ? lo0 + lo : r + 1;
            for (;;) {
              f = a.first[r];
              add = a.length[r];
              const int next = r + 1 < a.R ? min(a.first[r + 1], end) : end;
              stop = next;
              if (next > t + i) break;
              ++r;
            }
            const int held = add - (stop - f);      // served: length - its new tokens
            have = blocks_of(held, a.shift);
            before = a.before[r];
            shift_p = held - f;
          }
          s[i] = place(a, r, t + i + shift_p, have, before, n_free);
        }
      }
      if (vec && t + 4 <= a.max_tokens) {
        *reinterpret_cast<int4 *>(a.slot + t) = make_int4(s[0], s[1], s[2], s[3]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (t + i < a.max_tokens) a.slot[t + i] = s[i];
      }
    }
  }
}

__device__ __forceinline__ int returned(const BlockArgs &a, int r, int *held) {
  *held = a.held[r];
  const bool ok = *held >= 0 && *held <= ((long long)a.MB << a.shift);
  return a.done[r] && ok ? blocks_of(*held, a.shift) : 0;
}

__global__ void __launch_bounds__(kChunk) k_release_sums(BlockArgs a) {
  __shared__ long long lds[kChunk / 64];
  const int r = blockIdx.x * kChunk + threadIdx.x;
  int held;
  long long B;
  scan<kChunk>(r < a.R ? returned(a, r, &held) : 0, lds, &B);
  if (threadIdx.x == 0) {
    a.sum_blocks[blockIdx.x] = B;
    if (blockIdx.x == 0) a.total[3] = free_count(a);
  }
}

// One chunk of requests: `n_free` ids lie on the list already, `B0` come from the chunks before it.
__device__ void give_back(const BlockArgs &a, int chunk, int n_free, long long B0, long long *lds, long long *ends) {
  const int r = chunk * kChunk + threadIdx.x;
  int held = 0;
  const int n = r < a.R ? returned(a, r, &held) : 0;
  long long all;
  ends[threadIdx.x] = scan<kChunk>(n, lds, &all);
  __syncthreads();
  for (long long i = threadIdx.x; i < all; i += kChunk) {
    int lo = -1, hi = kChunk - 1;                      // ends[lo] <= i < ends[hi]
    while (hi - lo > 1) {
      const int m = (lo + hi) >> 1;
      if (ends[m] <= i) lo = m; else hi = m;
    }
    const int c = (int)(i - (hi ? ends[hi - 1] : 0));
    const long long at = n_free + B0 + i;
    if (at < a.NB) a.free_ids[at] = a.table[(size_t)(chunk * kChunk + hi) * a.MB + c];
  }
  if (r < a.R) a.length[r] = a.done[r] ? 0 : held;
  if (chunk == (a.R - 1) / kChunk && threadIdx.x == 0)
    *a.n_free_out = (int)min(n_free + B0 + all, (long long)a.NB);
}

__global__ void __launch_bounds__(kChunk) k_release_fill(BlockArgs a) {
  __shared__ long long lds[kChunk / 64];
  __shared__ long long ends[kChunk];
  long long b = 0, B0;
  for (int i = threadIdx.x; i < (int)blockIdx.x; i += kChunk) b += a.sum_blocks[i];
  scan<kChunk>(b, lds, &B0);
  give_back(a, blockIdx.x, a.total[3], B0, lds, ends);
}

// One chunk alone: every thread has read held and n_free (the scan's barrier) before any writes.
__global__ void __launch_bounds__(kChunk) k_release_one(BlockArgs a) {
  __shared__ long long lds[kChunk / 64];
  __shared__ long long ends[kChunk];
  give_back(a, 0, free_count(a), 0, lds, ends);
}

struct Layout {
  size_t sum_blocks, sum_tokens, total, before, owner, bytes;
};

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

Layout layout(int R, int max_tokens) {
  Layout l;
  const size_t chunks = ((size_t)R + kChunk - 1) / kChunk, fills = ((size_t)max_tokens + kFill - 1) / kFill;
  l.sum_blocks = 0;
  l.sum_tokens = up(chunks * 8);
  l.total = l.sum_tokens + up(chunks * 8);
  l.before = l.total + 256;
  l.owner = l.before + up((size_t)R * 4);
  l.bytes = l.owner + up((fills + 1) * 4);
  return l;
}

// Checks what both calls share and fills the arguments; FESTINA_OK when there is work.
festina_status arguments(const festina_kv_requests *q, festina_kv_step *out, bool extend, void *ws, size_t ws_bytes,
                         BlockArgs *a) {
  if (!q || !out || q->n_requests < 0 || q->max_blocks < 1 || q->n_blocks < 1) return FESTINA_ERR_INVALID;
  const int bt = q->block_tokens;
  if (bt < 1 || (extend && out->max_tokens < 0)) return FESTINA_ERR_INVALID;
  if (bt < 16 || bt > 256 || (bt & (bt - 1))) return FESTINA_ERR_UNSUPPORTED;
  if ((long long)q->n_blocks * bt > INT_MAX || (long long)q->max_blocks * bt > INT_MAX || q->n_requests > kMaxRequests)
    return FESTINA_ERR_UNSUPPORTED;
  if (!q->n_free || !out->n_free_out) return FESTINA_ERR_INVALID;
  if (q->n_requests > 0) {
    if (!q->held || !q->block_table || !q->free_ids || !out->length) return FESTINA_ERR_INVALID;
    if (extend && (!q->add || !out->served)) return FESTINA_ERR_INVALID;
  }
  if (extend && (!out->first || (out->max_tokens > 0 && !out->slot))) return FESTINA_ERR_INVALID;
  const Layout l = layout(q->n_requests, extend ? out->max_tokens : 0);
  if (!ws || ws_bytes < l.bytes || (reinterpret_cast<uintptr_t>(ws) & 255)) return FESTINA_ERR_INVALID;
  char *w = static_cast<char *>(ws);
  *a = BlockArgs{};
  a->R = q->n_requests;
  a->MB = q->max_blocks;
  a->shift = __builtin_ctz((unsigned)bt);
  a->NB = q->n_blocks;
  a->max_tokens = extend ? out->max_tokens : 0;
  a->held = q->held;
  a->add = q->add;
  a->n_free = q->n_free;
  a->table = q->block_table;
  a->free_ids = q->free_ids;
  a->first = out->first;
  a->slot = out->slot;
  a->length = out->length;
  a->n_free_out = out->n_free_out;
  a->served = out->served;
  a->sum_blocks = reinterpret_cast<long long *>(w + l.sum_blocks);
  a->sum_tokens = reinterpret_cast<long long *>(w + l.sum_tokens);
  a->total = reinterpret_cast<int32_t *>(w + l.total);
  a->before = reinterpret_cast<int32_t *>(w + l.before);
  a->owner = reinterpret_cast<int32_t *>(w + l.owner);
  return FESTINA_OK;
}

}  // namespace

extern "C" size_t festina_blocks_workspace_bytes(int32_t n_requests, int32_t max_tokens) {
  if (n_requests < 0 || n_requests > kMaxRequests || max_tokens < 0) return 0;
  return layout(n_requests, max_tokens).bytes;
}

extern "C" festina_status festina_extend_blocks(const festina_kv_requests *req, festina_kv_step *out,
                                                void *workspace, size_t workspace_bytes, void *stream) {
  BlockArgs a;
  const festina_status bad = arguments(req, out, true, workspace, workspace_bytes, &a);
  if (bad != FESTINA_OK) return bad;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (a.R <= kSmall && a.max_tokens <= kSmallTokens) {
    k_extend_small<<<1, kSmall, 0, st>>>(a);
  } else {
    const int chunks = max((a.R + kChunk - 1) / kChunk, 1);
    const int fills = (a.max_tokens + kFill - 1) / kFill;
    const bool vec = (reinterpret_cast<uintptr_t>(a.slot) & 15) == 0;
    k_extend_sums<<<chunks, kChunk, 0, st>>>(a);
    k_extend_scan<<<chunks, kChunk, 0, st>>>(a);
    k_extend_fill<<<min(max(max(fills, chunks), 1), 4096), 256, 0, st>>>(a, fills, vec);
  }
  return hipGetLastError() == hipSuccess ? FESTINA_OK : FESTINA_ERR_DEVICE;
}

extern "C" festina_status festina_release_blocks(const festina_kv_requests *req, const uint8_t *done,
                                                 festina_kv_step *out, void *workspace, size_t workspace_bytes,
                                                 void *stream) {
  BlockArgs a;
  const festina_status bad = arguments(req, out, false, workspace, workspace_bytes, &a);
  if (bad != FESTINA_OK) return bad;
  if (a.R > 0 && !done) return FESTINA_ERR_INVALID;
  a.done = done;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int chunks = (a.R + kChunk - 1) / kChunk;
  if (chunks <= 1) {
    k_release_one<<<1, kChunk, 0, st>>>(a);
  } else {
    k_release_sums<<<chunks, kChunk, 0, st>>>(a);
    k_release_fill<<<chunks, kChunk, 0, st>>>(a);
  }
  return hipGetLastError() == hipSuccess ? FESTINA_OK : FESTINA_ERR_DEVICE;
}
