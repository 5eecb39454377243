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
// k_extend_scan    the running sums of kChunk requests a workgroup, after the sums of all requests before them:
//   from k_extend_sums, one number a chunk, or, for few requests, summed by the workgroup itself, which
//   saves a launch.  It leaves what the fill needs of a request, and for each stretch of kFill tokens the
//   request that its first token belongs to, so that no search crosses the whole list.
// k_extend_fill    the slots, a stretch of 256 or 1,024 tokens a wave.  Where they lie in one request, everything
//   about it is uniform, and a lane makes its slots four at a time from one or two block ids, with all loads in
//   flight together.  Where they do not, each lane searches the few requests of its stretch in LDS, in steps
//   that all groups of the stretch take together, so that their loads wait once (4,096 requests: 14.7 -> 13.9 us).
// k_release        a thread per returned id, after the same sums.
//
// All arithmetic is on integers, so results do not depend on order.  Bound by the bytes of the slot map on
// large steps (65,536 requests, 42.5 M slots: sums 5, scan 13, fill 57 us, 170 MB at 3.0 TB/s), by latency on small
// ones (4,096 prompts: scan 6, fill 9 us; the blocks of a third of 20,011 requests returned: 12 us).
#include <hip/hip_runtime.h>

#include <climits>
#include <cstddef>
#include <cstdint>

#include "festina.h"

namespace {

typedef int i4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 256;          // requests a workgroup of the sums and scans
constexpr int kGive = 64;            // requests a workgroup of the release
constexpr int kDirect = 16384;       // up to so many requests a workgroup sums all requests before its own
// Slots a wave of the fill, in groups of 256: long stretches from the size on that gives every wave slot of the chip
// one (2.2 M slots of 4,096 requests 13 us with long stretches, 10 with short ones; 42.5 M: 65 and 82).
constexpr int kGroupsMost = 4;
constexpr int kLongFills = 8 << 20;
constexpr int kSmall = 1024;         // threads of the one-workgroup kernel, a request each
constexpr int kSmallTokens = 8192;   // and its slots
constexpr int kMaxRequests = 1 << 20;
constexpr int kMaxTokens = INT_MAX - 4096;     // the last stretch of the fill is counted in 32 bits

struct BlockArgs {
  int32_t R, MB, shift, NB, max_tokens;
  const int32_t *held, *add, *n_free;
  int32_t *table, *free_ids;
  int32_t *first, *slot, *length, *n_free_out;
  uint8_t *served;
  const uint8_t *done;
  // workspace
  long long *sum_blocks, *sum_tokens;   // [chunks]
  int4 *ends;                           // served tokens, the last request with any, the blocks they take: of each chunk
                                        // of a direct scan, else of all in ends[0]
  int32_t *n_free_in;                   // [1] the count before the call
  int4 *about;                          // [R] see About
  int32_t *owner;                       // [fill stretches] request of a stretch's first token
  int32_t fill;                         // slots of a stretch
  bool vec;                             // held, add (and done) may be read four at a time
};

// What the fill needs of a request: token t stands at position t + shift; columns from `have` on are new, column c is
// free_ids[top - c]; its length afterwards.
struct About {
  int32_t shift, have, top, length;
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

__device__ __forceinline__ Demand demand_of(const BlockArgs &a, int held, int add) {
  Demand d;
  d.held = held;
  d.add = add;
  const int room = a.MB << a.shift;                    // fits 32 bits
  d.fits = held >= 0 && add >= 0 && held <= room && add <= room - held;
  d.have = d.fits ? blocks_of(d.held, a.shift) : 0;
  d.need = d.fits ? blocks_of(d.held + d.add, a.shift) - d.have : 0;
  d.takes = d.fits ? d.add : 0;
  return d;
}

__device__ __forceinline__ Demand demand(const BlockArgs &a, int r) { return demand_of(a, a.held[r], a.add[r]); }

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

// A wave's last served request, if it has one: the sums up to it and its index (the served ones come first).
__device__ __forceinline__ void last_served(bool served, int tokens, int r, int blocks, int (&out)[3]) {
  const unsigned long long m = __ballot(served);
  const int lane = threadIdx.x & 63;
  if (m ? lane == 63 - __builtin_clzll(m) : lane == 0) {
    out[0] = m ? tokens : 0;
    out[1] = m ? r : 0;
    out[2] = m ? blocks : 0;
  }
}

// The block of column c of a request; the table's entry is filled where the column's first token is `begins`.
__device__ __forceinline__ int block_at(const BlockArgs &a, int r, const About &q, int c, bool begins) {
  if (c < q.have) return a.table[(size_t)r * a.MB + c];
  const int id = a.free_ids[max(q.top - c, 0)];
  if (begins) a.table[(size_t)r * a.MB + c] = id;
  return id;
}
__device__ __forceinline__ int slot_of(const BlockArgs &a, int id, int o) {
  return (unsigned)id < (unsigned)a.NB ? (id << a.shift) + o : -1;
}

template <int N>
__global__ void __launch_bounds__(N) k_extend_small(BlockArgs a) {
  __shared__ long long lds[N / 64];
  __shared__ int first[N + 1];
  __shared__ About about[N];
  __shared__ int ends[N / 64][3];
  const int r = threadIdx.x;
  const int n_free = free_count(a);
  Demand d{0, 0, 0, 0, 0, false};
  if (r < a.R) d = demand(a, r);
  long long unused;
  const long long B = scan<N>(d.need, lds, &unused);
  const long long T = scan<N>(d.takes, lds, &unused);
  const bool served = d.fits && B <= n_free && T <= a.max_tokens;
  last_served(served, (int)T, r, (int)B, ends[threadIdx.x >> 6]);
  __syncthreads();
  int end = 0, taken = 0;
#pragma unroll
  for (int w = 0; w < N / 64; ++w) end = max(end, ends[w][0]), taken = max(taken, ends[w][2]);
  if (r < a.R) {
    const int f = (int)min(T - d.takes, (long long)end), len = served ? d.held + d.add : d.held;
    first[r] = f;
    about[r] = About{d.held - f, d.have, (int)(n_free - 1 - min(B - d.need, (long long)n_free) + d.have), len};
    a.first[r] = f;
    a.length[r] = len;
    a.served[r] = served;
  }
  if (r == 0) {
    first[a.R] = end;
    a.first[a.R] = end;
    *a.n_free_out = n_free - taken;
  }
  __syncthreads();
  for (int t = threadIdx.x; t < a.max_tokens; t += N) {
    int s = -1;
    if (t < end) {
      int lo = 0, hi = a.R;                        // first[lo] <= t < first[hi]
      while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (first[m] <= t) lo = m; else hi = m;
      }
      const About q = about[lo];
      const int p = t + q.shift, o = p & ((1 << a.shift) - 1);
      s = slot_of(a, block_at(a, lo, q, p >> a.shift, o == 0), o);
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
    if (blockIdx.x == 0) a.ends[0] = make_int4(0, 0, 0, 0);
  }
}

// The caller's arrays are only read here (length and n_free may be the ones to be overwritten): the fill writes them.
template <bool DIRECT>
__global__ void __launch_bounds__(kChunk) k_extend_scan(BlockArgs a) {
  __shared__ long long lds[kChunk / 64];
  __shared__ int ends[kChunk / 64][3];
  const int r = blockIdx.x * kChunk + threadIdx.x, r0 = blockIdx.x * kChunk;
  long long b = 0, t = 0, B0, T0, unused;
  const auto count = [&](int held, int add) {
    const Demand d = demand_of(a, held, add);
    b += d.need;
    t += d.takes;
  };
  Demand d{0, 0, 0, 0, 0, false};
  if (r < a.R) d = demand(a, r);
  const int n_free = free_count(a);
  if (DIRECT && a.vec) {
#pragma unroll 4
    for (int i = threadIdx.x * 4; i < r0; i += kChunk * 4) {
      const int4 h = *reinterpret_cast<const int4 *>(a.held + i), n = *reinterpret_cast<const int4 *>(a.add + i);
      count(h.x, n.x), count(h.y, n.y), count(h.z, n.z), count(h.w, n.w);
    }
  } else if (DIRECT) {
    for (int i = threadIdx.x; i < r0; i += kChunk) count(a.held[i], a.add[i]);
  } else {
    for (int i = threadIdx.x; i < (int)blockIdx.x; i += kChunk) {
      b += a.sum_blocks[i];
      t += a.sum_tokens[i];
    }
  }
  scan<kChunk>(b, lds, &B0);
  scan<kChunk>(t, lds, &T0);
  const long long B = B0 + scan<kChunk>(d.need, lds, &unused);
  const long long T = T0 + scan<kChunk>(d.takes, lds, &unused);
  const bool served = d.fits && B <= n_free && T <= a.max_tokens;
  if (r < a.R) {
    const int f = (int)min(T - d.takes, (long long)a.max_tokens);   // the fill takes the least of this and the total
    a.first[r] = f;
    const int top = (int)(n_free - 1 - min(B - d.need, (long long)n_free) + d.have);
    a.about[r] = make_int4(d.held - f, d.have, top, served ? d.held + d.add : d.held);
    a.served[r] = served;
  }
  if (served && d.takes) {
    const int f = (int)(T - d.takes), e = (int)T;
    for (int w = (int)(((unsigned)f + a.fill - 1) / a.fill); w * (long long)a.fill < e; ++w) a.owner[w] = r;
  }
  last_served(served && d.takes, (int)T, r, (int)B, ends[threadIdx.x >> 6]);
  __syncthreads();
  if (threadIdx.x == 0) {
    int4 e = make_int4(0, 0, 0, 0);
#pragma unroll
    for (int w = 0; w < kChunk / 64; ++w)
      e = make_int4(max(e.x, ends[w][0]), max(e.y, ends[w][1]), max(e.z, ends[w][2]), 0);
    if (DIRECT) {
      a.ends[blockIdx.x] = e;
    } else if (e.x) {                                  // one maximum a workgroup, whatever their order
      int *all = reinterpret_cast<int *>(a.ends);
      atomicMax(all, e.x), atomicMax(all + 1, e.y), atomicMax(all + 2, e.z);
    }
    if (blockIdx.x == 0) *a.n_free_in = n_free;
  }
}

template <int kGroups>
__global__ void __launch_bounds__(256) k_extend_fill(BlockArgs a, int32_t chunks, int32_t fills, int32_t vec) {
  constexpr int kFill = kGroups * 256, kList = kFill + 64;
  __shared__ int lists[4][kList];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bt = 1 << a.shift;
  int *first = lists[wave];
  int end = 0, last = 0, taken = 0;
  if (chunks == 1) {
    const int4 e = a.ends[0];
    end = e.x, last = e.y, taken = e.z;
  } else {
    for (int i = lane; i < chunks; i += 64) {
      const int4 e = a.ends[i];
      end = max(end, e.x), last = max(last, e.y), taken = max(taken, e.z);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      end = max(end, __shfl_xor(end, d));
      last = max(last, __shfl_xor(last, d));
      taken = max(taken, __shfl_xor(taken, d));
    }
  }
  end = __builtin_amdgcn_readfirstlane(end);
  const auto put = [&](int t, const int (&s)[4]) {
    if (vec && t + 4 <= a.max_tokens) {
      // past the caches, which such lists do not fit: 42.5 M slots with all launches 116 -> 72 us, 2.2 M 13.9 -> 13.5
      __builtin_nontemporal_store(i4{s[0], s[1], s[2], s[3]}, reinterpret_cast<i4 *>(a.slot + t));
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (t + i < a.max_tokens) a.slot[t + i] = s[i];
    }
  };
  for (int w = blockIdx.x * 4 + wave; w < fills; w += gridDim.x * 4) {
    const int t0 = w * kFill;
    // requests lo0 .. lo0 + n - 1 (what is read for stretches past the end is not used)
    int lo0 = __builtin_amdgcn_readfirstlane(a.owner[w]), n = __builtin_amdgcn_readfirstlane(a.owner[w + 1]);
    n = t0 >= end ? 0 : (t0 + kFill < end ? n : __builtin_amdgcn_readfirstlane(last)) - lo0 + 1;
    if (n == 0) lo0 = 0;
    // Four slots from the lane's token t on, all of request r; tokens past `tail` get none.
    const auto quad = [&](int r, const About &q, int t, int tail) {
      const int p = t + q.shift, c = p >> a.shift, o = p & (bt - 1), over = o + 3 - (bt - 1) - max(t + 3 - tail, 0);
      int2 id = make_int2(-1, -1);
      if (t <= tail) {
        id.x = block_at(a, r, q, c, o == 0);
        if (over > 0) id.y = block_at(a, r, q, c + 1, true);
      }
      return id;
    };
    const auto slots = [&](const About &q, int t, int tail, int2 id) {
      const int o = (t + q.shift) & (bt - 1);
      // the slot that the lane's first token has, or would have, in either block; none stays below 0 with 3 added
      const int in0 = (unsigned)id.x < (unsigned)a.NB ? (id.x << a.shift) + o : INT_MIN;
      const int in1 = (unsigned)id.y < (unsigned)a.NB ? (id.y << a.shift) + o - bt : INT_MIN;
      int s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = max((o + i < bt ? in0 : in1) + i, -1);
      if (t + 3 > tail)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = t + i > tail ? -1 : s[i];
      put(t, s);
    };
    if (n <= 1) {                                      // one request, or none
      const int4 q4 = n ? a.about[lo0] : make_int4(0, 0, 0, 0);
      const About q{q4.x, q4.y, q4.z, q4.w};
      const int tail = n ? min(t0 + kFill, end) - 1 : -1;
      int2 id[kGroups];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) id[g] = quad(lo0, q, t0 + g * 256 + lane * 4, tail);
#pragma unroll
      for (int g = 0; g < kGroups; ++g) slots(q, t0 + g * 256 + lane * 4, tail, id[g]);
      continue;
    }
    for (int i = lane; i < min(n, kList); i += 64) first[i] = a.first[lo0 + i];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    // where request lo0 + i's tokens begin, the end behind the last; a lane's four tokens lie in one request, in two, or
    // (single tokens side by side) in more, which is left for later
    const auto start = [&](int i) { return min(i >= n ? end : i < kList ? first[i] : a.first[lo0 + i], end); };
    // The request of token t, which is i's or a later one's: steps that double, then halve, so that a neighbour is found
    // at once and idle requests between, up to all of them, cost few reads (2^20 of them, all launches: 42 us; read
    // one after the other 121 ms).
    const auto owner_from = [&](int i, int t) {
      int s = 1;
      for (; i + s < n && start(i + s) <= t; s <<= 1) i += s;
      for (s >>= 1; s; s >>= 1)
        if (i + s < n && start(i + s) <= t) i += s;
      return i;
    };
    int of[kGroups], then[kGroups], stop[kGroups], stop2[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) of[g] = 0;
    for (int s = 1 << (31 - __builtin_clz(n)); s; s >>= 1)                // the last request that begins at or before t
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
        if (of[g] + s < n && start(of[g] + s) <= t0 + g * 256 + lane * 4) of[g] += s;
    int4 about[kGroups], about2[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int t = t0 + g * 256 + lane * 4;
      stop[g] = start(of[g] + 1);
      then[g] = of[g] + 1;
      stop2[g] = end;
      about[g] = about2[g] = make_int4(0, 0, 0, 0);
      if (t < end) about[g] = a.about[lo0 + of[g]];
      if (t + 3 >= stop[g] && stop[g] < end) {
        then[g] = owner_from(then[g], stop[g]);
        stop2[g] = start(then[g] + 1);
        about2[g] = a.about[lo0 + then[g]];
      }
    }
    int2 id[kGroups], id2[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int t = t0 + g * 256 + lane * 4;
      id[g] = quad(lo0 + of[g], About{about[g].x, about[g].y, about[g].z, about[g].w}, t, stop[g] - 1);
      id2[g] = make_int2(-1, -1);
      if (t + 3 >= stop[g] && stop[g] < end) {
        const About q{about2[g].x, about2[g].y, about2[g].z, about2[g].w};
        const int p = stop[g] + q.shift, c = p >> a.shift, p1 = min(t + 3, stop2[g] - 1) + q.shift;
        id2[g].x = block_at(a, lo0 + then[g], q, c, (p & (bt - 1)) == 0);
        if (p1 >> a.shift != c) id2[g].y = block_at(a, lo0 + then[g], q, c + 1, true);
      }
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const int t = t0 + g * 256 + lane * 4;
      if (t >= a.max_tokens) break;
      const int o = (t + about[g].x) & (bt - 1), c2 = (stop[g] + about2[g].x) >> a.shift;
      int s[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int p2 = t + k + about2[g].x;
        s[k] = t + k < stop[g] ? (o + k < bt ? slot_of(a, id[g].x, o + k) : slot_of(a, id[g].y, o + k - bt))
                               : slot_of(a, p2 >> a.shift == c2 ? id2[g].x : id2[g].y, p2 & (bt - 1));
        if (t + k >= end) s[k] = -1;
      }
      if (t + 3 >= stop2[g] && stop2[g] < end) {
        int i = then[g], r = -1, c = -1, block = 0, next = stop2[g];      // next: where request r's tokens end
        About q{};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (t + k < stop2[g] || t + k >= end) continue;
          if (t + k >= next || r < 0) {
            i = owner_from(i + 1, t + k);
            next = start(i + 1);
            r = lo0 + i;
            const int4 q4 = a.about[r];
            q = About{q4.x, q4.y, q4.z, q4.w};
            c = -1;
          }
          const int p = t + k + q.shift, at = p & (bt - 1);
          if (p >> a.shift != c) block = block_at(a, r, q, c = p >> a.shift, at == 0);
          s[k] = slot_of(a, block, at);
        }
      }
      put(t, s);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  // the scan's first tokens of requests that are not served lie past the end
  for (int i = blockIdx.x * 256 + threadIdx.x; i <= a.R; i += gridDim.x * 256) {
    if (i == a.R || a.first[i] > end) a.first[i] = end;
    if (i < a.R) a.length[i] = a.about[i].w;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.n_free_out = *a.n_free_in - taken;
}

// At most 2^27 blocks.
__device__ __forceinline__ int returned_of(const BlockArgs &a, int held, unsigned done) {
  return done && held >= 0 && held <= (a.MB << a.shift) ? blocks_of(held, a.shift) : 0;
}
__device__ __forceinline__ int returned(const BlockArgs &a, int r, int *held) {
  *held = a.held[r];
  return returned_of(a, *held, a.done[r]);
}

__global__ void __launch_bounds__(kChunk) k_release_sums(BlockArgs a) {
  __shared__ long long lds[kChunk / 64];
  const int r = blockIdx.x * kChunk + threadIdx.x;
  int held;
  long long B;
  scan<kChunk>(r < a.R ? returned(a, r, &held) : 0, lds, &B);
  if (threadIdx.x == 0) {
    a.sum_blocks[blockIdx.x] = B;
    if (blockIdx.x == 0) *a.n_free_in = free_count(a);
  }
}

// kGive requests a workgroup.  DIRECT: sums the requests before its own itself, where what is written is not what
// is read; otherwise whole chunks from k_release_sums, and only the requests of its own chunk, whose
// lengths this launch overwrites, from their own thread.
template <bool DIRECT>
__global__ void __launch_bounds__(kChunk) k_release(BlockArgs a) {
  constexpr int kOwn = DIRECT ? kGive : kChunk;
  __shared__ long long lds[kChunk / 64];
  __shared__ long long ends[kOwn];
  const int r0 = blockIdx.x * kOwn, r = r0 + threadIdx.x;
  const int n_free = DIRECT ? free_count(a) : *a.n_free_in;
  long long b = 0, B0, all;
  int held = 0;
  if (DIRECT && a.vec) {
#pragma unroll 8
    for (int i = threadIdx.x * 4; i < r0; i += kChunk * 4) {
      const int4 x = *reinterpret_cast<const int4 *>(a.held + i);
      const unsigned done = *reinterpret_cast<const unsigned *>(a.done + i);
      b += returned_of(a, x.x, done & 0xffu) + returned_of(a, x.y, done & 0xff00u) +
           returned_of(a, x.z, done & 0xff0000u) + returned_of(a, x.w, done & 0xff000000u);
    }
  } else if (DIRECT) {
    for (int i = threadIdx.x; i < r0; i += kChunk) b += returned(a, i, &held);
  } else {
    for (int i = threadIdx.x; i < (int)blockIdx.x; i += kChunk) b += a.sum_blocks[i];
  }
  scan<kChunk>(b, lds, &B0);
  const bool mine = threadIdx.x < kOwn && r < a.R;
  const long long own = scan<kChunk>(mine ? returned(a, r, &held) : 0, lds, &all);
  if (threadIdx.x < kOwn) ends[threadIdx.x] = own;
  __syncthreads();
  for (long long i0 = threadIdx.x; i0 < all; i0 += 4 * kChunk) {
    int id[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {                          // four ids in flight
      const long long i = i0 + k * kChunk;
      int lo = -1, hi = kOwn - 1;                          // ends[lo] <= i < ends[hi]
      while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (ends[m] <= i) lo = m; else hi = m;
      }
      const int c = (int)(i - (hi ? ends[hi - 1] : 0));
      if (i < all) id[k] = a.table[(size_t)(r0 + hi) * a.MB + c];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const long long i = i0 + k * kChunk, at = n_free + B0 + i;
      if (i < all && at < a.NB) a.free_ids[at] = id[k];
    }
  }
  if (mine) a.length[r] = a.done[r] ? 0 : held;
  if (threadIdx.x == 0 && r0 + kOwn >= a.R) *a.n_free_out = (int)min(n_free + B0 + all, (long long)a.NB);
}

struct Layout {
  size_t sum_blocks, sum_tokens, ends, n_free_in, about, owner, bytes;
};

size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

Layout layout(int R, int max_tokens) {
  Layout l;
  const size_t chunks = R > 0 ? ((size_t)R + kChunk - 1) / kChunk : 1, fills = ((size_t)max_tokens + 255) / 256;
  l.sum_blocks = 0;
  l.sum_tokens = up(chunks * 8);
  l.ends = l.sum_tokens + up(chunks * 8);
  l.n_free_in = l.ends + up(chunks * 16);
  l.about = l.n_free_in + 256;
  l.owner = l.about + up((size_t)R * 16);
  l.bytes = l.owner + up((fills + 2) * 4);
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
  if (extend && out->max_tokens > kMaxTokens) return FESTINA_ERR_UNSUPPORTED;
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
  a->ends = reinterpret_cast<int4 *>(w + l.ends);
  a->n_free_in = reinterpret_cast<int32_t *>(w + l.n_free_in);
  a->about = reinterpret_cast<int4 *>(w + l.about);
  a->owner = reinterpret_cast<int32_t *>(w + l.owner);
  return FESTINA_OK;
}

}  // namespace

extern "C" size_t festina_blocks_workspace_bytes(int32_t n_requests, int32_t max_tokens) {
  if (n_requests < 0 || n_requests > kMaxRequests || max_tokens < 0 || max_tokens > kMaxTokens) return 0;
  return layout(n_requests, max_tokens).bytes;
}

extern "C" festina_status festina_extend_blocks(const festina_kv_requests *req, festina_kv_step *out,
                                                void *workspace, size_t workspace_bytes, void *stream) {
  BlockArgs a;
  const festina_status bad = arguments(req, out, true, workspace, workspace_bytes, &a);
  if (bad != FESTINA_OK) return bad;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (a.R <= 64 && a.max_tokens <= 512) {
    k_extend_small<64><<<1, 64, 0, st>>>(a);
  } else if (a.R <= kSmall && a.max_tokens <= kSmallTokens) {
    k_extend_small<kSmall><<<1, kSmall, 0, st>>>(a);
  } else {
    const int chunks = max((a.R + kChunk - 1) / kChunk, 1);
    a.fill = a.max_tokens >= kLongFills ? kGroupsMost * 256 : 256;
    const int fills = (int)(((long long)a.max_tokens + a.fill - 1) / a.fill);
    const bool vec = (reinterpret_cast<uintptr_t>(a.slot) & 15) == 0;
    a.vec = ((reinterpret_cast<uintptr_t>(a.held) | reinterpret_cast<uintptr_t>(a.add)) & 15) == 0;
    if (a.R <= kDirect) {
      k_extend_scan<true><<<chunks, kChunk, 0, st>>>(a);
    } else {
      k_extend_sums<<<chunks, kChunk, 0, st>>>(a);
      k_extend_scan<false><<<chunks, kChunk, 0, st>>>(a);
    }
    const int grid = min(max(max((fills + 3) / 4, chunks), 1), 8192);
    const int ends = a.R <= kDirect ? chunks : 1;
    if (a.fill > 256) k_extend_fill<kGroupsMost><<<grid, 256, 0, st>>>(a, ends, fills, vec);
    else k_extend_fill<1><<<grid, 256, 0, st>>>(a, ends, fills, vec);
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
  a.vec = ((reinterpret_cast<uintptr_t>(a.held) & 15) | (reinterpret_cast<uintptr_t>(done) & 3)) == 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  // one workgroup reads everything before it writes anything; several may only where they write elsewhere
  const bool apart = a.length != a.held && a.n_free_out != a.n_free;
  if (a.R <= kGive || (a.R <= kDirect * 2 && apart)) {
    k_release<true><<<max((a.R + kGive - 1) / kGive, 1), kChunk, 0, st>>>(a);
  } else {
    const int chunks = (a.R + kChunk - 1) / kChunk;
    k_release_sums<<<chunks, kChunk, 0, st>>>(a);
    k_release<false><<<chunks, kChunk, 0, st>>>(a);
  }
  return hipGetLastError() == hipSuccess ? FESTINA_OK : FESTINA_ERR_DEVICE;
}
