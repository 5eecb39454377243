// What the serving step's kernels use of HIP and of the gfx950's instructions, on the host: a workgroup's lanes are fibers
// that run one at a time, and cross-lane operations, matrix instructions and barriers are rendezvous of the lanes that
// still run (all lanes of a wave have to come to the same one).  LDS is static memory.  So the kernels' own source runs under
// the address and undefined-behaviour sanitizers, its indexes against buffers of just the size that a caller owes.
// Not modelled: memory shared between workgroups while they run, timing, rounding of the exponential.
#pragma once
#include <array>
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <type_traits>
#include <vector>
#if defined(__has_feature)
#if __has_feature(address_sanitizer)
#define EMU_ASAN 1
#include <sanitizer/common_interface_defs.h>
#include <sanitizer/asan_interface.h>
#endif
#endif

#define __global__
#define __device__
#define __host__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)

struct dim3 { unsigned x, y, z; dim3(unsigned a = 1, unsigned b = 1, unsigned c = 1) : x(a), y(b), z(c) {} };
struct int2 { int x, y; };
struct int4 { int x, y, z, w; };
struct uint2 { unsigned x, y; };
struct alignas(16) uint4 { unsigned x, y, z, w; };
struct float2 { float x, y; };
inline int2 make_int2(int a, int b) { return {a, b}; }
inline int4 make_int4(int a, int b, int c, int d) { return {a, b, c, d}; }
inline uint2 make_uint2(unsigned a, unsigned b) { return {a, b}; }
inline uint4 make_uint4(unsigned a, unsigned b, unsigned c, unsigned d) { return {a, b, c, d}; }
typedef void *hipStream_t;
typedef int hipError_t;
constexpr int hipSuccess = 0;
inline int hipGetLastError() { return 0; }
template <typename A, typename B> inline std::common_type_t<A, B> max(A a, B b) { typedef std::common_type_t<A, B> C; return (C)a > (C)b ? (C)a : (C)b; }
template <typename A, typename B> inline std::common_type_t<A, B> min(A a, B b) { typedef std::common_type_t<A, B> C; return (C)b < (C)a ? (C)b : (C)a; }

// Saves the callee's registers and the stack pointer at *from and goes on where `to` was left (x86-64).
extern "C" void emu_switch(void **from, void *to);
asm(R"(
.text
.weak emu_switch
.type emu_switch, @function
emu_switch:
  pushq %rbp
  pushq %rbx
  pushq %r12
  pushq %r13
  pushq %r14
  pushq %r15
  movq %rsp, (%rdi)
  movq %rsi, %rsp
  popq %r15
  popq %r14
  popq %r13
  popq %r12
  popq %rbx
  popq %rbp
  ret
.size emu_switch, .-emu_switch
)");

namespace emu {
constexpr int kStack = 192 << 10;
struct Lane {
  void *at = nullptr;
  char *stack = nullptr;
  bool done = true;
  int wait = 0;                 // 0 runs, 1 at a wave operation, 2 at a barrier
  const char *what = "";
  unsigned count = 0;           // wave operations so far
  void *fake = nullptr;
};
struct Slot { alignas(16) unsigned char b[128]; };   // what a lane brings: two, since a lane may be one operation ahead
inline void *main_at;
inline std::vector<Lane> lanes;
inline Slot slots[1024][2];
inline int cur, live, size;
inline std::function<void()> body;
inline const void *main_stack; inline size_t main_size;
inline dim3 tid, bid, gdim, bdim;

inline void to_main(bool dying = false) {
  Lane &l = lanes[cur];
#ifdef EMU_ASAN
  __sanitizer_start_switch_fiber(dying ? nullptr : &l.fake, main_stack, main_size);
#endif
  emu_switch(&l.at, main_at);
#ifdef EMU_ASAN
  __sanitizer_finish_switch_fiber(l.fake, &main_stack, &main_size);
#endif
}
inline void entry() {
#ifdef EMU_ASAN
  __sanitizer_finish_switch_fiber(nullptr, &main_stack, &main_size);
#endif
  body();
  lanes[cur].done = true;
  to_main(true);
}
inline void resume(int i) {
  cur = i;
  tid = dim3(i, 0, 0);
#ifdef EMU_ASAN
  void *fake;
  __sanitizer_start_switch_fiber(&fake, lanes[i].stack, kStack);
#endif
  emu_switch(&main_at, lanes[i].at);
#ifdef EMU_ASAN
  __sanitizer_finish_switch_fiber(fake, nullptr, nullptr);
#endif
}
inline void wait(int kind, const char *what) {
  Lane &l = lanes[cur];
  l.wait = kind;
  l.what = what;
  to_main();
}
inline void fail(const char *m) { printf("EMU: %s\n", m); fflush(stdout); abort(); }

inline void run_group(int n) {
  if ((int)lanes.size() < n) lanes.resize(1024);
  size = n;
  for (int i = 0; i < n; ++i) {
    Lane &l = lanes[i];
    if (!l.stack) l.stack = (char *)malloc(kStack);
    // six registers, then where to go, as if called (the return address at 8 past a multiple of 16)
    void **top = (void **)(((uintptr_t)l.stack + kStack - 64) & ~(uintptr_t)15) + 2;
    *--top = nullptr;
    *--top = (void *)entry;
    for (int k = 0; k < 6; ++k) *--top = nullptr;
    l.at = top;
    l.done = false;
    l.wait = 0;
    l.count = 0;
  }
  int left = n;
  while (left) {
    bool moved = false;
    // waves in an order that changes, lanes of a wave one after the other
    static unsigned seed = 1;
    const int waves = (n + 63) / 64;
    seed = seed * 1664525u + 1013904223u;
    const int w0 = (seed >> 16) % waves;
    for (int k = 0; k < waves; ++k) {
      const int w = (w0 + k) % waves, lo = w * 64, hi = std::min(n, lo + 64);
      for (int i = lo; i < hi; ++i)
        if (!lanes[i].done && lanes[i].wait == 0) {
          resume(i);
          moved = true;
          if (lanes[i].done) --left;
        }
      // a wave operation that all of the wave's running lanes have come to
      const char *what = nullptr;
      bool all = true, any = false;
      int lead = lo;
      for (int i = lo; i < hi; ++i)
        if (!lanes[i].done) {
          if (lanes[i].wait != 1) { all = false; continue; }
          any = true;
          if (!what) what = lanes[i].what, lead = i;
          else if (strcmp(what, lanes[i].what) || lanes[i].count != lanes[lead].count) { printf("%s / %s\n", what, lanes[i].what); fail("lanes at different wave operations"); }
        }
      if (all && any) {
        moved = true;
        for (int i = lo; i < hi; ++i) lanes[i].wait = 0;
      }
    }
    bool all = left > 0;
    for (int i = 0; i < n; ++i) if (!lanes[i].done && lanes[i].wait != 2) all = false;
    if (all) {
      moved = true;
      for (int i = 0; i < n; ++i) lanes[i].wait = 0;
    }
    if (!moved && left) fail("no lane can move");
  }
}
template <typename F> void launch(F f, dim3 grid, int block) {
  body = f;
  gdim = grid;
  bdim = dim3(block, 1, 1);
  for (unsigned y = 0; y < grid.y; ++y)
    for (unsigned x = 0; x < grid.x; ++x) {
      bid = dim3(x, y, 0);
      run_group(block);
    }
}
// The value that each lane of this lane's wave has brought, and whether it did.
template <typename T> struct All {
  int base, par;
  unsigned c;
  T at(int l) const { T v; memcpy(&v, slots[base + l][par].b, sizeof(T)); return v; }
  bool has(int l) const { return base + l < size && lanes[base + l].count > c; }
};
template <typename T> inline All<T> exchange(const T &v, const char *what) {
  static_assert(sizeof(T) <= sizeof(Slot::b), "");
  const int me = cur;
  const unsigned c = lanes[me].count++;
  memcpy(slots[me][c & 1].b, &v, sizeof(T));
  const int base = me & ~63;
  wait(1, what);
  return All<T>{base, (int)(c & 1), c};
}
}  // namespace emu

#define threadIdx emu::tid
#define blockIdx emu::bid
#define gridDim emu::gdim
#define blockDim emu::bdim
inline void __syncthreads() { emu::wait(2, "syncthreads"); }
inline void emu_wave(const char *w) { emu::exchange<int>(0, w); }
#define __builtin_amdgcn_s_barrier() emu::wait(2, "barrier")
#define __builtin_amdgcn_wave_barrier() emu_wave("wave barrier")
inline void emu_fence(const char *scope) { if (!strcmp(scope, "wavefront")) emu_wave("fence"); }
#define __builtin_amdgcn_fence(order, scope, ...) emu_fence(scope)
#define __builtin_amdgcn_sched_barrier(x)
#define __builtin_amdgcn_sched_group_barrier(a, b, c)

// A lane that has left counts as not there (its bit is 0).  Lanes present at an exchange are those not done before it.
inline unsigned long long __ballot(bool p) {
  const auto a = emu::exchange<int>(p ? 1 : 0, "ballot");
  unsigned long long m = 0;
  for (int l = 0; l < 64; ++l)
    if (a.has(l) && a.at(l)) m |= 1ull << l;
  return m;
}
inline int __any(bool p) { return __ballot(p) != 0; }
template <typename T> inline T __shfl(T v, int l) { const auto a = emu::exchange(v, "shfl"); return a.has(l & 63) ? a.at(l & 63) : v; }
template <typename T> inline T __shfl_xor(T v, int d) { const int l = (emu::cur & 63) ^ d; const auto a = emu::exchange(v, "shfl_xor"); return a.has(l) ? a.at(l) : v; }
template <typename T> inline T __shfl_up(T v, int d) { const int l = (emu::cur & 63) - d; const auto a = emu::exchange(v, "shfl_up"); return l >= 0 ? a.at(l) : v; }
inline int emu_first(int v) {
  const auto a = emu::exchange(v, "readfirstlane");
  for (int l = 0; l < 64; ++l) if (a.has(l)) return a.at(l);
  return v;
}
#define __builtin_amdgcn_readfirstlane(v) emu_first((int)(v))
inline int emu_readlane(int v, int l) { const auto a = emu::exchange(v, "readlane"); return a.at(l); }
#define __builtin_amdgcn_readlane(v, l) emu_readlane(v, l)

struct emu_pair { unsigned v[2]; unsigned operator[](int i) const { return v[i]; } };
// The swaps exchange halves of two registers: first[32..63] with second[0..31]; of 16: odd rows of the first with even
// rows of the second.
inline emu_pair emu_swap(unsigned x, unsigned y, int d) {
  struct P { unsigned x, y; };
  const int me = emu::cur & 63;
  const auto a = emu::exchange(P{x, y}, "permlane swap");
  emu_pair r;
  if (me & d) { r.v[0] = a.at(me ^ d).y; r.v[1] = y; }
  else { r.v[0] = x; r.v[1] = a.at(me ^ d).x; }
  return r;
}
#define __builtin_amdgcn_permlane32_swap(a, b, c, d) emu_swap(a, b, 32)
#define __builtin_amdgcn_permlane16_swap(a, b, c, d) emu_swap(a, b, 16)

inline float __uint_as_float(unsigned x) { float f; memcpy(&f, &x, 4); return f; }
inline unsigned __float_as_uint(float x) { unsigned f; memcpy(&f, &x, 4); return f; }
inline float emu_flush(float x) { return std::fpclassify(x) == FP_SUBNORMAL ? 0.f : x; }
#define __builtin_amdgcn_exp2f(x) emu_flush(exp2f(x))
#define __builtin_amdgcn_logf(x) log2f(x)
#define __builtin_amdgcn_rcpf(x) (1.f / (x))

inline float emu_e4m3(unsigned c) {
  const int e = (c >> 3) & 15, f = c & 7;
  const float s = c & 0x80 ? -1.f : 1.f;
  if ((c & 0x7f) == 0x7f) return __builtin_nanf("");
  return s * (e == 0 ? f * 0x1p-9f : ldexpf(1.f + f / 8.f, e - 7));
}
typedef __bf16 emu_bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 emu_bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 emu_h2 __attribute__((ext_vector_type(2)));
typedef _Float16 emu_h8 __attribute__((ext_vector_type(8)));
typedef float emu_f2 __attribute__((ext_vector_type(2)));
typedef float emu_f4 __attribute__((ext_vector_type(4)));
typedef float emu_f16 __attribute__((ext_vector_type(16)));
inline emu_bf2 emu_cvt_bf(int c, float s, bool hi) { const unsigned u = (unsigned)c >> (hi ? 16 : 0); return emu_bf2{(__bf16)(emu_e4m3(u & 255) * s), (__bf16)(emu_e4m3(u >> 8 & 255) * s)}; }
inline emu_h2 emu_cvt_h(int c, float s, bool hi) { const unsigned u = (unsigned)c >> (hi ? 16 : 0); return emu_h2{(_Float16)(emu_e4m3(u & 255) * s), (_Float16)(emu_e4m3(u >> 8 & 255) * s)}; }
inline emu_f2 emu_cvt_f(int c, bool hi) { const unsigned u = (unsigned)c >> (hi ? 16 : 0); return emu_f2{emu_e4m3(u & 255), emu_e4m3(u >> 8 & 255)}; }
#define __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8 emu_cvt_bf
#define __builtin_amdgcn_cvt_scalef32_pk_f16_fp8 emu_cvt_h
#define __builtin_amdgcn_cvt_pk_f32_fp8 emu_cvt_f
inline unsigned emu_enc(float x) {
  if (x != x) return 0x7f;
  const unsigned s = std::signbit(x) ? 0x80 : 0;
  const float a = std::min(std::fabs(x), 448.f);
  if (std::fabs(x) > 464.f) return s | 0x7f;
  int e; frexpf(a, &e);
  e = a == 0 ? -6 : std::max(e - 1, -6);
  return s | ((e + 6) * 8 + (unsigned)std::nearbyintf(ldexpf(a, 3 - e)));      // ties to even, into the next power where full
}
inline int emu_cvt_pk(float a, float b, int old, bool hi) { const unsigned w = emu_enc(a) | emu_enc(b) << 8; return hi ? (old & 0xffff) | (int)(w << 16) : (int)((old & 0xffff0000) | w); }
#define __builtin_amdgcn_cvt_pk_fp8_f32 emu_cvt_pk
inline unsigned emu_perm(unsigned a, unsigned b, unsigned s) {
  const unsigned long long v = (unsigned long long)a << 32 | b;
  unsigned r = 0;
  for (int i = 0; i < 4; ++i) { const unsigned k = s >> (8 * i) & 255; if (k > 7) emu::fail("perm"); r |= (unsigned)(v >> (8 * k) & 255) << (8 * i); }
  return r;
}
#define __builtin_amdgcn_perm emu_perm

// 16 x 16 x 32: a lane holds row l % 16 of A (column of B), k = 8 (l / 16) + j; of the result column l % 16, rows 4 (l / 16) + i.
template <typename V> inline emu_f4 emu_mfma16(V a, V b, emu_f4 c) {
  struct P { V a, b; };
  const auto x = emu::exchange(P{a, b}, "mfma16");
  const int l = emu::cur & 63, n = l & 15;
  for (int i = 0; i < 4; ++i) {
    const int m = (l >> 4) * 4 + i;
    float s = 0;
    for (int g = 0; g < 4; ++g) {
      const V p = x.at(g * 16 + m).a, q = x.at(g * 16 + n).b;
      for (int j = 0; j < 8; ++j) s += (float)p[j] * (float)q[j];
    }
    c[i] += s;
  }
  return c;
}
template <typename V> inline emu_f16 emu_mfma32(V a, V b, emu_f16 c) {
  struct P { V a, b; };
  const auto x = emu::exchange(P{a, b}, "mfma32");
  const int l = emu::cur & 63, n = l & 31, h = l >> 5;
  for (int i = 0; i < 16; ++i) {
    const int m = (i >> 2) * 8 + h * 4 + (i & 3);
    float s = 0;
    for (int g = 0; g < 2; ++g) {
      const V p = x.at(g * 32 + m).a, q = x.at(g * 32 + n).b;
      for (int j = 0; j < 8; ++j) s += (float)p[j] * (float)q[j];
    }
    c[i] += s;
  }
  return c;
}
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) emu_mfma16<emu_bf8>(a, b, c)
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, x, y, z) emu_mfma16<emu_h8>(a, b, c)
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) emu_mfma32<emu_bf8>(a, b, c)
#define __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, x, y, z) emu_mfma32<emu_h8>(a, b, c)
template <typename T> inline void atomicMax(T *p, T v) { if (v > *p) *p = v; }
