// Pieces of the selective scan's kernels (tt_scan.hip, tt_scan_bwd.hip, tt_step.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <hip/hip_bf16.h>
#include <type_traits>
#include "tt_kernels.h"

namespace tt {
namespace scan {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float to_f(__hip_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(float v) { return v; }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ __hip_bfloat16 from_f<__hip_bfloat16>(float v) { return __float2bfloat16(v); }
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }

// ln(1 + e) for e in [0, 1]: the logarithm of the rounded sum w, and what its rounding took, e - (w - 1) (exact), so that small
// steps keep their relative precision.  (To first order the correction is divided by w; it is at most 2^-24, so that where w is
// not 1 to many digits the result is not small and the division does not show.)
__device__ __forceinline__ float log1p_unit(float e) {
  const float w = 1.f + e;
  return fmaf(LN2, __builtin_amdgcn_logf(w), e - (w - 1.f));
}
__device__ __forceinline__ float softplus(float r) { return fmaxf(r, 0.f) + log1p_unit(ex2(-LOG2E * fabsf(r))); }
// softplus or the value itself, by a selection (a branch here cuts the loops into pieces that the loads cannot be moved across)
__device__ __forceinline__ float step_size(float r, bool use_softplus) {
  float s = softplus(r);
  asm volatile("" : "+v"(s));
  return use_softplus ? s : r;
}
// its derivative (0 where the exponential is past fp32), without the cancellation of 1 - exp(-softplus(r))
__device__ __forceinline__ float sigmoid(float r) { return __builtin_amdgcn_rcpf(1.f + ex2(-LOG2E * r)); }

// A vector B or C of one token and group is the same for all lanes: read through the scalar cache, its elements are scalar operands.
template <typename T, int N>
struct Words {                                  // as they lie in memory: bf16 in pairs
  static constexpr int W = N * (int)sizeof(T) / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const void* p) {
    typedef const __attribute__((address_space(4))) uint32_t* Scalar;
    const Scalar q = (Scalar)(uintptr_t)p;
#pragma unroll
    for (int i = 0; i < W; i++) w[i] = q[i];
  }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (sizeof(T) == 2) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    else return __uint_as_float(w[i]);
  }
};

template <int NS>
__device__ __forceinline__ void load_rates(const float* A, int64_t c, float (&a2)[NS]) {      // rates in base 2
#pragma unroll
  for (int n = 0; n < NS; n++) a2[n] = A[c * NS + n] * LOG2E;
}

// Whether anything starts from the state that chunk u leaves.
__device__ __forceinline__ bool state_is_used(const ScanArgs& a, int u) {
  return a.chunk_dst[u] >= 0 || (a.chunk_cap && a.chunk_cap[u] >= 0) || (u + 1 < a.n_chunks && a.chunk_src[u + 1] == -2);
}

constexpr int THREADS = 256;
constexpr int AHEAD = 4;                   // tokens whose loads are in flight behind the ones worked on

// Workgroup `block` of a grid of chunks x channel blocks.
struct Place { int chunk, c; bool valid; int64_t cc; int group; };
__device__ __forceinline__ Place place(const ScanArgs& a, int blocks) {
  Place p;
  p.chunk = blockIdx.x / (unsigned)blocks;
  p.c = (int)(blockIdx.x % (unsigned)blocks) * THREADS + threadIdx.x;
  p.valid = p.c < a.channels;
  p.cc = p.valid ? p.c : a.channels - 1;
  p.group = __builtin_amdgcn_readfirstlane((int)p.cc) / (a.channels / a.groups);     // a wave's channels are of one group
  return p;
}

// Rows of a chunk, one element per lane: buffer accesses, whose address is a scalar base, the lane's 32-bit offset and a scalar row
// offset that one addition steps.  (As pointers, the multiples of every stride are worked out ahead of the loops and spilled, and
// each access costs a 64-bit vector addition.)  A row offset stays below 2^31: strides are below 2^19 elements, chunks of at most
// TT_SCAN_CHUNK_MAX = 2^10 rows.
template <typename T>
struct Feed {
  __amdgpu_buffer_rsrc_t r;
  int step, so;
  __device__ __forceinline__ Feed(const void* base, int64_t stride, int64_t row0, int row = 0)
      : r(__builtin_amdgcn_make_buffer_rsrc((char*)const_cast<void*>(base) + row0 * stride * (int64_t)sizeof(T), (short)0, -1, 0x00020000)),
        step((int)stride * (int)sizeof(T)), so(row * ((int)stride * (int)sizeof(T))) {}
  // the lane's element of this row, then on to the next row if `more`
  __device__ __forceinline__ T next(uint32_t lane_bytes, bool more) {
    T v;
    if constexpr (sizeof(T) == 2) v = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b16(r, lane_bytes, so, 0));
    else v = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(r, lane_bytes, so, 0));
    so += more ? step : 0;
    return v;
  }
  __device__ __forceinline__ void put(uint32_t lane_bytes, float f) {
    const T v = from_f<T>(f);
    if constexpr (sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, v), r, lane_bytes, so, 0);
    else __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned int, v), r, lane_bytes, so, 0);
  }
};
// vectors of rows that are the same for all lanes
template <typename T, int N>
struct UniformFeed {
  const char* p;
  int step;
  __device__ __forceinline__ UniformFeed(const void* base, int64_t stride, int64_t row, int at)
      : p((const char*)base + (row * stride + at) * (int64_t)sizeof(T)), step((int)stride * (int)sizeof(T)) {}
  __device__ __forceinline__ void next(Words<T, N>& v) { v.load(p); p += step; }
  __device__ __forceinline__ void prev(Words<T, N>& v) { v.load(p); p -= step; }
};

// Tokens 0 .. len in blocks of AHEAD, the loads of a block issued before the one in front of it is worked on.
template <typename In, typename Request, typename Work>
__device__ __forceinline__ void stream(int len, Request request, Work work) {
  In buf[2][AHEAD];
  request(0, buf[0]);
  int t = 0;
  for (; t + 2 * AHEAD <= len; t += 2 * AHEAD) {
    request(t + AHEAD, buf[1]);
#pragma unroll
    for (int j = 0; j < AHEAD; j++) work(t + j, buf[0][j]);
    request(t + 2 * AHEAD, buf[0]);
#pragma unroll
    for (int j = 0; j < AHEAD; j++) work(t + AHEAD + j, buf[1][j]);
  }
  if (t + AHEAD <= len) {
    request(t + AHEAD, buf[1]);
#pragma unroll
    for (int j = 0; j < AHEAD; j++) work(t + j, buf[0][j]);
    t += AHEAD;
#pragma unroll
    for (int j = 0; j < AHEAD; j++) buf[0][j] = buf[1][j];
  }
#pragma unroll
  for (int j = 0; j < AHEAD; j++)
    if (t + j < len) work(t + j, buf[0][j]);
}

// The walks along the chunk program (one lane per channel and state): what a chunk contributes does not depend on the walk, so a
// block of WALK chunks is requested before the one in front of it is walked, and its results are stored in one go behind it: no
// branch lies between a load and its use, where the wait for it would become a wait for everything.  The program's entries come 64
// at a time, a lane each.
constexpr int WALK = 16;
constexpr int WALK_THREADS = 256;
constexpr int LDS_SLOTS = 64;                   // saved states held in LDS: up to 64 KB a workgroup; more live in the workspace
struct Program {
  int src, dst, cap;
  __device__ __forceinline__ void load(const ScanArgs& a, int base, bool with_cap) {
    const int u = min(base + (int)(threadIdx.x & 63), a.n_chunks - 1);
    src = a.chunk_src[u];
    dst = a.chunk_dst[u];
    cap = with_cap ? a.chunk_cap[u] : -1;
  }
  static __device__ __forceinline__ int at(int v, int u) { return __builtin_amdgcn_readlane(v, u & 63); }
};
// Whether a wave of a walk has no entry at all.  In one that has some, the lanes past the last entry stand in for it, in step with the
// lane that is on it: they write what it writes.  A whole wave of such lanes would not be in step and add to the saved gradients again.
__device__ __forceinline__ bool walk_is_empty(int64_t width) {
  return (int64_t)blockIdx.x * WALK_THREADS + (int64_t)(threadIdx.x & ~63u) >= width;
}
template <bool LDS>
struct Slots {
  float* p;
  int64_t step;
  __device__ __forceinline__ Slots(float* lds, float* global, int64_t width, int64_t at)
      : p(LDS ? lds + threadIdx.x : global + at), step(LDS ? WALK_THREADS : width) {}
  __device__ __forceinline__ float& operator[](int s) const { return p[s * step]; }
};

// WALK rows of [n_chunks][width] and [n_chunks][channels] arrays from row u0 on; rows past the end are the last one again.
struct WalkRows {
  int n_chunks, channels;
  int64_t width;
  uint32_t at, c;                               // the lane's offsets in bytes
  __device__ __forceinline__ WalkRows(const ScanArgs& a, int64_t w, int64_t at_, int c_)
      : n_chunks(a.n_chunks), channels(a.channels), width(w), at((uint32_t)at_ * 4u), c((uint32_t)c_ * 4u) {}
  __device__ __forceinline__ void load(const float* values, const float* steps, int u0, float (&h)[WALK], float (&d)[WALK]) const {
    const int first = min(u0, n_chunks - 1);
    Feed<float> x(values, width, first), y(steps, channels, first);
#pragma unroll
    for (int j = 0; j < WALK; j++) {
      const bool more = u0 + j < n_chunks - 1;
      h[j] = x.next(at, more);
      d[j] = y.next(c, more);
    }
  }
  __device__ __forceinline__ void store(float* values, int u0, const float (&h)[WALK]) const {
    Feed<float> x(values, width, u0);
#pragma unroll
    for (int j = 0; j < WALK; j++, x.so += x.step)
      if (u0 + j < n_chunks) x.put(at, h[j]);
  }
};

// Down the tree: replaces add[chunk] by the state entering the chunk.  leave(cap, state) sees the captured states.
template <bool LDS, typename Leave>
__device__ __forceinline__ void walk_down(const ScanArgs& a, float* local, const float* __restrict__ steps, int64_t width, int64_t at, int c,
                                          float a2, float first, const Slots<LDS>& slots, bool with_cap, Leave leave) {
  Program prog;
  float s = first, add[2][WALK], len[2][WALK];
  const WalkRows rows(a, width, at, c);
  auto request = [&](int u0, float (&h)[WALK], float (&d)[WALK]) { rows.load(local, steps, u0, h, d); };
  auto walk = [&](int u0, const float (&h)[WALK], const float (&d)[WALK]) {
    float entering[WALK];
#pragma unroll
    for (int j = 0; j < WALK; j++) {
      const int u = u0 + j;
      if (u < a.n_chunks) {
        const int src = Program::at(prog.src, u), dst = Program::at(prog.dst, u), cap = Program::at(prog.cap, u);
        if (src == -1) s = first;
        else if (src >= 0) s = slots[src];
        entering[j] = s;
        s = fmaf(ex2(d[j] * a2), s, h[j]);
        if (dst >= 0) slots[dst] = s;
        if (cap >= 0) leave(cap, s);
      }
    }
    rows.store(local, u0, entering);
  };
  request(0, add[0], len[0]);
  for (int u0 = 0; u0 < a.n_chunks; u0 += 2 * WALK) {
    if (u0 % 64 == 0) prog.load(a, u0, with_cap);
    if (u0 + WALK < a.n_chunks) request(u0 + WALK, add[1], len[1]);
    walk(u0, add[0], len[0]);
    if (u0 + 2 * WALK < a.n_chunks) request(u0 + 2 * WALK, add[0], len[0]);
    walk(u0 + WALK, add[1], len[1]);
  }
}

template <typename F>
hipError_t by_type(bool bf16, int n_state, F f) {
  auto typed = [&](auto z) -> hipError_t {
    switch (n_state) {
      case 4: return f(z, std::integral_constant<int, 4>{});
      case 8: return f(z, std::integral_constant<int, 8>{});
      case 16: return f(z, std::integral_constant<int, 16>{});
    }
    return hipErrorInvalidValue;
  };
  return bf16 ? typed(__hip_bfloat16{}) : typed(float{});
}

}  // namespace scan
}  // namespace tt
