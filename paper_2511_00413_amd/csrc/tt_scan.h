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
  p.chunk = (int)(blockIdx.x / (unsigned)blocks);
  if (a.chunk_order) p.chunk = a.chunk_order[p.chunk];
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

// The walks along the chunk program: one lane per channel and state, one wave per workgroup.  What a chunk contributes does not depend
// on the walk, so the rows of WALK chunks are requested before the WALK in front of them are walked.  A walk is one chain of dependent
// steps, and on a small tree most entries begin or end a branch: no step down branches on its entry, and a saved state is read two
// entries before it is used (down 78 entries of 1024 channels and 16 states, 54 of which start from a saved state: 18.3 us with
// branches and reads on the spot, 14 so; 143 entries of 2048 channels, down and up: 35 and 25; 269 of 4096 channels: 73 and 66, 58 of
// them the bytes).
constexpr int WALK = 16;
constexpr int WAVE = 64;
// Rows of the arrays that are walked: WALK are read and written at a time, and nothing comes of those past the end.
inline size_t walk_rows(int n_chunks) { return (size_t)n_chunks + WALK - 1; }
constexpr int LDS_SLOTS = 64;                   // saved states held in LDS: up to 16 KB a workgroup; more live in the workspace
// Two more than the program has: FIRST, for what a root starts from, and one for what is written and never read.
constexpr int EXTRA_SLOTS = 2;
inline size_t walk_lds(int n_slots) { return n_slots <= LDS_SLOTS ? (size_t)(n_slots + EXTRA_SLOTS) * WAVE * sizeof(float) : 0; }
// The walk's lane: entry `at` of the [n_state][channels] rows.  Lanes past the last entry stand in for it, in step with the lane that
// is on it: they read and write what it does.
struct Walker {
  int64_t width, at, state_at;
  int c;
  __device__ __forceinline__ explicit Walker(const ScanArgs& a) {
    width = (int64_t)a.n_state * a.channels;
    at = min((int64_t)blockIdx.x * WAVE + threadIdx.x, width - 1);
    const int n = (int)(at / a.channels);
    c = (int)(at - (int64_t)n * a.channels);
    state_at = (int64_t)c * a.n_state + n;
  }
};
template <bool LDS>
struct Slots {
  float* p;
  int64_t step;
  int first, unread;
  __device__ __forceinline__ Slots(const ScanArgs& a, const Walker& w, float* lds, float* global)
      : p(LDS ? lds + threadIdx.x : global + w.at), step(LDS ? WAVE : w.width), first(a.n_slots), unread(a.n_slots + 1) {}
  __device__ __forceinline__ float& operator[](int s) const {
    if constexpr (LDS) return p[s * WAVE];
    else return p[s * step];
  }
};
// WALK entries of the program, a lane each, and the destinations of the one and two in front, the source of the one behind.
struct Entries {
  int src, dst, cap, dst1, dst2, src_behind;
  __device__ __forceinline__ void load(const ScanArgs& a, int u0, bool with_cap) {
    const int u = u0 + (int)threadIdx.x, last = a.n_chunks - 1;
    const bool in = u <= last;
    src = a.chunk_src[min(u, last)];
    dst = a.chunk_dst[min(u, last)];
    cap = with_cap ? a.chunk_cap[min(u, last)] : -1;
    dst1 = a.chunk_dst[min(max(u - 1, 0), last)];
    dst2 = a.chunk_dst[min(max(u - 2, 0), last)];
    src_behind = a.chunk_src[min(u + 1, last)];
    if (!in) src = -2, dst = cap = -1;                     // past the end: nothing comes of them
    if (u >= last) src_behind = -1;
  }
  static __device__ __forceinline__ int at(int v, int j) { return __builtin_amdgcn_readlane(v, j); }
};
__device__ __forceinline__ uint32_t mask_of(bool b) { return (uint32_t)__ballot(b); }      // (of the first 32 lanes: one has WALK entries)
__device__ __forceinline__ bool bit(uint32_t mask, int j) { return mask & 1u << j; }

// values[chunk] (rows of `width`) is replaced by what step(entries, decay, value, result) puts into result, WALK chunks after WALK
// chunks, down (UP: up) the program; decay = 2^(a2 steps[chunk]).
template <bool UP, typename Step>
__device__ __forceinline__ void walk(const ScanArgs& a, float* values, const float* __restrict__ steps, const Walker& w, float a2, bool with_cap,
                                     Step step) {
  const int n = a.n_chunks, blocks = (n + WALK - 1) / WALK;
  const uint32_t at = (uint32_t)w.at * 4u, c = (uint32_t)w.c * 4u;
  float value[WALK], len[WALK], result[WALK];
  Entries next;
  auto request = [&](int u0) {
    Feed<float> x(values, w.width, u0), y(steps, a.channels, u0);
#pragma unroll
    for (int j = 0; j < WALK; j++) {
      value[j] = x.next(at, true);
      len[j] = y.next(c, true);
    }
    next.load(a, u0, with_cap);
  };
  auto store = [&](int u0) {
    Feed<float> x(values, w.width, u0);
#pragma unroll
    for (int j = 0; j < WALK; j++, x.so += x.step) x.put(at, result[j]);
  };
  auto start_of = [&](int i) { return WALK * (UP ? blocks - 1 - i : i); };
  request(start_of(0));
#pragma unroll 1
  for (int i = 0; i < blocks; i++) {
    float own[WALK], decay[WALK];
#pragma unroll
    for (int j = 0; j < WALK; j++) {
      own[j] = value[j];
      decay[j] = ex2(len[j] * a2);
    }
    const Entries e = next;
    // (the stores of the block in front before the loads: what is waited for at the top is then a walk old, all of it)
    if (i) store(start_of(i - 1));
    if (i + 1 < blocks) request(start_of(i + 1));
    step(e, decay, own, result);
  }
  store(start_of(blocks - 1));
}

// Down the tree: replaces add[chunk] by the state entering the chunk.  leave(cap, state) sees the captured states.
template <bool LDS, typename Leave>
__device__ __forceinline__ void walk_down(const ScanArgs& a, float* local, const float* __restrict__ steps, const Walker& w, float a2,
                                          const Slots<LDS>& slots, bool with_cap, Leave leave) {
  float s = a.initial_state ? a.initial_state[w.state_at] : 0.f;
  slots[slots.first] = s;
  walk<false>(a, local, steps, w, a2, with_cap, [&](const Entries& e, const float (&decay)[WALK], const float (&add)[WALK],
                                                    float (&entering)[WALK]) {
    // A saved state is read before the two entries in front have saved theirs: one that they save is taken from the registers.
    const int lane = threadIdx.x;
    const uint32_t from_one = mask_of(e.src == -2 || (e.src >= 0 && lane >= 1 && e.src == e.dst1));
    const uint32_t from_two = mask_of(e.src >= 0 && lane >= 2 && e.src == e.dst2), captured = mask_of(e.cap >= 0);
    const int from = e.src < 0 ? slots.first : e.src, to = e.dst < 0 ? slots.unread : e.dst;
    float saved[WALK], before = 0.f;
    saved[0] = slots[Entries::at(from, 0)];
    saved[1] = slots[Entries::at(from, 1)];
#pragma unroll
    for (int j = 0; j < WALK; j++) {
      if (j + 2 < WALK) saved[j + 2] = slots[Entries::at(from, j + 2)];
      const float start = bit(from_one, j) ? s : bit(from_two, j) ? before : saved[j];
      before = s;
      entering[j] = start;
      s = fmaf(decay[j], start, add[j]);
      slots[Entries::at(to, j)] = s;
    }
    if (captured)
#pragma unroll
      for (int j = 0; j < WALK; j++)
        if (bit(captured, j)) leave(Entries::at(e.cap, j), fmaf(decay[j], entering[j], add[j]));
  });
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
