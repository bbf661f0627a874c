// Selective state space scan with tree state routing, forward.
//
// Per channel c and state n, token t with predecessor p on its own root-to-token sequence:
//   delta = softplus(dt_t + bias);  h_t = exp(delta A) h_p + delta x_t B_t;  y_t = (sum_n C_t h_t + D x_t) silu(z_t).
// The state is linear in the state it starts from, so the chunks of the tree's chunk program are independent up to their
// entering states:
//   carry   every chunk that something goes on from: the state it would leave from zero, and the sum of its steps (the decay over
//           the chunk is exp(A sum delta), one exponential)
//   states  down the tree, one lane per (channel, state): entering state of every chunk
//   out     every chunk again from its entering state, with the outputs
// One lane holds one channel with all its states in registers; B and C are the same for a wave's 64 channels and come as scalar
// operands.  Nothing is shared between lanes, and everything is fp32 until the output is rounded.
//
// Bound by the vector ALU: 16 states cost an exponential (two issue slots) and four to five plain instructions each, against 8
// bytes of bf16 per token and channel.
#include <algorithm>
#include "tt_scan.h"

namespace tt {
namespace {
using namespace scan;

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
  p.group = __builtin_amdgcn_readfirstlane((int)p.cc / (a.channels / a.groups));     // a wave's channels are of one group
  return p;
}

template <typename T, int NS>
__global__ void __launch_bounds__(THREADS)
scan_carry_kernel(ScanArgs a, int blocks, float* __restrict__ local, float* __restrict__ steps) {
  const Place p = place(a, blocks);
  if (!state_is_used(a, p.chunk)) return;
  const int t0 = a.chunk_tok0[p.chunk], len = a.chunk_len[p.chunk];
  const T* x = (const T*)a.x + (int64_t)t0 * a.x_stride;
  const T* dt = (const T*)a.dt + (int64_t)t0 * a.dt_stride;
  const T* b = (const T*)a.b + (int64_t)t0 * a.b_stride + p.group * NS;
  float a2[NS], h[NS], total = 0.f;
  load_rates<NS>(a.A, p.cc, a2);
#pragma unroll
  for (int n = 0; n < NS; n++) h[n] = 0.f;
  const float bias = a.dt_bias ? a.dt_bias[p.cc] : 0.f;
  T xs[2][AHEAD], ds[2][AHEAD];
  auto request = [&](int t, T (&xv)[AHEAD], T (&dv)[AHEAD]) {
#pragma unroll
    for (int j = 0; j < AHEAD; j++) {
      const int64_t s = min(t + j, len - 1);
      xv[j] = (x + s * a.x_stride)[p.cc];
      dv[j] = (dt + s * a.dt_stride)[p.cc];
    }
  };
  auto work = [&](int t, const T (&xv)[AHEAD], const T (&dv)[AHEAD]) {
#pragma unroll
    for (int j = 0; j < AHEAD; j++) {
      if (t + j >= len) break;
      float bv[NS];
      load_uniform<T, NS>(b + (int64_t)(t + j) * a.b_stride, bv);
      const float raw = to_f(dv[j]) + bias, delta = a.use_softplus ? softplus(raw) : raw;
      const float u = delta * to_f(xv[j]);
      total += delta;
#pragma unroll
      for (int n = 0; n < NS; n++) h[n] = fmaf(ex2(delta * a2[n]), h[n], u * bv[n]);
    }
  };
  request(0, xs[0], ds[0]);
  for (int t = 0; t < len; t += 2 * AHEAD) {
    request(t + AHEAD, xs[1], ds[1]);
    work(t, xs[0], ds[0]);
    request(t + 2 * AHEAD, xs[0], ds[0]);
    work(t + AHEAD, xs[1], ds[1]);
  }
  if (!p.valid) return;
  float* out = local + (int64_t)p.chunk * NS * a.channels + p.c;
#pragma unroll
  for (int n = 0; n < NS; n++) out[(int64_t)n * a.channels] = h[n];
  steps[(int64_t)p.chunk * a.channels + p.c] = total;
}

// One lane per (state, channel) walks the chunk program.  local[chunk] is replaced by the chunk's entering state.
// What a chunk contributes does not depend on the walk, so it is requested WALK chunks ahead.
constexpr int WALK = 8;
__global__ void __launch_bounds__(THREADS)
scan_states_kernel(ScanArgs a, float* local, const float* __restrict__ steps, float* slots) {
  const int64_t width = (int64_t)a.n_state * a.channels;
  const int64_t at = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (at >= width) return;
  const int n = (int)(at / a.channels), c = (int)(at - (int64_t)n * a.channels);
  const float a2 = a.A[(int64_t)c * a.n_state + n] * LOG2E;
  const float first = a.initial_state ? a.initial_state[(int64_t)c * a.n_state + n] : 0.f;
  float s = first, add[WALK], len[WALK];
  auto request = [&](int u, float& h, float& d) {
    u = min(u, a.n_chunks - 1);
    h = local[u * width + at];
    d = steps[(int64_t)u * a.channels + c];
  };
#pragma unroll
  for (int j = 0; j < WALK; j++) request(j, add[j], len[j]);
  for (int u0 = 0; u0 < a.n_chunks; u0 += WALK) {
#pragma unroll
    for (int j = 0; j < WALK; j++) {
      const int u = u0 + j;
      if (u >= a.n_chunks) break;
      const int src = a.chunk_src[u], dst = a.chunk_dst[u], cap = a.chunk_cap ? a.chunk_cap[u] : -1;
      if (src == -1) s = first;
      else if (src >= 0) s = slots[src * width + at];
      local[u * width + at] = s;
      s = fmaf(ex2(len[j] * a2), s, add[j]);
      if (dst >= 0) slots[dst * width + at] = s;
      if (cap >= 0) a.state_out[((int64_t)cap * a.channels + c) * a.n_state + n] = s;
      if (u + WALK < a.n_chunks) request(u + WALK, add[j], len[j]);
    }
  }
}

template <typename T, int NS, bool GATED>
__global__ void __launch_bounds__(THREADS)
scan_out_kernel(ScanArgs a, int blocks, const float* __restrict__ states) {
  const Place p = place(a, blocks);
  const int t0 = a.chunk_tok0[p.chunk], len = a.chunk_len[p.chunk];
  const T* x = (const T*)a.x + (int64_t)t0 * a.x_stride;
  const T* dt = (const T*)a.dt + (int64_t)t0 * a.dt_stride;
  const T* z = GATED ? (const T*)a.z + (int64_t)t0 * a.z_stride : nullptr;
  const T* b = (const T*)a.b + (int64_t)t0 * a.b_stride + p.group * NS;
  const T* c = (const T*)a.c + (int64_t)t0 * a.c_stride + p.group * NS;
  T* y = (T*)a.y + (int64_t)t0 * a.y_stride;
  float a2[NS], h[NS];
  load_rates<NS>(a.A, p.cc, a2);
#pragma unroll
  for (int n = 0; n < NS; n++) h[n] = states[((int64_t)p.chunk * NS + n) * a.channels + p.cc];
  const float bias = a.dt_bias ? a.dt_bias[p.cc] : 0.f, skip = a.D ? a.D[p.cc] : 0.f;
  struct In { T x, dt, z; };
  In buf[2][AHEAD];
  auto request = [&](int t, In (&v)[AHEAD]) {
#pragma unroll
    for (int j = 0; j < AHEAD; j++) {
      const int64_t s = min(t + j, len - 1);
      v[j].x = (x + s * a.x_stride)[p.cc];
      v[j].dt = (dt + s * a.dt_stride)[p.cc];
      if constexpr (GATED) v[j].z = (z + s * a.z_stride)[p.cc];
    }
  };
  auto work = [&](int t, const In (&v)[AHEAD]) {
#pragma unroll
    for (int j = 0; j < AHEAD; j++) {
      if (t + j >= len) break;
      float bv[NS], cv[NS];
      load_uniform<T, NS>(b + (int64_t)(t + j) * a.b_stride, bv);
      load_uniform<T, NS>(c + (int64_t)(t + j) * a.c_stride, cv);
      const float raw = to_f(v[j].dt) + bias, delta = a.use_softplus ? softplus(raw) : raw;
      const float xv = to_f(v[j].x), u = delta * xv;
      float out = skip * xv;
#pragma unroll
      for (int n = 0; n < NS; n++) {
        h[n] = fmaf(ex2(delta * a2[n]), h[n], u * bv[n]);
        out = fmaf(cv[n], h[n], out);
      }
      if constexpr (GATED) {
        const float zv = to_f(v[j].z);
        out *= zv * sigmoid(zv);
      }
      if (p.valid) (y + (int64_t)(t + j) * a.y_stride)[p.c] = from_f<T>(out);
    }
  };
  request(0, buf[0]);
  for (int t = 0; t < len; t += 2 * AHEAD) {
    request(t + AHEAD, buf[1]);
    work(t, buf[0]);
    request(t + 2 * AHEAD, buf[0]);
    work(t + AHEAD, buf[1]);
  }
}

size_t up(size_t v) { return (v + 255) & ~(size_t)255; }

}  // namespace

size_t scan_fwd_workspace(int channels, int n_state, int n_chunks, int n_slots) {
  const size_t width = (size_t)channels * n_state * sizeof(float);
  return up(width * n_chunks) + up((size_t)channels * n_chunks * sizeof(float)) + up(width * n_slots) + 256;
}

hipError_t scan_fwd(const ScanArgs& a, hipStream_t st) {
  if (a.n_chunks == 0) return hipSuccess;
  const size_t width = (size_t)a.channels * a.n_state * sizeof(float);
  float* local = (float*)a.workspace;
  float* steps = (float*)((char*)local + up(width * a.n_chunks));
  float* slots = (float*)((char*)steps + up((size_t)a.channels * a.n_chunks * sizeof(float)));
  const int blocks = (a.channels + THREADS - 1) / THREADS;
  const unsigned grid = (unsigned)blocks * (unsigned)a.n_chunks;
  return by_type(a.bf16, a.n_state, [&](auto zero, auto ns) -> hipError_t {
    using T = decltype(zero);
    constexpr int NS = decltype(ns)::value;
    {
      KernelTimer timer(TT_KERNEL_SCAN_CARRY, st);
      scan_carry_kernel<T, NS><<<grid, THREADS, 0, st>>>(a, blocks, local, steps);
    }
    if (hipError_t e = hipGetLastError()) return e;
    {
      KernelTimer timer(TT_KERNEL_SCAN_STATES, st);
      scan_states_kernel<<<(unsigned)((NS * (int64_t)a.channels + THREADS - 1) / THREADS), THREADS, 0, st>>>(a, local, steps, slots);
    }
    if (hipError_t e = hipGetLastError()) return e;
    KernelTimer timer(TT_KERNEL_SCAN_OUT, st);
    if (a.z) scan_out_kernel<T, NS, true><<<grid, THREADS, 0, st>>>(a, blocks, local);
    else scan_out_kernel<T, NS, false><<<grid, THREADS, 0, st>>>(a, blocks, local);
    return hipGetLastError();
  });
}

}  // namespace tt
