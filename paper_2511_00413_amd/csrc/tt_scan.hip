// Selective state space scan with tree state routing, forward.
//
// Per channel c and state n, token t with predecessor p on its own root-to-token sequence:
//   delta = softplus(dt_t + bias);  h_t = exp(delta A) h_p + delta x_t B_t;  y_t = (sum_n C_t h_t + D x_t) silu(z_t).
// The state is linear in the state it starts from, so the chunks of the tree's chunk program are independent up to their
// entering states:
//   carry   every chunk that something goes on from: the state it would leave from zero, and the sum of its steps (the decay over
//           the chunk is exp(A sum delta), one exponential)
//   states  down the tree, one lane per (channel, state): entering state of every chunk
//   out     every chunk again from its entering state, with the outputs; the longest first, if the caller says which
// One lane holds one channel with all its states in registers; B and C are the same for a wave's 64 channels and come as scalar
// operands.  Nothing is shared between lanes, and everything is fp32 until the output is rounded.
//
// Bound by the vector ALU: 16 states cost an exponential (two issue slots) and four to five plain instructions each, against 8
// bytes of bf16 per token and channel.  16406 tokens of 8192 channels: carry 188 us over 58 % of the tokens, states 26, out 405, in passes
// one after the other (619 of their 623; the first few after a pause, at a lower clock, take a sixth longer).
#include <algorithm>
#include "tt_scan.h"

namespace tt {
namespace {
using namespace scan;

template <typename T, int NS>
__global__ void __launch_bounds__(THREADS)
scan_carry_kernel(ScanArgs a, int blocks, float* __restrict__ local, float* __restrict__ steps) {
  const Place p = place(a, blocks);
  const int t0 = a.chunk_tok0[p.chunk], len = min(a.chunk_len[p.chunk], TT_SCAN_CHUNK_MAX);
  if (!state_is_used(a, p.chunk)) return;
  Feed<T> x(a.x, a.x_stride, t0), dt(a.dt, a.dt_stride, t0);
  UniformFeed<T, NS> b(a.b, a.b_stride, t0, p.group * NS);
  float a2[NS], h[NS], total = 0.f;
  load_rates<NS>(a.A, p.cc, a2);
#pragma unroll
  for (int n = 0; n < NS; n++) h[n] = 0.f;
  const float bias = a.dt_bias ? a.dt_bias[p.cc] : 0.f;
  const uint32_t off = (uint32_t)p.cc * sizeof(T);
  struct In { T x, dt; };
  stream<In>(
      len,
      [&](int t, In (&v)[AHEAD]) {
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
          const bool more = t + j < len - 1;
          v[j].x = x.next(off, more);
          v[j].dt = dt.next(off, more);
        }
      },
      [&](int, const In& v) {
        Words<T, NS> bv;
        b.next(bv);
        const float raw = to_f(v.dt) + bias, delta = step_size(raw, a.use_softplus);
        const float u = delta * to_f(v.x);
        total += delta;
#pragma unroll
        for (int n = 0; n < NS; n++) h[n] = fmaf(ex2(delta * a2[n]), h[n], u * bv[n]);
      });
  if (!p.valid) return;
  float* out = local + (int64_t)p.chunk * NS * a.channels + p.c;
#pragma unroll
  for (int n = 0; n < NS; n++) out[(int64_t)n * a.channels] = h[n];
  steps[(int64_t)p.chunk * a.channels + p.c] = total;
}

// One lane per (state, channel) walks the chunk program.  local[chunk] is replaced by the chunk's entering state.
template <bool LDS>
__global__ void __launch_bounds__(WAVE)
scan_states_kernel(ScanArgs a, float* local, const float* __restrict__ steps, float* saved) {
  extern __shared__ float lds[];
  const Walker w(a);
  walk_down<LDS>(a, local, steps, w, a.A[w.state_at] * LOG2E, Slots<LDS>(a, w, lds, saved), a.chunk_cap != nullptr,
                 [&](int cap, float s) { a.state_out[cap * w.width + w.state_at] = s; });
}

template <typename T, int NS, bool GATED>
__global__ void __launch_bounds__(THREADS)
scan_out_kernel(ScanArgs a, int blocks, const float* __restrict__ states) {
  const Place p = place(a, blocks);
  const int t0 = a.chunk_tok0[p.chunk], len = min(a.chunk_len[p.chunk], TT_SCAN_CHUNK_MAX);
  Feed<T> x(a.x, a.x_stride, t0), dt(a.dt, a.dt_stride, t0), z(a.z, a.z_stride, t0);
  UniformFeed<T, NS> b(a.b, a.b_stride, t0, p.group * NS), c(a.c, a.c_stride, t0, p.group * NS);
  Feed<T> y(a.y, a.y_stride, t0);
  float a2[NS], h[NS];
  load_rates<NS>(a.A, p.cc, a2);
#pragma unroll
  for (int n = 0; n < NS; n++) h[n] = states[((int64_t)p.chunk * NS + n) * a.channels + p.cc];
  const float bias = a.dt_bias ? a.dt_bias[p.cc] : 0.f, skip = a.D ? a.D[p.cc] : 0.f;
  const uint32_t off = (uint32_t)p.cc * sizeof(T);
  struct In { T x, dt, z; };
  stream<In>(
      len,
      [&](int t, In (&v)[AHEAD]) {
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
          const bool more = t + j < len - 1;
          v[j].x = x.next(off, more);
          v[j].dt = dt.next(off, more);
          if constexpr (GATED) v[j].z = z.next(off, more);
        }
      },
      [&](int, const In& v) {
        Words<T, NS> bv, cv;
        b.next(bv);
        c.next(cv);
        const float raw = to_f(v.dt) + bias, delta = step_size(raw, a.use_softplus);
        const float xv = to_f(v.x), u = delta * xv;
        float out = skip * xv;
#pragma unroll
        for (int n = 0; n < NS; n++) {
          h[n] = fmaf(ex2(delta * a2[n]), h[n], u * bv[n]);
          out = fmaf(cv[n], h[n], out);
        }
        if constexpr (GATED) {
          const float zv = to_f(v.z);
          out *= zv * sigmoid(zv);
        }
        if (p.valid) y.put(off, out);
        y.so += y.step;
      });
}

size_t up(size_t v) { return (v + 255) & ~(size_t)255; }

}  // namespace

size_t scan_fwd_workspace(int channels, int n_state, int n_chunks, int n_slots) {
  const size_t width = (size_t)channels * n_state * sizeof(float);
  return up(width * walk_rows(n_chunks)) + up(channels * walk_rows(n_chunks) * sizeof(float)) + up(width * (n_slots + EXTRA_SLOTS)) + 256;
}

hipError_t scan_fwd(const ScanArgs& a, hipStream_t st) {
  if (a.n_chunks == 0) return hipSuccess;
  const size_t width = (size_t)a.channels * a.n_state * sizeof(float);
  float* local = (float*)a.workspace;
  float* steps = (float*)((char*)local + up(width * walk_rows(a.n_chunks)));
  float* slots = (float*)((char*)steps + up(a.channels * walk_rows(a.n_chunks) * sizeof(float)));
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
      const unsigned walkers = (unsigned)((NS * (int64_t)a.channels + WAVE - 1) / WAVE);
      if (a.n_slots <= LDS_SLOTS) scan_states_kernel<true><<<walkers, WAVE, walk_lds(a.n_slots), st>>>(a, local, steps, slots);
      else scan_states_kernel<false><<<walkers, WAVE, walk_lds(a.n_slots), st>>>(a, local, steps, slots);
    }
    if (hipError_t e = hipGetLastError()) return e;
    KernelTimer timer(TT_KERNEL_SCAN_OUT, st);
    if (a.z) scan_out_kernel<T, NS, true><<<grid, THREADS, 0, st>>>(a, blocks, local);
    else scan_out_kernel<T, NS, false><<<grid, THREADS, 0, st>>>(a, blocks, local);
    return hipGetLastError();
  });
}

}  // namespace tt
