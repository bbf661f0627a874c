// One token per row from saved states: the causal convolution and the selective scan of a decoding step.
// Row r goes on from state index[r] (several rows may go on from the same one: branches of a tree node) and leaves its new
// state in row r of the output.  An index outside the saved states stands for the start of a sequence: zero.
// Bound by the states' bytes; a single row by the launch.
#include "tt_scan.h"

namespace tt {
namespace {
using namespace scan;


template <typename T> struct alignas(4 * sizeof(T)) Four { T v[4]; };

// Four states per lane: 16 bytes of state each, neighbouring lanes neighbouring bytes; the NS / 4 lanes of a channel add their
// parts of the output.
template <typename T, int NS>
__global__ void __launch_bounds__(THREADS)
scan_step_kernel(ScanStepArgs a, int64_t row0) {
  constexpr int LANES = NS / 4;
  const int64_t r = row0 + blockIdx.y;
  const int at = blockIdx.x * THREADS + threadIdx.x;
  const int c = at / LANES, part = at % LANES;
  if (c >= a.channels) return;
  const int64_t slot = a.index ? a.index[r] : r;
  const int group = c / (a.channels / a.groups);
  const int64_t st = (int64_t)c * NS + 4 * part;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (slot >= 0 && slot < a.n_slots) s = *(const float4*)(a.state + slot * a.channels * NS + st);
  const float4 rate = *(const float4*)(a.A + st);
  const Four<T> b = *(const Four<T>*)((const T*)a.b + r * a.b_stride + group * NS + 4 * part);
  const Four<T> o = *(const Four<T>*)((const T*)a.c + r * a.c_stride + group * NS + 4 * part);
  const float x = to_f(((const T*)a.x)[r * a.x_stride + c]);
  const float raw = to_f(((const T*)a.dt)[r * a.dt_stride + c]) + (a.dt_bias ? a.dt_bias[c] : 0.f);
  const float gate = a.z ? to_f(((const T*)a.z)[r * a.z_stride + c]) : 0.f;
  const float delta = a.use_softplus ? softplus(raw) : raw, u = delta * x, d2 = delta * LOG2E;
  s.x = fmaf(ex2(d2 * rate.x), s.x, u * to_f(b.v[0]));
  s.y = fmaf(ex2(d2 * rate.y), s.y, u * to_f(b.v[1]));
  s.z = fmaf(ex2(d2 * rate.z), s.z, u * to_f(b.v[2]));
  s.w = fmaf(ex2(d2 * rate.w), s.w, u * to_f(b.v[3]));
  *(float4*)(a.state_out + r * a.channels * NS + st) = s;
  float y = fmaf(s.x, to_f(o.v[0]), s.y * to_f(o.v[1])) + fmaf(s.z, to_f(o.v[2]), s.w * to_f(o.v[3]));
#pragma unroll
  for (int m = 1; m < LANES; m <<= 1) y += __shfl_xor(y, m);
  if (part) return;
  if (a.D) y = fmaf(a.D[c], x, y);
  if (a.z) y *= gate * sigmoid(gate);
  ((T*)a.y)[r * a.y_stride + c] = from_f<T>(y);
}

// Four channels per lane; the K - 1 rows of a state are the inputs before the token, the oldest first.
template <typename T, int K>
__global__ void __launch_bounds__(THREADS)
conv_step_kernel(ConvStepArgs a, int64_t row0) {
  const int64_t r = row0 + blockIdx.y;
  const int c = 4 * (blockIdx.x * THREADS + threadIdx.x);
  if (c >= a.channels) return;
  const int64_t slot = a.index ? a.index[r] : r;
  const bool saved = slot >= 0 && slot < a.n_slots;
  Four<T> w[K];
#pragma unroll
  for (int j = 0; j < K - 1; j++) {
    if (saved) w[j] = *(const Four<T>*)((const T*)a.state + (slot * (K - 1) + j) * a.channels + c);
    else
      for (int i = 0; i < 4; i++) w[j].v[i] = from_f<T>(0.f);
  }
  w[K - 1] = *(const Four<T>*)((const T*)a.x + r * a.x_stride + c);
  Four<T> y;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    float acc = a.bias ? a.bias[c + i] : 0.f;
#pragma unroll
    for (int j = 0; j < K; j++) acc = fmaf(a.weight[(int64_t)(c + i) * K + j], to_f(w[j].v[i]), acc);
    y.v[i] = from_f<T>(a.silu ? acc * sigmoid(acc) : acc);
  }
  *(Four<T>*)((T*)a.y + r * a.y_stride + c) = y;
#pragma unroll
  for (int j = 0; j < K - 1; j++) *(Four<T>*)((T*)a.state_out + (r * (K - 1) + j) * a.channels + c) = w[j + 1];
}

constexpr int64_t ROWS = 32768;            // rows per launch (the second dimension of a grid)

}  // namespace

hipError_t scan_step(const ScanStepArgs& a, bool bf16, hipStream_t st) {
  for (int64_t row0 = 0; row0 < a.n_rows; row0 += ROWS) {
    const unsigned rows = (unsigned)(a.n_rows - row0 < ROWS ? a.n_rows - row0 : ROWS);
    KernelTimer timer(TT_KERNEL_SCAN_STEP, st);
    const hipError_t e = by_type(bf16, a.n_state, [&](auto zero, auto ns) -> hipError_t {
      constexpr int NS = decltype(ns)::value;
      const dim3 grid((unsigned)(((int64_t)a.channels * (NS / 4) + THREADS - 1) / THREADS), rows);
      scan_step_kernel<decltype(zero), NS><<<grid, THREADS, 0, st>>>(a, row0);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t conv_step(const ConvStepArgs& a, int kernel_size, bool bf16, hipStream_t st) {
  for (int64_t row0 = 0; row0 < a.n_rows; row0 += ROWS) {
    const unsigned rows = (unsigned)(a.n_rows - row0 < ROWS ? a.n_rows - row0 : ROWS);
    const dim3 grid((unsigned)((a.channels / 4 + THREADS - 1) / THREADS), rows);
    KernelTimer timer(TT_KERNEL_CONV_STEP, st);
    auto run = [&](auto zero) {
      using T = decltype(zero);
      if (kernel_size == 2) conv_step_kernel<T, 2><<<grid, THREADS, 0, st>>>(a, row0);
      else if (kernel_size == 3) conv_step_kernel<T, 3><<<grid, THREADS, 0, st>>>(a, row0);
      else conv_step_kernel<T, 4><<<grid, THREADS, 0, st>>>(a, row0);
      return hipGetLastError();
    };
    if (hipError_t e = bf16 ? run(__hip_bfloat16{}) : run(float{})) return e;
  }
  return hipSuccess;
}

}  // namespace tt
