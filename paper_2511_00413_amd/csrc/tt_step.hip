// One token per row from saved states: the causal convolution and the selective scan of a decoding step.
// Row r goes on from state index[r] (several rows may go on from the same one: branches of a tree node) and leaves its new
// state in row r of the output.  An index outside the saved states stands for the start of a sequence: zero.
// Bound by the states' bytes; a single row by the launch.
#include "tt_scan.h"

namespace tt {
namespace {
using namespace scan;


typedef float f32x4 __attribute__((ext_vector_type(4)));
template <typename T> struct alignas(4 * sizeof(T)) Four { T v[4]; };

// Rows a workgroup takes: the layer's parameters (a third of what one row moves) are read once for all of them, and their states are
// in flight together; the new states are streamed out.  256 rows of 8192 channels, 16 states: one row 43 us, four 41, streamed 34 (153
// MB, 4.5 TB/s).  Few rows go one by one, to fill the chip.
constexpr int MANY = 4;
constexpr int MANY_FROM = 32;

// Four states per lane: 16 bytes of state each, neighbouring lanes neighbouring bytes; the NS / 4 lanes of a channel add their
// parts of the output.
template <typename T, int NS, int R>
__global__ void __launch_bounds__(THREADS)
scan_step_kernel(ScanStepArgs a, int64_t row0) {
  constexpr int LANES = NS / 4;
  const int64_t first = row0 + (int64_t)blockIdx.y * R;
  const int at = blockIdx.x * THREADS + threadIdx.x;
  const int c = at / LANES, part = at % LANES;
  if (c >= a.channels) return;
  const int group = c / (a.channels / a.groups);
  const int64_t st = (int64_t)c * NS + 4 * part, width = (int64_t)a.channels * NS;
  float4 s[R];
  Four<T> b[R], o[R];
  float x[R], raw[R], gate[R];
#pragma unroll
  for (int i = 0; i < R; i++) {                  // (rows past the end are the last one again, and not stored)
    const int64_t r = min(first + i, (int64_t)a.n_rows - 1);
    const int64_t slot = a.index ? a.index[r] : r;
    s[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (slot >= 0 && slot < a.n_slots) s[i] = *(const float4*)(a.state + slot * width + st);
    b[i] = *(const Four<T>*)((const T*)a.b + r * a.b_stride + group * NS + 4 * part);
    o[i] = *(const Four<T>*)((const T*)a.c + r * a.c_stride + group * NS + 4 * part);
    x[i] = to_f(((const T*)a.x)[r * a.x_stride + c]);
    raw[i] = to_f(((const T*)a.dt)[r * a.dt_stride + c]);
    gate[i] = a.z ? to_f(((const T*)a.z)[r * a.z_stride + c]) : 0.f;
  }
  const float4 rate = *(const float4*)(a.A + st);
  const float bias = a.dt_bias ? a.dt_bias[c] : 0.f, skip = a.D ? a.D[c] : 0.f;
#pragma unroll
  for (int i = 0; i < R; i++) {
    const float delta = step_size(raw[i] + bias, a.use_softplus), u = delta * x[i], d2 = delta * LOG2E;
    s[i].x = fmaf(ex2(d2 * rate.x), s[i].x, u * to_f(b[i].v[0]));
    s[i].y = fmaf(ex2(d2 * rate.y), s[i].y, u * to_f(b[i].v[1]));
    s[i].z = fmaf(ex2(d2 * rate.z), s[i].z, u * to_f(b[i].v[2]));
    s[i].w = fmaf(ex2(d2 * rate.w), s[i].w, u * to_f(b[i].v[3]));
    float y = fmaf(s[i].x, to_f(o[i].v[0]), s[i].y * to_f(o[i].v[1])) + fmaf(s[i].z, to_f(o[i].v[2]), s[i].w * to_f(o[i].v[3]));
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) y += __shfl_xor(y, m);
    y = fmaf(skip, x[i], y);
    if (a.z) y *= gate[i] * sigmoid(gate[i]);
    const int64_t r = first + i;
    if (r < a.n_rows) {
      const f32x4 v = {s[i].x, s[i].y, s[i].z, s[i].w};
      f32x4* to = (f32x4*)(a.state_out + r * width + st);
      if constexpr (R > 1) __builtin_nontemporal_store(v, to);
      else *to = v;
      if (part == 0) ((T*)a.y)[r * a.y_stride + c] = from_f<T>(y);
    }
  }
}

// Four channels per lane; the K - 1 rows of a state are the inputs before the token, the oldest first.
template <typename T, int K, int R>
__global__ void __launch_bounds__(THREADS)
conv_step_kernel(ConvStepArgs a, int64_t row0) {
  const int64_t first = row0 + (int64_t)blockIdx.y * R;
  const int c = 4 * (blockIdx.x * THREADS + threadIdx.x);
  if (c >= a.channels) return;
  Four<T> w[R][K];
#pragma unroll
  for (int i = 0; i < R; i++) {
    const int64_t r = min(first + i, (int64_t)a.n_rows - 1);
    const int64_t slot = a.index ? a.index[r] : r;
    const bool saved = slot >= 0 && slot < a.n_slots;
#pragma unroll
    for (int j = 0; j < K - 1; j++) {
      w[i][j] = Four<T>{from_f<T>(0.f), from_f<T>(0.f), from_f<T>(0.f), from_f<T>(0.f)};
      if (saved) w[i][j] = *(const Four<T>*)((const T*)a.state + (slot * (K - 1) + j) * a.channels + c);
    }
    w[i][K - 1] = *(const Four<T>*)((const T*)a.x + r * a.x_stride + c);
  }
  float weight[4][K], bias[4];
#pragma unroll
  for (int e = 0; e < 4; e++) {
    bias[e] = a.bias ? a.bias[c + e] : 0.f;
#pragma unroll
    for (int j = 0; j < K; j++) weight[e][j] = a.weight[(int64_t)(c + e) * K + j];
  }
#pragma unroll
  for (int i = 0; i < R; i++) {
    const int64_t r = first + i;
    if (r >= a.n_rows) break;
    Four<T> y;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      float acc = bias[e];
#pragma unroll
      for (int j = 0; j < K; j++) acc = fmaf(weight[e][j], to_f(w[i][j].v[e]), acc);
      y.v[e] = from_f<T>(a.silu ? acc * sigmoid(acc) : acc);
    }
    *(Four<T>*)((T*)a.y + r * a.y_stride + c) = y;
#pragma unroll
    for (int j = 0; j < K - 1; j++) *(Four<T>*)((T*)a.state_out + (r * (K - 1) + j) * a.channels + c) = w[i][j + 1];
  }
}

constexpr int64_t ROWS = 32768;            // rows per launch (the second dimension of a grid)

}  // namespace

hipError_t scan_step(const ScanStepArgs& a, bool bf16, hipStream_t st) {
  for (int64_t row0 = 0; row0 < a.n_rows; row0 += ROWS) {
    const int64_t rows = a.n_rows - row0 < ROWS ? a.n_rows - row0 : ROWS;
    KernelTimer timer(TT_KERNEL_SCAN_STEP, st);
    const hipError_t e = by_type(bf16, a.n_state, [&](auto zero, auto ns) -> hipError_t {
      using T = decltype(zero);
      constexpr int NS = decltype(ns)::value;
      const unsigned blocks = (unsigned)(((int64_t)a.channels * (NS / 4) + THREADS - 1) / THREADS);
      if (a.n_rows >= MANY_FROM) scan_step_kernel<T, NS, MANY><<<dim3(blocks, (unsigned)((rows + MANY - 1) / MANY)), THREADS, 0, st>>>(a, row0);
      else scan_step_kernel<T, NS, 1><<<dim3(blocks, (unsigned)rows), THREADS, 0, st>>>(a, row0);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t conv_step(const ConvStepArgs& a, int kernel_size, bool bf16, hipStream_t st) {
  for (int64_t row0 = 0; row0 < a.n_rows; row0 += ROWS) {
    const int64_t rows = a.n_rows - row0 < ROWS ? a.n_rows - row0 : ROWS;
    const unsigned blocks = (unsigned)((a.channels / 4 + THREADS - 1) / THREADS);
    KernelTimer timer(TT_KERNEL_CONV_STEP, st);
    auto sized = [&](auto zero, auto k) {
      using T = decltype(zero);
      constexpr int K = decltype(k)::value;
      if (a.n_rows >= MANY_FROM) conv_step_kernel<T, K, MANY><<<dim3(blocks, (unsigned)((rows + MANY - 1) / MANY)), THREADS, 0, st>>>(a, row0);
      else conv_step_kernel<T, K, 1><<<dim3(blocks, (unsigned)rows), THREADS, 0, st>>>(a, row0);
      return hipGetLastError();
    };
    auto run = [&](auto zero) {
      if (kernel_size == 2) return sized(zero, std::integral_constant<int, 2>{});
      if (kernel_size == 3) return sized(zero, std::integral_constant<int, 3>{});
      return sized(zero, std::integral_constant<int, 4>{});
    };
    if (hipError_t e = bf16 ? run(__hip_bfloat16{}) : run(float{})) return e;
  }
  return hipSuccess;
}

}  // namespace tt
