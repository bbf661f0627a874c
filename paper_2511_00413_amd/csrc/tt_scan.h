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

// ln(1 + e) for e in [0, 1]: the logarithm of the rounded sum w = 1 + e, corrected by e / (w - 1) for what the rounding took
// (Kahan), so that small steps keep their relative precision.
__device__ __forceinline__ float log1p_unit(float e) {
  const float w = 1.f + e, d = w - 1.f;
  return d == 0.f ? e : LN2 * __builtin_amdgcn_logf(w) * (e * __builtin_amdgcn_rcpf(d));
}
__device__ __forceinline__ float softplus(float r) { return fmaxf(r, 0.f) + log1p_unit(ex2(-LOG2E * fabsf(r))); }
// its derivative, without the cancellation of 1 - exp(-softplus(r))
__device__ __forceinline__ float sigmoid(float r) {
  const float e = ex2(-LOG2E * fabsf(r)), q = __builtin_amdgcn_rcpf(1.f + e);
  return r >= 0.f ? q : e * q;
}

// A vector of NS inputs B or outputs C of one token, the same for all lanes: read through the scalar cache, so that its
// elements are scalar operands.
template <typename T, int NS>
__device__ __forceinline__ void load_uniform(const T* p, float (&v)[NS]) {
  typedef const __attribute__((address_space(4))) uint32_t* Words;
  const Words w = (Words)(uintptr_t)p;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < NS / 2; i++) {
      const uint32_t q = w[i];
      v[2 * i] = __uint_as_float(q << 16);
      v[2 * i + 1] = __uint_as_float(q & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < NS; i++) v[i] = __uint_as_float(w[i]);
  }
}

template <int NS>
__device__ __forceinline__ void load_rates(const float* A, int64_t c, float (&a2)[NS]) {      // rates in base 2
#pragma unroll
  for (int n = 0; n < NS; n++) a2[n] = A[c * NS + n] * LOG2E;
}

// Whether anything starts from the state that chunk u leaves.
__device__ __forceinline__ bool state_is_used(const ScanArgs& a, int u) {
  return a.chunk_dst[u] >= 0 || (a.chunk_cap && a.chunk_cap[u] >= 0) || (u + 1 < a.n_chunks && a.chunk_src[u + 1] == -2);
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
