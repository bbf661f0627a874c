// Log-probability of given tokens with the entropy and the most probable alternatives, and the gradient of the first two.
//
// Per row of logits z, in powers of two (x = z log2 e) against a whole number r just above the maximum of x (by what its product
// rounds, at most one below it):
//   s = sum 2^(x - r),  u = sum 2^(x - r) (x - r);
//   lse = ln 2 (r + log2 s),  logp = ln 2 ((x_y - r) - log2 s),  entropy = -sum p ln p = ln 2 (log2 s - u / s),
// all in one pass over the row: when r becomes r', s becomes s f and u becomes f (u + s (r - r')), f = 2^(r - r').  r being whole, x - r
// is one fused multiply-add with a single rounding, and the differences lose nothing.  Gradient of d_logp logp + d_entropy entropy:
//   dz_v = d_logp ([v = y] - p_v) - d_entropy p_v (ln p_v + entropy).
//
// Top alternatives without a second pass: in the same pass every thread leaves the maximum of each four of its vectors in LDS.  The
// k-th largest of the threads' own maxima is a lower bound of the k-th largest entry (k threads hold an entry that large), so only the
// vectors that reach it are read again: a little more than k times four.  Keys are 64 bits -- the value in an order of whole numbers
// above the complement of the index -- so no two are equal, ties go to the lowest index, and the order in which candidates are
// collected does not matter.  Where more candidates tie at the bound than the list holds, the row is read again once per alternative.
//
// Bound by HBM, every logit being read once: 4096 rows of 151936 in bf16 188 us (6.6 TB/s), their gradient 400 us (6.2 TB/s).  With
// alternatives the vector ALU is 89 % busy: 8191 rows of 32003, five, 103 us (5.1 TB/s; 125 some milliseconds into passes without a
// pause, when the clock is lower).  Few rows are cut into parts for one workgroup each, joined by a second launch.
#include <hip/hip_runtime.h>
#include <algorithm>
#include <type_traits>
#include <hip/hip_bf16.h>
#include "tt_kernels.h"

namespace tt {
namespace {

constexpr int THREADS = 256;
constexpr int WAVES = THREADS / 64;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr int LIST = 1024;                 // candidates held in LDS
constexpr int ROUNDS = 4;                  // a thread's vectors per entry of the maxima kept in LDS: 4 bytes per 64 of the row
constexpr int PART_VECS_MAX = 32768;       // 32 KB of them
constexpr int64_t LAUNCH_GROUPS = 1 << 22; // workgroups per launch: a dimension holds less than 2^32 work-items

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float ex2(float x) { return __builtin_amdgcn_exp2f(x); }     // arguments <= 1: what flushes to 0 is 0 in a sum

// r comes from the rounded product, x - r holds the exact one: what the rounding took, half a step of the largest x, is added to every
// exponent.  Within +-2^24 that is at most one.  (Unbounded it is hundreds at masks of -1e10, whose exponentials overflow.)  So r starts
// at START: logits below that, masks, add nothing and never set it; and a row whose r ends up past +-EXTREME, masked throughout or far
// from zero as a whole, is done again by far_row.  A term far below r is 0 in s and, its exponent cut at FAR, a zero in u as well.
// NaN passes the maxima and stays in s.
struct Stat { float r, s, u; };
constexpr float START = -0x1p24f, EXTREME = 0x1p23f, FAR = -300.f;

__device__ __forceinline__ void raise(Stat& st, float r) {
  const float d = st.r - r, f = ex2(d);
  st.u = f * (st.u + st.s * fmaxf(d, FAR));
  st.s *= f;
  st.r = r;
}
// N logits whose largest is `most`
template <int N>
__device__ __forceinline__ void add(Stat& st, const float (&z)[N], float most) {
  const float top = most * LOG2E;
  if (top > st.r) raise(st, ceilf(top));
  float x[N], e[N], u = 0.f;
#pragma unroll
  for (int i = 0; i < N; i++) {
    x[i] = fmaf(z[i], LOG2E, -st.r);
    e[i] = ex2(x[i]);
    st.s += e[i];
    u = fmaf(e[i], x[i], u);
  }
  if (u != u) {                              // 0 times -inf (or NaN, which stays): few vectors of few rows
    u = 0.f;
#pragma unroll
    for (int i = 0; i < N; i++) u = fmaf(e[i], fmaxf(x[i], FAR), u);
  }
  st.u += u;
}

template <typename T> struct Row;
template <> struct Row<__hip_bfloat16> {
  static constexpr int EPV = 8;
  static __device__ __forceinline__ void unpack(const u32x4& v, float (&z)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; i++) { z[2 * i] = __uint_as_float(w[i] << 16); z[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&g)[8]) {
    f32x8 f;
#pragma unroll
    for (int e = 0; e < 8; e++) f[e] = g[e];
    return __builtin_bit_cast(u32x4, __builtin_convertvector(f, bf16x8));              // round to nearest even
  }
  static __device__ __forceinline__ float at(const __hip_bfloat16* p, int64_t i) { return __bfloat162float(p[i]); }
  static __device__ __forceinline__ void put(__hip_bfloat16* p, int64_t i, float g) { p[i] = __float2bfloat16(g); }
};
template <> struct Row<float> {
  static constexpr int EPV = 4;
  static __device__ __forceinline__ void unpack(const u32x4& v, float (&z)[4]) {
    z[0] = __uint_as_float(v.x); z[1] = __uint_as_float(v.y); z[2] = __uint_as_float(v.z); z[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ u32x4 pack(const float (&g)[4]) {
    u32x4 o;
    o.x = __float_as_uint(g[0]); o.y = __float_as_uint(g[1]); o.z = __float_as_uint(g[2]); o.w = __float_as_uint(g[3]);
    return o;
  }
  static __device__ __forceinline__ float at(const float* p, int64_t i) { return p[i]; }
  static __device__ __forceinline__ void put(float* p, int64_t i, float g) { p[i] = g; }
};

// Values as unsigned numbers of the same order; NaN counts as -inf, -0 as +0.
__device__ __forceinline__ uint32_t order_of(float z) {
  z = z == z ? z + 0.f : -INFINITY;
  const uint32_t b = __float_as_uint(z);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
typedef unsigned long long Key;           // never 0
__device__ __forceinline__ Key key_of(float z, int index) { return (Key)order_of(z) << 32 | (uint32_t)~index; }

// lane ^ 1, ^ 2, mirrored in eight, ^ 8 (in sixteen)
template <int CTRL>
__device__ __forceinline__ float dpp(float v) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true)); }
constexpr int XOR1 = 0xb1, XOR2 = 0x4e, HALF_MIRROR = 0x141, ROR8 = 0x128;
template <typename Op>
__device__ __forceinline__ float wave_all(float v, Op op) {       // over the wave
  v = op(v, dpp<XOR1>(v));
  v = op(v, dpp<XOR2>(v));
  v = op(v, dpp<HALF_MIRROR>(v));
  v = op(v, dpp<ROR8>(v));
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

struct Shared {
  Stat part[WAVES];
  uint32_t lane_max[THREADS];
  uint32_t bound;
  int count;
  Key best[WAVES];
  Key last;
  alignas(16) Key list[LIST];
};

// The workgroup's sums from the threads': raised to the wave's maximum and added, then the same for the waves.
__device__ Stat join(Stat (&part)[WAVES], Stat st) {
  raise(st, wave_all(st.r, [](float a, float b) { return fmaxf(a, b); }));
  st.s = wave_all(st.s, [](float a, float b) { return a + b; });
  st.u = wave_all(st.u, [](float a, float b) { return a + b; });
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = st;
  __syncthreads();
  Stat all = {part[0].r, 0.f, 0.f};
  for (int w = 1; w < WAVES; w++) all.r = fmaxf(all.r, part[w].r);
  for (int w = 0; w < WAVES; w++) {
    Stat p = part[w];
    raise(p, all.r);
    all.s += p.s;
    all.u += p.u;
  }
  return all;
}

// What a row's outputs are made of: ln p of a logit is ln 2 ((x - r) - log2 s), or, for a row of extreme logits, (z - m) - ln s.
struct Result {
  bool far;
  float ref, log_s, entropy;                 // r or m; log2 s or ln s
  __device__ __forceinline__ float lse() const { return far ? ref + log_s : LN2 * (ref + log_s); }
  __device__ __forceinline__ float logp(float z) const {
    if (far) return (z - ref) - log_s;
    if (!(fabsf(z) < EXTREME)) return z - lse();          // a masked logit: one rounding, where its x may overflow
    return LN2 * (fmaf(z, LOG2E, -ref) - log_s);
  }
};

// f(z) for a thread's entries of a row: whole vectors, four in flight, behind a scalar head.
template <typename T, typename F>
__device__ __forceinline__ void each_entry(const T* row, int vocab, F f) {
  constexpr int EPV = Row<T>::EPV;
  const int t = threadIdx.x;
  const int head = min((int)(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(T)), vocab), nvec = (vocab - head) / EPV;
  const u32x4* vp = reinterpret_cast<const u32x4*>(row + head);
  auto vec = [&](const u32x4& v) {
    float z[EPV];
    Row<T>::unpack(v, z);
#pragma unroll
    for (int e = 0; e < EPV; e++) f(z[e]);
  };
  for (int e = t; e < head; e += THREADS) f(Row<T>::at(row, e));
  int i = t;
  for (; i + 3 * THREADS < nvec; i += 4 * THREADS) {
    const u32x4 a = vp[i], b = vp[i + THREADS], c = vp[i + 2 * THREADS], d = vp[i + 3 * THREADS];
    vec(a); vec(b); vec(c); vec(d);
  }
  for (; i < nvec; i += THREADS) vec(vp[i]);
  for (int e = head + nvec * EPV + t; e < vocab; e += THREADS) f(Row<T>::at(row, e));
}

// The sums of a row of extreme logits against its maximum, differences taken before they are scaled: two more passes.
template <typename T>
__device__ Result far_row(Stat (&part)[WAVES], const T* row, int vocab) {
  const int t = threadIdx.x;
  float m = -INFINITY;
  each_entry(row, vocab, [&](float z) { m = fmaxf(m, z); });
  m = wave_all(m, [](float a, float b) { return fmaxf(a, b); });
  __syncthreads();                           // (the sums in part have been read)
  if ((t & 63) == 0) part[t >> 6].r = m;
  __syncthreads();
  for (int w = 0; w < WAVES; w++) m = fmaxf(m, part[w].r);
  Stat st = {0.f, 0.f, 0.f};
  each_entry(row, vocab, [&](float z) {
    const float d = z - m, p = ex2(d * LOG2E);
    st.s += p;
    st.u = fmaf(p, fmaxf(d, FAR), st.u);
  });
  __syncthreads();
  st = join(part, st);
  const float ln_s = LN2 * log2f(st.s);
  return {true, m, ln_s, ln_s - st.u / st.s};
}

template <typename T>
__device__ __forceinline__ Result result_of(Stat (&part)[WAVES], const Stat& all, const T* row, int vocab) {
  if (!(fabsf(all.r) < EXTREME)) return far_row(part, row, vocab);          // (all threads hold the same r)
  const float log_s = log2f(all.s);
  return {false, all.r, log_s, LN2 * (log_s - all.u / all.s)};
}

// Bound from the threads' largest entries (order_of; 0 = none): the largest multiple T of 2^16 that at least k of them reach.
// Found bit by bit by the first wave; the lower halves are left out, which keeps T a lower bound (and loses nothing in bf16).
__device__ void find_bound(Shared& sh, uint32_t mine, int k) {
  const int t = threadIdx.x;
  sh.lane_max[t] = mine;
  if (t == 0) sh.count = 0;
  __syncthreads();
  if (t < 64) {
    uint32_t v[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; w++) v[w] = sh.lane_max[w * 64 + t];
    uint32_t T = 0;
    for (int bit = 31; bit >= 16; bit--) {
      const uint32_t c = T | 1u << bit;
      int n = 0;
#pragma unroll
      for (int w = 0; w < WAVES; w++) n += __popcll(__ballot(v[w] >= c));
      if (n >= k) T = c;
    }
    if (t == 0) sh.bound = T;
  }
  __syncthreads();
}

__device__ __forceinline__ void offer(Shared& sh, Key key) {
  const int at = atomicAdd(&sh.count, 1);
  if (at < LIST) sh.list[at] = key;
}

// The k largest keys in descending order, given to emit(rank, key) by one thread each.  offer_all offers every key whose value
// reaches sh.bound; largest_below(limit) is the thread's largest key below limit (0 = none), for the rows that need the long way.
// Called by all threads behind find_bound.
template <typename OfferAll, typename LargestBelow, typename Emit>
__device__ void select_top(Shared& sh, int k, OfferAll offer_all, LargestBelow largest_below, Emit emit) {
  const int t = threadIdx.x;
  offer_all();
  __syncthreads();
  const int n = sh.count;
  if (n >= k && n <= LIST) {
    for (int c = t; c < n; c += THREADS) {                 // a key's place is the number of larger ones
      const Key key = sh.list[c];
      int rank = 0;
      for (int o = 0; o < n; o++) rank += sh.list[o] > key;
      if (rank < k) emit(rank, key);
    }
    return;
  }
  Key limit = ~(Key)0;
  for (int r = 0; r < k; r++) {
    Key best = largest_below(limit);
    for (int o = 32; o > 0; o >>= 1) {
      const Key other = __shfl_xor(best, o);
      best = other > best ? other : best;
    }
    if ((t & 63) == 0) sh.best[t >> 6] = best;
    __syncthreads();
    if (t == 0) {
      for (int w = 1; w < WAVES; w++) best = sh.best[w] > best ? sh.best[w] : best;
      sh.last = best;
      emit(r, best);
    }
    __syncthreads();
    limit = sh.last;
  }
}

struct Outs {
  float *logp, *entropy, *lse;
  int32_t* top_index;
  float* top_logp;
};
struct Partial { Stat st; };

// Part `part` of a row: whole 16-byte vectors [part * part_vecs, ..) behind the head that lies in front of the first 16-byte
// boundary; the head goes with the first part, what is left behind the last vector with the last.
// parts == 1: the row's results; otherwise its sums and k keys go to `partial` and `keys`.
template <typename T, bool TOP>
__global__ void __launch_bounds__(THREADS)
entropy_rows_kernel(int64_t row0, int vocab, const T* __restrict__ logits, int64_t row_stride, const int32_t* __restrict__ target,
                    int k, int parts, int part_vecs, Outs out, Partial* __restrict__ partial, Key* __restrict__ keys) {
  constexpr int EPV = Row<T>::EPV;
  __shared__ Shared sh;
  extern __shared__ float four_max[];
  const int64_t r = row0 + (parts == 1 ? (int64_t)blockIdx.x : (int64_t)(blockIdx.x / (unsigned)parts));
  const int part = parts == 1 ? 0 : (int)(blockIdx.x % (unsigned)parts);
  const T* row = logits + r * row_stride;
  const int t = threadIdx.x;
  const int head = min((int)(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(T)), vocab);
  const int nvec = (vocab - head) / EPV;
  const int v0 = part * part_vecs, v1 = part == parts - 1 ? nvec : min(nvec, v0 + part_vecs);
  const int tail0 = head + nvec * EPV;
  const bool first = part == 0, last = part == parts - 1;
  const u32x4* vp = reinterpret_cast<const u32x4*>(row + head);

  Stat st = {START, 0.f, 0.f};
  [[maybe_unused]] float top = -INFINITY;                  // largest of the thread's entries
  auto single = [&](int e) {
    const float z[1] = {Row<T>::at(row, e)};
    if (TOP) top = fmaxf(top, z[0]);
    add<1>(st, z, z[0]);
  };
  auto vec = [&](const u32x4& v) {
    float z[EPV];
    Row<T>::unpack(v, z);
    float vm = z[0];
#pragma unroll
    for (int e = 1; e < EPV; e++) vm = fmaxf(vm, z[e]);
    add<EPV>(st, z, vm);
    return vm;
  };
  [[maybe_unused]] auto keep = [&](int r4, float m) {
    top = fmaxf(top, m);
    four_max[r4 / ROUNDS * THREADS + t] = m;
  };
  if (first) for (int e = t; e < head; e += THREADS) single(e);
  // Rounds of 256 vectors, four in flight; of the last four, what lies past the end stands in as -inf.
  const int rounds = (v1 - v0 + THREADS - 1) / THREADS;
  int r4 = 0;
  for (; r4 + 4 < rounds; r4 += 4) {
    const int i = v0 + r4 * THREADS + t;
    const u32x4 a = __builtin_nontemporal_load(vp + i);
    const u32x4 b = __builtin_nontemporal_load(vp + i + THREADS);
    const u32x4 c = __builtin_nontemporal_load(vp + i + 2 * THREADS);
    const u32x4 d = __builtin_nontemporal_load(vp + i + 3 * THREADS);
    const float m0 = vec(a), m1 = vec(b), m2 = vec(c), m3 = vec(d);
    if constexpr (TOP) keep(r4, fmaxf(fmaxf(m0, m1), fmaxf(m2, m3)));
  }
  if (r4 < rounds) {
    const uint32_t none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;      // -inf
    u32x4 v[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      v[j] = u32x4{none, none, none, none};
      const int i = v0 + (r4 + j) * THREADS + t;
      if (i < v1) v[j] = __builtin_nontemporal_load(vp + i);
    }
    float m = -INFINITY;
#pragma unroll
    for (int j = 0; j < 4; j++)
      if (r4 + j < rounds) m = fmaxf(m, vec(v[j]));
    if constexpr (TOP) keep(r4, m);
  }
  if (last) for (int e = tail0 + t; e < vocab; e += THREADS) single(e);

  const Stat all = join(sh.part, st);
  Result res{};
  if (parts == 1) {
    res = result_of(sh.part, all, row, vocab);
    if (t == 0) {
      const int y = target[r];
      const bool used = y >= 0 && y < vocab;
      out.logp[r] = used ? res.logp(Row<T>::at(row, y)) : 0.f;
      out.entropy[r] = used ? res.entropy : 0.f;
      if (out.lse) out.lse[r] = res.lse();
    }
  } else if (t == 0) {
    partial[r * parts + part].st = all;
  }
  if constexpr (TOP) {
    const bool any = (v0 + t < v1) || (first && t < head) || (last && tail0 + t < vocab);
    find_bound(sh, any ? order_of(top) : 0u, k);
    const uint32_t bound = sh.bound;
    auto offer_all = [&]() {
      auto try_one = [&](int e) {
        const float z = Row<T>::at(row, e);
        if (order_of(z) >= bound) offer(sh, key_of(z, e));
      };
      if (first) for (int e = t; e < head; e += THREADS) try_one(e);
      if (last) for (int e = tail0 + t; e < vocab; e += THREADS) try_one(e);
      const float floor_value = value_of(bound);              // (bounds below -inf's give NaN, which passes everything)
      for (int r4 = 0; r4 < rounds; r4 += ROUNDS) {
        if (four_max[r4 / ROUNDS * THREADS + t] < floor_value) continue;
        const int j0 = v0 + r4 * THREADS + t;
        const uint32_t none = sizeof(T) == 2 ? 0xff80ff80u : 0xff800000u;
        u32x4 v[ROUNDS];
#pragma unroll
        for (int q = 0; q < ROUNDS; q++) {
          v[q] = u32x4{none, none, none, none};
          if (j0 + q * THREADS < v1) v[q] = vp[j0 + q * THREADS];
        }
#pragma unroll 1
        for (int q = 0; q < ROUNDS; q++) {
          const int j = j0 + q * THREADS;
          float z[EPV];
          Row<T>::unpack(q == 0 ? v[0] : q == 1 ? v[1] : q == 2 ? v[2] : v[3], z);
          float m = z[0];
#pragma unroll
          for (int e = 1; e < EPV; e++) m = fmaxf(m, z[e]);
          if (j >= v1 || m < floor_value) continue;
#pragma unroll
          for (int e = 0; e < EPV; e++)
            if (order_of(z[e]) >= bound) offer(sh, key_of(z[e], head + j * EPV + e));
        }
      }
    };
    auto largest_below = [&](Key limit) {
      Key best = 0;
      auto see = [&](float z, int e) {
        const Key key = key_of(z, e);
        if (key < limit && key > best) best = key;
      };
      if (first) for (int e = t; e < head; e += THREADS) see(Row<T>::at(row, e), e);
      if (last) for (int e = tail0 + t; e < vocab; e += THREADS) see(Row<T>::at(row, e), e);
      for (int j = v0 + t; j < v1; j += THREADS) {
        float z[EPV];
        Row<T>::unpack(vp[j], z);
#pragma unroll
        for (int e = 0; e < EPV; e++) see(z[e], head + j * EPV + e);
      }
      return best;
    };
    auto emit = [&](int rank, Key key) {
      if (parts == 1) {
        out.top_index[r * k + rank] = (int32_t)~(uint32_t)key;
        out.top_logp[r * k + rank] = res.logp(value_of((uint32_t)(key >> 32)));
      } else {
        keys[(r * parts + part) * k + rank] = key;          // 0 where the part has fewer than k entries
      }
    };
    select_top(sh, k, offer_all, largest_below, emit);
  }
}

// One workgroup per row: the parts' sums in their order, and the k largest of their keys.
template <typename T, bool TOP>
__global__ void __launch_bounds__(THREADS)
entropy_join_kernel(int64_t row0, int vocab, const T* __restrict__ logits, int64_t row_stride, const int32_t* __restrict__ target,
                    int k, int parts, Outs out, const Partial* __restrict__ partial, const Key* __restrict__ keys) {
  __shared__ Shared sh;
  const int64_t r = row0 + blockIdx.x;
  const int t = threadIdx.x;
  Stat st = {START, 0.f, 0.f};
  for (int p = t; p < parts; p += THREADS) {
    Stat q = partial[r * parts + p].st;
    const float m = fmaxf(st.r, q.r);
    raise(st, m);
    raise(q, m);
    st.s += q.s;
    st.u += q.u;
  }
  const Stat all = join(sh.part, st);
  const T* row = logits + r * row_stride;
  const Result res = result_of(sh.part, all, row, vocab);
  if (t == 0) {
    const int y = target[r];
    const bool used = y >= 0 && y < vocab;
    out.logp[r] = used ? res.logp(Row<T>::at(row, y)) : 0.f;
    out.entropy[r] = used ? res.entropy : 0.f;
    if (out.lse) out.lse[r] = res.lse();
  }
  if constexpr (TOP) {
    const Key* mine = keys + r * parts * k;
    const int n = parts * k;
    uint32_t top = 0;
    for (int c = t; c < n; c += THREADS) top = max(top, (uint32_t)(mine[c] >> 32));
    find_bound(sh, top, k);
    const Key bound = max((Key)sh.bound << 32, (Key)1);      // 0 = no key
    select_top(
        sh, k, [&]() { for (int c = t; c < n; c += THREADS) if (mine[c] >= bound) offer(sh, mine[c]); },
        [&](Key limit) {
          Key best = 0;
          for (int c = t; c < n; c += THREADS) if (mine[c] < limit && mine[c] > best) best = mine[c];
          return best;
        },
        [&](int rank, Key key) {
          out.top_index[r * k + rank] = (int32_t)~(uint32_t)key;
          out.top_logp[r * k + rank] = res.logp(value_of((uint32_t)(key >> 32)));
        });
  }
}

// ---- gradient ------------------------------------------------------------------------------------
// A row is cut into parts of 16 KB, one workgroup each, four vectors in flight per thread.
// Gradient and logits rows the same distance from a 16-byte boundary go in vectors behind a scalar head.
// p = exp(z - lse) is off by what lse is rounded by, some |lse| 2^-23: 10^-4 of it at SUM_AGAIN (a twentieth of half a step in bf16), all
// of it where ln s does not reach lse's last digit.  In rows from there on, which no trained model has, and rows without a distribution
// the workgroup of one part adds up p once more and takes the whole row: lse lies within 33 of the exact one (half its last digit,
// or, where ln s does not reach that, ln s itself), so the sum stays in range, and its logarithm is what lse is off by.  4096 rows of
// 32003 in fp32: 242 us instead of 189 (their forward, three reads, 234 instead of 87).
constexpr float SUM_AGAIN = 1024.f;
template <typename T>
__global__ void __launch_bounds__(THREADS)
entropy_bwd_kernel(int64_t row0, int vocab, const T* logits, int64_t row_stride, const int32_t* __restrict__ target,
                   const float* __restrict__ lse_in, const float* __restrict__ entropy, const float* __restrict__ d_logp,
                   const float* __restrict__ d_entropy, T* dlogits, int64_t out_stride, int parts, int part_vecs) {
  constexpr int EPV = Row<T>::EPV;
  const int64_t r = row0 + (int64_t)(blockIdx.x / (unsigned)parts);
  int part = (int)(blockIdx.x % (unsigned)parts);
  const T* row = logits + r * row_stride;
  T* out = dlogits + r * out_stride;
  const int t = threadIdx.x;
  const int y = target[r];
  const bool used = y >= 0 && y < vocab;
  const float a = used && d_logp ? d_logp[r] : 0.f, b = used && d_entropy ? d_entropy[r] : 0.f;
  const float lse = used ? lse_in[r] : 0.f;
  const float c = a + b * (used ? entropy[r] : 0.f);
  __shared__ Stat sums[WAVES];
  float off = 0.f;                          // what lse is off by
  if (used && !(fabsf(lse) < SUM_AGAIN)) {
    if (part != (int)(r / 8 % parts)) return;               // (workgroups go round the eight XCDs: always the same part may be one of them)
    float s = 0.f;
    each_entry(row, vocab, [&](float z) { s += ex2((z - lse) * LOG2E); });
    off = LN2 * log2f(join(sums, {0.f, s, 0.f}).s);           // (the barrier in join: the row may be written from here on)
    part = 0;
    parts = 1;
  }
  const bool vec_ok = ((reinterpret_cast<uintptr_t>(row) ^ reinterpret_cast<uintptr_t>(out)) & 15) == 0;
  const int head = vec_ok ? min((int)(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(T)), vocab) : 0;
  const int nvec = vec_ok ? (vocab - head) / EPV : 0;
  const u32x4* vp = reinterpret_cast<const u32x4*>(row + head);
  u32x4* op = reinterpret_cast<u32x4*>(out + head);
  // -p (a + b (ln p + entropy)); far below the maximum p is 0 and the cut keeps the other factor finite
  auto grad1 = [&](float z) {
    const float d = (z - lse) - off;
    return -ex2(d * LOG2E) * fmaf(b, fmaxf(d, FAR), c);
  };
  auto grad = [&](const u32x4& v, int i) {
    float z[EPV];
    Row<T>::unpack(v, z);
#pragma unroll
    for (int e = 0; e < EPV; e++) z[e] = grad1(z[e]);
    const int base = head + i * EPV;
    if ((unsigned)(y - base) < (unsigned)EPV) {
#pragma unroll
      for (int e = 0; e < EPV; e++) z[e] += base + e == y ? a : 0.f;
    }
    return Row<T>::pack(z);
  };
  const int v1 = part == parts - 1 ? nvec : min(nvec, (part + 1) * part_vecs);
  int i = part * part_vecs + t;
  if (!used) {                              // an ignored row: zero, whatever its logits are
    const u32x4 zero = {0, 0, 0, 0};
    for (; i < v1; i += THREADS) __builtin_nontemporal_store(zero, op + i);
  } else {
    for (; i + 3 * THREADS < v1; i += 4 * THREADS) {
      const u32x4 q0 = __builtin_nontemporal_load(vp + i);
      const u32x4 q1 = __builtin_nontemporal_load(vp + i + THREADS);
      const u32x4 q2 = __builtin_nontemporal_load(vp + i + 2 * THREADS);
      const u32x4 q3 = __builtin_nontemporal_load(vp + i + 3 * THREADS);
      __builtin_nontemporal_store(grad(q0, i), op + i);
      __builtin_nontemporal_store(grad(q1, i + THREADS), op + i + THREADS);
      __builtin_nontemporal_store(grad(q2, i + 2 * THREADS), op + i + 2 * THREADS);
      __builtin_nontemporal_store(grad(q3, i + 3 * THREADS), op + i + 3 * THREADS);
    }
    for (; i < v1; i += THREADS) __builtin_nontemporal_store(grad(__builtin_nontemporal_load(vp + i), i), op + i);
  }
  auto single = [&](int e) { Row<T>::put(out, e, used ? grad1(Row<T>::at(row, e)) + (e == y ? a : 0.f) : 0.f); };
  if (part == 0) for (int e = t; e < head; e += THREADS) single(e);
  // behind the last vector (rows of unequal distance: everything), shared by the parts
  for (int e = head + nvec * EPV + part * THREADS + t; e < vocab; e += parts * THREADS) single(e);
}

// Parts per row: one, unless the row is longer than the kept maxima have room for or there are too few rows to fill the chip;
// then as many as make about 512 workgroups, of at least 512 vectors (two per thread) each.  A part is whole rounds of 256 vectors.
struct Split { int parts, part_vecs; };
Split split_rows(int64_t n_rows, int vocab, bool bf16) {
  const int64_t nvec = std::max(vocab / (bf16 ? 8 : 4), 1);
  int64_t parts = (nvec + PART_VECS_MAX - 1) / PART_VECS_MAX;
  if (n_rows < 512) parts = std::max(parts, std::min((int64_t)512 / std::max(n_rows, (int64_t)1), nvec / 512));
  if (parts <= 1) return {1, (int)nvec};
  const int64_t part_vecs = ((nvec + parts - 1) / parts + THREADS - 1) / THREADS * THREADS;
  return {(int)((nvec + part_vecs - 1) / part_vecs), (int)part_vecs};
}

}  // namespace

size_t logprob_entropy_workspace(int64_t n_rows, int vocab, bool bf16, int top_k) {
  const int parts = split_rows(n_rows, vocab, bf16).parts;
  if (parts == 1) return 256;
  const size_t sums = ((size_t)n_rows * parts * sizeof(Partial) + 255) & ~(size_t)255;
  return sums + (size_t)n_rows * parts * top_k * sizeof(Key) + 256;
}

hipError_t logprob_entropy(int64_t n_rows, int vocab, bool bf16, const void* logits, int64_t row_stride, const int32_t* target,
                           int top_k, float* logp, float* entropy, float* lse, int32_t* top_index, float* top_logp, void* workspace,
                           hipStream_t st) {
  if (n_rows == 0) return hipSuccess;
  const auto [parts, part_vecs] = split_rows(n_rows, vocab, bf16);
  const size_t lds = top_k ? ((size_t)part_vecs / (ROUNDS * THREADS) + 1) * THREADS * sizeof(float) : 0;
  Partial* partial = (Partial*)workspace;
  Key* keys = (Key*)((char*)workspace + (((size_t)n_rows * parts * sizeof(Partial) + 255) & ~(size_t)255));
  const Outs out{logp, entropy, lse, top_index, top_logp};
  const int64_t rows_per_launch = std::max(LAUNCH_GROUPS / parts, (int64_t)1);
  for (int64_t row0 = 0; row0 < n_rows; row0 += rows_per_launch) {
    const int64_t rows = std::min(rows_per_launch, n_rows - row0);
    auto run = [&, parts = parts, part_vecs = part_vecs](auto* z) -> hipError_t {
      using T = std::remove_const_t<std::remove_pointer_t<decltype(z)>>;
      {
        KernelTimer timer(TT_KERNEL_ENTROPY_ROWS, st);
        if (top_k)
          entropy_rows_kernel<T, true><<<(unsigned)(rows * parts), THREADS, lds, st>>>(row0, vocab, z, row_stride, target, top_k, parts,
                                                                                       part_vecs, out, partial, keys);
        else
          entropy_rows_kernel<T, false><<<(unsigned)(rows * parts), THREADS, 0, st>>>(row0, vocab, z, row_stride, target, 0, parts,
                                                                                      part_vecs, out, partial, keys);
      }
      if (hipError_t e = hipGetLastError()) return e;
      if (parts == 1) return hipSuccess;
      KernelTimer timer(TT_KERNEL_ENTROPY_JOIN, st);
      if (top_k)
        entropy_join_kernel<T, true><<<(unsigned)rows, THREADS, 0, st>>>(row0, vocab, z, row_stride, target, top_k, parts, out, partial, keys);
      else
        entropy_join_kernel<T, false><<<(unsigned)rows, THREADS, 0, st>>>(row0, vocab, z, row_stride, target, 0, parts, out, partial, keys);
      return hipGetLastError();
    };
    if (hipError_t e = bf16 ? run((const __hip_bfloat16*)logits) : run((const float*)logits)) return e;
  }
  return hipSuccess;
}

hipError_t logprob_entropy_bwd(int64_t n_rows, int vocab, bool bf16, const void* logits, int64_t row_stride, const int32_t* target,
                               const float* lse, const float* entropy, const float* d_logp, const float* d_entropy, void* dlogits,
                               int64_t out_stride, hipStream_t st) {
  if (n_rows == 0) return hipSuccess;
  const int nvec = vocab / (bf16 ? 8 : 4);
  const int part_vecs = 4 * THREADS;
  const int parts = std::max(1, (nvec + part_vecs - 1) / part_vecs);
  const int64_t rows_per_launch = std::max(LAUNCH_GROUPS / parts, (int64_t)1);
  for (int64_t row0 = 0; row0 < n_rows; row0 += rows_per_launch) {
    const int64_t rows = std::min(rows_per_launch, n_rows - row0);
    KernelTimer timer(TT_KERNEL_ENTROPY_BWD, st);
    if (bf16)
      entropy_bwd_kernel<__hip_bfloat16><<<(unsigned)(rows * parts), THREADS, 0, st>>>(
          row0, vocab, (const __hip_bfloat16*)logits, row_stride, target, lse, entropy, d_logp, d_entropy, (__hip_bfloat16*)dlogits,
          out_stride, parts, part_vecs);
    else
      entropy_bwd_kernel<float><<<(unsigned)(rows * parts), THREADS, 0, st>>>(
          row0, vocab, (const float*)logits, row_stride, target, lse, entropy, d_logp, d_entropy, (float*)dlogits, out_stride, parts,
          part_vecs);
    if (hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace tt
