// Selective state space scan with tree state routing, backward.
//
// With a = exp(delta A), u = delta x, dy' = dy silu(z) and G_t the gradient of h_t (its own token's C_t dy'_t and what every
// successor on any branch sends back, a G):
//   dC_t = sum_c h dy'          dB_t = sum_c G u            du = sum_n G B           q = G a h_p
//   ddelta = x du + sum_n A q   dA = sum_t delta q          dx = delta du + D dy'    ddt = ddelta sigmoid(dt + bias)
// Chunks are independent up to the state entering them and the gradient of the state leaving them:
//   ends    per chunk, one pass: the state it leaves from zero, the sum of its steps, and the gradient of its entering state
//           that its own outputs give, sum_t (prod_{s<=t} a_s) C_t dy'_t
//   states  down the tree, then up again, one lane per (channel, state): entering states, gradients of the leaving states
//   grads   every chunk once more with the two known: eight tokens at a time from the last, their states worked out again from
//           the state in front of them, which a first pass over the chunk left in LDS
//   sums    of what the waves and strips of chunks left: dB, dC over the channels, dA, dD and the bias over the strips
// No atomics: every sum has a fixed order.  One lane holds one channel; the sums over a wave's 64 channels for the 2 NS entries of
// dB and dC are taken together, the lanes halving the entries they keep at every step (70 instructions for 32 sums).
//
// Bound by the vector ALU, as the forward.
#include <algorithm>
#include "tt_scan.h"

namespace tt {
namespace {
using namespace scan;

constexpr int THREADS = 256;
constexpr int WAVE = 64;
constexpr int SUB = 8;                          // tokens whose states are held in registers
constexpr int CHUNK = TT_GDN_CHUNK;
constexpr int SAVED = CHUNK / SUB - 1;          // states in front of the second and later groups of a chunk

// ---- ends ----------------------------------------------------------------------------------------
template <typename T, int NS, bool GATED>
__global__ void __launch_bounds__(THREADS)
scan_ends_kernel(ScanArgs a, int blocks, float* __restrict__ local, float* __restrict__ steps, float* __restrict__ back) {
  constexpr int AHEAD = 4;
  const int chunk = blockIdx.x / (unsigned)blocks;
  const int ch = (int)(blockIdx.x % (unsigned)blocks) * THREADS + threadIdx.x;
  const int64_t cc = min(ch, a.channels - 1);
  const int group = __builtin_amdgcn_readfirstlane((int)cc / (a.channels / a.groups));
  if (!state_is_used(a, chunk) && a.chunk_src[chunk] == -1 && !a.d_initial_state) return;
  const int t0 = a.chunk_tok0[chunk], len = min(a.chunk_len[chunk], CHUNK);
  const T* x = (const T*)a.x + (int64_t)t0 * a.x_stride;
  const T* dt = (const T*)a.dt + (int64_t)t0 * a.dt_stride;
  const T* z = GATED ? (const T*)a.z + (int64_t)t0 * a.z_stride : nullptr;
  const T* dy = (const T*)a.dy + (int64_t)t0 * a.dy_stride;
  const T* b = (const T*)a.b + (int64_t)t0 * a.b_stride + group * NS;
  const T* c = (const T*)a.c + (int64_t)t0 * a.c_stride + group * NS;
  float a2[NS], h[NS], along[NS], r[NS], total = 0.f;
  load_rates<NS>(a.A, cc, a2);
#pragma unroll
  for (int n = 0; n < NS; n++) { h[n] = 0.f; along[n] = 1.f; r[n] = 0.f; }
  const float bias = a.dt_bias ? a.dt_bias[cc] : 0.f;
  struct In { T x, dt, z, dy; };
  In buf[2][AHEAD];
  auto request = [&](int t, In (&v)[AHEAD]) {
#pragma unroll
    for (int j = 0; j < AHEAD; j++) {
      const int64_t s = min(t + j, len - 1);
      v[j].x = (x + s * a.x_stride)[cc];
      v[j].dt = (dt + s * a.dt_stride)[cc];
      if constexpr (GATED) v[j].z = (z + s * a.z_stride)[cc];
      v[j].dy = (dy + s * a.dy_stride)[cc];
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
      const float u = delta * to_f(v[j].x);
      float g = to_f(v[j].dy);
      if constexpr (GATED) {
        const float zv = to_f(v[j].z);
        g *= zv * sigmoid(zv);
      }
      total += delta;
#pragma unroll
      for (int n = 0; n < NS; n++) {
        const float d = ex2(delta * a2[n]);
        h[n] = fmaf(d, h[n], u * bv[n]);
        along[n] *= d;
        r[n] = fmaf(along[n], g * cv[n], r[n]);
      }
    }
  };
  request(0, buf[0]);
  for (int t = 0; t < len; t += 2 * AHEAD) {
    request(t + AHEAD, buf[1]);
    work(t, buf[0]);
    request(t + 2 * AHEAD, buf[0]);
    work(t + AHEAD, buf[1]);
  }
  if (ch >= a.channels) return;
  const int64_t at = (int64_t)chunk * NS * a.channels + ch;
#pragma unroll
  for (int n = 0; n < NS; n++) {
    local[at + (int64_t)n * a.channels] = h[n];
    back[at + (int64_t)n * a.channels] = r[n];
  }
  steps[(int64_t)chunk * a.channels + ch] = total;
}

// ---- states --------------------------------------------------------------------------------------
// local[chunk]: entering state; back[chunk]: gradient of the leaving state.
constexpr int WALK = 8;
__global__ void __launch_bounds__(THREADS)
scan_bwd_states_kernel(ScanArgs a, float* local, float* back, const float* __restrict__ steps, float* slots) {
  const int64_t width = (int64_t)a.n_state * a.channels;
  const int64_t at = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (at >= width) return;
  const int n = (int)(at / a.channels), c = (int)(at - (int64_t)n * a.channels);
  const float a2 = a.A[(int64_t)c * a.n_state + n] * LOG2E;
  const float first = a.initial_state ? a.initial_state[(int64_t)c * a.n_state + n] : 0.f;
  if (a.n_chunks == 0) {
    a.d_initial_state[(int64_t)c * a.n_state + n] = 0.f;
    return;
  }
  {
    float s = first, add[WALK], len[WALK];
    auto request = [&](int u, float& h, float& d) {
      h = local[u * width + at];
      d = steps[(int64_t)u * a.channels + c];
    };
#pragma unroll
    for (int j = 0; j < WALK; j++) request(min(j, a.n_chunks - 1), add[j], len[j]);
    for (int u0 = 0; u0 < a.n_chunks; u0 += WALK) {
#pragma unroll
      for (int j = 0; j < WALK; j++) {
        const int u = u0 + j;
        if (u >= a.n_chunks) break;
        const int src = a.chunk_src[u], dst = a.chunk_dst[u];
        if (src == -1) s = first;
        else if (src >= 0) s = slots[src * width + at];
        local[u * width + at] = s;
        s = fmaf(ex2(len[j] * a2), s, add[j]);
        if (dst >= 0) slots[dst * width + at] = s;
        if (u + WALK < a.n_chunks) request(u + WALK, add[j], len[j]);
      }
    }
  }
  for (int s = 0; s < a.n_slots; s++) slots[s * width + at] = 0.f;          // from here on: gradients of the saved states
  float sent = 0.f, d_first = 0.f, add[WALK], len[WALK];
  int nxt_src = -1;                                                          // of the chunk behind
  auto request = [&](int u, float& r, float& d) {
    r = back[u * width + at];
    d = steps[(int64_t)u * a.channels + c];
  };
#pragma unroll
  for (int j = 0; j < WALK; j++) request(max(a.n_chunks - 1 - j, 0), add[j], len[j]);
  for (int u0 = a.n_chunks - 1; u0 >= 0; u0 -= WALK) {
#pragma unroll
    for (int j = 0; j < WALK; j++) {
      const int u = u0 - j;
      if (u < 0) break;
      const int src = a.chunk_src[u], dst = a.chunk_dst[u], cap = a.d_state_out ? a.chunk_cap[u] : -1;
      float g = nxt_src == -2 ? sent : 0.f;
      bool used = nxt_src == -2;
      if (dst >= 0) { g += slots[dst * width + at]; used = true; }
      if (cap >= 0) { g += a.d_state_out[((int64_t)cap * a.channels + c) * a.n_state + n]; used = true; }
      back[u * width + at] = g;
      sent = used ? fmaf(ex2(len[j] * a2), g, add[j]) : add[j];              // (steps are not there where no state is used)
      if (src == -1) d_first += sent;
      else if (src >= 0) slots[src * width + at] += sent;
      nxt_src = src;
      if (u - WALK >= 0) request(u - WALK, add[j], len[j]);
    }
  }
  if (a.d_initial_state) a.d_initial_state[(int64_t)c * a.n_state + n] = d_first;
}

// ---- grads ---------------------------------------------------------------------------------------
__device__ __forceinline__ float dpp_ror8(float v) {      // lane ^ 8
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x128, 0xf, 0xf, true));
}
__device__ __forceinline__ float dpp_half_mirror(float v) {      // lane ^ 7
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x141, 0xf, 0xf, true));
}
__device__ __forceinline__ float dpp_xor2(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0x4e, 0xf, 0xf, true));
}
__device__ __forceinline__ float dpp_xor1(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), 0xb1, 0xf, 0xf, true));
}

// Sums of M values over the wave: lane l returns the sum of value l * M / 64 (M = 8, 16, 32).  Every step adds the two halves of
// the lanes for half of the values each, so the values halve with the lanes that share them.
template <int M>
__device__ __forceinline__ float wave_sums(float (&v)[M], int lane) {
#pragma unroll
  for (int i = 0; i < M / 2; i++) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + M / 2]), false, false);
    v[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
#pragma unroll
  for (int i = 0; i < M / 4; i++) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + M / 4]), false, false);
    v[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
#pragma unroll
  for (int i = 0; i < M / 8; i++) {
    const bool up = lane & 8;
    const float keep = up ? v[i + M / 8] : v[i], give = up ? v[i] : v[i + M / 8];
    v[i] = keep + dpp_ror8(give);
  }
  if constexpr (M >= 16) {
#pragma unroll
    for (int i = 0; i < M / 16; i++) {
      const bool up = lane & 4;
      const float keep = up ? v[i + M / 16] : v[i], give = up ? v[i] : v[i + M / 16];
      v[i] = keep + dpp_half_mirror(give);
    }
  } else {
    v[0] += dpp_half_mirror(v[0]);
  }
  if constexpr (M >= 32) {
    const bool up = lane & 2;
    const float keep = up ? v[1] : v[0], give = up ? v[0] : v[1];
    v[0] = keep + dpp_xor2(give);
  } else {
    v[0] += dpp_xor2(v[0]);
  }
  return v[0] + dpp_xor1(v[0]);
}

struct GradBuffers {
  const float *states, *back;      // [n_chunks][NS][channels]
  float* bc;                       // [channel blocks of 64][n_tokens][2 NS]: dB, dC of the block
  float* rates;                    // [strips][NS][channels]: dA
  float* sums;                     // [strips][2][channels]: dD, ddt_bias
};

template <typename T, int NS, bool GATED>
__global__ void __launch_bounds__(WAVE)
scan_grads_kernel(ScanArgs a, int blocks, int strips, GradBuffers buf) {
  __shared__ float4 saved[SAVED][NS / 4][WAVE];
  const int lane = threadIdx.x;
  const int block = blockIdx.x % (unsigned)blocks, strip = blockIdx.x / (unsigned)blocks;
  const int ch = block * WAVE + lane;
  const bool valid = ch < a.channels;
  const int64_t cc = valid ? ch : a.channels - 1;
  const int group = __builtin_amdgcn_readfirstlane((int)cc / (a.channels / a.groups));
  float a2[NS], dA[NS], G[NS];
  load_rates<NS>(a.A, cc, a2);
#pragma unroll
  for (int n = 0; n < NS; n++) dA[n] = 0.f;
  const float bias = a.dt_bias ? a.dt_bias[cc] : 0.f, skip = a.D ? a.D[cc] : 0.f;
  float dD = 0.f, dbias = 0.f;
  struct In { T x, dt, z, dy; };

  for (int chunk = strip; chunk < a.n_chunks; chunk += strips) {
    const int t0 = a.chunk_tok0[chunk], len = min(a.chunk_len[chunk], CHUNK);
    const int groups_of = (len + SUB - 1) / SUB;
    const T* x = (const T*)a.x + (int64_t)t0 * a.x_stride;
    const T* dt = (const T*)a.dt + (int64_t)t0 * a.dt_stride;
    const T* z = GATED ? (const T*)a.z + (int64_t)t0 * a.z_stride : nullptr;
    const T* dy = (const T*)a.dy + (int64_t)t0 * a.dy_stride;
    const T* b = (const T*)a.b + (int64_t)t0 * a.b_stride + group * NS;
    const T* c = (const T*)a.c + (int64_t)t0 * a.c_stride + group * NS;
    const int64_t at = (int64_t)chunk * NS * a.channels + cc;
    auto enter = [&](float (&h)[NS]) {
#pragma unroll
      for (int n = 0; n < NS; n++) h[n] = buf.states[at + (int64_t)n * a.channels];
    };
    auto step = [&](float (&h)[NS], float delta, float u, int t) {
      float bv[NS];
      load_uniform<T, NS>(b + (int64_t)t * a.b_stride, bv);
#pragma unroll
      for (int n = 0; n < NS; n++) h[n] = fmaf(ex2(delta * a2[n]), h[n], u * bv[n]);
    };
    auto delta_of = [&](T raw) { const float r = to_f(raw) + bias; return a.use_softplus ? softplus(r) : r; };

    // the states in front of the second and later groups
    float h0[NS];
    enter(h0);
    for (int s = 0; s + 1 < groups_of; s++) {
      T xv[SUB], dv[SUB];
#pragma unroll
      for (int j = 0; j < SUB; j++) {
        const int64_t t = s * SUB + j;
        xv[j] = (x + t * a.x_stride)[cc];
        dv[j] = (dt + t * a.dt_stride)[cc];
      }
#pragma unroll
      for (int j = 0; j < SUB; j++) {
        const float delta = delta_of(dv[j]);
        step(h0, delta, delta * to_f(xv[j]), s * SUB + j);
      }
#pragma unroll
      for (int q = 0; q < NS / 4; q++) saved[s][q][lane] = make_float4(h0[4 * q], h0[4 * q + 1], h0[4 * q + 2], h0[4 * q + 3]);
    }
#pragma unroll
    for (int n = 0; n < NS; n++) G[n] = buf.back[at + (int64_t)n * a.channels];

    for (int s = groups_of - 1; s >= 0; s--) {
      const int base = s * SUB, m = min(SUB, len - base);
      In in[SUB];
#pragma unroll
      for (int j = 0; j < SUB; j++) {
        const int64_t t = min(base + j, len - 1);
        in[j].x = (x + t * a.x_stride)[cc];
        in[j].dt = (dt + t * a.dt_stride)[cc];
        if constexpr (GATED) in[j].z = (z + t * a.z_stride)[cc];
        in[j].dy = (dy + t * a.dy_stride)[cc];
      }
      float h[SUB + 1][NS], delta[SUB];
      if (s) {
#pragma unroll
        for (int q = 0; q < NS / 4; q++) {
          const float4 v = saved[s - 1][q][lane];
          h[0][4 * q] = v.x; h[0][4 * q + 1] = v.y; h[0][4 * q + 2] = v.z; h[0][4 * q + 3] = v.w;
        }
      } else {
        enter(h[0]);
      }
#pragma unroll
      for (int j = 0; j < SUB; j++) {
        if (j >= m) break;
        delta[j] = delta_of(in[j].dt);
#pragma unroll
        for (int n = 0; n < NS; n++) h[j + 1][n] = h[j][n];
        step(h[j + 1], delta[j], delta[j] * (valid ? to_f(in[j].x) : 0.f), base + j);
      }
#pragma unroll
      for (int j = SUB - 1; j >= 0; j--) {
        if (j >= m) continue;
        const int t = base + j;
        float bv[NS], cv[NS], red[2 * NS];
        load_uniform<T, NS>(b + (int64_t)t * a.b_stride, bv);
        load_uniform<T, NS>(c + (int64_t)t * a.c_stride, cv);
        const float xv = valid ? to_f(in[j].x) : 0.f, up = valid ? to_f(in[j].dy) : 0.f;
        float g = up, zv = 0.f, sig = 0.f;
        if constexpr (GATED) {
          zv = to_f(in[j].z);
          sig = sigmoid(zv);
          g *= zv * sig;
        }
        const float u = delta[j] * xv;
        float du = 0.f, dd = 0.f, y = skip * xv;
#pragma unroll
        for (int n = 0; n < NS; n++) {
          const float hn = h[j + 1][n];
          G[n] = fmaf(cv[n], g, G[n]);
          if constexpr (GATED) y = fmaf(cv[n], hn, y);
          red[n] = G[n] * u;
          red[NS + n] = hn * g;
          du = fmaf(G[n], bv[n], du);
          G[n] *= ex2(delta[j] * a2[n]);
          const float q = G[n] * h[j][n];
          dd = fmaf(a2[n], q, dd);
          dA[n] = fmaf(delta[j], q, dA[n]);
        }
        const float sum = wave_sums<2 * NS>(red, lane);
        constexpr int SHARE = WAVE / (2 * NS);
        if (lane % SHARE == 0) buf.bc[((int64_t)block * a.n_tokens + t0 + t) * (2 * NS) + lane / SHARE] = sum;
        dD = fmaf(g, xv, dD);
        dd = fmaf(xv, du, dd * LN2);
        if (a.use_softplus) dd *= sigmoid(to_f(in[j].dt) + bias);
        dbias += dd;
        if (valid) {
          const int64_t o = (int64_t)(t0 + t) * a.channels + ch;
          ((T*)a.dx)[o] = from_f<T>(fmaf(delta[j], du, skip * g));
          ((T*)a.ddt)[o] = from_f<T>(dd);
          if constexpr (GATED) ((T*)a.dz)[o] = from_f<T>(up * y * sig * (1.f + zv * (1.f - sig)));
        }
      }
    }
  }
  if (!valid) return;
#pragma unroll
  for (int n = 0; n < NS; n++) buf.rates[((int64_t)strip * NS + n) * a.channels + ch] = dA[n];
  buf.sums[(int64_t)(2 * strip) * a.channels + ch] = dD;
  buf.sums[(int64_t)(2 * strip + 1) * a.channels + ch] = dbias;
}

// ---- sums ----------------------------------------------------------------------------------------
// Entry j of token t and group: the sum over the group's channel blocks.  Then, in the workgroups behind those: dA, dD, bias.
template <typename T, int NS>
__global__ void __launch_bounds__(THREADS)
scan_sums_kernel(ScanArgs a, int blocks, int strips, GradBuffers buf, int64_t bc_groups) {
  if ((int64_t)blockIdx.x < bc_groups) {
    const int64_t at = (int64_t)blockIdx.x * THREADS + threadIdx.x;
    const int64_t per_group = (int64_t)a.n_tokens * 2 * NS;
    if (at >= per_group * a.groups) return;
    const int group = (int)(at / per_group);
    const int64_t i = at - group * per_group;
    const int b0 = (int)((int64_t)blocks * group / a.groups), b1 = (int)((int64_t)blocks * (group + 1) / a.groups);
    float s = 0.f;
    for (int b = b0; b < b1; b++) s += buf.bc[b * per_group + i];
    const int64_t t = i / (2 * NS);
    const int j = (int)(i - t * 2 * NS);
    T* out = (T*)(j < NS ? a.db : a.dc);
    out[(t * a.groups + group) * NS + j % NS] = from_f<T>(s);
    return;
  }
  const int64_t at = ((int64_t)blockIdx.x - bc_groups) * THREADS + threadIdx.x;
  const int64_t n = at / a.channels;
  const int64_t c = at - n * a.channels;
  if (n >= NS + 2) return;
  const float* in = n < NS ? buf.rates + n * a.channels + c : buf.sums + (n - NS) * a.channels + c;
  const int64_t step = (int64_t)(n < NS ? NS : 2) * a.channels;
  float s = 0.f;
  for (int k = 0; k < strips; k++) s += in[k * step];
  if (n < NS) a.dA[c * NS + n] = s;
  else if (n == NS) { if (a.dD) a.dD[c] = s; }
  else if (a.ddt_bias) a.ddt_bias[c] = s;
}

size_t up(size_t v) { return (v + 255) & ~(size_t)255; }

// Strips of chunks that one wave per channel block takes one after the other, keeping dA in registers: as many as give the chip
// 2560 waves, ten per compute unit.
int strips_of(int channels, int n_chunks) {
  const int blocks = (channels + WAVE - 1) / WAVE;
  return std::max(1, std::min(n_chunks, (2560 + blocks - 1) / blocks));
}

}  // namespace

size_t scan_bwd_workspace(int64_t n_tokens, int channels, int n_state, int groups, int n_chunks, int n_slots) {
  const size_t width = (size_t)channels * n_state * sizeof(float);
  const size_t blocks = (channels + WAVE - 1) / WAVE, strips = strips_of(channels, n_chunks);
  return 2 * up(width * n_chunks) + up((size_t)channels * n_chunks * sizeof(float)) + up(width * n_slots) +
         up(blocks * n_tokens * 2 * n_state * sizeof(float)) + up(strips * width) + up(strips * 2 * channels * sizeof(float)) + 256;
}

hipError_t scan_bwd(const ScanArgs& a, hipStream_t st) {
  const size_t width = (size_t)a.channels * a.n_state * sizeof(float);
  const int blocks = (a.channels + WAVE - 1) / WAVE, strips = strips_of(a.channels, a.n_chunks);
  char* w = (char*)a.workspace;
  auto take = [&](size_t bytes) { float* p = (float*)w; w += up(bytes); return p; };
  float* local = take(width * a.n_chunks);
  float* back = take(width * a.n_chunks);
  float* steps = take((size_t)a.channels * a.n_chunks * sizeof(float));
  float* slots = take(width * a.n_slots);
  GradBuffers buf{local, back, nullptr, nullptr, nullptr};
  buf.bc = take((size_t)blocks * a.n_tokens * 2 * a.n_state * sizeof(float));
  buf.rates = take(strips * width);
  buf.sums = take((size_t)strips * 2 * a.channels * sizeof(float));
  const int wide = (a.channels + THREADS - 1) / THREADS;
  return by_type(a.bf16, a.n_state, [&](auto zero, auto ns) -> hipError_t {
    using T = decltype(zero);
    constexpr int NS = decltype(ns)::value;
    if (a.n_chunks > 0) {
      KernelTimer timer(TT_KERNEL_SCAN_CARRY, st);
      const unsigned grid = (unsigned)wide * (unsigned)a.n_chunks;
      if (a.z) scan_ends_kernel<T, NS, true><<<grid, THREADS, 0, st>>>(a, wide, local, steps, back);
      else scan_ends_kernel<T, NS, false><<<grid, THREADS, 0, st>>>(a, wide, local, steps, back);
    }
    if (hipError_t e = hipGetLastError()) return e;
    if (a.n_chunks > 0 || a.d_initial_state) {
      KernelTimer timer(TT_KERNEL_SCAN_STATES, st);
      scan_bwd_states_kernel<<<(unsigned)((NS * (int64_t)a.channels + THREADS - 1) / THREADS), THREADS, 0, st>>>(a, local, back, steps, slots);
    }
    if (hipError_t e = hipGetLastError()) return e;
    {
      KernelTimer timer(TT_KERNEL_SCAN_GRADS, st);
      const unsigned grid = (unsigned)blocks * (unsigned)strips;      // (no chunks: the strip's sums are zero)
      if (a.z) scan_grads_kernel<T, NS, true><<<grid, WAVE, 0, st>>>(a, blocks, strips, buf);
      else scan_grads_kernel<T, NS, false><<<grid, WAVE, 0, st>>>(a, blocks, strips, buf);
    }
    if (hipError_t e = hipGetLastError()) return e;
    KernelTimer timer(TT_KERNEL_SCAN_SUMS, st);
    const int64_t bc = ((int64_t)a.n_tokens * 2 * NS * a.groups + THREADS - 1) / THREADS;
    const int64_t rest = ((int64_t)(NS + 2) * a.channels + THREADS - 1) / THREADS;
    scan_sums_kernel<T, NS><<<(unsigned)(bc + rest), THREADS, 0, st>>>(a, blocks, strips, buf, bc);
    return hipGetLastError();
  });
}

}  // namespace tt
