// Selective state space scan with tree state routing, backward.
//
// With a = exp(delta A), u = delta x, dy' = dy silu(z) and G_t the gradient of h_t (its own token's C_t dy'_t and what every
// successor on any branch sends back, a G):
//   dC_t = sum_c h dy'          dB_t = sum_c G u            du = sum_n G B           q = G a h_p
//   ddelta = x du + sum_n A q   dA = sum_t delta q          dx = delta du + D dy'    ddt = ddelta sigmoid(dt + bias)
// Chunks are independent up to the state entering them and the gradient of the state leaving them:
//   ends    per chunk, one pass: the state it leaves from zero, the sum of its steps, and the gradient of its entering state
//           that its own outputs give, sum_t (prod_{s<=t} a_s) C_t dy'_t; also the states from zero and the sums of steps in
//           front of every eighth token
//   states  down the tree, then up again, one lane per (channel, state): entering states, gradients of the leaving states
//   grads   every chunk once more with the two known: eight tokens at a time from the last, their states worked out again from
//           the state in front of them, h = (state from zero) + exp(A (sum of steps)) (entering state)
//   sums    of what the waves and strips of chunks left: dB, dC over the channels, dA, dD and the bias over the strips
// No atomics: every sum has a fixed order.  One lane holds one channel; the sums over a wave's 64 channels for the 2 NS entries of
// dB and dC are taken together, the lanes halving the entries they keep at every step (70 instructions for 32 sums).
//
// Bound by the vector ALU, as the forward: 16406 tokens of 4096 channels, ends 260 us (105 % busy), states 65, grads 877 (87 %), sums 32
// (1234 of a pass of 1238).  In fp32, where grads spills 26 registers at 16 gated states, the pass takes 1598.
#include <algorithm>
#include "tt_scan.h"

namespace tt {
namespace {
using namespace scan;

constexpr int CHUNK = TT_GDN_CHUNK;
// Tokens whose states are held in registers at a time.  The states in front of them cost 64 bytes of workspace per eight tokens and
// channel, written once and read once; worked out again from the chunk's start (kept in LDS for every 16 tokens) they were a quarter
// of the grads kernel's instructions.
constexpr int SUB = 8;
static_assert(SUB == 2 * AHEAD, "the ends kernel saves a state every two blocks of loads");
// Place of the state in front of token t0 + 8 s (s > 0) of the chunk that starts at t0: no two chunks share one.
__device__ __forceinline__ int64_t front(int t0, int s) { return t0 / SUB + s; }
__host__ inline int64_t fronts(int64_t n_tokens) { return n_tokens / SUB + 1; }

// ---- ends ----------------------------------------------------------------------------------------
template <typename T, int NS, bool GATED>
__global__ void __launch_bounds__(THREADS)
scan_ends_kernel(ScanArgs a, int blocks, float* __restrict__ local, float* __restrict__ steps, float* __restrict__ back,
                 float* __restrict__ fronts, float* __restrict__ front_steps) {
  const Place p = place(a, blocks);
  const int t0 = a.chunk_tok0[p.chunk], len = min(a.chunk_len[p.chunk], CHUNK);
  Feed<T> x(a.x, a.x_stride, t0), dt(a.dt, a.dt_stride, t0), z(a.z, a.z_stride, t0), dy(a.dy, a.dy_stride, t0);
  UniformFeed<T, NS> b(a.b, a.b_stride, t0, p.group * NS), c(a.c, a.c_stride, t0, p.group * NS);
  float a2[NS], h[NS], along[NS], r[NS], total = 0.f;
  load_rates<NS>(a.A, p.cc, a2);
#pragma unroll
  for (int n = 0; n < NS; n++) { h[n] = 0.f; along[n] = 1.f; r[n] = 0.f; }
  const float bias = a.dt_bias ? a.dt_bias[p.cc] : 0.f;
  const uint32_t off = (uint32_t)p.cc * sizeof(T);
  struct In { T x, dt, z, dy; };
  stream<In>(
      len,
      [&](int t, In (&v)[AHEAD]) {
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
          const bool more = t + j < len - 1;
          v[j].x = x.next(off, more);
          v[j].dt = dt.next(off, more);
          if constexpr (GATED) v[j].z = z.next(off, more);
          v[j].dy = dy.next(off, more);
        }
      },
      [&](int t, const In& v) {
        if (t % SUB == 0 && t > 0 && p.valid) {
          const int64_t f = front(t0, t / SUB);
          Feed<float> out(fronts + f * NS * a.channels, a.channels, 0);
#pragma unroll
          for (int n = 0; n < NS; n++, out.so += out.step) out.put((uint32_t)p.c * 4u, h[n]);
          front_steps[f * a.channels + p.c] = total;
        }
        Words<T, NS> bv, cv;
        b.next(bv);
        c.next(cv);
        const float raw = to_f(v.dt) + bias, delta = step_size(raw, a.use_softplus);
        const float u = delta * to_f(v.x);
        float g = to_f(v.dy);
        if constexpr (GATED) {
          const float zv = to_f(v.z);
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
      });
  if (!p.valid) return;
  const int64_t at = (int64_t)p.chunk * NS * a.channels + p.c;
#pragma unroll
  for (int n = 0; n < NS; n++) {
    local[at + (int64_t)n * a.channels] = h[n];
    back[at + (int64_t)n * a.channels] = r[n];
  }
  steps[(int64_t)p.chunk * a.channels + p.c] = total;
}

// ---- states --------------------------------------------------------------------------------------
// local[chunk]: entering state; back[chunk]: gradient of the leaving state.
template <bool LDS>
__global__ void __launch_bounds__(WAVE)
scan_bwd_states_kernel(ScanArgs a, float* local, float* back, const float* __restrict__ steps, float* saved) {
  extern __shared__ float lds[];
  const Walker w(a);
  if (a.n_chunks == 0) {
    if (blockIdx.y) a.d_initial_state[w.state_at] = 0.f;
    return;
  }
  // the two walks do not depend on each other: one half of the workgroups takes the way down, the other the way up
  const Slots<LDS> slots(a, w, lds, saved + (blockIdx.y ? (a.n_slots + EXTRA_SLOTS) * w.width : 0));
  const float a2 = a.A[w.state_at] * LOG2E;
  if (blockIdx.y == 0) {
    walk_down<LDS>(a, local, steps, w, a2, slots, false, [](int, float) {});
    return;
  }
  // up the tree: back[chunk] (the gradient of the entering state that the chunk's outputs give) becomes that of the leaving state
  for (int s = 0; s <= slots.first; s++) slots[s] = 0.f;                       // gradients of the saved states, and of the first
  float sent = 0.f;                                                            // by the chunk behind
  walk<true>(a, back, steps, w, a2, a.d_state_out != nullptr, [&](const Entries& e, const float (&decay)[WALK], const float (&own)[WALK],
                                                                  float (&leaving)[WALK]) {
    const uint32_t continued = mask_of(e.src_behind == -2), saves = mask_of(e.dst >= 0), captured = mask_of(e.cap >= 0);
    const uint32_t used = continued | saves | captured;        // (elsewhere g is 0, and steps as given below 0 may make the decay infinite)
    const uint32_t starts = mask_of(e.src != -2);
    const int to = e.src < 0 ? slots.first : e.src;
    float given[WALK];
#pragma unroll
    for (int j = 0; j < WALK; j++) given[j] = 0.f;
    if (captured)
#pragma unroll
      for (int j = 0; j < WALK; j++)
        if (bit(captured, j)) given[j] = a.d_state_out[Entries::at(e.cap, j) * w.width + w.state_at];
#pragma unroll
    for (int j = WALK - 1; j >= 0; j--) {
      float g = bit(continued, j) ? sent : 0.f;
      if (bit(saves, j)) g += slots[Entries::at(e.dst, j)];
      g += given[j];
      leaving[j] = g;
      sent = bit(used, j) ? fmaf(decay[j], g, own[j]) : own[j];
      if (bit(starts, j)) slots[Entries::at(to, j)] += sent;
    }
  });
  if (a.d_initial_state) a.d_initial_state[w.state_at] = slots[slots.first];
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

// Sums of M values over the wave: lane l returns the sum of value l / (64 / M) (M = 4, 8, 16).  Every step adds the two halves of
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
  if constexpr (M >= 8) {
#pragma unroll
    for (int i = 0; i < M / 8; i++) {
      const bool up = lane & 8;
      const float keep = up ? v[i + M / 8] : v[i], give = up ? v[i] : v[i + M / 8];
      v[i] = keep + dpp_ror8(give);
    }
  } else {
    v[0] += dpp_ror8(v[0]);
  }
  if constexpr (M >= 16) {
    const bool up = lane & 4;
    const float keep = up ? v[1] : v[0], give = up ? v[0] : v[1];
    v[0] = keep + dpp_half_mirror(give);
  } else {
    v[0] += dpp_half_mirror(v[0]);
  }
  v[0] += dpp_xor2(v[0]);
  return v[0] + dpp_xor1(v[0]);
}

struct GradBuffers {
  const float *states, *back;      // [n_chunks][NS][channels]
  const float *fronts, *front_steps;      // [tokens / SUB + 1][NS][channels], [..][channels]
  float* bc;                       // [channel blocks of 64][n_tokens][2 NS]: dB, dC of the block
  float* rates;                    // [strips][NS][channels]: dA
  float* sums;                     // [strips][2][channels]: dD, ddt_bias
};

template <typename T, int NS, bool GATED>
__global__ void __launch_bounds__(WAVE, 2)
scan_grads_kernel(ScanArgs a, int blocks, int strips, GradBuffers buf) {
  __shared__ float4 entering[NS / 4][WAVE], before[NS / 4][WAVE];       // the chunk's entering state; the state in front of the SUB tokens
  // the lanes that hold the same entry of the sums over the wave: one half of them stores its dB, the other its dC
  constexpr int SHARE = WAVE / NS, HALF = SHARE / 2;
  struct In { T x, dt, z, dy; };
  __shared__ In inputs[SUB][WAVE];
  __shared__ float sizes[SUB][WAVE];                                    // the steps' (in registers they would be spilled)
  const int lane = threadIdx.x;
  const int block = blockIdx.x % (unsigned)blocks, strip = blockIdx.x / (unsigned)blocks;
  const int ch = block * WAVE + lane;
  const bool valid = ch < a.channels;
  const int cc = valid ? ch : a.channels - 1;
  const int group = __builtin_amdgcn_readfirstlane(cc / (a.channels / a.groups));
  const uint32_t off = (uint32_t)cc * sizeof(T), bc_off = 4u * ((lane & HALF ? NS : 0) + lane / SHARE);
  float a2[NS], dA[NS], G[NS];
  load_rates<NS>(a.A, cc, a2);
#pragma unroll
  for (int n = 0; n < NS; n++) dA[n] = 0.f;
  const float bias = a.dt_bias ? a.dt_bias[cc] : 0.f, skip = a.D ? a.D[cc] : 0.f;
  float dD = 0.f, dbias = 0.f;
  auto save = [&](float4 (&to)[NS / 4][WAVE], const float (&h)[NS]) {
#pragma unroll
    for (int q = 0; q < NS / 4; q++) to[q][lane] = make_float4(h[4 * q], h[4 * q + 1], h[4 * q + 2], h[4 * q + 3]);
  };
  auto restore = [&](const float4 (&from)[NS / 4][WAVE], float (&h)[NS]) {
#pragma unroll
    for (int q = 0; q < NS / 4; q++) {
      const float4 v = from[q][lane];
      h[4 * q] = v.x; h[4 * q + 1] = v.y; h[4 * q + 2] = v.z; h[4 * q + 3] = v.w;
    }
  };
  auto per_state = [&](const float* p, int64_t block_of, float (&h)[NS]) {
    Feed<float> f(p + block_of * NS * a.channels, a.channels, 0);
#pragma unroll
    for (int n = 0; n < NS; n++) h[n] = f.next((uint32_t)cc * 4u, true);
  };
  auto delta_of = [&](T raw) { return step_size(to_f(raw) + bias, a.use_softplus); };
  auto step = [&](const float (&from)[NS], float (&h)[NS], const Words<T, NS>& bv, float delta, float u) {
#pragma unroll
    for (int n = 0; n < NS; n++) h[n] = fmaf(ex2(delta * a2[n]), from[n], u * bv[n]);
  };

  for (int chunk = strip; chunk < a.n_chunks; chunk += strips) {
    const int t0 = __builtin_amdgcn_readfirstlane(a.chunk_tok0[chunk]), len = __builtin_amdgcn_readfirstlane(min(a.chunk_len[chunk], CHUNK));
    Feed<float> bc(buf.bc, 2 * NS, (int64_t)block * a.n_tokens + t0);
    Feed<T> dx(a.dx, a.channels, t0), ddt(a.ddt, a.channels, t0), dz(a.dz, a.channels, t0);
    float h0[NS];
    per_state(buf.states, chunk, h0);
    per_state(buf.back, chunk, G);
    save(entering, h0);

    // the inputs of SUB tokens and the state from zero in front of them
    In in[SUB];
    float from_zero[NS], along = 0.f;
    auto request = [&](int s) {
      const int base = s * SUB, m = min(SUB, len - base);
      Feed<T> x(a.x, a.x_stride, t0, base), dt(a.dt, a.dt_stride, t0, base), z(a.z, a.z_stride, t0, base), dy(a.dy, a.dy_stride, t0, base);
#pragma unroll
      for (int j = 0; j < SUB; j++) {
        const bool more = j < m - 1;
        in[j].x = x.next(off, more);
        in[j].dt = dt.next(off, more);
        if constexpr (GATED) in[j].z = z.next(off, more);
        in[j].dy = dy.next(off, more);
      }
      if (s) {
        per_state(buf.fronts, front(t0, s), from_zero);
        along = buf.front_steps[front(t0, s) * a.channels + cc];
      }
    };
    request((len - 1) / SUB);

    for (int s = (len - 1) / SUB; s >= 0; s--) {
      const int base = s * SUB, m = min(SUB, len - base);
      // the inputs wait in LDS: with all states of these tokens in registers there is no room for them there
#pragma unroll
      for (int j = 0; j < SUB; j++) inputs[j][lane] = in[j];
      restore(entering, h0);
      if (s)
#pragma unroll
        for (int n = 0; n < NS; n++) h0[n] = fmaf(ex2(along * a2[n]), h0[n], from_zero[n]);
      save(before, h0);
      float h[SUB][NS];
      UniformFeed<T, NS> b(a.b, a.b_stride, t0 + base, group * NS), c(a.c, a.c_stride, t0 + base + m - 1, group * NS);
#pragma unroll
      for (int j = 0; j < SUB; j++) {
        if (j >= m) break;
        Words<T, NS> bv;
        b.next(bv);
        const float delta = delta_of(inputs[j][lane].dt);
        sizes[j][lane] = delta;
        step(j ? h[j - 1] : h0, h[j], bv, delta, delta * to_f(inputs[j][lane].x));
      }
      b.p -= b.step;                             // both from the last token back
      asm volatile("" : "+s"(b.p));              // (the vectors kept from above would be spilled)
      // the vectors of a token are requested while the one behind it is worked on
      Words<T, NS> bv, cv, next_b, next_c;
      b.prev(next_b);
      c.prev(next_c);
      // The next group is requested as soon as the states of half the tokens are used up: there its registers come from.
      if (s && m <= SUB / 2) request(s - 1);
#pragma unroll
      for (int j = SUB - 1; j >= 0; j--) {
        if (j >= m) continue;
        if (j == SUB / 2 - 1 && s && m > SUB / 2) request(s - 1);
        bv = next_b;
        cv = next_c;
        const In in = inputs[j][lane];
        const float xv = to_f(in.x), up = to_f(in.dy), delta = sizes[j][lane];
        if (j) {
          b.prev(next_b);
          c.prev(next_c);
        }
        float g = up, zv = 0.f, sig = 0.f, red[NS];
        if constexpr (GATED) {
          zv = to_f(in.z);
          sig = sigmoid(zv);
          g *= zv * sig;
        }
        // (a lane past the last channel stands in for it and writes what it writes, but must not be in the sums over the channels)
        const float u = delta * xv, u_in = valid ? u : 0.f, g_in = valid ? g : 0.f;
        float y = skip * xv;
#pragma unroll
        for (int n = 0; n < NS; n++) {
          if constexpr (GATED) y = fmaf(cv[n], h[j][n], y);
          G[n] = fmaf(cv[n], g, G[n]);
          red[n] = h[j][n] * g_in;
        }
        const float sum_c = wave_sums<NS>(red, lane);
        if (j == 0) restore(before, h0);
        const float (&hp)[NS] = j ? h[j - 1] : h0;
        float du = 0.f, dd = 0.f;
#pragma unroll
        for (int n = 0; n < NS; n++) {
          red[n] = G[n] * u_in;
          du = fmaf(G[n], bv[n], du);
          G[n] *= ex2(delta * a2[n]);
          const float r = G[n] * hp[n];
          dd = fmaf(a2[n], r, dd);
          dA[n] = fmaf(delta, r, dA[n]);
        }
        const float sum_b = wave_sums<NS>(red, lane);
        bc.so = (base + j) * bc.step;
        bc.put(bc_off, lane & HALF ? sum_c : sum_b);
        dD = fmaf(g, xv, dD);
        dd = fmaf(xv, du, dd * LN2);
        float slope = sigmoid(to_f(in.dt) + bias);
        asm volatile("" : "+v"(slope));
        dd *= a.use_softplus ? slope : 1.f;
        dbias += dd;
        dx.so = ddt.so = dz.so = (base + j) * dx.step;
        dx.put(off, fmaf(delta, du, skip * g));
        ddt.put(off, dd);
        if constexpr (GATED) dz.put(off, up * y * sig * (1.f + zv * (1.f - sig)));
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
// Four entries of dB, dC of a token and group per thread: the sum over the group's channel blocks.  Then, in the workgroups behind
// those: dA, dD, ddt_bias of a channel, the sum over the strips.
template <typename T, int NS>
__global__ void __launch_bounds__(THREADS)
scan_sums_kernel(ScanArgs a, int blocks, int strips, GradBuffers buf, int64_t bc_groups) {
  if ((int64_t)blockIdx.x < bc_groups) {
    const int64_t at = (int64_t)blockIdx.x * THREADS + threadIdx.x;
    const int64_t per_group = (int64_t)a.n_tokens * (2 * NS / 4);
    if (at >= per_group * a.groups) return;
    const int group = (int)(at / per_group);
    const int64_t i = at - group * per_group;
    const int n = blocks / a.groups;                                         // (several groups are whole blocks)
    const float4* in = (const float4*)buf.bc + (int64_t)group * n * per_group + i;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int b = 0; b < n; b++) {
      const float4 v = in[b * per_group];
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    const int64_t t = i / (2 * NS / 4);
    const int j = 4 * (int)(i - t * (2 * NS / 4));
    T* out = (T*)(j < NS ? a.db : a.dc) + (t * a.groups + group) * NS + j % NS;
    out[0] = from_f<T>(s.x); out[1] = from_f<T>(s.y); out[2] = from_f<T>(s.z); out[3] = from_f<T>(s.w);
    return;
  }
  const int64_t at = ((int64_t)blockIdx.x - bc_groups) * THREADS + threadIdx.x;
  const int64_t n = at / a.channels;
  const int64_t c = at - n * a.channels;
  if (n >= NS + 2) return;
  const float* in = n < NS ? buf.rates + n * a.channels + c : buf.sums + (n - NS) * a.channels + c;
  const int64_t step = (int64_t)(n < NS ? NS : 2) * a.channels;
  float s = 0.f;
#pragma unroll 8
  for (int k = 0; k < strips; k++) s += in[k * step];
  if (n < NS) a.dA[c * NS + n] = s;
  else if (n == NS) { if (a.dD) a.dD[c] = s; }
  else if (a.ddt_bias) a.ddt_bias[c] = s;
}

size_t up(size_t v) { return (v + 255) & ~(size_t)255; }

// Strips of chunks that one wave per channel block takes one after the other, keeping dA in registers: as many as give the chip
// 6144 waves, three times what it holds at a time (2048 / 4096 / 6144 / 8192 waves and one chunk each, with the sums over the strips,
// 16406 tokens of 4096 channels, first passes after a pause: 1014 / 1004 / 946 / 998 / 983 us).
int strips_of(int channels, int n_chunks) {
  const int blocks = (channels + WAVE - 1) / WAVE;
  return std::max(1, std::min(n_chunks, (6144 + blocks - 1) / blocks));
}

}  // namespace

size_t scan_bwd_workspace(int64_t n_tokens, int channels, int n_state, int n_chunks, int n_slots) {
  const size_t width = (size_t)channels * n_state * sizeof(float);
  const size_t blocks = (channels + WAVE - 1) / WAVE, strips = strips_of(channels, n_chunks);
  return 2 * up(width * walk_rows(n_chunks)) + up(channels * walk_rows(n_chunks) * sizeof(float)) + up(2 * width * (n_slots + EXTRA_SLOTS)) +
         up(width * fronts(n_tokens)) + up((size_t)channels * fronts(n_tokens) * sizeof(float)) +
         up(blocks * n_tokens * 2 * n_state * sizeof(float)) + up(strips * width) + up(strips * 2 * channels * sizeof(float)) + 256;
}

hipError_t scan_bwd(const ScanArgs& a, hipStream_t st) {
  const size_t width = (size_t)a.channels * a.n_state * sizeof(float);
  const int blocks = (a.channels + WAVE - 1) / WAVE, strips = strips_of(a.channels, a.n_chunks);
  char* w = (char*)a.workspace;
  auto take = [&](size_t bytes) { float* p = (float*)w; w += up(bytes); return p; };
  float* local = take(width * walk_rows(a.n_chunks));
  float* back = take(width * walk_rows(a.n_chunks));
  float* steps = take(a.channels * walk_rows(a.n_chunks) * sizeof(float));
  float* slots = take(2 * width * (a.n_slots + EXTRA_SLOTS));
  float* front_states = take(width * fronts(a.n_tokens));
  float* front_steps = take((size_t)a.channels * fronts(a.n_tokens) * sizeof(float));
  GradBuffers buf{local, back, front_states, front_steps, nullptr, nullptr, nullptr};
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
      if (a.z) scan_ends_kernel<T, NS, true><<<grid, THREADS, 0, st>>>(a, wide, local, steps, back, front_states, front_steps);
      else scan_ends_kernel<T, NS, false><<<grid, THREADS, 0, st>>>(a, wide, local, steps, back, front_states, front_steps);
    }
    if (hipError_t e = hipGetLastError()) return e;
    if (a.n_chunks > 0 || a.d_initial_state) {
      KernelTimer timer(TT_KERNEL_SCAN_STATES, st);
      const dim3 walkers((unsigned)((NS * (int64_t)a.channels + WAVE - 1) / WAVE), 2);
      if (a.n_slots <= LDS_SLOTS) scan_bwd_states_kernel<true><<<walkers, WAVE, walk_lds(a.n_slots), st>>>(a, local, back, steps, slots);
      else scan_bwd_states_kernel<false><<<walkers, WAVE, walk_lds(a.n_slots), st>>>(a, local, back, steps, slots);
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
    const int64_t bc = ((int64_t)a.n_tokens * (2 * NS / 4) * a.groups + THREADS - 1) / THREADS;
    const int64_t rest = ((int64_t)(NS + 2) * a.channels + THREADS - 1) / THREADS;
    scan_sums_kernel<T, NS><<<(unsigned)(bc + rest), THREADS, 0, st>>>(a, blocks, strips, buf, bc);
    return hipGetLastError();
  });
}

}  // namespace tt
