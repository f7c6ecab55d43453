// The gradient of the selective state space scan (paac_selective_scan_backward).
//
// With G_t = dL/dh_t, dy' = dy silu(z) and g = exp(delta_t A) (0 at a restart):
//   G_t = C_t dy'_t + g_{t+1} G_{t+1},   through_t = G_t g_t h_{t-1}   (what comes through the exponential, divided by delta A)
//   dx = D dy' + delta sum_s G B,   ddelta = sum_s through A + x sum_s G B,   dz = dy (C h + D x) silu'(z),   ddt = ddelta softplus'
//   dB_t = sum over the group's channels of G delta x,   dC_t = of dy' h,   dA = sum over steps of through delta,   dh0 = g_0 G_0.
// A window of SPAN steps begins at a state that the forward pass has kept.  From there it is walked once, and the state before every SUB-th step
// put aside in shared memory; then SUB steps at a time, the last first, are walked again with states and decays in registers, and
// back.  So a decay is worked out 1 + 3/4 times, and no state but the kept ones comes from memory.  Sums over channels: the thread's
// own two, then by halves over the lanes (a lane ends with one or a few of the 16 sums, so that 16 take 15 exchanges), over the
// block's warps in shared memory, and over blocks by a second kernel in a fixed order.
//
// What bounds it: instructions; of every element of the state a step takes 1.75 exponentials and some 13 other operations, most of them two at a time.
#include "per_device.h"
#include "selective.cuh"

namespace {
using namespace paac::selective;
using paac::bf16;

constexpr int SUB = 4, SUBS = SPAN / SUB;
constexpr float LN2 = 0.693147182f;

template <int SL> __host__ __device__ constexpr int sums_of() { return 2 * EACH * SL; }       // a step's sums over channels: dB, then dC

// Sums of v over the lanes with the same states; the lane is left with `left` of them, from `first` on, in v[0..left).
template <int SL> struct OverChannels {
  static constexpr int COUNT = 2 * EACH, LANES = 32 / SL, LEFT = COUNT > LANES ? COUNT / LANES : 1;
  __device__ __forceinline__ static int sum(float (&v)[COUNT]) {
    const int lane = threadIdx.x & 31;
    int first = 0;
#pragma unroll
    for (int d = 16, count = COUNT; d >= SL; d /= 2) {
      if (count > 1) {
        const bool upper = (lane & d) != 0;
        count /= 2;
#pragma unroll
        for (int i = 0; i < COUNT / 2; ++i)
          if (i < count) {
            const float keep = upper ? v[i + count] : v[i], send = upper ? v[i] : v[i + count];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, send, d);
          }
        if (upper) first += count;
      } else {
        v[0] += __shfl_xor_sync(0xffffffffu, v[0], d);
      }
    }
    return first;
  }
};

// dy', the gradient behind the gate
template <class T, int VEC> __device__ __forceinline__ void behind_gate(float (&dy)[VEC], const Args& a, int k, int seq, int channel) {
  if (a.z.data == nullptr) return;
  float z[VEC], s, rest;
  load_vec<T, VEC>(z, paac::row_at<T>(a.z, k, seq) + channel);
#pragma unroll
  for (int j = 0; j < VEC; ++j) { paac::logistic<T>(z[j], s, rest); dy[j] *= z[j] * s; }
}

// What a chunk passes on from nothing (the last from dh_last) to the one before it, and its deltas' sum.
template <class T, int SL, int VEC>
__global__ void __launch_bounds__(32 * MOST_WARPS)
selective_back_ends_kernel(const __grid_constant__ Args a) {
  paac::pdl_entry();
  extern __shared__ float4 shared[];
  Place<SL> at(a);
  at.chunk += 1;                                                  // the first passes on to nobody
  constexpr int WIDE = EACH * SL;
  float2* slot = reinterpret_cast<float2*>(shared);                 // [SPAN][width]: delta, dy'
  float* Cs = reinterpret_cast<float*>(slot + SPAN * at.width);
  float A[PAIR][EACH], carry[PAIR][EACH], sum[PAIR];
  load_rates<SL>(A, a, at);
  zero<SL>(carry);
#pragma unroll
  for (int i = 0; i < PAIR; ++i) {
    sum[i] = 0.f;
    if (at.chunk == a.chunks - 1 && a.first != nullptr)
      load_states(carry[i], a.first + state_at(a, at.seq, at.channel(i)), at.sl * EACH, a.state, a.wide, at.has(i));
  }
  const int k0 = at.chunk * a.chunk, end = a.t - k0 < a.chunk ? a.t : k0 + a.chunk;
  bool any_cut = false;
  for (int k = k0 + (end - k0 - 1) / SPAN * SPAN; k >= k0; k -= SPAN) {
    const int steps = end - k < SPAN ? end - k : SPAN;
    __syncthreads();
    for_tile<VEC>(steps, at.room, at.width, [&](int q, int ch) {
      float dy[VEC], dt[VEC];
      load_vec<T, VEC>(dt, paac::row_at<T>(a.dt, k + q, at.seq) + at.base + ch);
      load_vec<T, VEC>(dy, paac::row_at<T>(a.dy, k + q, at.seq) + at.base + ch);
      behind_gate<T, VEC>(dy, a, k + q, at.seq, at.base + ch);
#pragma unroll
      for (int j = 0; j < VEC; ++j) slot[q * at.width + ch + j] = make_float2(delta_of<T>(a, dt[j], at.base + ch + j), dy[j]);
    });
    load_inputs<T, SL>(Cs, a, a.c, k, steps, at.seq, at.group);
    const uint32_t cuts = restarts(a, k, steps, at.seq);
    __syncthreads();
    for (int q = steps - 1; q >= 0; --q) {
      const float4 d = reinterpret_cast<const float4*>(slot + q * at.width)[at.pair];
      float C[EACH], keep[EACH];
      load_each(C, Cs + q * WIDE + at.sl * EACH);
#pragma unroll
      for (int i = 0; i < PAIR; ++i) {
        const float delta = i == 0 ? d.x : d.z, dy = i == 0 ? d.y : d.w;
        decay(keep, A[i], delta);
#pragma unroll
        for (int j = 0; j < EACH; j += 2) {
          paac::fma2(carry[i][j], carry[i][j + 1], C[j], C[j + 1], dy, dy);
          paac::mul2(carry[i][j], carry[i][j + 1], keep[j], keep[j + 1]);
        }
        sum[i] += delta;
      }
      if ((cuts >> q & 1u) != 0) { zero<SL>(carry); any_cut = true; }
    }
  }
#pragma unroll
  for (int i = 0; i < PAIR; ++i)
    if (at.has(i)) {
      store_states(a.ends + (int64_t)at.chunk * all_states(a) + state_at(a, at.seq, at.channel(i)), carry[i], at.sl * EACH, a.state, a.wide);
      if (at.sl == 0) a.sums[((int64_t)at.chunk * a.n + at.seq) * a.channels + at.channel(i)] = sum[i];
    }
  if (threadIdx.x == 0 && at.tile == 0 && at.group == 0) a.cuts[(int64_t)at.chunk * a.n + at.seq] = any_cut;
}

template <class T, int SL, int VEC>
__global__ void __launch_bounds__(32 * MOST_WARPS)
selective_back_kernel(const __grid_constant__ Args a) {
  paac::pdl_entry();
  extern __shared__ float4 shared[];
  const Place<SL> at(a);
  constexpr int WIDE = EACH * SL, SUMS = sums_of<SL>();
  const int threads = blockDim.x, warps = threads / 32;
  float4* aside = shared;                                                     // [SUBS - 1][4][thread]: the states before SUB steps
  float2* slot = reinterpret_cast<float2*>(aside + (SUBS - 1) * 4 * threads);   // [SPAN][width]: delta, delta x; then sum of G B, of through A
  float* dys = reinterpret_cast<float*>(slot + SPAN * at.width);                // [SPAN][width]: dy'; then C h
  float* Bs = dys + SPAN * at.width;
  float* Cs = Bs + SPAN * WIDE;
  float* bc = Cs + SPAN * WIDE;                                               // [warp][SPAN][SUMS]

  float A[PAIR][EACH], carry[PAIR][EACH], dA[PAIR][EACH], of_channel[2][2] = {};
  load_rates<SL>(A, a, at);
  zero<SL>(carry);
  zero<SL>(dA);
  if (at.chunk < a.chunks - 1) {
    fold_chunks<SL>(carry, A, a, at, a.chunks - 1, -1);
  } else if (a.first != nullptr) {
#pragma unroll
    for (int i = 0; i < PAIR; ++i) load_states(carry[i], a.first + state_at(a, at.seq, at.channel(i)), at.sl * EACH, a.state, a.wide, at.has(i));
  }
  const int k0 = at.chunk * a.chunk, end = a.t - k0 < a.chunk ? a.t : k0 + a.chunk;
  for (int k = k0 + (end - k0 - 1) / SPAN * SPAN; k >= k0; k -= SPAN) {
    const int steps = end - k < SPAN ? end - k : SPAN;
    __syncthreads();                                              // the window before has been written
    for_tile<VEC>(steps, at.room, at.width, [&](int q, int ch) {
      float x[VEC], dt[VEC], dy[VEC];
      load_vec<T, VEC>(x, paac::row_at<T>(a.x, k + q, at.seq) + at.base + ch);
      load_vec<T, VEC>(dt, paac::row_at<T>(a.dt, k + q, at.seq) + at.base + ch);
      load_vec<T, VEC>(dy, paac::row_at<T>(a.dy, k + q, at.seq) + at.base + ch);
      behind_gate<T, VEC>(dy, a, k + q, at.seq, at.base + ch);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float delta = delta_of<T>(a, dt[j], at.base + ch + j);
        slot[q * at.width + ch + j] = make_float2(delta, delta * x[j]);
        dys[q * at.width + ch + j] = dy[j];
      }
    });
    // what channels beyond the last leave in the sums over channels
    for (int i = threadIdx.x; i < steps * (at.width - at.room); i += threads) {
      const int q = i / (at.width - at.room), ch = at.room + i % (at.width - at.room);
      slot[q * at.width + ch] = make_float2(0.f, 0.f);
      dys[q * at.width + ch] = 0.f;
    }
    load_inputs<T, SL>(Bs, a, a.b, k, steps, at.seq, at.group);
    load_inputs<T, SL>(Cs, a, a.c, k, steps, at.seq, at.group);
    const uint32_t cuts = restarts(a, k, steps, at.seq);
    float h[PAIR][EACH];
    const float* mark = a.states + (int64_t)(k / SPAN) * all_states(a);
#pragma unroll
    for (int i = 0; i < PAIR; ++i) load_states(h[i], mark + state_at(a, at.seq, at.channel(i)), at.sl * EACH, a.state, a.wide, at.has(i));
    __syncthreads();

    const int subs = (steps + SUB - 1) / SUB;
    for (int q = 0; q < (subs - 1) * SUB; ++q) {
      const float4 d = reinterpret_cast<const float4*>(slot + q * at.width)[at.pair];
      float B[EACH], keep[EACH];
      load_each(B, Bs + q * WIDE + at.sl * EACH);
      const bool cut = (cuts >> q & 1u) != 0;
      if (cut) zero<SL>(h);
      decay(keep, A[0], d.x);
      if (cut) advance(h[0], h[0], d.y, B); else advance(h[0], keep, d.y, B);
      decay(keep, A[1], d.z);
      if (cut) advance(h[1], h[1], d.w, B); else advance(h[1], keep, d.w, B);
      if (q % SUB == SUB - 1) {
        float4* to = aside + (q / SUB) * 4 * threads + threadIdx.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i * threads] = make_float4(h[i / 2][i % 2 * 4], h[i / 2][i % 2 * 4 + 1], h[i / 2][i % 2 * 4 + 2], h[i / 2][i % 2 * 4 + 3]);
      }
    }
    for (int sub = subs - 1; sub >= 0; --sub) {
      if (sub < subs - 1) {
        if (sub > 0) {
          const float4* from = aside + (sub - 1) * 4 * threads + threadIdx.x;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float4 v = from[i * threads];
            h[i / 2][i % 2 * 4] = v.x; h[i / 2][i % 2 * 4 + 1] = v.y; h[i / 2][i % 2 * 4 + 2] = v.z; h[i / 2][i % 2 * 4 + 3] = v.w;
          }
        } else {
#pragma unroll
          for (int i = 0; i < PAIR; ++i) load_states(h[i], mark + state_at(a, at.seq, at.channel(i)), at.sl * EACH, a.state, a.wide, at.has(i));
        }
      }
      const int q0 = sub * SUB;
      float after[SUB][PAIR][EACH], keep[SUB][PAIR][EACH];
#pragma unroll
      for (int u = 0; u < SUB; ++u)
        if (q0 + u < steps) {
          const int q = q0 + u;
          const float4 d = reinterpret_cast<const float4*>(slot + q * at.width)[at.pair];
          float B[EACH];
          load_each(B, Bs + q * WIDE + at.sl * EACH);
          const bool cut = (cuts >> q & 1u) != 0;
#pragma unroll
          for (int i = 0; i < PAIR; ++i) {
            decay(keep[u][i], A[i], i == 0 ? d.x : d.z);
#pragma unroll
            for (int j = 0; j < EACH; ++j) after[u][i][j] = cut ? 0.f : (u == 0 ? h[i][j] : after[u - 1][i][j]);
            if (cut) {
#pragma unroll
              for (int j = 0; j < EACH; ++j) keep[u][i][j] = 0.f;
            }
            advance(after[u][i], keep[u][i], i == 0 ? d.y : d.w, B);
          }
        }
#pragma unroll
      for (int u = SUB - 1; u >= 0; --u)
        if (q0 + u < steps) {
          const int q = q0 + u;
          const float4 d = reinterpret_cast<const float4*>(slot + q * at.width)[at.pair];
          const float2 dy = reinterpret_cast<const float2*>(dys + q * at.width)[at.pair];
          float B[EACH], C[EACH], over[2 * EACH], y[PAIR], gB[PAIR], rate[PAIR];
          load_each(B, Bs + q * WIDE + at.sl * EACH);
          load_each(C, Cs + q * WIDE + at.sl * EACH);
          const bool cut = (cuts >> q & 1u) != 0;
#pragma unroll
          for (int j = 0; j < 2 * EACH; ++j) over[j] = 0.f;
#pragma unroll
          for (int i = 0; i < PAIR; ++i) {
            const float delta = i == 0 ? d.x : d.z, take = i == 0 ? d.y : d.w, dyi = i == 0 ? dy.x : dy.y;
            y[i] = dot(after[u][i], C);
            float g0 = 0.f, g1 = 0.f, r0 = 0.f, r1 = 0.f;
#pragma unroll
            for (int j = 0; j < EACH; j += 2) {
              float (&G)[EACH] = carry[i];
              paac::fma2(G[j], G[j + 1], C[j], C[j + 1], dyi, dyi);
              paac::fma2(g0, g1, G[j], G[j + 1], B[j], B[j + 1]);
              paac::fma2(over[j], over[j + 1], G[j], G[j + 1], take, take);
              paac::fma2(over[EACH + j], over[EACH + j + 1], after[u][i][j], after[u][i][j + 1], dyi, dyi);
              float t0 = u == 0 ? h[i][j] : after[u == 0 ? 0 : u - 1][i][j], t1 = u == 0 ? h[i][j + 1] : after[u == 0 ? 0 : u - 1][i][j + 1];
              if (cut) t0 = t1 = 0.f;
              paac::mul2(G[j], G[j + 1], keep[u][i][j], keep[u][i][j + 1]);     // what goes on to the step before
              if (cut) G[j] = G[j + 1] = 0.f;
              paac::mul2(t0, t1, G[j], G[j + 1]);                              // through
              paac::fma2(r0, r1, t0, t1, A[i][j], A[i][j + 1]);
              paac::fma2(dA[i][j], dA[i][j + 1], t0, t1, delta, delta);
            }
            gB[i] = g0 + g1;
            rate[i] = r0 + r1;
          }
          const int first = OverChannels<SL>::sum(over);
#pragma unroll
          for (int i = 0; i < OverChannels<SL>::LEFT; ++i) {
            const int s = first + i;
            bc[((threadIdx.x >> 5) * SPAN + q) * SUMS + (s / EACH) * WIDE + at.sl * EACH + s % EACH] = over[i];
          }
          float2* to = slot + q * at.width + at.pair * PAIR;
          float* toy = dys + q * at.width + at.pair * PAIR;
          if (SL == 1) {
            to[0] = make_float2(gB[0], rate[0]);
            to[1] = make_float2(gB[1], rate[1]);
            toy[0] = y[0];
            toy[1] = y[1];
          } else {
            const float g = over_states<SL>(gB[0], gB[1], at.sl), r = over_states<SL>(rate[0], rate[1], at.sl), yy = over_states<SL>(y[0], y[1], at.sl);
            if (at.sl < 2) { to[at.sl] = make_float2(g, r); toy[at.sl] = yy; }
          }
        }
    }
    __syncthreads();

    for (int i = threadIdx.x; i < steps * 2 * a.state; i += threads) {
      const int q = i / (2 * a.state), s = i - q * 2 * a.state, which = s / a.state, of = s - which * a.state;
      float sum = 0.f;
      for (int w = 0; w < warps; ++w) sum += bc[(w * SPAN + q) * SUMS + which * WIDE + of];
      a.bc_sums[((((int64_t)at.tile * a.t + k + q) * a.n + at.seq) * a.groups + at.group) * 2 * a.state + s] = sum;
    }
    for_tile<VEC>(steps, at.room, at.width, [&](int q, int ch) {
      const int c = at.base + ch;
      float x[VEC], dt[VEC], dy[VEC], z[VEC], dx[VEC], dz[VEC];
      load_vec<T, VEC>(x, paac::row_at<T>(a.x, k + q, at.seq) + c);
      load_vec<T, VEC>(dt, paac::row_at<T>(a.dt, k + q, at.seq) + c);
      load_vec<T, VEC>(dy, paac::row_at<T>(a.dy, k + q, at.seq) + c);
      if (a.z.data != nullptr) load_vec<T, VEC>(z, paac::row_at<T>(a.z, k + q, at.seq) + c);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float2 v = slot[q * at.width + ch + j];                 // sum of G B, of through A log2(e)
        const float y = dys[q * at.width + ch + j], D = a.D != nullptr ? a.D[c + j] : 0.f;
        if (a.z.data != nullptr) {
          float s, rest;
          paac::logistic<T>(z[j], s, rest);
          dz[j] = dy[j] * fmaf(D, x[j], y) * fmaf(z[j] * s, rest, s);
          dy[j] *= z[j] * s;
        }
        const float delta = delta_of<T>(a, dt[j], c + j);
        dx[j] = fmaf(D, dy[j], delta * v.x);
        float ddt = fmaf(x[j], v.x, v.y * LN2);
        if (a.softplus) {
          float s, rest;
          paac::logistic<T>(a.bias != nullptr ? dt[j] + a.bias[c + j] : dt[j], s, rest);
          ddt *= s;
        }
        dt[j] = ddt;
        slot[q * at.width + ch + j] = make_float2(dy[j] * x[j], ddt);
      }
      paac::Pack<T, VEC> p;
      if (a.dx.data != nullptr) { p.round(dx); p.store(paac::row_to<T>(a.dx, k + q, at.seq) + c); }
      if (a.ddt.data != nullptr) { p.round(dt); p.store(paac::row_to<T>(a.ddt, k + q, at.seq) + c); }
      if (a.dz.data != nullptr) { p.round(dz); p.store(paac::row_to<T>(a.dz, k + q, at.seq) + c); }
    });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int ch = threadIdx.x + i * threads;
      if (ch < at.room) {
        float d = 0.f, b = 0.f;
        for (int q = 0; q < steps; ++q) {
          const float2 v = slot[q * at.width + ch];
          d += v.x;
          b += v.y;
        }
        of_channel[i][0] += d;
        of_channel[i][1] += b;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < PAIR; ++i)
    if (at.has(i)) {
      store_states(a.a_sums + (int64_t)at.chunk * all_states(a) + state_at(a, at.seq, at.channel(i)), dA[i], at.sl * EACH, a.state, a.wide);
      if (at.chunk == 0 && a.last != nullptr) store_states(a.last + state_at(a, at.seq, at.channel(i)), carry[i], at.sl * EACH, a.state, a.wide);
    }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int ch = threadIdx.x + i * threads;
    if (ch < at.room) {
      float* to = a.d_sums + (((int64_t)at.chunk * a.n + at.seq) * a.channels + at.base + ch) * 2;
      to[0] = of_channel[i][0];
      to[1] = of_channel[i][1];
    }
  }
}

// The blocks' sums added up, in 64 bits: first 32 sums a block over the chunks and sequences (dA; dD and ddt_bias), then dB and dC over the tiles.
struct Finish { float *dA, *dD, *dbias; paac::StepRows db, dc; int a_blocks, d_blocks; };
template <class T>
__global__ void __launch_bounds__(256)
selective_sums_kernel(const __grid_constant__ Args a, const __grid_constant__ Finish f) {
  paac::pdl_entry();
  int block = blockIdx.x;
  if (block < f.a_blocks + f.d_blocks) {
    __shared__ double of_warp[8][32];
    const bool rates = block < f.a_blocks;
    if (!rates) block -= f.a_blocks;
    const int64_t count = (int64_t)a.channels * (rates ? a.state : 2), i = (int64_t)block * 32 + (threadIdx.x & 31), rows = (int64_t)a.chunks * a.n;
    const float* from = rates ? a.a_sums : a.d_sums;
    double sum = 0.0;
    if (i < count)
      for (int64_t r = threadIdx.x >> 5; r < rows; r += 8) sum += from[r * count + i];
    of_warp[threadIdx.x >> 5][threadIdx.x & 31] = sum;
    __syncthreads();
    if (threadIdx.x >= 32 || i >= count) return;
    sum = 0.0;
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += of_warp[u][threadIdx.x];
    if (rates) f.dA[i] = (float)sum;
    else if ((i & 1) == 0) { if (f.dD != nullptr) f.dD[i / 2] = (float)sum; }
    else if (f.dbias != nullptr) f.dbias[i / 2] = (float)sum;
    return;
  }
  block -= f.a_blocks + f.d_blocks;
  const int64_t row = (int64_t)a.groups * 2 * a.state, count = (int64_t)a.t * a.n * row, i = (int64_t)block * 256 + threadIdx.x;
  if (i >= count) return;
  const int64_t at = i / row;
  const int s = (int)(i - at * row), group = s / (2 * a.state), of = s - group * 2 * a.state, which = of / a.state;
  const paac::StepRows& to = which == 0 ? f.db : f.dc;
  if (to.data == nullptr) return;
  double sum = 0.0;
  for (int tile = 0; tile < a.tiles; ++tile) sum += a.bc_sums[tile * count + i];
  paac::row_to<T>(to, at / a.n, at % a.n)[group * a.state + of - which * a.state] = paac::from_f<T>((float)sum);
}

template <class T, int SL, int VEC> cudaError_t backward(const Args& a, const Shape& h, const Finish& f, cudaStream_t st) {
  const dim3 block(32 * h.warps);
  if (h.chunks > 1) {
    const size_t smem = (size_t)SPAN * (h.width * 8 + EACH * SL * 4);
    const cudaError_t e = paac::launch_overlapped_on(st, selective_back_ends_kernel<T, SL, VEC>, dim3((unsigned)(h.blocks / h.chunks * (h.chunks - 1))), block, smem, a);
    if (e != cudaSuccess) return e;
  }
  const size_t smem = (size_t)(SUBS - 1) * 4 * 16 * block.x + (size_t)SPAN * (h.width * 12 + 2 * EACH * SL * 4 + h.warps * sums_of<SL>() * 4);
  static paac::PerDevice<bool> ready;
  int device = -1;
  const bool ok = cudaGetDevice(&device) == cudaSuccess && ready.get(device, [](bool&) {
    return cudaFuncSetAttribute(selective_back_kernel<T, SL, VEC>, cudaFuncAttributeMaxDynamicSharedMemorySize, 160 << 10) == cudaSuccess;
  }) != nullptr;
  if (!ok) return cudaErrorUnknown;
  cudaError_t e = paac::launch_overlapped_on(st, selective_back_kernel<T, SL, VEC>, dim3((unsigned)h.blocks), block, smem, a);
  if (e != cudaSuccess) return e;
  const int64_t inputs = f.db.data != nullptr || f.dc.data != nullptr ? (int64_t)a.t * a.n * a.groups * 2 * a.state : 0;
  const int64_t blocks = f.a_blocks + f.d_blocks + (inputs + 255) / 256;
  if (blocks == 0) return e;
  return paac::launch_overlapped_on(st, selective_sums_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, a, f);
}

}  // namespace

extern "C" int paac_selective_scan_backward(const paac_selective* s, paac_rows x, paac_rows dt, const float* A, paac_rows B, paac_rows C, const float* D,
                                            paac_rows z, const float* dt_bias, const float* states, paac_rows dy, const float* dh_last,
                                            const paac_selective_grads* g, void* workspace, size_t workspace_bytes, void* stream) {
  if (!shape_ok(s) || g == nullptr) return PAAC_ERR_ARG;
  if (g->dx.data == nullptr && g->ddt.data == nullptr && g->dB.data == nullptr && g->dC.data == nullptr && g->dz.data == nullptr && g->dA == nullptr &&
      g->dD == nullptr && g->ddt_bias == nullptr && g->dh0 == nullptr)
    return PAAC_ERR_ARG;
  if (z.data == nullptr && g->dz.data != nullptr) return PAAC_ERR_ARG;
  const int64_t all = (int64_t)s->n * s->c * s->state, inputs = (int64_t)s->groups * s->state;
  paac::StepCheck check(s->t, s->n, size_of(*s), s->restart, s->restart_n, s->restart_t);
  check.steps(x, s->c, false, true);
  check.steps(dt, s->c, false, true);
  check.steps(B, inputs, false, true, false);
  check.steps(C, inputs, false, true, false);
  check.steps(z, s->c, false, false);
  check.steps(dy, s->c, false, true);
  check.steps(g->dx, s->c, true, false);
  check.steps(g->ddt, s->c, true, false);
  check.steps(g->dz, s->c, true, false);
  check.steps(g->dB, inputs, true, false, false);
  check.steps(g->dC, inputs, true, false, false);
  check.floats(A, (int64_t)s->c * s->state, false, true);
  check.floats(D, s->c, false);
  check.floats(dt_bias, s->c, false);
  check.floats(states, all * (((int64_t)s->t + SPAN - 1) / SPAN), false, true);
  check.floats(dh_last, all, false);
  check.floats(g->dA, (int64_t)s->c * s->state, true);
  check.floats(g->dD, s->c, true);
  check.floats(g->ddt_bias, s->c, true);
  check.floats(g->dh0, all, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  const Shape h = shape_of(*s);
  const Room room = room_of(*s, h, true);
  if (workspace == nullptr || ((uintptr_t)workspace & 15u) != 0 || workspace_bytes < room.total) return PAAC_ERR_WORKSPACE;
  check.arrays.keep(workspace, (int64_t)room.total, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  Args a = common_args(*s, h, x, dt, A, B, C, D, z, dt_bias);
  a.dy = paac::step_rows(dy, s->t, s->n); a.dx = paac::step_rows(g->dx, s->t, s->n); a.ddt = paac::step_rows(g->ddt, s->t, s->n);
  a.dz = paac::step_rows(g->dz, s->t, s->n);
  a.first = dh_last; a.last = g->dh0; a.states = const_cast<float*>(states);
  a.wide = states_wide(*s, A, dh_last, g->dh0) && ((uintptr_t)states & 15u) == 0;
  place_room(a, room, h, true, workspace);
  Finish f{};
  f.dA = g->dA; f.dD = g->dD; f.dbias = g->ddt_bias;
  f.db = paac::step_rows(g->dB, s->t, s->n); f.dc = paac::step_rows(g->dC, s->t, s->n);
  f.a_blocks = g->dA != nullptr ? (int)(((int64_t)s->c * s->state + 31) / 32) : 0;
  f.d_blocks = g->dD != nullptr || g->ddt_bias != nullptr ? (int)(((int64_t)s->c * 2 + 31) / 32) : 0;
  const bool four = four_wide(*s, check.align);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return paac::launch_status(by_lanes(h.sl, [&](auto lanes) {
    constexpr int SL = decltype(lanes)::value;
    if (s->type == PAAC_BF16) return four ? backward<bf16, SL, 4>(a, h, f, st) : backward<bf16, SL, 1>(a, h, f, st);
    return four ? backward<float, SL, 4>(a, h, f, st) : backward<float, SL, 1>(a, h, f, st);
  }));
}
