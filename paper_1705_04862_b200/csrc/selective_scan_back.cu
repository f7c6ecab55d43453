// The gradient of the selective state space scan (paac_selective_scan_backward).
//
// With G_t = dL/dh_t, dy' = dy silu(z) and g = exp(delta_t A) (0 at a restart):
//   G_t = C_t dy'_t + g_{t+1} G_{t+1},   through_t = G_t g_t h_{t-1}   (what comes through the exponential, divided by delta A)
//   dx = D dy' + delta sum_s G B,   ddelta = sum_s through A + x sum_s G B,   dz = dy (C h + D x) silu'(z),   ddt = ddelta softplus'
//   dB_t = sum over the group's channels of G delta x,   dC_t = of dy' h,   dA = sum over steps of through delta,   dh0 = g_0 G_0.
// A window of SPAN steps begins at a state that the forward pass has kept.  From there it is walked once, and the state before every SUB-th step
// put aside in shared memory; then SUB steps at a time, the last first, are walked again with states and decays in registers, and
// back.  So a decay is worked out 1 + 7/8 times, and no state but the kept ones comes from memory.  Sums over channels: the thread's
// own two, then by halves over the lanes, over the block's warps in shared memory, and over blocks by a second kernel in a fixed order.
//
// What bounds it: instructions and their latencies; a step takes some 300 for a thread's eight elements of the state, at 2.2 a clock and multiprocessor with the 12
// warps that 168 registers allow.  Measured in a graph (bf16, 16 states, gate): 2048 steps of 8 sequences with 1024 channels 626 us (one by one, with cold caches: what
// the chunks pass on 103, this 513, the sums 18), in float 850 (86 KB of shared memory a block instead of 70: two a multiprocessor, not three).  Tried there: eight states and two channels a thread 1013 (255 registers), one channel 636, four blocks a multiprocessor with spills
// 851.  Left out to see: the first walk 570, writing 588, sums over channels or states 615 to 620.
// Three sequences of 1003 steps with 200 channels of eight states in float 66 us; five steps of 1024 with 512 channels of 16 states 197 (in float 184), one step of
// 550 with 1765 channels of 64 states 269 (264).
#include "per_device.h"
#include "selective.cuh"

namespace {
using namespace paac::selective;
using paac::bf16;

constexpr int SUB = 2, SUBS = SPAN / SUB;
constexpr float LN2 = 0.693147182f;

// The thread's cells of a window's arrays, two windows under way or in use: [2][array][COUNT][thread].
template <class T, class L, int VEC, int ARRAYS> struct Raws {
  typedef Ahead<T, VEC> Way;
  typedef Cells<L, VEC> C;
  static constexpr int COUNT = C::COUNT;
  typename Way::Raw* ring;
  int threads;
  static int bytes(int threads) { return 2 * ARRAYS * COUNT * VEC * (int)sizeof(T) * threads; }
  __device__ __forceinline__ Raws(void* p) : ring((typename Way::Raw*)p + threadIdx.x), threads(blockDim.x) {}
  // `from`: the first row of the window, from the tile's first channel on
  __device__ __forceinline__ void get(int half, int array, const C& cells, const T* from, int64_t step, int steps, int room) const {
    typename Way::Raw* to = ring + (half * ARRAYS + array) * COUNT * threads;
    if constexpr (Way::BYTES >= 4) {
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
        if (cells.there(i, steps, room)) Way::get(to + i * threads, from + cells.step(i) * step + cells.channel(i));
    } else {
      // no asynchronous copy is as small: all loads, then all stores
      typename Way::Raw v[COUNT];
#pragma unroll
      for (int i = 0; i < COUNT; ++i)
        v[i] = cells.there(i, steps, room) ? *reinterpret_cast<const typename Way::Raw*>(from + cells.step(i) * step + cells.channel(i)) : (typename Way::Raw)0;
#pragma unroll
      for (int i = 0; i < COUNT; ++i) to[i * threads] = v[i];
    }
  }
  __device__ __forceinline__ void widen(float (&v)[VEC], int half, int array, int i) const { Way::widen(v, ring + ((half * ARRAYS + array) * COUNT + i) * threads); }
};

// What a chunk passes on from nothing (the last from dh_last) to the one before it, and its deltas' sum.
template <class T, class L, int VEC> int ends_bytes(int width, int threads) { return SPAN * (width * 8 + L::WIDE * 4) + Raws<T, L, VEC, 3>::bytes(threads); }
template <class T, class L, int VEC>
__global__ void __launch_bounds__(32 * MOST_WARPS, 5)
selective_back_ends_kernel(const __grid_constant__ Args a) {
  paac::pdl_entry();
  extern __shared__ float4 shared[];
  Place<L> at(a);
  at.chunk += 1;                                                  // the first passes on to nobody
  typedef Cells<L, VEC> C;
  constexpr int PAIR = L::PAIR, TWOS = L::TWOS, WIDE = L::WIDE;
  float2* slot = reinterpret_cast<float2*>(shared);                 // [SPAN][width]: delta, dy'
  float* Cs = reinterpret_cast<float*>(slot + SPAN * at.width);
  const Raws<T, L, VEC, 3> raws(Cs + SPAN * WIDE);
  const C cells(at.width);
  const bool gate = a.z.data != nullptr;
  const int k0 = at.chunk * a.chunk, end = a.t - k0 < a.chunk ? a.t : k0 + a.chunk;
  const auto fetch = [&](int k, int half) {
    if (k >= k0) {
      const int steps = end - k;
      raws.get(half, 0, cells, paac::row_at<T>(a.dt, k, at.seq) + at.base, a.dt.step, steps, at.room);
      raws.get(half, 1, cells, paac::row_at<T>(a.dy, k, at.seq) + at.base, a.dy.step, steps, at.room);
      if (gate) raws.get(half, 2, cells, paac::row_at<T>(a.z, k, at.seq) + at.base, a.z.step, steps, at.room);
    }
    paac::copies_end_step();
  };
  int k = k0 + (end - k0 - 1) / SPAN * SPAN, half = 0;
  Inputs<T, L> c;
  fetch(k, 0);
  c.fetch(a, a.c, k, end - k, at.seq, at.group);
  float bias[C::TURNS][VEC];
#pragma unroll
  for (int u = 0; u < C::TURNS; ++u) load_of_channels(bias[u], a.bias, at.base + cells.ch + u * (int)blockDim.x, cells.ch + u * (int)blockDim.x < at.room);
  States<L> A, carry;
  float sum[PAIR];
  load_rates<L>(A, a, at);
  zero(carry);
#pragma unroll
  for (int i = 0; i < PAIR; ++i) sum[i] = 0.f;
  if (at.chunk == a.chunks - 1 && a.first != nullptr) load_all<L>(carry, a.first, a, at);
  bool any_cut = false;
  uint32_t mine = restart_of(a, k, end - k, at.seq);
  for (; k >= k0; k -= SPAN, half ^= 1) {
    const int steps = end - k < SPAN ? end - k : SPAN;
    const uint32_t cuts = restarts(mine);
    if (k - SPAN >= k0) mine = restart_of(a, k - SPAN, SPAN, at.seq);
    any_cut = any_cut || cuts != 0;
    fetch(k - SPAN, half ^ 1);
    paac::copies_wait<1>();
    __syncthreads();                                              // the window behind has been walked
    C::each([&](int i, int u) {
      if (cells.there(i, steps, at.room)) {
        float dt[VEC], dy[VEC], z[VEC];
        raws.widen(dt, half, 0, i);
        raws.widen(dy, half, 1, i);
        if (gate) raws.widen(z, half, 2, i);
        float2* to = slot + cells.step(i) * at.width + cells.channel(i);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float v = dt[j] + bias[u][j];
          dt[j] = a.softplus ? paac::softplus<T>(v) : v;
          if (gate) dy[j] *= paac::silu<T>(z[j]);
        }
        if constexpr (VEC == 4) {
          reinterpret_cast<float4*>(to)[0] = make_float4(dt[0], dy[0], dt[1], dy[1]);
          reinterpret_cast<float4*>(to)[1] = make_float4(dt[2], dy[2], dt[3], dy[3]);
        } else {
          to[0] = make_float2(dt[0], dy[0]);
        }
      }
    });
    c.put(Cs, a, a.c, k, steps, at.seq, at.group);
    if (k - SPAN >= k0) c.fetch(a, a.c, k - SPAN, SPAN, at.seq, at.group);
    __syncthreads();
    const auto step = [&](int q) {
      f2 Cq[TWOS], keep[TWOS];
      load_each(Cq, Cs + q * WIDE + at.state0());
#pragma unroll
      for (int i = 0; i < PAIR; ++i) {
        const float2 d = slot[q * at.width + at.pair * PAIR + i];
        const f2 dy = both(d.y);
        decay(keep, A[i], d.x);
#pragma unroll
        for (int j = 0; j < TWOS; ++j) carry[i][j] = mul(keep[j], fma(Cq[j], dy, carry[i][j]));
        sum[i] += d.x;
      }
    };
    if (steps == SPAN && cuts == 0) {
#pragma unroll 4
      for (int q = SPAN - 1; q >= 0; --q) step(q);
    } else {
      for (int q = steps - 1; q >= 0; --q) {
        step(q);
        if ((cuts >> q & 1u) != 0) zero(carry);
      }
    }
  }
  leave_chunk<L>(carry, sum, any_cut, a, at);
}

// SUB steps from `q0` on, from the state h before them: forward with states and decays in registers, and back.  CUTS: with restarts among them, or with less
// steps in the window than it has places for.  slot: [SPAN][width] delta, delta x, dy' -> delta, sum of G B, C h, sum of through A log2(e).
template <class L, bool CUTS>
__device__ __forceinline__ void sub_steps(States<L>& carry, States<L>& dA, const States<L>& h, const States<L>& A, float4* slot, const float* Bs, const float* Cs, float* bc,
                                          const Place<L>& at, int q0, int steps, uint32_t cuts) {
  constexpr int PAIR = L::PAIR, TWOS = L::TWOS, EACH = L::EACH, WIDE = L::WIDE;
  f2 after[SUB][PAIR][TWOS], keep[SUB][PAIR][TWOS];
#pragma unroll
  for (int u = 0; u < SUB; ++u)
    if (!CUTS || q0 + u < steps) {
      const int q = q0 + u;
      f2 B[TWOS];
      load_each(B, Bs + q * WIDE + at.state0());
#pragma unroll
      for (int i = 0; i < PAIR; ++i) {
        const float2 d = *reinterpret_cast<const float2*>(slot + q * at.width + at.pair * PAIR + i);
        const f2 take = both(d.y);
        if (CUTS && (cuts >> q & 1u) != 0) {
#pragma unroll
          for (int j = 0; j < TWOS; ++j) keep[u][i][j] = 0;
          begin(after[u][i], d.y, B);
        } else {
          decay(keep[u][i], A[i], d.x);
#pragma unroll
          for (int j = 0; j < TWOS; ++j) after[u][i][j] = fma(keep[u][i][j], u == 0 ? h[i][j] : after[u == 0 ? 0 : u - 1][i][j], mul(B[j], take));
        }
      }
    }
#pragma unroll
  for (int u = SUB - 1; u >= 0; --u)
    if (!CUTS || q0 + u < steps) {
      const int q = q0 + u;
      f2 B[TWOS], C[TWOS], ofB[TWOS], ofC[TWOS];
      float y[PAIR], gB[PAIR], rate[PAIR];
      load_each(B, Bs + q * WIDE + at.state0());
      load_each(C, Cs + q * WIDE + at.state0());
      const bool cut = CUTS && (cuts >> q & 1u) != 0;
      float4* cell = slot + q * at.width + at.pair * PAIR;
#pragma unroll
      for (int i = 0; i < PAIR; ++i) {
        const float4 d = cell[i];
        const f2 delta = both(d.x), take = both(d.y), dy = both(d.z);
        y[i] = dot(after[u][i], C);
        f2 g = 0, r = 0;
#pragma unroll
        for (int j = 0; j < TWOS; ++j) {
          const f2 G = fma(C[j], dy, carry[i][j]);
          g = j == 0 ? mul(G, B[j]) : fma(G, B[j], g);
          ofB[j] = i == 0 ? mul(G, take) : fma(G, take, ofB[j]);
          ofC[j] = i == 0 ? mul(after[u][i][j], dy) : fma(after[u][i][j], dy, ofC[j]);
          if (cut) {
            carry[i][j] = 0;
          } else {
            carry[i][j] = mul(keep[u][i][j], G);                   // what goes on to the step before
            const f2 through = mul(u == 0 ? h[i][j] : after[u == 0 ? 0 : u - 1][i][j], carry[i][j]);
            r = j == 0 ? mul(through, A[i][j]) : fma(through, A[i][j], r);
            dA[i][j] = fma(through, delta, dA[i][j]);
          }
        }
        gB[i] = sum_of(g);
        rate[i] = cut ? 0.f : sum_of(r);
      }
      {
        float over[2 * EACH];
#pragma unroll
        for (int j = 0; j < TWOS; ++j) { unpack2(ofB[j], over[2 * j], over[2 * j + 1]); unpack2(ofC[j], over[EACH + 2 * j], over[EACH + 2 * j + 1]); }
        typedef Halves<2 * EACH, 16, L::SL> H;
        const int first = H::sum(over);
        float* to = bc + ((threadIdx.x >> 5) * SPAN + q) * 2 * WIDE + (first / EACH) * WIDE + at.state0() + first % EACH;
#pragma unroll
        for (int i = 0; i < H::LEFT; ++i) to[i / EACH * WIDE + i % EACH] = over[i];
      }
      typedef Halves<PAIR, L::SL / 2, 1> H;
      H::sum(gB);
      H::sum(rate);
      const int first = H::sum(y);
#pragma unroll
      for (int i = 0; i < H::LEFT; ++i) {                            // (the lanes of a channel have read the cell when they meet above)
        if (at.pair * PAIR + first + i >= at.room) continue;          // (what is beyond the last stays 0)
        cell[first + i].y = gB[i];
        *reinterpret_cast<float2*>(&cell[first + i].z) = make_float2(y[i], rate[i]);
      }
    }
}

template <class T, class L, int VEC> int back_bytes(int width, int threads) {
  return (SUBS - 1) * L::PAIR * L::EACH * 4 * threads + SPAN * (width * 16 + 2 * L::WIDE * 4 + threads / 32 * 2 * L::WIDE * 4) + Raws<T, L, VEC, 4>::bytes(threads);
}
template <class T, class L, int VEC>
__global__ void __launch_bounds__(32 * MOST_WARPS, 3)
selective_back_kernel(const __grid_constant__ Args a) {
  paac::pdl_entry();
  extern __shared__ float4 shared[];
  const Place<L> at(a);
  typedef Cells<L, VEC> C;
  constexpr int PAIR = L::PAIR, TWOS = L::TWOS, WIDE = L::WIDE, ASIDE = PAIR * TWOS / 2;
  const int threads = blockDim.x, warps = threads / 32, width = at.width;
  ulonglong2* aside = reinterpret_cast<ulonglong2*>(shared) + threadIdx.x;          // [SUBS - 1][ASIDE][thread]: the states before SUB steps
  float4* slot = shared + (SUBS - 1) * ASIDE * threads;
  float* Bs = reinterpret_cast<float*>(slot + SPAN * width);
  float* Cs = Bs + SPAN * WIDE;
  float* bc = Cs + SPAN * WIDE;                                                   // [warp][SPAN][2 WIDE]
  const Raws<T, L, VEC, 4> raws(bc + warps * SPAN * 2 * WIDE);
  const C cells(width);
  const bool gate = a.z.data != nullptr;
  const int k0 = at.chunk * a.chunk, end = a.t - k0 < a.chunk ? a.t : k0 + a.chunk;
  const auto fetch = [&](int k, int half) {
    if (k >= k0) {
      const int steps = end - k;
      raws.get(half, 0, cells, paac::row_at<T>(a.x, k, at.seq) + at.base, a.x.step, steps, at.room);
      raws.get(half, 1, cells, paac::row_at<T>(a.dt, k, at.seq) + at.base, a.dt.step, steps, at.room);
      raws.get(half, 2, cells, paac::row_at<T>(a.dy, k, at.seq) + at.base, a.dy.step, steps, at.room);
      if (gate) raws.get(half, 3, cells, paac::row_at<T>(a.z, k, at.seq) + at.base, a.z.step, steps, at.room);
    }
    paac::copies_end_step();
  };
  int k = k0 + (end - k0 - 1) / SPAN * SPAN, half = 0;
  Inputs<T, L> b, c;
  fetch(k, 0);
  b.fetch(a, a.b, k, end - k, at.seq, at.group);
  c.fetch(a, a.c, k, end - k, at.seq, at.group);
  float bias[C::TURNS][VEC], D[C::TURNS][VEC], dD[C::TURNS][VEC], dbias[C::TURNS][VEC];
#pragma unroll
  for (int u = 0; u < C::TURNS; ++u) {
    const int ch = cells.ch + u * threads;
    load_of_channels(bias[u], a.bias, at.base + ch, ch < at.room);
    load_of_channels(D[u], a.D, at.base + ch, ch < at.room);
#pragma unroll
    for (int j = 0; j < VEC; ++j) dD[u][j] = dbias[u][j] = 0.f;
  }
  States<L> A, carry, dA;
  load_rates<L>(A, a, at);
  zero(carry);
  zero(dA);
  if (at.chunk < a.chunks - 1) fold_chunks<L>(carry, A, a, at, a.chunks - 1, -1);
  else if (a.first != nullptr) load_all<L>(carry, a.first, a, at);
  // what channels beyond the last leave in the sums over channels: nothing
  for (int i = threadIdx.x; i < SPAN * (width - at.room); i += threads) slot[i / (width - at.room) * width + at.room + i % (width - at.room)] = make_float4(0.f, 0.f, 0.f, 0.f);

  uint32_t mine = restart_of(a, k, end - k, at.seq);
  States<L> kept;                                                 // the state before the window's first step
  load_all<L>(kept, a.states + (int64_t)(k / SPAN) * all_states(a), a, at);
  for (; k >= k0; k -= SPAN, half ^= 1) {
    const int steps = end - k < SPAN ? end - k : SPAN;
    const uint32_t cuts = restarts(mine);
    if (k - SPAN >= k0) mine = restart_of(a, k - SPAN, SPAN, at.seq);
    const float* mark = a.states + (int64_t)(k / SPAN) * all_states(a);
    States<L> h;
#pragma unroll
    for (int i = 0; i < PAIR; ++i)
#pragma unroll
      for (int j = 0; j < TWOS; ++j) h[i][j] = kept[i][j];
    fetch(k - SPAN, half ^ 1);
    paac::copies_wait<1>();
    __syncthreads();                                              // the window behind has been written
    C::each([&](int i, int u) {
      if (cells.there(i, steps, at.room)) {
        float x[VEC], dt[VEC], dy[VEC], z[VEC];
        raws.widen(x, half, 0, i);
        raws.widen(dt, half, 1, i);
        raws.widen(dy, half, 2, i);
        if (gate) raws.widen(z, half, 3, i);
        float4* to = slot + cells.step(i) * width + cells.channel(i);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float v = dt[j] + bias[u][j], delta = a.softplus ? paac::softplus<T>(v) : v;
          if (gate) dy[j] *= paac::silu<T>(z[j]);
          to[j] = make_float4(delta, delta * x[j], dy[j], 0.f);
        }
      }
    });
    b.put(Bs, a, a.b, k, steps, at.seq, at.group);
    c.put(Cs, a, a.c, k, steps, at.seq, at.group);
    if (k - SPAN >= k0) {
      b.fetch(a, a.b, k - SPAN, SPAN, at.seq, at.group);
      c.fetch(a, a.c, k - SPAN, SPAN, at.seq, at.group);
    }
    __syncthreads();

    const bool plain = steps == SPAN && cuts == 0;
    const int subs = (steps + SUB - 1) / SUB;
    const auto step = [&](int q, bool cut) {
      f2 B[TWOS];
      load_each(B, Bs + q * WIDE + at.state0());
#pragma unroll
      for (int i = 0; i < PAIR; ++i) {
        const float2 d = *reinterpret_cast<const float2*>(slot + q * width + at.pair * PAIR + i);
        if (cut) {
          begin(h[i], d.y, B);
        } else {
          f2 keep[TWOS];
          decay(keep, A[i], d.x);
          advance(h[i], keep, d.y, B);
        }
      }
    };
    for (int sub = 0; sub + 1 < subs; ++sub) {
      if (plain) {
#pragma unroll
        for (int u = 0; u < SUB; ++u) step(sub * SUB + u, false);
      } else {
        for (int u = 0; u < SUB; ++u) step(sub * SUB + u, (cuts >> (sub * SUB + u) & 1u) != 0);
      }
#pragma unroll
      for (int i = 0; i < ASIDE; ++i) aside[(sub * ASIDE + i) * threads] = make_ulonglong2(h[i * 2 / TWOS][i * 2 % TWOS], h[i * 2 / TWOS][i * 2 % TWOS + 1]);
    }
    for (int sub = subs - 1; sub >= 0; --sub) {
      if (sub == 0) {
        load_all<L>(h, mark, a, at);
      } else if (sub < subs - 1) {
#pragma unroll
        for (int i = 0; i < ASIDE; ++i) {
          const ulonglong2 v = aside[((sub - 1) * ASIDE + i) * threads];
          h[i * 2 / TWOS][i * 2 % TWOS] = v.x;
          h[i * 2 / TWOS][i * 2 % TWOS + 1] = v.y;
        }
      }
      if (sub == 0 && k - SPAN >= k0) load_all<L>(kept, mark - all_states(a), a, at);
      if (plain) sub_steps<L, false>(carry, dA, h, A, slot, Bs, Cs, bc, at, sub * SUB, steps, cuts);
      else sub_steps<L, true>(carry, dA, h, A, slot, Bs, Cs, bc, at, sub * SUB, steps, cuts);
    }
    __syncthreads();

    {
      float* to = a.bc_sums + ((((int64_t)at.tile * a.t + k) * a.n + at.seq) * a.groups + at.group) * 2 * a.state;
      const int64_t row = (int64_t)a.n * a.groups * 2 * a.state;
      for (int i = threadIdx.x; i < steps * 2 * WIDE; i += threads) {
        const int q = i / (2 * WIDE), s = i % (2 * WIDE), which = s / WIDE, of = s % WIDE;
        if (of >= a.state) continue;
        float sum = 0.f;
        for (int w = 0; w < warps; ++w) sum += bc[(w * SPAN + q) * 2 * WIDE + s];
        to[q * row + which * a.state + of] = sum;
      }
    }
    T *dx_at = paac::row_to<T>(a.dx, k, at.seq) + at.base, *ddt_at = paac::row_to<T>(a.ddt, k, at.seq) + at.base, *dz_at = paac::row_to<T>(a.dz, k, at.seq) + at.base;
    C::each([&](int i, int u) {
      if (cells.there(i, steps, at.room)) {
        const int q = cells.step(i), ch = cells.channel(i);
        float x[VEC], dt[VEC], dy[VEC], z[VEC], dx[VEC], ddt[VEC], dz[VEC];
        raws.widen(x, half, 0, i);
        raws.widen(dt, half, 1, i);
        raws.widen(dy, half, 2, i);
        if (gate) raws.widen(z, half, 3, i);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float4 v = slot[q * width + ch + j];                   // delta, sum of G B, C h, sum of through A log2(e)
          if (gate) {
            float s, rest;
            paac::logistic<T>(z[j], s, rest);
            dz[j] = dy[j] * fmaf(D[u][j], x[j], v.z) * fmaf(z[j] * s, rest, s);
            dy[j] *= z[j] * s;
          }
          dx[j] = fmaf(D[u][j], dy[j], v.x * v.y);
          ddt[j] = fmaf(x[j], v.y, v.w * LN2);
          if (a.softplus) {
            float s, rest;
            paac::logistic<T>(dt[j] + bias[u][j], s, rest);
            ddt[j] *= s;
          }
          dD[u][j] = fmaf(dy[j], x[j], dD[u][j]);
          dbias[u][j] += ddt[j];
        }
        paac::Pack<T, VEC> p;
        if (a.dx.data != nullptr) { p.round(dx); p.store(dx_at + q * a.dx.step + ch); }
        if (a.ddt.data != nullptr) { p.round(ddt); p.store(ddt_at + q * a.ddt.step + ch); }
        if (a.dz.data != nullptr) { p.round(dz); p.store(dz_at + q * a.dz.step + ch); }
      }
    });
  }
  store_all<L>(a.a_sums + (int64_t)at.chunk * all_states(a), dA, a, at);
  if (at.chunk == 0 && a.last != nullptr) store_all<L>(a.last, carry, a, at);
  // sums over the threads with the same channels, in the slots' place: [row][width]
  __syncthreads();
  float2* sums = reinterpret_cast<float2*>(slot);
  constexpr int ROWS = C::ROWS < SPAN ? C::ROWS : SPAN;
#pragma unroll
  for (int u = 0; u < C::TURNS; ++u)
    if (cells.row < ROWS)
#pragma unroll
      for (int j = 0; j < VEC; ++j) sums[cells.row * width + cells.ch + u * threads + j] = make_float2(dD[u][j], dbias[u][j]);
  __syncthreads();
  for (int ch = threadIdx.x; ch < at.room; ch += threads) {
    float2 sum = make_float2(0.f, 0.f);
    for (int r = 0; r < ROWS; ++r) { sum.x += sums[r * width + ch].x; sum.y += sums[r * width + ch].y; }
    reinterpret_cast<float2*>(a.d_sums)[((int64_t)at.chunk * a.n + at.seq) * a.channels + at.base + ch] = sum;
  }
}

// A few steps: a channel's states over LANES threads side by side, eight to each, with the states behind every step in registers.  A lane works out what every
// LANES-th step needs and, once sums over states are there, writes those steps' gradients.  A block takes its channels through several sequences one after another, so
// that the sums over steps and sequences are few.
constexpr int FEW_THREADS = 128, FEW_EACH = 8, MOST_FEW = 8;
template <class T, int LANES, int STEPS>
__global__ void __launch_bounds__(FEW_THREADS, STEPS == 1 ? 6 : 2)
selective_few_back_kernel(const __grid_constant__ Args a, int sequences) {
  paac::pdl_entry();
  constexpr int COLUMNS = FEW_THREADS / LANES, WIDE = FEW_EACH * LANES, TWOS = FEW_EACH / 2, OWN = (STEPS + LANES - 1) / LANES, WARPS = FEW_THREADS / 32;
  __shared__ __align__(16) float Bs[STEPS][WIDE], Cs[STEPS][WIDE], bc[WARPS][STEPS][2 * WIDE];
  const uint32_t tiles = (uint32_t)a.tiles * a.groups, split = blockIdx.x / tiles, in = blockIdx.x - split * tiles;
  const int group = (int)in / a.tiles, tile = (int)in % a.tiles, of_group = a.channels / a.groups;
  const int column = tile * COLUMNS + threadIdx.x / LANES, sl = threadIdx.x % LANES, s0 = FEW_EACH * sl;
  const bool there = column < of_group;
  const int ch = group * of_group + (there ? column : 0), steps = a.t;
  const float bias = a.bias != nullptr ? a.bias[ch] : 0.f, D = a.D != nullptr ? a.D[ch] : 0.f;
  f2 A[TWOS], dA[TWOS] = {};
  load_states(A, a.A + (int64_t)ch * a.state, s0, a.state, a.wide, there);
#pragma unroll
  for (int j = 0; j < TWOS; ++j) A[j] = mul(A[j], both(LOG2E));
  float dD = 0.f, dbias = 0.f;
  const int64_t first = (int64_t)split * sequences, beyond = first + sequences < a.n ? first + sequences : a.n;
  for (int64_t seq = first; seq < beyond; ++seq) {
    const int64_t at = (seq * a.channels + ch) * a.state;
    // the lane's own steps
    float x[OWN], dt[OWN], dy[OWN], z[OWN], delta[OWN];
    uint32_t mine = 0;
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
      const int q = o * LANES + sl;
      const bool own = q < steps;
      x[o] = own ? paac::to_f(paac::row_at<T>(a.x, q, seq)[ch]) : 0.f;
      dt[o] = own ? paac::to_f(paac::row_at<T>(a.dt, q, seq)[ch]) + bias : 0.f;
      dy[o] = own && there ? paac::to_f(paac::row_at<T>(a.dy, q, seq)[ch]) : 0.f;
      z[o] = own && a.z.data != nullptr ? paac::to_f(paac::row_at<T>(a.z, q, seq)[ch]) : 0.f;
      if (own && a.restart.data != nullptr && a.restart.data[q * a.restart.step + seq * a.restart.seq] != 0) mine |= 1u << q;
    }
    f2 h[TWOS], carry[TWOS] = {};
    load_states(h, a.states + at, s0, a.state, a.wide, there);
    if (a.first != nullptr) load_states(carry, a.first + at, s0, a.state, a.wide, there);
    __syncthreads();                     // the sequence before has been worked on
    {
      const T *b = paac::row_at<T>(a.b, 0, seq) + group * a.state, *c = paac::row_at<T>(a.c, 0, seq) + group * a.state;
      for (int i = threadIdx.x; i < steps * WIDE; i += FEW_THREADS) {
        const int q = i / WIDE, s = i % WIDE;
        Bs[q][s] = s < a.state ? paac::to_f(b[q * a.b.step + s]) : 0.f;
        Cs[q][s] = s < a.state ? paac::to_f(c[q * a.c.step + s]) : 0.f;
      }
    }
    uint32_t cuts = mine;                // (the lanes of a channel have them between them)
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) cuts |= __shfl_xor_sync(0xffffffffu, cuts, d);
    float gated[OWN], take[OWN];
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
      const float soft = paac::softplus<T>(dt[o]);
      delta[o] = there ? (a.softplus ? soft : dt[o]) : 0.f;
      take[o] = delta[o] * x[o];
      gated[o] = a.z.data != nullptr ? dy[o] * paac::silu<T>(z[o]) : dy[o];
    }
    __syncthreads();
    f2 after[STEPS][TWOS];
#pragma unroll
    for (int q = 0; q < STEPS; ++q)
      if (q < steps) {
        const float d = __shfl_sync(0xffffffffu, delta[q / LANES], q % LANES, LANES), t = __shfl_sync(0xffffffffu, take[q / LANES], q % LANES, LANES);
        f2 B[TWOS], keep[TWOS];
        load_each(B, &Bs[q][s0]);
        if ((cuts >> q & 1u) != 0) {
          begin(after[q], t, B);
        } else {
          decay(keep, A, d);
#pragma unroll
          for (int j = 0; j < TWOS; ++j) after[q][j] = fma(keep[j], q == 0 ? h[j] : after[q == 0 ? 0 : q - 1][j], mul(B[j], both(t)));
        }
      }
    float y[OWN * LANES] = {}, gB[OWN * LANES] = {}, rate[OWN * LANES] = {};
#pragma unroll
    for (int q = STEPS - 1; q >= 0; --q) {
      if (q >= steps) continue;
      const float d = __shfl_sync(0xffffffffu, delta[q / LANES], q % LANES, LANES), t = __shfl_sync(0xffffffffu, take[q / LANES], q % LANES, LANES),
                  g = __shfl_sync(0xffffffffu, gated[q / LANES], q % LANES, LANES);
      const bool cut = (cuts >> q & 1u) != 0;
      f2 B[TWOS], C[TWOS], keep[TWOS], sumB = 0, sumR = 0;
      load_each(B, &Bs[q][s0]);
      load_each(C, &Cs[q][s0]);
      decay(keep, A, d);
      y[q] = dot(after[q], C);
      float over[2 * FEW_EACH];
#pragma unroll
      for (int j = 0; j < TWOS; ++j) {
        const f2 G = fma(C[j], both(g), carry[j]);
        sumB = fma(G, B[j], sumB);
        unpack2(mul(G, both(t)), over[2 * j], over[2 * j + 1]);
        unpack2(mul(after[q][j], both(g)), over[FEW_EACH + 2 * j], over[FEW_EACH + 2 * j + 1]);
        if (cut) {
          carry[j] = 0;
        } else {
          carry[j] = mul(keep[j], G);
          const f2 through = mul(q == 0 ? h[j] : after[q == 0 ? 0 : q - 1][j], carry[j]);
          sumR = fma(through, A[j], sumR);
          dA[j] = fma(through, both(d), dA[j]);
        }
      }
      gB[q] = sum_of(sumB);
      rate[q] = cut ? 0.f : sum_of(sumR);
      if (!there) {                      // (a column beyond the last is in no sum)
#pragma unroll
        for (int j = 0; j < 2 * FEW_EACH; ++j) over[j] = 0.f;
      }
      typedef Halves<2 * FEW_EACH, 16, LANES> H;
      const int from = H::sum(over);
#pragma unroll
      for (int i = 0; i < H::LEFT; ++i) bc[threadIdx.x / 32][q][(from + i) / FEW_EACH * WIDE + s0 + (from + i) % FEW_EACH] = over[i];
    }
#pragma unroll
    for (int o = 0; o < OWN; ++o) {
      float v[3][LANES];
#pragma unroll
      for (int u = 0; u < LANES; ++u) { v[0][u] = y[o * LANES + u]; v[1][u] = gB[o * LANES + u]; v[2][u] = rate[o * LANES + u]; }
#pragma unroll
      for (int i = 0; i < 3; ++i) Halves<LANES, LANES / 2, 1>::sum(v[i]);      // (lane sl is left with step o LANES + sl's)
      const int q = o * LANES + sl;
      if (!there || q >= steps) continue;
      if (a.dz.data != nullptr) {
        float s, rest;
        paac::logistic<T>(z[o], s, rest);
        paac::row_to<T>(a.dz, q, seq)[ch] = paac::from_f<T>(dy[o] * fmaf(D, x[o], v[0][0]) * fmaf(z[o] * s, rest, s));
      }
      float ddt = fmaf(x[o], v[1][0], v[2][0] * LN2);
      if (a.softplus) {
        float s, rest;
        paac::logistic<T>(dt[o], s, rest);
        ddt *= s;
      }
      if (a.dx.data != nullptr) paac::row_to<T>(a.dx, q, seq)[ch] = paac::from_f<T>(fmaf(D, gated[o], delta[o] * v[1][0]));
      if (a.ddt.data != nullptr) paac::row_to<T>(a.ddt, q, seq)[ch] = paac::from_f<T>(ddt);
      dD = fmaf(gated[o], x[o], dD);
      dbias += ddt;
    }
    if (a.last != nullptr && there) store_states(a.last + at, carry, s0, a.state, a.wide);
    __syncthreads();
    for (int i = threadIdx.x; i < steps * 2 * WIDE; i += FEW_THREADS) {
      const int q = i / (2 * WIDE), s = i % (2 * WIDE), which = s / WIDE, of = s % WIDE;
      if (of >= a.state) continue;
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) sum += bc[w][q][s];
      a.bc_sums[(((((int64_t)tile * a.t + q) * a.n + seq) * a.groups + group) * 2 + which) * a.state + of] = sum;
    }
  }
  if (there) store_states(a.a_sums + ((int64_t)split * a.channels + ch) * a.state, dA, s0, a.state, a.wide);
#pragma unroll
  for (int d = 1; d < LANES; d *= 2) {
    dD += __shfl_xor_sync(0xffffffffu, dD, d);
    dbias += __shfl_xor_sync(0xffffffffu, dbias, d);
  }
  if (there && sl == 0) reinterpret_cast<float2*>(a.d_sums)[(int64_t)split * a.channels + ch] = make_float2(dD, dbias);
}

// The blocks' sums added up, in 64 bits: first 32 sums a block over their rows (dA; dD and ddt_bias), then dB and dC over the tiles.
struct Finish { float *dA, *dD, *dbias; paac::StepRows db, dc; int a_blocks, d_blocks; int64_t rows; };      // rows: of sums over steps
template <class T>
__global__ void __launch_bounds__(256)
selective_sums_kernel(const __grid_constant__ Args a, const __grid_constant__ Finish f) {
  paac::pdl_entry();
  int64_t block = blockIdx.x;
  if (block < f.a_blocks + f.d_blocks) {
    __shared__ double of_warp[8][32];
    const bool rates = block < f.a_blocks;
    if (!rates) block -= f.a_blocks;
    const int64_t count = (int64_t)a.channels * (rates ? a.state : 2), i = block * 32 + (threadIdx.x & 31), rows = f.rows;
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
  const int64_t row = (int64_t)a.groups * 2 * a.state, count = (int64_t)a.t * a.n * row, i = block * 256 + threadIdx.x;
  if (i >= count) return;
  const int64_t at = i / row;
  const int s = (int)(i - at * row), group = s / (2 * a.state), of = s - group * 2 * a.state, which = of / a.state;
  const paac::StepRows& to = which == 0 ? f.db : f.dc;
  if (to.data == nullptr) return;
  double sum = 0.0;
  for (int tile = 0; tile < a.tiles; ++tile) sum += a.bc_sums[tile * count + i];
  paac::row_to<T>(to, at / a.n, at % a.n)[group * a.state + of - which * a.state] = paac::from_f<T>((float)sum);
}

// Layouts: the gradient's, and that of the kernel that works out what chunks pass on, whose tiles are its own.
template <int SL> using Back = Layout<4, 2, SL>;
template <int PAIR, int SL> using Ends = Layout<8, PAIR, SL>;
Shape shape_of(const paac_selective& s) {
  if (s.t > MOST_FEW) {
    Shape h = tiled(s, 4, 2, 128);
    cut_steps(h, s, 148 * 36, 2);                           // (three times what is resident: waves that fill, and chunks for the kernel before)
    h.rows = (int64_t)h.chunks * s.n;
    return h;
  }
  // few steps: a block takes as many sequences one after another as leave 16 blocks to a multiprocessor
  Shape h = tiled(s, FEW_EACH, 1, 128 * FEW_THREADS);
  h.warps = FEW_THREADS / 32;
  h.width = FEW_THREADS / h.sl;
  h.tiles = (s.c / s.groups + h.width - 1) / h.width;
  const int64_t rows = 148 * 16 / ((int64_t)h.tiles * s.groups) + 1;
  h.each = (int)((s.n + rows - 1) / rows);
  h.rows = (s.n + (int64_t)h.each - 1) / h.each;
  h.blocks = (int64_t)h.tiles * s.groups * h.rows;
  return h;
}

template <class K> bool may_take(K kernel) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 << 10) == cudaSuccess; }
template <class T, class L, int VEC> cudaError_t ends(Args a, const paac_selective& s, cudaStream_t st) {
  const Shape h = tiled(s, L::EACH, L::PAIR, 128);
  a.tiles = h.tiles;
  static paac::PerDevice<bool> ready;
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess || ready.get(device, [](bool&) { return may_take(selective_back_ends_kernel<T, L, VEC>); }) == nullptr) return cudaErrorUnknown;
  const int threads = 32 * h.warps;
  return paac::launch_overlapped_on(st, selective_back_ends_kernel<T, L, VEC>, dim3((unsigned)(h.blocks * (a.chunks - 1))), dim3(threads), (ends_bytes<T, L, VEC>(h.width, threads)), a);
}
template <class T, class L, int VEC> cudaError_t steps(const Args& a, const Shape& h, cudaStream_t st) {
  static paac::PerDevice<bool> ready;
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess || ready.get(device, [](bool&) { return may_take(selective_back_kernel<T, L, VEC>); }) == nullptr) return cudaErrorUnknown;
  const int threads = 32 * h.warps;
  return paac::launch_overlapped_on(st, selective_back_kernel<T, L, VEC>, dim3((unsigned)h.blocks), dim3(threads), (back_bytes<T, L, VEC>(h.width, threads)), a);
}
template <class T> cudaError_t finish(const Args& a, const Finish& f, cudaStream_t st) {
  const int64_t inputs = f.db.data != nullptr || f.dc.data != nullptr ? (int64_t)a.t * a.n * a.groups * 2 * a.state : 0;
  const int64_t blocks = f.a_blocks + f.d_blocks + (inputs + 255) / 256;
  if (blocks == 0) return cudaSuccess;
  return paac::launch_overlapped_on(st, selective_sums_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, a, f);
}
template <class T, int VEC> cudaError_t backward(const Args& a, const paac_selective& s, const Shape& h, const Finish& f, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  if (s.t <= MOST_FEW) {
    e = by_lanes<8>(h.sl, [&](auto lanes) {
      constexpr int LANES = decltype(lanes)::value;
      return paac::launch_overlapped_on(st, s.t == 1 ? selective_few_back_kernel<T, LANES, 1> : selective_few_back_kernel<T, LANES, MOST_FEW>, dim3((unsigned)h.blocks),
                                        dim3(FEW_THREADS), 0, a, h.each);
    });
    return e != cudaSuccess ? e : finish<T>(a, f, st);
  }
  if (h.chunks > 1)
    e = by_lanes<8>(tiled(s, 8, 2, 128).sl, [&](auto lanes) {
      constexpr int SL = decltype(lanes)::value;
      // (two channels a thread where that leaves no lane of a warp without any)
      return s.c / s.groups * SL <= 32 ? ends<T, Ends<1, SL>, VEC>(a, s, st) : ends<T, Ends<2, SL>, VEC>(a, s, st);
    });
  if (e != cudaSuccess) return e;
  e = by_lanes<16>(h.sl, [&](auto lanes) { return steps<T, Back<decltype(lanes)::value>, VEC>(a, h, st); });
  if (e != cudaSuccess) return e;
  return finish<T>(a, f, st);
}

}  // namespace

size_t paac::selective::gradient_room(const paac_selective& s) { return room_of(s, ::shape_of(s), true).total; }

extern "C" int paac_selective_scan_backward(const paac_selective* s, const paac_selective_grads* g, void* stream) {
  if (!shape_ok(s) || g == nullptr) return PAAC_ERR_ARG;
  if (g->dx.data == nullptr && g->ddt.data == nullptr && g->dB.data == nullptr && g->dC.data == nullptr && g->dz.data == nullptr && g->dA == nullptr &&
      g->dD == nullptr && g->ddt_bias == nullptr && g->dh0 == nullptr)
    return PAAC_ERR_ARG;
  if (s->z.data == nullptr && g->dz.data != nullptr) return PAAC_ERR_ARG;
  const int64_t all = (int64_t)s->n * s->c * s->state, inputs = (int64_t)s->groups * s->state;
  paac::StepCheck check(s->t, s->n, size_of(*s), s->restart, s->restart_n, s->restart_t);
  check.steps(s->x, s->c, false, true);
  check.steps(s->dt, s->c, false, true);
  check.steps(s->B, inputs, false, true, false);
  check.steps(s->C, inputs, false, true, false);
  check.steps(s->z, s->c, false, false);
  check.steps(g->dy, s->c, false, true);
  check.steps(g->dx, s->c, true, false);
  check.steps(g->ddt, s->c, true, false);
  check.steps(g->dz, s->c, true, false);
  check.steps(g->dB, inputs, true, false, false);
  check.steps(g->dC, inputs, true, false, false);
  check.floats(s->A, (int64_t)s->c * s->state, false, true);
  check.floats(s->D, s->c, false);
  check.floats(s->dt_bias, s->c, false);
  check.floats(g->states, all * (((int64_t)s->t + SPAN - 1) / SPAN), false, true);
  check.floats(g->dh_last, all, false);
  check.floats(g->dA, (int64_t)s->c * s->state, true);
  check.floats(g->dD, s->c, true);
  check.floats(g->ddt_bias, s->c, true);
  check.floats(g->dh0, all, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  const Shape h = ::shape_of(*s);
  const Room room = room_of(*s, h, true);
  if (g->workspace == nullptr || ((uintptr_t)g->workspace & 15u) != 0 || g->workspace_bytes < room.total) return PAAC_ERR_WORKSPACE;
  check.arrays.keep(g->workspace, (int64_t)room.total, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  Args a = common_args(*s, h);
  a.dy = paac::step_rows(g->dy, s->t, s->n); a.dx = paac::step_rows(g->dx, s->t, s->n); a.ddt = paac::step_rows(g->ddt, s->t, s->n);
  a.dz = paac::step_rows(g->dz, s->t, s->n);
  a.first = g->dh_last; a.last = g->dh0; a.states = const_cast<float*>(g->states);
  a.wide = states_wide(*s, s->A, g->dh_last, g->dh0) && ((uintptr_t)g->states & 15u) == 0;
  place_room(a, room, h, true, g->workspace);
  Finish f{};
  f.dA = g->dA; f.dD = g->dD; f.dbias = g->ddt_bias;
  f.db = paac::step_rows(g->dB, s->t, s->n); f.dc = paac::step_rows(g->dC, s->t, s->n);
  f.rows = h.rows;
  f.a_blocks = g->dA != nullptr ? (int)(((int64_t)s->c * s->state + 31) / 32) : 0;
  f.d_blocks = g->dD != nullptr || g->ddt_bias != nullptr ? (int)(((int64_t)s->c * 2 + 31) / 32) : 0;
  const bool four = four_wide(*s, check.align);
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (s->type == PAAC_BF16) return paac::launch_status(four ? backward<bf16, 4>(a, *s, h, f, st) : backward<bf16, 1>(a, *s, h, f, st));
  return paac::launch_status(four ? backward<float, 4>(a, *s, h, f, st) : backward<float, 1>(a, *s, h, f, st));
}
