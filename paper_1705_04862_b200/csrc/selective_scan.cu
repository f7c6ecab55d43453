// The selective state space scan forward (paac_selective_scan): h_t = exp(delta_t A) h_{t-1} + delta_t B_t x_t, y_t = (C_t h_t + D x_t) silu(z_t).
//
// Of every element of the state a step takes an exponential and four multiply-adds; the exponentials, 16 a clock and multiprocessor, bound
// it where channels have 16 states: memory has four values to move for 16 of them.
//
// While the steps of a window are walked, the window before it is written and the one behind it made ready (delta and delta x), a few of either's
// channels behind every four steps, so that one barrier does for a window and no unit waits for the others; arrays are copied to
// shared memory some windows before that.
//
// Few channels are walked by threads with four states, in one go, or by threads with eight whose steps are cut into chunks: a first kernel finds
// what every chunk passes on (its exponentials are worked out again by the second), from which the second makes every chunk's beginning.
//
// Measured in a graph (bf16, 16 states, gate, inputs in turn that L2 does not hold together): 8192 steps of 2 sequences with 2048 channels 425 us (0.54 G
// exponentials twice, which alone are 240; issue slots 48 and 57 %), 2048 steps of 8 with 1024, with the states for the way back, 248 (in one go 262), five steps of
// 1024 with 512 40 (122 MB at 3.0 TB/s, issue slots 67 %), a step of 32 with 1024 3.0; that call through the binding 12.6.
#include "per_device.h"
#include "selective.cuh"

namespace {
using namespace paac::selective;
using paac::bf16;

constexpr int FOUR = 4;                // steps walked at a time

// Windows of x that are under way or in use, and of dt and z: x is needed when a window is made ready and two windows later when it is written, dt for the first
// alone and z for the second, so that each of these is fetched where the last one of it was.  With four states a thread a block has a multiprocessor almost to
// itself and looks further ahead.
template <class L, bool ENDS> constexpr int ring_of() { return ENDS ? 2 : L::EACH == 4 ? 4 : 3; }
template <class L, bool ENDS> constexpr int spare_of() { return ENDS ? 2 : ring_of<L, ENDS>() - 2; }
// Bytes of shared memory of a block.
template <class T, class L, int VEC, bool ENDS> int shared_bytes(int width, int threads) {
  return 2 * SPAN * (width * 8 + L::WIDE * 4 * (ENDS ? 1 : 2)) + (ring_of<L, ENDS>() + (ENDS ? 1 : 2) * spare_of<L, ENDS>()) * Cells<L, VEC>::COUNT * VEC * (int)sizeof(T) * threads;
}

// ENDS: what a chunk passes on from nothing (the first from h0), and its deltas' sum; otherwise all that is written.
template <class T, class L, int VEC, bool ENDS>
__global__ void __launch_bounds__(32 * MOST_WARPS, 4)
selective_scan_kernel(const __grid_constant__ Args a) {
  paac::pdl_entry();
  extern __shared__ float4 shared[];
  const Place<L> at(a);
  typedef Ahead<T, VEC> Way;
  typedef Cells<L, VEC> C;
  constexpr int PAIR = L::PAIR, TWOS = L::TWOS, WIDE = L::WIDE, COUNT = C::COUNT, RING = ring_of<L, ENDS>(), SPARE = spare_of<L, ENDS>();
  const int threads = blockDim.x, width = at.width;
  float2* slots = reinterpret_cast<float2*>(shared);                // [2][SPAN][width]: delta, delta x; then y in the second's place
  float* Bs = reinterpret_cast<float*>(slots + 2 * SPAN * width);     // [2][SPAN][WIDE]
  float* Cs = Bs + 2 * SPAN * WIDE;
  typename Way::Raw* ring = reinterpret_cast<typename Way::Raw*>(ENDS ? Cs : Cs + 2 * SPAN * WIDE) + threadIdx.x;      // [RING] x, [SPARE] dt, [SPARE] z, of [COUNT][thread]
  const int ring_step = COUNT * threads;
  typename Way::Raw *dt_ring = ring + RING * ring_step, *z_ring = dt_ring + SPARE * ring_step;

  const int k0 = at.chunk * a.chunk, end = a.t - k0 < a.chunk ? a.t : k0 + a.chunk;
  const C cells(width);
  const bool gate = !ENDS && a.z.data != nullptr;
  const T* x_at = paac::row_at<T>(a.x, k0 + cells.row, at.seq) + at.base + cells.ch;
  const T* dt_at = paac::row_at<T>(a.dt, k0 + cells.row, at.seq) + at.base + cells.ch;
  const T* z_at = paac::row_at<T>(a.z, gate ? k0 + cells.row : 0, gate ? at.seq : 0) + at.base + cells.ch;
  T* y_at = ENDS ? nullptr : paac::row_to<T>(a.y, k0 + cells.row, at.seq) + at.base + cells.ch;
  // elements from the thread's first cell of the chunk to cell i of the window that begins at step k
  const auto from_first = [&](int k, int i, int64_t step) { return (int64_t)(k - k0 + i % C::OF_TURN * C::ROWS) * step + C::turn(i) * threads; };
  // x and dt of the window that begins at step k, and z of the one that lies two before it
  const auto fetch = [&](int k, int place, int spare, int i) {
    if (cells.there(i, end - k, at.room)) {
      Way::get(ring + place * ring_step + i * threads, x_at + from_first(k, i, a.x.step));
      Way::get(dt_ring + spare * ring_step + i * threads, dt_at + from_first(k, i, a.dt.step));
    }
    k -= 2 * SPAN;
    if (gate && k >= k0 && cells.there(i, end - k, at.room)) Way::get(z_ring + spare * ring_step + i * threads, z_at + from_first(k, i, a.z.step));
  };
  // all cells of a window; where no asynchronous copy is as small as an access, the loads of a few at a time, then their stores
  const auto fetch_window = [&](int k, int place, int spare) {
    if constexpr (Way::BYTES >= 4) {
#pragma unroll
      for (int i = 0; i < COUNT; ++i) fetch(k, place, spare, i);
    } else {
      typedef typename Way::Raw Raw;
      constexpr int FEW = COUNT < 4 ? COUNT : 4;
      const auto one = [&](const T* p, bool in) { return in ? *reinterpret_cast<const Raw*>(p) : (Raw)0; };
#pragma unroll
      for (int i0 = 0; i0 < COUNT; i0 += FEW) {
        Raw v[FEW][3];
#pragma unroll
        for (int u = 0; u < FEW; ++u) {
          const int i = i0 + u;
          const bool in = cells.there(i, end - k, at.room), in_z = gate && k - 2 * SPAN >= k0 && cells.there(i, end - k + 2 * SPAN, at.room);
          v[u][0] = one(x_at + from_first(k, i, a.x.step), in);
          v[u][1] = one(dt_at + from_first(k, i, a.dt.step), in);
          v[u][2] = one(z_at + from_first(k - 2 * SPAN, i, a.z.step), in_z);
        }
#pragma unroll
        for (int u = 0; u < FEW; ++u) {
          const int i = (i0 + u) * threads;
          ring[place * ring_step + i] = v[u][0];
          dt_ring[spare * ring_step + i] = v[u][1];
          if (!ENDS) z_ring[spare * ring_step + i] = v[u][2];
        }
      }
    }
  };
  float bias[C::TURNS][VEC], D[C::TURNS][VEC];
#pragma unroll
  for (int u = 0; u < C::TURNS; ++u) {
    const int ch = cells.ch + u * threads;
    load_of_channels(bias[u], a.bias, at.base + ch, ch < at.room);
    load_of_channels(D[u], a.D, at.base + ch, ch < at.room);
  }
  // delta and delta x of a cell
  const auto ready = [&](float2* slot, int place, int spare, int i) {
    float x[VEC], dt[VEC];
    Way::widen(x, ring + place * ring_step + i * threads);
    Way::widen(dt, dt_ring + spare * ring_step + i * threads);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float v = dt[j] + bias[C::turn(i)][j], soft = paac::softplus<T>(v);
      dt[j] = a.softplus ? soft : v;
      x[j] *= dt[j];
    }
    float2* to = slot + cells.step(i) * width + cells.channel(i);
    if constexpr (VEC == 4) {
      reinterpret_cast<float4*>(to)[0] = make_float4(dt[0], x[0], dt[1], x[1]);
      reinterpret_cast<float4*>(to)[1] = make_float4(dt[2], x[2], dt[3], x[3]);
    } else {
      to[0] = make_float2(dt[0], x[0]);
    }
  };
  // y of a cell of the window that begins at step k
  const auto write = [&](const float2* slot, int place, int spare, int k, int i) {
    float y[VEC], x[VEC], z[VEC];
    const float2* from = slot + cells.step(i) * width + cells.channel(i);
    if constexpr (VEC == 4) {
      const float4 u = reinterpret_cast<const float4*>(from)[0], v = reinterpret_cast<const float4*>(from)[1];
      y[0] = u.y; y[1] = u.w; y[2] = v.y; y[3] = v.w;
    } else {
      y[0] = from[0].y;
    }
    Way::widen(x, ring + place * ring_step + i * threads);
    Way::widen(z, z_ring + spare * ring_step + i * threads);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      y[j] = a.D != nullptr ? fmaf(D[C::turn(i)][j], x[j], y[j]) : y[j];
      const float g = paac::silu<T>(z[j]);
      y[j] = gate ? y[j] * g : y[j];
    }
    paac::Pack<T, VEC> p;
    p.round(y);
    p.store(y_at + from_first(k, i, a.y.step));
  };

  Inputs<T, L> b, c;
#pragma unroll
  for (int v = 0; v < SPARE; ++v) {
    fetch_window(k0 + v * SPAN, v, v);
    paac::copies_end_step();
  }
  b.fetch(a, a.b, k0, end - k0, at.seq, at.group);
  if (!ENDS) c.fetch(a, a.c, k0, end - k0, at.seq, at.group);
  uint32_t mine = restart_of(a, k0, end - k0, at.seq);

  States<L> A, h;
  float sum[PAIR];
  load_rates<L>(A, a, at);
#pragma unroll
  for (int i = 0; i < PAIR; ++i) sum[i] = 0.f;
  zero(h);
  if (at.chunk == 0) {
    if (a.first != nullptr) {
      load_all<L>(h, ENDS || a.start == nullptr ? a.first : a.start, a, at);
      if (ENDS) store_all<L>(a.start, h, a, at);
    }
  } else if (!ENDS) {
    fold_chunks<L>(h, A, a, at, 0, 1);
  }

  // the first window made ready
  paac::copies_wait<SPARE - 1>();
  C::each([&](int i, int) { if (cells.there(i, end - k0, at.room)) ready(slots, 0, 0, i); });
  fetch_window(k0 + SPARE * SPAN, SPARE % RING, 0);
  paac::copies_end_step();
  b.put(Bs, a, a.b, k0, end - k0, at.seq, at.group);
  if (!ENDS) c.put(Cs, a, a.c, k0, end - k0, at.seq, at.group);
  b.fetch(a, a.b, k0 + SPAN, end - k0 - SPAN, at.seq, at.group);
  if (!ENDS) c.fetch(a, a.c, k0 + SPAN, end - k0 - SPAN, at.seq, at.group);

  bool any_cut = false;
  int half = 0, next = 1 % RING, last = RING - 1;      // of the slots; places in the ring of the window behind this one and of the one before
  int k = k0;
  for (; k < end; k += SPAN, half ^= 1) {
    const int steps = end - k < SPAN ? end - k : SPAN, behind = end - k - SPAN;
    const uint32_t cuts = restarts(mine);
    any_cut = any_cut || cuts != 0;
    mine = restart_of(a, k + SPAN, behind, at.seq);
    float2 *slot = slots + half * SPAN * width, *other = slots + (half ^ 1) * SPAN * width;
    const float *B_at = Bs + half * SPAN * WIDE + at.state0(), *C_at = Cs + half * SPAN * WIDE + at.state0();
    const int spare = ENDS ? next : SPARE == 1 ? 0 : half ^ 1;      // of this window's neighbours
    if (!ENDS && a.states != nullptr) store_all<L>(a.states + (int64_t)(k / SPAN) * all_states(a), h, a, at);
    paac::copies_wait<ENDS ? RING - 1 : RING - 3>();                // the next window's are there
    __syncthreads();
    const auto step = [&](int q, float (&y)[PAIR], bool cut) {
      float2 d[PAIR];
#pragma unroll
      for (int i = 0; i < PAIR; ++i) d[i] = slot[q * width + at.pair * PAIR + i];
      f2 B[TWOS], Cq[TWOS];
      load_each(B, B_at + q * WIDE);
      if (!ENDS) load_each(Cq, C_at + q * WIDE);
#pragma unroll
      for (int i = 0; i < PAIR; ++i) {
        if (cut) {
          begin(h[i], d[i].y, B);
        } else {
          f2 keep[TWOS];
          decay(keep, A[i], d[i].x);
          advance(h[i], keep, d[i].y, B);
        }
        if (ENDS) sum[i] += d[i].x; else y[i] = dot(h[i], Cq);
      }
    };
    // (places beyond the tile's last channel are worked on with whatever is there, and not written)
    if (steps == SPAN && cuts == 0 && behind >= SPAN && (ENDS || k > k0)) {
#pragma unroll
      for (int g = 0; g < SPAN / FOUR; ++g) {
        float y[FOUR * PAIR];
#pragma unroll
        for (int u = 0; u < FOUR; ++u) {
          float of[PAIR];
          step(g * FOUR + u, of, false);
          if (!ENDS)
#pragma unroll
            for (int i = 0; i < PAIR; ++i) y[u * PAIR + i] = of[i];
        }
        if (!ENDS) {
          typedef Halves<FOUR * PAIR, L::SL / 2, 1> H;
          const int first = H::sum(y);
#pragma unroll
          for (int i = 0; i < H::LEFT; ++i) slot[(g * FOUR + (first + i) / PAIR) * width + at.pair * PAIR + (first + i) % PAIR].y = y[i];
        }
        // (behind the first steps where a thread has less cells than there are fours)
#pragma unroll
        for (int i = 0; i < COUNT; ++i)
          if (COUNT < FOUR ? i == g : i / (COUNT / FOUR) == g) {
            if (cells.row >= SPAN) continue;
            if (!ENDS && cells.channel(i) < at.room) write(other, last, spare, k - SPAN, i);
            ready(other, next, spare, i);
            if (Way::BYTES >= 4) fetch(k + (ENDS ? 1 + RING : RING - 1) * SPAN, ENDS ? next : last, spare, i);
          }
      }
      if (Way::BYTES < 4) fetch_window(k + (ENDS ? 1 + RING : RING - 1) * SPAN, ENDS ? next : last, spare);
    } else {
      for (int q = 0; q < steps; ++q) {
        float y[PAIR];
        step(q, y, (cuts >> q & 1u) != 0);
        if (!ENDS) {
          typedef Halves<PAIR, L::SL / 2, 1> H;
          const int first = H::sum(y);
#pragma unroll
          for (int i = 0; i < H::LEFT; ++i) slot[q * width + at.pair * PAIR + first + i].y = y[i];
        }
      }
      C::each([&](int i, int) {
        if (!ENDS && k > k0 && cells.there(i, SPAN, at.room)) write(other, last, spare, k - SPAN, i);
        if (cells.there(i, behind, at.room)) ready(other, next, spare, i);
      });
      fetch_window(k + (ENDS ? 1 + RING : RING - 1) * SPAN, ENDS ? next : last, spare);
    }
    paac::copies_end_step();
    b.put(Bs + (half ^ 1) * SPAN * WIDE, a, a.b, k + SPAN, behind, at.seq, at.group);
    if (!ENDS) c.put(Cs + (half ^ 1) * SPAN * WIDE, a, a.c, k + SPAN, behind, at.seq, at.group);
    b.fetch(a, a.b, k + 2 * SPAN, behind - SPAN, at.seq, at.group);
    if (!ENDS) c.fetch(a, a.c, k + 2 * SPAN, behind - SPAN, at.seq, at.group);
    next = next + 1 == RING ? 0 : next + 1;
    last = last + 1 == RING ? 0 : last + 1;
  }
  if (ENDS) {
    leave_chunk<L>(h, sum, any_cut, a, at);
    return;
  }
  paac::copies_wait<0>();                                           // the last window's z
  __syncthreads();
  k -= SPAN;
  C::each([&](int i, int) { if (cells.there(i, end - k, at.room)) write(slots + (half ^ 1) * SPAN * width, last, SPARE == 1 ? 0 : half ^ 1, k, i); });
  if (a.last != nullptr && at.chunk == a.chunks - 1) store_all<L>(a.last, h, a, at);
}

// A few steps: a channel's states over LANES threads side by side, eight to each, so that states are read and written as they lie in memory.  A lane
// works out what one of LANES steps needs and, once their outputs are summed by halves, writes that step's.  The block's B and C are in shared memory where
// its channels are of one sequence and group.
constexpr int FEW_THREADS = 128, FEW_EACH = 8, MOST_FEW = SPAN;
template <class T, int LANES>
__global__ void __launch_bounds__(FEW_THREADS, 7)
selective_few_kernel(const __grid_constant__ Args a, int per_row) {
  paac::pdl_entry();
  constexpr int COLUMNS = FEW_THREADS / LANES, WIDE = FEW_EACH * LANES, TWOS = FEW_EACH / 2;
  __shared__ __align__(16) float Bs[MOST_FEW][WIDE], Cs[MOST_FEW][WIDE];
  // blocks of a sequence's group
  const uint32_t row = blockIdx.x / (uint32_t)per_row;
  const int seq = (int)(row / (uint32_t)a.groups), group = (int)(row - (uint32_t)seq * a.groups), of_group = a.channels / a.groups;
  const int column = (int)(blockIdx.x - row * per_row) * COLUMNS + threadIdx.x / LANES, sl = threadIdx.x % LANES, s0 = FEW_EACH * sl;
  const bool there = column < of_group;
  const int ch = group * of_group + (there ? column : 0);
  const int64_t at = ((int64_t)seq * a.channels + ch) * a.state;
  f2 A[TWOS], h[TWOS] = {};
  load_states(A, a.A + (int64_t)ch * a.state, s0, a.state, a.wide, there);
#pragma unroll
  for (int j = 0; j < TWOS; ++j) A[j] = mul(A[j], both(LOG2E));
  if (a.first != nullptr) load_states(h, a.first + at, s0, a.state, a.wide, there);
  const T *x_at = paac::row_at<T>(a.x, sl, seq) + ch, *dt_at = paac::row_at<T>(a.dt, sl, seq) + ch, *z_at = paac::row_at<T>(a.z, sl, seq) + ch;
  T* y_at = paac::row_to<T>(a.y, sl, seq) + ch;
  // the lane's step among those from k on, as it is: asked for while the ones before are worked on
  struct Step { paac::Pack<T, 1> x, dt, z; uint32_t cut; } next;
  const auto fetch = [&](int k) {
    next.x.zero(); next.dt.zero(); next.z.zero();
    next.cut = 0;
    if (k + sl >= a.t) return;
    next.x.load(x_at + k * a.x.step);
    next.dt.load(dt_at + k * a.dt.step);
    if (a.z.data != nullptr) next.z.load(z_at + k * a.z.step);
    if (a.restart.data != nullptr) next.cut = a.restart.data[(k + sl) * a.restart.step + seq * a.restart.seq];
  };
  fetch(0);
  {
    const T *b = paac::row_at<T>(a.b, 0, seq) + group * a.state, *c = paac::row_at<T>(a.c, 0, seq) + group * a.state;
    for (int i = threadIdx.x; i < a.t * WIDE; i += FEW_THREADS) {
      const int q = i / WIDE, s = i % WIDE;
      const bool in = s < a.state;
      Bs[q][s] = in ? paac::to_f(b[q * a.b.step + s]) : 0.f;
      Cs[q][s] = in ? paac::to_f(c[q * a.c.step + s]) : 0.f;
    }
  }
  const float bias = a.bias != nullptr ? a.bias[ch] : 0.f, D = a.D != nullptr ? a.D[ch] : 0.f;
  if (a.states != nullptr && there) store_states(a.states + at, h, s0, a.state, a.wide);
  __syncthreads();
  Step now = next;
  for (int k = 0; k < a.t; k += LANES) {
    const int mine = k + sl, steps = a.t - k < LANES ? a.t - k : LANES;
    if (k + LANES < a.t) fetch(k + LANES);
    float x[1], dt[1], z[1];
    now.x.widen(x);
    now.dt.widen(dt);
    now.z.widen(z);
    const float v = dt[0] + bias, soft = paac::softplus<T>(v), delta = a.softplus ? soft : v, take = delta * x[0];
    const uint32_t cuts = __ballot_sync(0xffffffffu, now.cut != 0);      // (the same in every group of lanes)
    now = next;
    float y[LANES];
#pragma unroll
    for (int u = 0; u < LANES; ++u) {
      y[u] = 0.f;
      if (u < steps) {
        const float d = __shfl_sync(0xffffffffu, delta, u, LANES), t = __shfl_sync(0xffffffffu, take, u, LANES);
        f2 B[TWOS], C[TWOS];
        load_each(B, &Bs[k + u][s0]);
        load_each(C, &Cs[k + u][s0]);
        if ((cuts >> u & 1u) != 0) {
          begin(h, t, B);
        } else {
          f2 keep[TWOS];
          decay(keep, A, d);
          advance(h, keep, t, B);
        }
        y[u] = dot(h, C);
      }
    }
    Halves<LANES, LANES / 2, 1>::sum(y);                            // (lane sl is left with step sl's)
    if (there && mine < a.t) {
      float v = y[0];
      if (a.D != nullptr) v = fmaf(D, x[0], v);
      if (a.z.data != nullptr) v *= paac::silu<T>(z[0]);
      y_at[k * a.y.step] = paac::from_f<T>(v);
    }
  }
  if (a.last != nullptr && there) store_states(a.last + at, h, s0, a.state, a.wide);
}

template <class T> cudaError_t few(const Args& a, cudaStream_t st) {
  int lanes = 1;
  while (lanes * FEW_EACH < a.state) lanes *= 2;
  return by_lanes<8>(lanes, [&](auto l) {
    constexpr int LANES = decltype(l)::value, COLUMNS = FEW_THREADS / LANES;
    const int per_row = (a.channels / a.groups + COLUMNS - 1) / COLUMNS;
    return paac::launch_overlapped_on(st, selective_few_kernel<T, LANES>, dim3((unsigned)((int64_t)a.n * a.groups * per_row)), dim3(FEW_THREADS), 0, a, per_row);
  });
}
template <class T, class L, int VEC, bool ENDS> cudaError_t launch(const Args& a, const Shape& h, int64_t blocks, cudaStream_t st) {
  const int threads = 32 * h.warps, bytes = shared_bytes<T, L, VEC, ENDS>(h.width, threads);
  static paac::PerDevice<bool> ready;
  int device = -1;
  const bool ok = cudaGetDevice(&device) == cudaSuccess && ready.get(device, [](bool&) {
    return cudaFuncSetAttribute(selective_scan_kernel<T, L, VEC, ENDS>, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 << 10) == cudaSuccess;
  }) != nullptr;
  if (!ok) return cudaErrorUnknown;
  return paac::launch_overlapped_on(st, selective_scan_kernel<T, L, VEC, ENDS>, dim3((unsigned)blocks), dim3(threads), bytes, a);
}
template <class T, int VEC> cudaError_t scan(const Args& a, const Shape& h, cudaStream_t st) {
  if (h.narrow)
    return by_lanes<16>(h.sl, [&](auto lanes) { return launch<T, Layout<4, 1, decltype(lanes)::value>, VEC, false>(a, h, h.blocks, st); });
  return by_lanes<8>(h.sl, [&](auto lanes) {
    typedef Layout<8, 1, decltype(lanes)::value> L;
    if (h.chunks > 1) {
      const cudaError_t e = launch<T, L, VEC, true>(a, h, h.blocks / h.chunks * (h.chunks - 1), st);      // (the last chunk's end is nobody's begin)
      if (e != cudaSuccess) return e;
    }
    return launch<T, L, VEC, false>(a, h, h.blocks, st);
  });
}
// Which layout, and whether steps are cut: by the warps that are resident at 128 registers, 16 a multiprocessor.  Eight states a thread without a cut where they
// fill it; four without a cut where they fill ten of the 16; chunks of four windows or more otherwise, where there are three of them.  Measured with 16 states
// (us; four in one go, cut into chunks of eight, eight in one go): 2048 steps of 1024 channels of 4, 8, 12, 14 and 20 sequences, 512 to 2560 warps of the first kind: 235, 125, 308;
// 262, 247, 315; 350, 326, 361; 358, -, 367; 560, -, 532; 300 steps of 10 and 12: 58, 62, 59; 57, 66, 60.
Shape shape_of(const paac_selective& s) {
  Shape wide = tiled(s, 8, 1, 128), narrow = tiled(s, 4, 1, 128);
  narrow.narrow = true;
  if (wide.blocks * wide.warps >= 148 * 16) return wide;
  if (narrow.blocks * narrow.warps >= 148 * 10) return narrow;
  cut_steps(wide, s, 148 * 16, 4);
  return wide.chunks > 1 ? wide : narrow;
}

}  // namespace

extern "C" size_t paac_selective_scan_workspace_bytes(const paac_selective* s, int backward) {
  if (!shape_ok(s) || (s->t <= MOST_FEW && !backward)) return 0;
  return backward ? gradient_room(*s) : room_of(*s, shape_of(*s), false).total;
}

extern "C" int paac_selective_scan(const paac_selective* s, const paac_selective_out* out, void* stream) {
  if (!shape_ok(s) || out == nullptr) return PAAC_ERR_ARG;
  const float* h0 = out->h0;
  float *h_last = out->h_last, *states = out->states;
  const int64_t all = (int64_t)s->n * s->c * s->state, inputs = (int64_t)s->groups * s->state;
  paac::StepCheck check(s->t, s->n, size_of(*s), s->restart, s->restart_n, s->restart_t);
  check.steps(s->x, s->c, false, true);
  check.steps(s->dt, s->c, false, true);
  check.steps(s->B, inputs, false, true, false);
  check.steps(s->C, inputs, false, true, false);
  check.steps(s->z, s->c, false, false);
  check.steps(out->y, s->c, true, true);
  check.floats(s->A, (int64_t)s->c * s->state, false, true);
  check.floats(s->D, s->c, false);
  check.floats(s->dt_bias, s->c, false);
  if (h0 != h_last) check.floats(h0, all, false);
  check.floats(h_last, all, true);
  check.floats(states, all * (((int64_t)s->t + SPAN - 1) / SPAN), true);
  if (!check.fit()) return PAAC_ERR_ARG;
  const Shape h = shape_of(*s);
  Args a = common_args(*s, h);
  a.y = paac::step_rows(out->y, s->t, s->n);
  a.first = h0; a.last = h_last; a.states = states;
  a.wide = states_wide(*s, s->A, h0, h_last) && ((uintptr_t)states & 15u) == 0;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (s->t <= MOST_FEW) return paac::launch_status(s->type == PAAC_BF16 ? few<bf16>(a, st) : few<float>(a, st));
  const Room room = room_of(*s, h, false);
  if (room.total > 0) {
    if (out->workspace == nullptr || ((uintptr_t)out->workspace & 15u) != 0 || out->workspace_bytes < room.total) return PAAC_ERR_WORKSPACE;
    check.arrays.keep(out->workspace, (int64_t)room.total, true);
    if (!check.fit()) return PAAC_ERR_ARG;
    place_room(a, room, h, false, out->workspace);
  }
  const bool four = four_wide(*s, check.align);
  if (s->type == PAAC_BF16) return paac::launch_status(four ? scan<bf16, 4>(a, h, st) : scan<bf16, 1>(a, h, st));
  return paac::launch_status(four ? scan<float, 4>(a, h, st) : scan<float, 1>(a, h, st));
}
