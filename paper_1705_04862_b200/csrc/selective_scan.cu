// The selective state space scan forward (paac_selective_scan): h_t = exp(delta_t A) h_{t-1} + delta_t B_t x_t, y_t = (C_t h_t + D x_t) silu(z_t).
//
// Of every element of the state a step takes an exponential and four multiply-adds; the exponentials, 16 a clock and multiprocessor, bound
// it where channels have 16 states: memory has four values to move for 16 of them.
#include "selective.cuh"

namespace {
using namespace paac::selective;
using paac::bf16;

// ENDS: what a chunk passes on from nothing (the first from h0), and its deltas' sum; otherwise all that is written.
template <class T, int SL, int VEC, bool ENDS>
__global__ void __launch_bounds__(32 * MOST_WARPS)
selective_scan_kernel(const __grid_constant__ Args a) {
  paac::pdl_entry();
  extern __shared__ float4 shared[];
  const Place<SL> at(a);
  constexpr int WIDE = EACH * SL;
  float2* slot = reinterpret_cast<float2*>(shared);                 // [SPAN][width]: delta, delta x; then y in the second's place
  float* Bs = reinterpret_cast<float*>(slot + SPAN * at.width);
  float* Cs = Bs + SPAN * WIDE;

  float A[PAIR][EACH], h[PAIR][EACH], sum[PAIR];
  load_rates<SL>(A, a, at);
#pragma unroll
  for (int i = 0; i < PAIR; ++i) sum[i] = 0.f;
  zero<SL>(h);
  if (at.chunk == 0) {
    const float* from = ENDS || a.start == nullptr ? a.first : a.start;
    if (a.first != nullptr)
#pragma unroll
      for (int i = 0; i < PAIR; ++i) load_states(h[i], from + state_at(a, at.seq, at.channel(i)), at.sl * EACH, a.state, a.wide, at.has(i));
    if (ENDS && a.first != nullptr)
#pragma unroll
      for (int i = 0; i < PAIR; ++i)
        if (at.has(i)) store_states(a.start + state_at(a, at.seq, at.channel(i)), h[i], at.sl * EACH, a.state, a.wide);
  } else if (!ENDS) {
    fold_chunks<SL>(h, A, a, at, 0, 1);
  }
  const int k0 = at.chunk * a.chunk, end = a.t - k0 < a.chunk ? a.t : k0 + a.chunk;
  bool any_cut = false;
  for (int k = k0; k < end; k += SPAN) {
    const int steps = end - k < SPAN ? end - k : SPAN;
    __syncthreads();                                              // the window before has been written
    for_tile<VEC>(steps, at.room, at.width, [&](int q, int ch) {
      float x[VEC], dt[VEC];
      load_vec<T, VEC>(x, paac::row_at<T>(a.x, k + q, at.seq) + at.base + ch);
      load_vec<T, VEC>(dt, paac::row_at<T>(a.dt, k + q, at.seq) + at.base + ch);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float delta = delta_of<T>(a, dt[j], at.base + ch + j);
        slot[q * at.width + ch + j] = make_float2(delta, delta * x[j]);
      }
    });
    load_inputs<T, SL>(Bs, a, a.b, k, steps, at.seq, at.group);
    if (!ENDS) load_inputs<T, SL>(Cs, a, a.c, k, steps, at.seq, at.group);
    const uint32_t cuts = restarts(a, k, steps, at.seq);
    if (!ENDS && a.states != nullptr)
#pragma unroll
      for (int i = 0; i < PAIR; ++i)
        if (at.has(i)) store_states(a.states + (int64_t)(k / SPAN) * all_states(a) + state_at(a, at.seq, at.channel(i)), h[i], at.sl * EACH, a.state, a.wide);
    __syncthreads();
    for (int q = 0; q < steps; ++q) {
      const float4 d = reinterpret_cast<const float4*>(slot + q * at.width)[at.pair];
      float B[EACH], keep[EACH];
      load_each(B, Bs + q * WIDE + at.sl * EACH);
      const bool cut = (cuts >> q & 1u) != 0;
      if (cut) { zero<SL>(h); any_cut = true; }
      decay(keep, A[0], d.x);
      if (cut) advance(h[0], h[0], d.y, B); else advance(h[0], keep, d.y, B);
      decay(keep, A[1], d.z);
      if (cut) advance(h[1], h[1], d.w, B); else advance(h[1], keep, d.w, B);
      if (ENDS) {
        sum[0] += d.x;
        sum[1] += d.z;
      } else {
        float C[EACH];
        load_each(C, Cs + q * WIDE + at.sl * EACH);
        const float y0 = dot(h[0], C), y1 = dot(h[1], C);
        float2* to = slot + q * at.width + at.pair * PAIR;
        if (SL == 1) {
          to[0].y = y0;
          to[1].y = y1;
        } else {
          const float y = over_states<SL>(y0, y1, at.sl);         // (the lanes of a channel have read the slot when they meet here)
          if (at.sl < 2) to[at.sl].y = y;
        }
      }
    }
    if (ENDS) continue;
    __syncthreads();
    for_tile<VEC>(steps, at.room, at.width, [&](int q, int ch) {
      float y[VEC];
#pragma unroll
      for (int j = 0; j < VEC; ++j) y[j] = slot[q * at.width + ch + j].y;
      if (a.D != nullptr) {
        float x[VEC];
        load_vec<T, VEC>(x, paac::row_at<T>(a.x, k + q, at.seq) + at.base + ch);
#pragma unroll
        for (int j = 0; j < VEC; ++j) y[j] = fmaf(a.D[at.base + ch + j], x[j], y[j]);
      }
      if (a.z.data != nullptr) {
        float z[VEC], s, rest;
        load_vec<T, VEC>(z, paac::row_at<T>(a.z, k + q, at.seq) + at.base + ch);
#pragma unroll
        for (int j = 0; j < VEC; ++j) { paac::logistic<T>(z[j], s, rest); y[j] *= z[j] * s; }
      }
      paac::Pack<T, VEC> p;
      p.round(y);
      p.store(paac::row_to<T>(a.y, k + q, at.seq) + at.base + ch);
    });
  }
  if (ENDS) {
#pragma unroll
    for (int i = 0; i < PAIR; ++i)
      if (at.has(i)) {
        store_states(a.ends + (int64_t)at.chunk * all_states(a) + state_at(a, at.seq, at.channel(i)), h[i], at.sl * EACH, a.state, a.wide);
        if (at.sl == 0) a.sums[((int64_t)at.chunk * a.n + at.seq) * a.channels + at.channel(i)] = sum[i];
      }
    if (threadIdx.x == 0 && at.tile == 0 && at.group == 0) a.cuts[(int64_t)at.chunk * a.n + at.seq] = any_cut;
  } else if (a.last != nullptr && at.chunk == a.chunks - 1) {
#pragma unroll
    for (int i = 0; i < PAIR; ++i)
      if (at.has(i)) store_states(a.last + state_at(a, at.seq, at.channel(i)), h[i], at.sl * EACH, a.state, a.wide);
  }
}

// One step: a channel's states over `lanes` threads side by side, four to each, so that states are read and written as they lie in memory.
constexpr int STEP_THREADS = 256;
template <class T>
__global__ void __launch_bounds__(STEP_THREADS)
selective_step_kernel(const __grid_constant__ Args a, int lanes) {
  paac::pdl_entry();
  const int64_t i = ((int64_t)blockIdx.x * STEP_THREADS + threadIdx.x) / lanes, columns = (int64_t)a.n * a.channels;
  const int sl = threadIdx.x % lanes;
  const bool there = i < columns;
  const int seq = there ? (int)(i / a.channels) : 0, ch = there ? (int)(i - (int64_t)seq * a.channels) : 0;
  const int group = ch / (a.channels / a.groups), first = a.wide ? 4 * sl : sl, by = a.wide ? 1 : lanes;
  const bool cut = a.restart.data != nullptr && a.restart.data[seq * a.restart.seq] != 0;
  const float x = paac::to_f(paac::row_at<T>(a.x, 0, seq)[ch]), delta = delta_of<T>(a, paac::to_f(paac::row_at<T>(a.dt, 0, seq)[ch]), ch);
  const T *b = paac::row_at<T>(a.b, 0, seq) + group * a.state, *c = paac::row_at<T>(a.c, 0, seq) + group * a.state;
  const int64_t at = state_at(a, seq, ch);
  float h[4], A[4], B[4], C[4], y = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int s = first + j * by;
    const bool in = there && s < a.state;
    B[j] = in ? paac::to_f(b[s]) : 0.f;
    C[j] = in ? paac::to_f(c[s]) : 0.f;
    h[j] = A[j] = 0.f;
    if (!a.wide && in) {
      A[j] = a.A[(int64_t)ch * a.state + s];
      if (a.first != nullptr) h[j] = a.first[at + s];
    }
  }
  if (a.wide && there && first < a.state) {
    paac::load_floats(A, a.A + (int64_t)ch * a.state + first);
    if (a.first != nullptr) paac::load_floats(h, a.first + at + first);
  }
  if (a.states != nullptr && there) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (first + j * by < a.state) a.states[at + first + j * by] = h[j];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float take = delta * x * B[j];
    h[j] = cut ? take : fmaf(exp2_fast(delta * (A[j] * LOG2E)), h[j], take);
    y = fmaf(C[j], h[j], y);
  }
  if (a.last != nullptr && there) {
    if (a.wide) {
      if (first < a.state) paac::store_floats(a.last + at + first, h);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (first + j * by < a.state) a.last[at + first + j * by] = h[j];
    }
  }
  for (int d = lanes / 2; d > 0; d /= 2) y += __shfl_xor_sync(0xffffffffu, y, d);
  if (there && sl == 0) {
    if (a.D != nullptr) y = fmaf(a.D[ch], x, y);
    if (a.z.data != nullptr) {
      const float z = paac::to_f(paac::row_at<T>(a.z, 0, seq)[ch]);
      float s, rest;
      paac::logistic<T>(z, s, rest);
      y *= z * s;
    }
    paac::row_to<T>(a.y, 0, seq)[ch] = paac::from_f<T>(y);
  }
}

template <class T> cudaError_t step(const Args& a, cudaStream_t st) {
  int lanes = 1;
  while (lanes * 4 < a.state) lanes *= 2;
  const int64_t threads = (int64_t)a.n * a.channels * lanes;
  return paac::launch_overlapped_on(st, selective_step_kernel<T>, dim3((unsigned)((threads + STEP_THREADS - 1) / STEP_THREADS)), dim3(STEP_THREADS), 0, a, lanes);
}
template <class T, int SL, int VEC> cudaError_t scan(const Args& a, const Shape& h, cudaStream_t st) {
  const size_t smem = (size_t)SPAN * (h.width * 8 + 2 * EACH * SL * 4);
  const dim3 block(32 * h.warps);
  if (h.chunks > 1) {
    // (the last chunk's end is nobody's begin)
    const cudaError_t e = paac::launch_overlapped_on(st, selective_scan_kernel<T, SL, VEC, true>, dim3((unsigned)(h.blocks / h.chunks * (h.chunks - 1))), block, smem, a);
    if (e != cudaSuccess) return e;
  }
  return paac::launch_overlapped_on(st, selective_scan_kernel<T, SL, VEC, false>, dim3((unsigned)h.blocks), block, smem, a);
}

}  // namespace

extern "C" size_t paac_selective_scan_workspace_bytes(const paac_selective* s, int backward) {
  if (!shape_ok(s) || (s->t == 1 && !backward)) return 0;
  return room_of(*s, shape_of(*s), backward != 0).total;
}

extern "C" int paac_selective_scan(const paac_selective* s, paac_rows x, paac_rows dt, const float* A, paac_rows B, paac_rows C, const float* D, paac_rows z,
                                   const float* dt_bias, const float* h0, paac_rows y, float* h_last, float* states, void* workspace,
                                   size_t workspace_bytes, void* stream) {
  if (!shape_ok(s)) return PAAC_ERR_ARG;
  const int64_t all = (int64_t)s->n * s->c * s->state, inputs = (int64_t)s->groups * s->state;
  paac::StepCheck check(s->t, s->n, size_of(*s), s->restart, s->restart_n, s->restart_t);
  check.steps(x, s->c, false, true);
  check.steps(dt, s->c, false, true);
  check.steps(B, inputs, false, true, false);
  check.steps(C, inputs, false, true, false);
  check.steps(z, s->c, false, false);
  check.steps(y, s->c, true, true);
  check.floats(A, (int64_t)s->c * s->state, false, true);
  check.floats(D, s->c, false);
  check.floats(dt_bias, s->c, false);
  if (h0 != h_last) check.floats(h0, all, false);
  check.floats(h_last, all, true);
  check.floats(states, all * (((int64_t)s->t + SPAN - 1) / SPAN), true);
  if (!check.fit()) return PAAC_ERR_ARG;
  const Shape h = shape_of(*s);
  Args a = common_args(*s, h, x, dt, A, B, C, D, z, dt_bias);
  a.y = paac::step_rows(y, s->t, s->n);
  a.first = h0; a.last = h_last; a.states = states;
  a.wide = states_wide(*s, A, h0, h_last) && ((uintptr_t)states & 15u) == 0;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (s->t == 1) return paac::launch_status(s->type == PAAC_BF16 ? step<bf16>(a, st) : step<float>(a, st));
  const Room room = room_of(*s, h, false);
  if (room.total > 0) {
    if (workspace == nullptr || ((uintptr_t)workspace & 15u) != 0 || workspace_bytes < room.total) return PAAC_ERR_WORKSPACE;
    check.arrays.keep(workspace, (int64_t)room.total, true);
    if (!check.fit()) return PAAC_ERR_ARG;
    place_room(a, room, h, false, workspace);
  }
  const bool four = four_wide(*s, check.align);
  return paac::launch_status(by_lanes(h.sl, [&](auto lanes) {
    constexpr int SL = decltype(lanes)::value;
    if (s->type == PAAC_BF16) return four ? scan<bf16, SL, 4>(a, h, st) : scan<bf16, SL, 1>(a, h, st);
    return four ? scan<float, SL, 4>(a, h, st) : scan<float, SL, 1>(a, h, st);
  }));
}
