// What the selective scan's forward and backward kernels share: how channels and states lie over threads, a window of steps in shared memory, and
// how the steps of few channels are cut into chunks.
//
// A block has one sequence, a tile of neighbouring channels of one group and a chunk of steps, which it takes in windows of
// SPAN steps.  A thread has eight states of PAIR neighbouring channels; SL lanes side by side have a channel's up to 8 SL states.  What a step needs of
// a channel (delta, delta x) is worked out once by all threads together, in the order of the arrays in memory, and left in shared memory, where the
// threads with that channel's states find it; B and C, which all channels of the tile take, too.
#pragma once
#include "sequence.cuh"

namespace paac {
namespace selective {

constexpr int SPAN = PAAC_SELECTIVE_SPAN, EACH = 8, PAIR = 2, MOST_WARPS = 4;
constexpr float LOG2E = 1.44269504f;

struct Args {
  StepRows x, dt, b, c, z, y;          // y: forward only
  StepRows dy, dx, ddt, dz;
  StepFlags restart;
  const float *A, *D, *bias;
  const float* first;                  // forward: h0; backward: dh_last
  float* last;                         // forward: h_last; backward: dh0
  float* states;
  float *ends, *sums;                  // of chunks: [chunk][n][c][state] what a chunk passes on from nothing; [chunk][n][c] its deltas' sum
  uint32_t* cuts;                      // [chunk][n] whether a restart is in it
  float* start;                        // [n][c][state]: a copy of `first`, which `last` may replace
  float *bc_sums, *a_sums, *d_sums;    // backward: [tile][t][n][group][2][state], [chunk][n][c][state], [chunk][n][c][2]
  int t, n, channels, state, groups;
  int softplus, wide;                  // wide: states may be accessed four at a time
  int tiles;                           // of a group
  int chunks, chunk;                   // how many, and their steps (a multiple of SPAN)
};

__device__ __forceinline__ float exp2_fast(float v) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v));
  return e;
}

// Where a thread is.
template <int SL> struct Place {
  int sl, pair, seq, chunk, group, tile, base, room, width;       // room: channels of the tile from `base` on, of `width` places
  __device__ __forceinline__ explicit Place(const Args& a) {
    const int lane = threadIdx.x & 31;
    sl = lane % SL;
    pair = (threadIdx.x >> 5) * (32 / SL) + lane / SL;
    width = (int)blockDim.x / SL * PAIR;
    uint32_t at = blockIdx.x;
    const uint32_t tiles = (uint32_t)a.tiles * a.groups, in_group = at % tiles;
    at /= tiles;
    seq = (int)(at % (uint32_t)a.n);
    chunk = (int)(at / (uint32_t)a.n);
    group = (int)in_group / a.tiles;
    tile = (int)in_group % a.tiles;
    const int of_group = a.channels / a.groups;
    base = group * of_group + tile * width;
    room = of_group - tile * width < width ? of_group - tile * width : width;
  }
  __device__ __forceinline__ bool has(int j) const { return pair * PAIR + j < room; }
  __device__ __forceinline__ int channel(int j) const { return base + pair * PAIR + j; }
};

// eight of the states of a channel, from `s0` on; 0 beyond the last
__device__ __forceinline__ void load_states(float (&v)[EACH], const float* p, int s0, int state, int wide, bool there) {
  if (wide) {
#pragma unroll
    for (int j = 0; j < EACH; j += 4) {
      const float4 q = there && s0 + j < state ? *reinterpret_cast<const float4*>(p + s0 + j) : make_float4(0.f, 0.f, 0.f, 0.f);
      v[j] = q.x; v[j + 1] = q.y; v[j + 2] = q.z; v[j + 3] = q.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < EACH; ++j) v[j] = there && s0 + j < state ? p[s0 + j] : 0.f;
  }
}
__device__ __forceinline__ void store_states(float* p, const float (&v)[EACH], int s0, int state, int wide) {
  if (wide) {
#pragma unroll
    for (int j = 0; j < EACH; j += 4)
      if (s0 + j < state) *reinterpret_cast<float4*>(p + s0 + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
  } else {
#pragma unroll
    for (int j = 0; j < EACH; ++j)
      if (s0 + j < state) p[s0 + j] = v[j];
  }
}

// the restarts of steps [k, k + steps) of a window, a bit a step
__device__ __forceinline__ uint32_t restarts(const Args& a, int k, int steps, int seq) {
  if (a.restart.data == nullptr) return 0;
  const int lane = threadIdx.x & 31;
  const bool cut = lane < steps && a.restart.data[(int64_t)(k + lane) * a.restart.step + seq * a.restart.seq] != 0;
  return __ballot_sync(0xffffffffu, cut);
}

// f(step of the window, first of VEC channels within the tile) for all there are, spread over the block in the order of memory
template <int VEC, class F> __device__ __forceinline__ void for_tile(int steps, int room, int width, F f) {
  const int per = width / VEC;
  for (int i = threadIdx.x; i < steps * per; i += blockDim.x) {
    const int q = i / per, ch = (i - q * per) * VEC;
    if (ch < room) f(q, ch);
  }
}
template <class T, int VEC> __device__ __forceinline__ void load_vec(float (&v)[VEC], const T* p) {
  Pack<T, VEC> q;
  q.load(p);
  q.widen(v);
}

// the step of a state's channel
template <class T> __device__ __forceinline__ float delta_of(const Args& a, float dt, int channel) {
  const float v = a.bias != nullptr ? dt + a.bias[channel] : dt;
  return a.softplus ? softplus<T>(v) : v;
}

// B or C of a window's steps into [SPAN][8 SL], 0 beyond the last state
template <class T, int SL> __device__ __forceinline__ void load_inputs(float* to, const Args& a, const StepRows& r, int k, int steps, int seq, int group) {
  constexpr int WIDE = EACH * SL;
  for (int i = threadIdx.x; i < steps * WIDE; i += blockDim.x) {
    const int q = i / WIDE, s = i - q * WIDE;
    to[i] = s < a.state ? to_f(row_at<T>(r, k + q, seq)[group * a.state + s]) : 0.f;
  }
}
__device__ __forceinline__ void load_each(float (&v)[EACH], const float* p) { load_floats(v, p); }

// keep = exp(delta A), A times log2(e)
__device__ __forceinline__ void decay(float (&keep)[EACH], const float (&A)[EACH], float delta) {
#pragma unroll
  for (int j = 0; j < EACH; j += 2) {
    keep[j] = A[j]; keep[j + 1] = A[j + 1];
    mul2(keep[j], keep[j + 1], delta, delta);
  }
#pragma unroll
  for (int j = 0; j < EACH; ++j) keep[j] = exp2_fast(keep[j]);
}
// h = keep h + take B
__device__ __forceinline__ void advance(float (&h)[EACH], const float (&keep)[EACH], float take, const float (&B)[EACH]) {
#pragma unroll
  for (int j = 0; j < EACH; j += 2) {
    float b0 = B[j], b1 = B[j + 1];
    mul2(b0, b1, take, take);
    fma2_to(h[j], h[j + 1], keep[j], keep[j + 1], h[j], h[j + 1], b0, b1);
  }
}
__device__ __forceinline__ float dot(const float (&v)[EACH], const float (&w)[EACH]) {
  float s0 = 0.f, s1 = 0.f;
#pragma unroll
  for (int j = 0; j < EACH; j += 2) fma2(s0, s1, v[j], v[j + 1], w[j], w[j + 1]);
  return s0 + s1;
}
// Sums over the SL lanes of a channel: lane 0 gets the first's, lane 1 the second's (with one lane, both stay).
template <int SL> __device__ __forceinline__ float over_states(float first, float second, int sl) {
  const bool odd = (sl & 1) != 0;
  float keep = odd ? second : first;
  keep += __shfl_xor_sync(0xffffffffu, odd ? first : second, 1);
#pragma unroll
  for (int d = 2; d < SL; d *= 2) keep += __shfl_xor_sync(0xffffffffu, keep, d);
  return keep;
}
template <int SL> __device__ __forceinline__ void zero(float (&v)[PAIR][EACH]) {
#pragma unroll
  for (int i = 0; i < PAIR; ++i)
#pragma unroll
    for (int j = 0; j < EACH; ++j) v[i][j] = 0.f;
}
// A of the thread's states, times log2(e)
template <int SL> __device__ __forceinline__ void load_rates(float (&A)[PAIR][EACH], const Args& a, const Place<SL>& at) {
#pragma unroll
  for (int i = 0; i < PAIR; ++i) {
    load_states(A[i], a.A + (int64_t)at.channel(i) * a.state, at.sl * EACH, a.state, a.wide, at.has(i));
#pragma unroll
    for (int j = 0; j < EACH; ++j) A[i][j] *= LOG2E;
  }
}
__device__ __forceinline__ int64_t state_at(const Args& a, int seq, int channel) { return ((int64_t)seq * a.channels + channel) * a.state; }
__device__ __forceinline__ int64_t all_states(const Args& a) { return (int64_t)a.n * a.channels * a.state; }

// What the chunks one after another pass on, from `from` on (towards the chunk of the block, by `way`): h = exp(A sum) h + end.
template <int SL> __device__ __forceinline__ void fold_chunks(float (&h)[PAIR][EACH], const float (&A)[PAIR][EACH], const Args& a, const Place<SL>& at, int from, int way) {
  for (int j = from; j != at.chunk; j += way) {
    const bool cut = j == from || a.cuts[(int64_t)j * a.n + at.seq] != 0;      // the first of them began from what there was
#pragma unroll
    for (int i = 0; i < PAIR; ++i) {
      float end[EACH], keep[EACH];
      load_states(end, a.ends + (int64_t)j * all_states(a) + state_at(a, at.seq, at.channel(i)), at.sl * EACH, a.state, a.wide, at.has(i));
      const float sum = at.has(i) ? a.sums[((int64_t)j * a.n + at.seq) * a.channels + at.channel(i)] : 0.f;
      decay(keep, A[i], sum);
#pragma unroll
      for (int s = 0; s < EACH; ++s) h[i][s] = cut ? end[s] : fmaf(keep[s], h[i][s], end[s]);
    }
  }
}

// ---- the host's part -------------------------------------------------------------------------------------------------------------------

struct Shape {
  int sl, warps, width, tiles, chunks, chunk;
  int64_t blocks;
};
// Lanes for a channel's states, warps for a group's channels, and chunks.  Every block walks its chunk twice where there are more than one, so
// steps are cut only where the blocks would leave most of the multiprocessors empty.
inline Shape shape_of(const paac_selective& s) {
  Shape h;
  h.sl = 1;
  while (h.sl * EACH < s.state) h.sl *= 2;
  const int per_warp = 32 / h.sl * PAIR, of_group = s.c / s.groups;
  h.warps = (of_group + per_warp - 1) / per_warp;
  if (h.warps > MOST_WARPS) h.warps = MOST_WARPS;
  h.width = h.warps * per_warp;
  h.tiles = (of_group + h.width - 1) / h.width;
  const int64_t walks = (int64_t)h.tiles * s.groups * s.n, spans = ((int64_t)s.t + SPAN - 1) / SPAN;
  const int64_t warps = walks * h.warps, room = 148 * 16;
  int64_t chunks = warps * 2 <= room ? room / warps : 1;
  if (chunks > spans / 2) chunks = spans / 2;
  if (chunks > 64) chunks = 64;
  if (chunks < 3) chunks = 1;                            // two chunks take as long as one
  const int64_t each = (spans + chunks - 1) / chunks;
  h.chunk = chunks == 1 ? s.t : (int)each * SPAN;
  h.chunks = chunks == 1 ? 1 : (int)((spans + each - 1) / each);
  h.blocks = walks * h.chunks;
  return h;
}
inline size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

// Scratch of a call, in pieces.
struct Room { size_t ends, sums, cuts, start, bc, a, d, total; };
inline Room room_of(const paac_selective& s, const Shape& h, bool backward) {
  Room r{};
  size_t at = 0;
  auto piece = [&](size_t bytes) { const size_t here = at; at += round_up(bytes); return here; };
  const size_t states = (size_t)s.n * s.c * s.state * 4, columns = (size_t)s.n * s.c * 4;
  if (h.chunks > 1) {
    r.ends = piece(states * h.chunks);
    r.sums = piece(columns * h.chunks);
    r.cuts = piece((size_t)h.chunks * s.n * 4);
    if (!backward) r.start = piece(states);
  }
  if (backward) {
    r.bc = piece((size_t)h.tiles * s.t * s.n * s.groups * 2 * s.state * 4);
    r.a = piece(states * h.chunks);
    r.d = piece(columns * 2 * h.chunks);
  }
  r.total = at;
  return r;
}
inline void place_room(Args& a, const Room& r, const Shape& h, bool backward, void* workspace) {
  char* p = (char*)workspace;
  if (h.chunks > 1) {
    a.ends = (float*)(p + r.ends); a.sums = (float*)(p + r.sums); a.cuts = (uint32_t*)(p + r.cuts);
    if (!backward) a.start = (float*)(p + r.start);
  }
  if (backward) { a.bc_sums = (float*)(p + r.bc); a.a_sums = (float*)(p + r.a); a.d_sums = (float*)(p + r.d); }
}

inline bool shape_ok(const paac_selective* s) {
  return s != nullptr && s->t >= 1 && s->t <= (1 << 30) && s->n >= 1 && s->c >= 1 && (int64_t)s->n * s->c < ((int64_t)1 << 31) && s->state >= 1 && s->state <= 64 &&
         s->groups >= 1 && s->c % s->groups == 0 && (s->type == PAAC_FP32 || s->type == PAAC_BF16);
}
inline int size_of(const paac_selective& s) { return s.type == PAAC_BF16 ? 2 : 4; }

inline Args common_args(const paac_selective& s, const Shape& h, const paac_rows& x, const paac_rows& dt, const float* A, const paac_rows& B, const paac_rows& C,
                        const float* D, const paac_rows& z, const float* bias) {
  Args a{};
  a.x = step_rows(x, s.t, s.n); a.dt = step_rows(dt, s.t, s.n); a.b = step_rows(B, s.t, s.n); a.c = step_rows(C, s.t, s.n); a.z = step_rows(z, s.t, s.n);
  a.restart = {s.restart, s.t > 1 ? s.restart_t : 0, s.n > 1 ? s.restart_n : 0};
  a.A = A; a.D = D; a.bias = bias;
  a.t = s.t; a.n = s.n; a.channels = s.c; a.state = s.state; a.groups = s.groups; a.softplus = s.softplus != 0;
  a.tiles = h.tiles; a.chunks = h.chunks; a.chunk = h.chunk;
  return a;
}
// Accesses of four channels where places, channels and groups allow it.
inline bool four_wide(const paac_selective& s, int align) { return align >= 4 * size_of(s) && (s.c / s.groups) % 4 == 0; }
inline bool states_wide(const paac_selective& s, const void* p, const void* q, const void* r) {
  return s.state % 4 == 0 && (((uintptr_t)p | (uintptr_t)q | (uintptr_t)r) & 15u) == 0;
}
template <class F> cudaError_t by_lanes(int sl, F f) {
  if (sl == 1) return f(std::integral_constant<int, 1>());
  if (sl == 2) return f(std::integral_constant<int, 2>());
  if (sl == 4) return f(std::integral_constant<int, 4>());
  return f(std::integral_constant<int, 8>());
}

}  // namespace selective
}  // namespace paac
