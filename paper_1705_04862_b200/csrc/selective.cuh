// What the selective scan's forward and backward kernels share: how channels and states lie over threads, a window of steps in shared memory, and
// how the steps of few channels are cut into chunks.
//
// A block has one sequence, a tile of neighbouring channels of one group and a chunk of steps, which it takes in windows of
// SPAN steps.  A thread has EACH states of PAIR neighbouring channels; SL lanes side by side have a channel's up to EACH SL states.  What a step needs of
// a channel (delta, delta x) is worked out once by all threads together, in the order of the arrays in memory, and left in shared memory, where the
// threads with that channel's states find it; B and C, which all channels of the tile take, too.
#pragma once
#include "sequence.cuh"

namespace paac {
namespace selective {

constexpr int SPAN = PAAC_SELECTIVE_SPAN, MOST_WARPS = 4;
constexpr float LOG2E = 1.44269504f;

template <int EACH_, int PAIR_, int SL_> struct Layout {
  static constexpr int EACH = EACH_, TWOS = EACH_ / 2, PAIR = PAIR_, SL = SL_, WIDE = EACH_ * SL_, PER_WARP = 32 / SL_ * PAIR_;
};

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
  float *bc_sums, *a_sums, *d_sums;    // backward: [tile][t][n][group][2][state], [row][c][state], [row][c][2], a row for chunk and sequence or several of these
  int t, n, channels, state, groups;
  int softplus, wide;                  // wide: states may be accessed four at a time
  int tiles;                           // of a group
  int chunks, chunk;                   // how many, and their steps (a multiple of SPAN)
};

// The decays' power of two, whatever the storage: one instruction, off by up to 2^-22 of it, below 2^-126 0 (expf is several, where exponentials bound the scan already).  What that
// adds up to, float storage, relative: states behind 1000 steps 4.3e-7 where step-by-step torch with its exp is 2.1e-7 off, with a hundredth of the rates 1.8e-6 and 2.4e-6.
__device__ __forceinline__ float exp2_fast(float v) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v));
  return e;
}
// Two floats in a register pair, as the packed instructions take them; each result is rounded once.
typedef unsigned long long f2;
__device__ __forceinline__ f2 pack2(float x, float y) { f2 v; asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y)); return v; }
__device__ __forceinline__ void unpack2(f2 v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ f2 both(float x) { return pack2(x, x); }
__device__ __forceinline__ f2 mul(f2 a, f2 b) { f2 v; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b)); return v; }
__device__ __forceinline__ f2 fma(f2 a, f2 b, f2 c) { f2 v; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c)); return v; }
__device__ __forceinline__ float sum_of(f2 v) { float x, y; unpack2(v, x, y); return x + y; }

// Where a thread is.
template <class L> struct Place {
  int sl, pair, seq, chunk, group, tile, base, room, width;       // room: channels of the tile from `base` on, of `width` places
  __device__ __forceinline__ explicit Place(const Args& a) {
    const int lane = threadIdx.x & 31;
    sl = lane % L::SL;
    pair = (threadIdx.x >> 5) * (32 / L::SL) + lane / L::SL;
    width = (int)blockDim.x / L::SL * L::PAIR;
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
  __device__ __forceinline__ bool has(int j) const { return pair * L::PAIR + j < room; }
  __device__ __forceinline__ int channel(int j) const { return base + pair * L::PAIR + j; }
  __device__ __forceinline__ int state0() const { return sl * L::EACH; }
};

// 2 TWOS of the states of a channel, from `s0` on; 0 beyond the last
template <int TWOS> __device__ __forceinline__ void load_states(f2 (&v)[TWOS], const float* p, int s0, int state, int wide, bool there) {
  if (wide) {
#pragma unroll
    for (int j = 0; j < TWOS; j += 2) {
      const ulonglong2 q = there && s0 + 2 * j < state ? *reinterpret_cast<const ulonglong2*>(p + s0 + 2 * j) : make_ulonglong2(0, 0);
      v[j] = q.x;
      v[j + 1] = q.y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < TWOS; ++j)
      v[j] = pack2(there && s0 + 2 * j < state ? p[s0 + 2 * j] : 0.f, there && s0 + 2 * j + 1 < state ? p[s0 + 2 * j + 1] : 0.f);
  }
}
template <int TWOS> __device__ __forceinline__ void store_states(float* p, const f2 (&v)[TWOS], int s0, int state, int wide) {
  if (wide) {
#pragma unroll
    for (int j = 0; j < TWOS; j += 2)
      if (s0 + 2 * j < state) *reinterpret_cast<ulonglong2*>(p + s0 + 2 * j) = make_ulonglong2(v[j], v[j + 1]);
  } else {
#pragma unroll
    for (int j = 0; j < TWOS; ++j) {
      float x, y;
      unpack2(v[j], x, y);
      if (s0 + 2 * j < state) p[s0 + 2 * j] = x;
      if (s0 + 2 * j + 1 < state) p[s0 + 2 * j + 1] = y;
    }
  }
}

// The restart byte of this lane's step of a window, and all that are set, a bit a step.  (The byte as it is: a comparison would wait for it.)
__device__ __forceinline__ uint32_t restart_of(const Args& a, int k, int steps, int seq) {
  const int lane = threadIdx.x & 31;
  return a.restart.data != nullptr && lane < SPAN && lane < steps ? a.restart.data[(int64_t)(k + lane) * a.restart.step + seq * a.restart.seq] : 0;
}
__device__ __forceinline__ uint32_t restarts(uint32_t mine) { return __ballot_sync(0xffffffffu, mine != 0); }

// The part of a tile's channels and steps that a thread works on when arrays are read and written in the order of memory: VEC channels from `ch` on,
// of every ROWS-th step from `row` on (TURNS such columns where a block has less threads than its tile channels).
template <class L, int VEC> struct Cells {
  static constexpr int TURNS = VEC * L::SL < L::PAIR ? 2 : 1, ROWS = TURNS == 2 ? 1 : VEC * L::SL / L::PAIR;
  static constexpr int OF_TURN = ROWS < SPAN ? SPAN / ROWS : 1, COUNT = TURNS * OF_TURN;
  int ch, row;
  __device__ __forceinline__ explicit Cells(int width) {
    const int per = width / (VEC * TURNS);
    row = threadIdx.x / per;
    ch = (threadIdx.x - row * per) * VEC;
  }
  __device__ __forceinline__ int step(int i) const { return row + i % OF_TURN * ROWS; }
  static __device__ __forceinline__ constexpr int turn(int i) { return TURNS == 1 ? 0 : i / OF_TURN; }
  __device__ __forceinline__ int channel(int i) const { return ch + turn(i) * (int)blockDim.x; }
  __device__ __forceinline__ bool there(int i, int steps, int room) const { return step(i) < steps && step(i) < SPAN && channel(i) < room; }
  // f(cell, its turn) for all of them, a few at a time: sixteen side by side (accesses of one channel) are more instructions than are kept at hand
  template <class F> static __device__ __forceinline__ void each(F f) {
    constexpr int FEW = OF_TURN < 4 ? OF_TURN : 4;
#pragma unroll
    for (int u = 0; u < TURNS; ++u)
#pragma unroll FEW
      for (int i = 0; i < OF_TURN; ++i) f(u * OF_TURN + i, u);
  }
};
// A thread's own cells of an array on their way to shared memory: asynchronously where an access has four bytes or more, so that a window's are under
// way while others are worked on, and need no barrier.
template <class T, int VEC> struct Ahead {
  static constexpr int BYTES = VEC * sizeof(T);
  typedef typename Word<BYTES>::type Raw;
  static __device__ __forceinline__ void get(Raw* to, const T* from) {
    if constexpr (BYTES >= 4) copy_to<BYTES>(to, from); else *to = *reinterpret_cast<const Raw*>(from);
  }
  static __device__ __forceinline__ void widen(float (&v)[VEC], const Raw* from) {
    Pack<T, VEC> q;
    q.raw = *from;
    q.widen(v);
  }
};
// a number of each of VEC channels, 0 where there are none
template <int VEC> __device__ __forceinline__ void load_of_channels(float (&v)[VEC], const float* p, int channel, bool there) {
#pragma unroll
  for (int j = 0; j < VEC; ++j) v[j] = p != nullptr && there ? p[channel + j] : 0.f;
}

// B or C of a window's steps into [SPAN][WIDE], 0 beyond the last state.  A thread's first elements are read a window ahead.
template <class T, class L> struct Inputs {
  static constexpr int WIDE = L::WIDE, KEPT = SPAN * WIDE / (32 * MOST_WARPS) < 1 ? 1 : SPAN * WIDE / (32 * MOST_WARPS);
  Pack<T, 1> kept[KEPT];               // (as they are: a conversion would wait for them)
  static __device__ __forceinline__ Pack<T, 1> one(const Args& a, const T* from, const StepRows& r, int i, int steps) {
    const int q = i / WIDE, s = i % WIDE;
    Pack<T, 1> v;
    v.zero();
    if (q < steps && q < SPAN && s < a.state) v.load(from + q * r.step + s);
    return v;
  }
  static __device__ __forceinline__ float number(const Pack<T, 1>& p) {
    float v[1];
    p.widen(v);
    return v[0];
  }
  static __device__ __forceinline__ const T* rows(const Args& a, const StepRows& r, int k, int seq, int group) { return row_at<T>(r, k, seq) + group * a.state; }
  __device__ __forceinline__ void fetch(const Args& a, const StepRows& r, int k, int steps, int seq, int group) {
    const T* from = rows(a, r, k, seq, group);
#pragma unroll
    for (int u = 0; u < KEPT; ++u) kept[u] = one(a, from, r, threadIdx.x + u * blockDim.x, steps);
  }
  __device__ __forceinline__ void put(float* to, const Args& a, const StepRows& r, int k, int steps, int seq, int group) const {
#pragma unroll
    for (int u = 0; u < KEPT; ++u) {
      const int i = threadIdx.x + u * blockDim.x;
      if (i < SPAN * WIDE) to[i] = number(kept[u]);
    }
    if (blockDim.x == 32 * MOST_WARPS) return;
    const T* from = rows(a, r, k, seq, group);
    for (int i = threadIdx.x + KEPT * blockDim.x; i < SPAN * WIDE; i += blockDim.x) to[i] = number(one(a, from, r, i, steps));
  }
};
// a step's B or C for the thread's states, out of shared memory
template <int TWOS> __device__ __forceinline__ void load_each(f2 (&v)[TWOS], const float* p) {
#pragma unroll
  for (int j = 0; j < TWOS; j += 2) {
    const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(p + 2 * j);
    v[j] = q.x;
    v[j + 1] = q.y;
  }
}

// keep = exp(delta A), A times log2(e)
template <int TWOS> __device__ __forceinline__ void decay(f2 (&keep)[TWOS], const f2 (&A)[TWOS], float delta) {
  const f2 d = both(delta);
#pragma unroll
  for (int j = 0; j < TWOS; ++j) {
    float x, y;
    unpack2(mul(A[j], d), x, y);
    keep[j] = pack2(exp2_fast(x), exp2_fast(y));
  }
}
// h = keep h + take B
template <int TWOS> __device__ __forceinline__ void advance(f2 (&h)[TWOS], const f2 (&keep)[TWOS], float take, const f2 (&B)[TWOS]) {
  const f2 t = both(take);
#pragma unroll
  for (int j = 0; j < TWOS; ++j) h[j] = fma(keep[j], h[j], mul(B[j], t));
}
// h = take B: nothing of the state is taken
template <int TWOS> __device__ __forceinline__ void begin(f2 (&h)[TWOS], float take, const f2 (&B)[TWOS]) {
#pragma unroll
  for (int j = 0; j < TWOS; ++j) h[j] = mul(B[j], both(take));
}
template <int TWOS> __device__ __forceinline__ float dot(const f2 (&v)[TWOS], const f2 (&w)[TWOS]) {
  f2 s = mul(v[0], w[0]);
#pragma unroll
  for (int j = 1; j < TWOS; ++j) s = fma(v[j], w[j], s);
  return sum_of(s);
}

// Sums of COUNT values over the lanes that differ in the bits FROM, FROM / 2, ..., TO of their number, by halves: where a lane has more than one value
// it hands one half over and keeps the other.  It is left with LEFT of the sums, from the returned one on, in v[0..LEFT).
template <int COUNT, int FROM, int TO> struct Halves {
  static constexpr int LANES = FROM < TO ? 1 : 2 * FROM / TO, LEFT = COUNT > LANES ? COUNT / LANES : 1;
  __device__ __forceinline__ static int sum(float (&v)[COUNT]) {
    const int lane = threadIdx.x & 31;
    int first = 0;
#pragma unroll
    for (int d = FROM, count = COUNT; d >= TO && d > 0; d /= 2) {
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

template <int PAIR, int TWOS> __device__ __forceinline__ void zero(f2 (&v)[PAIR][TWOS]) {
#pragma unroll
  for (int i = 0; i < PAIR; ++i)
#pragma unroll
    for (int j = 0; j < TWOS; ++j) v[i][j] = 0;
}
template <class L> using States = f2[L::PAIR][L::TWOS];
// A of the thread's states, times log2(e)
template <class L> __device__ __forceinline__ void load_rates(States<L>& A, const Args& a, const Place<L>& at) {
#pragma unroll
  for (int i = 0; i < L::PAIR; ++i) {
    load_states(A[i], a.A + (int64_t)at.channel(i) * a.state, at.state0(), a.state, a.wide, at.has(i));
#pragma unroll
    for (int j = 0; j < L::TWOS; ++j) A[i][j] = mul(A[i][j], both(LOG2E));
  }
}
__device__ __forceinline__ int64_t all_states(const Args& a) { return (int64_t)a.n * a.channels * a.state; }
// the thread's states of an array [n][c][state]
template <class L> __device__ __forceinline__ void load_all(States<L>& v, const float* p, const Args& a, const Place<L>& at) {
#pragma unroll
  for (int i = 0; i < L::PAIR; ++i)
    load_states(v[i], p + ((int64_t)at.seq * a.channels + at.channel(i)) * a.state, at.state0(), a.state, a.wide, at.has(i));
}
template <class L> __device__ __forceinline__ void store_all(float* p, const States<L>& v, const Args& a, const Place<L>& at) {
#pragma unroll
  for (int i = 0; i < L::PAIR; ++i)
    if (at.has(i)) store_states(p + ((int64_t)at.seq * a.channels + at.channel(i)) * a.state, v[i], at.state0(), a.state, a.wide);
}

// The decays of a chunk as its steps one by one would have it: where their product is below a float's and the state infinite, that stays what it is.
__device__ __forceinline__ f2 held(f2 keep, f2 h) {
  float x, y, p, q;
  unpack2(keep, x, y);
  unpack2(h, p, q);
  return pack2(x == 0.f && fabsf(p) == INFINITY ? 1.f : x, y == 0.f && fabsf(q) == INFINITY ? 1.f : y);
}
// What the chunks one after another pass on, from `from` on (towards the chunk of the block, by `way`): h = exp(A sum) h + end.  Those of several chunks are
// asked for at a time.
template <class L> __device__ __forceinline__ void fold_chunks(States<L>& h, const States<L>& A, const Args& a, const Place<L>& at, int from, int way) {
  constexpr int BATCH = 4;
  for (int j0 = from; j0 != at.chunk;) {
    const int left = way > 0 ? at.chunk - j0 : j0 - at.chunk, count = left < BATCH ? left : BATCH;
    States<L> end[BATCH];
    float sum[BATCH][L::PAIR];
    bool cut[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (u < count) {
        const int j = j0 + u * way;
        cut[u] = j == from || a.cuts[(int64_t)j * a.n + at.seq] != 0;      // the first of them began from what there was
        load_all<L>(end[u], a.ends + (int64_t)j * all_states(a), a, at);
#pragma unroll
        for (int i = 0; i < L::PAIR; ++i) sum[u][i] = at.has(i) ? a.sums[((int64_t)j * a.n + at.seq) * a.channels + at.channel(i)] : 0.f;
      }
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (u < count)
#pragma unroll
        for (int i = 0; i < L::PAIR; ++i) {
          f2 keep[L::TWOS];
          decay(keep, A[i], sum[u][i]);
#pragma unroll
          for (int s = 0; s < L::TWOS; ++s) h[i][s] = cut[u] ? end[u][i][s] : fma(held(keep[s], h[i][s]), h[i][s], end[u][i][s]);
        }
    j0 += count * way;
  }
}
// What a chunk leaves for them.
template <class L> __device__ __forceinline__ void leave_chunk(const States<L>& h, const float (&sum)[L::PAIR], bool cut, const Args& a, const Place<L>& at) {
  store_all<L>(a.ends + (int64_t)at.chunk * all_states(a), h, a, at);
#pragma unroll
  for (int i = 0; i < L::PAIR; ++i)
    if (at.has(i) && at.sl == 0) a.sums[((int64_t)at.chunk * a.n + at.seq) * a.channels + at.channel(i)] = sum[i];
  if (threadIdx.x == 0 && at.tile == 0 && at.group == 0) a.cuts[(int64_t)at.chunk * a.n + at.seq] = cut;
}

// ---- the host's part -------------------------------------------------------------------------------------------------------------------

struct Shape {
  bool narrow;                         // a thread has few states, so that few channels fill the device
  int sl, warps, width, tiles, chunks, chunk;
  int each;                            // few steps backward: sequences of a block
  int64_t blocks, rows;                // backward: rows of sums over steps
};
// Lanes for a channel's states of `each`, warps (a power of two) for a group's channels of which a thread has `pair`, up to `most_width` together (shared
// memory).
inline Shape tiled(const paac_selective& s, int each, int pair, int most_width) {
  Shape h{};
  h.sl = 1;
  while (h.sl * each < s.state) h.sl *= 2;
  const int per_warp = 32 / h.sl * pair, of_group = s.c / s.groups;
  h.warps = 1;
  while (h.warps < MOST_WARPS && h.warps * per_warp < of_group && h.warps * per_warp * 2 <= most_width) h.warps *= 2;
  h.width = h.warps * per_warp;
  h.tiles = (of_group + h.width - 1) / h.width;
  h.chunks = 1;
  h.chunk = s.t;
  h.blocks = (int64_t)h.tiles * s.groups * s.n;
  return h;
}
// Steps cut into chunks of `least` windows or more, so that about `room` warps are at work, or not at all if that leaves less than three: every block walks its
// chunk twice then.
inline void cut_steps(Shape& h, const paac_selective& s, int64_t room, int least) {
  const int64_t spans = ((int64_t)s.t + SPAN - 1) / SPAN;
  int64_t chunks = room / (h.blocks * h.warps);
  if (chunks > spans / least) chunks = spans / least;
  if (chunks > 64) chunks = 64;
  if (chunks < 3) return;
  const int64_t each = (spans + chunks - 1) / chunks;
  h.chunk = (int)each * SPAN;
  h.chunks = (int)((spans + each - 1) / each);
  h.blocks *= h.chunks;
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
    r.a = piece((size_t)h.rows * s.c * s.state * 4);
    r.d = piece((size_t)h.rows * s.c * 8);
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

size_t gradient_room(const paac_selective& s);      // of the gradient's scratch (selective_scan_back.cu)

inline bool shape_ok(const paac_selective* s) {
  return s != nullptr && s->t >= 1 && s->t <= (1 << 30) && s->n >= 1 && s->c >= 1 && (int64_t)s->n * s->c < ((int64_t)1 << 31) && s->state >= 1 && s->state <= 64 &&
         s->groups >= 1 && s->c % s->groups == 0 && (s->type == PAAC_FP32 || s->type == PAAC_BF16);
}
inline int size_of(const paac_selective& s) { return s.type == PAAC_BF16 ? 2 : 4; }

inline Args common_args(const paac_selective& s, const Shape& h) {
  Args a{};
  a.x = step_rows(s.x, s.t, s.n); a.dt = step_rows(s.dt, s.t, s.n); a.b = step_rows(s.B, s.t, s.n); a.c = step_rows(s.C, s.t, s.n); a.z = step_rows(s.z, s.t, s.n);
  a.restart = {s.restart, s.t > 1 ? s.restart_t : 0, s.n > 1 ? s.restart_n : 0};
  a.A = s.A; a.D = s.D; a.bias = s.dt_bias;
  a.t = s.t; a.n = s.n; a.channels = s.c; a.state = s.state; a.groups = s.groups; a.softplus = s.softplus != 0;
  a.tiles = h.tiles; a.chunks = h.chunks; a.chunk = h.chunk;
  return a;
}
// Accesses of four channels where places, channels and groups allow it.
inline bool four_wide(const paac_selective& s, int align) { return align >= 4 * size_of(s) && (s.c / s.groups) % 4 == 0; }
inline bool states_wide(const paac_selective& s, const void* p, const void* q, const void* r) {
  return s.state % 4 == 0 && (((uintptr_t)p | (uintptr_t)q | (uintptr_t)r) & 15u) == 0;
}
// f(a layout's lanes as a constant), up to MOST
template <int MOST, class F> cudaError_t by_lanes(int sl, F f) {
  if (sl == 1) return f(std::integral_constant<int, 1>());
  if (sl == 2) return f(std::integral_constant<int, 2>());
  if (sl == 4) return f(std::integral_constant<int, 4>());
  if constexpr (MOST == 16) if (sl == 16) return f(std::integral_constant<int, 16>());
  return f(std::integral_constant<int, 8>());
}

}  // namespace selective
}  // namespace paac
