// A gated linear recurrence over the steps of many sequences, and its gradient (paac_gated_scan, paac_gated_scan_backward).
//
// Every channel is a chain of its own, h_t = a_t h_{t-1} + b_t.  Backward, what step t passes on to the one before it is
// r_t = a_t (dh_t + r_{t+1}): the same chain in the state r, with the coefficients a_t and a_t dh_t, run the other way.
// A step that restarts takes nothing of the state: the state is left out there, not multiplied by 0.
//
// What bounds it: memory (three arrays forward, five or six backward, a few operations for each element), latency for few columns.
// Measured (the kernels back to back in a graph, inputs in turn that L2 does not hold together; bf16 unless said): 5 steps of 1024 sequences
// with 512 channels 5.7 us forward (20 MB; 4.1 where L2 holds them) and 8.1 backward (31 MB; 6.1), calls through the binding 9.8 and 12;
// 2 sequences of 32,768 steps with 512 channels 69 us (201 MB at 2.9 TB/s: both walks work out the gates, half of all issue
// slots, and a round's begin and joins leave memory idle); 3 of 20,011 steps with 200 channels of floats backward 59 us (240 MB at
// 4.0 TB/s, waits for loads); returns of 5 steps of 32 environments 1.5 us, of 64 steps of 1024 4.1, calls 8.
#include "cluster.cuh"
#include "pack.cuh"
#include "per_device.h"
#include "rows.h"

namespace {
using paac::bf16;
using paac::Pack;

// Arrays as the kernels walk them: k counts the steps in the order of the recurrence (backward: of the gradient's), so that pointers are
// to the first of those and strides along the steps may be negative.
struct Rows { void* data; int64_t step, seq; };
struct Args {
  Rows gate, x, h, dh, out, dgate;     // forward: out is h; backward: out is dx, h the stored states
  const uint8_t* restart;
  int64_t restart_step, restart_seq;
  const float* first;                  // forward: h0; backward: dh_last
  float* last;                         // forward: h_last; backward: dh0
  const float* h0;                     // backward: the state before the sequence's first step
  int t, n, c;
};

// z = 1 / (1 + e^-g) and 1 - z = e^-g z, both right to float rounding: g is kept above -87, where e^-g is still a float (z is 1.6e-38
// there and below).  max.NaN keeps a NaN; what e^-g or z is below 2^-126 counts as 0.  bf16 storage takes the faster exponential, whose
// argument is a rounded product with log2(e), so that e^-g is off by up to (2 + 1.2 |g|) 2^-23 of its value: 2^-19 at 10.  The
// storage's rounding hides that in h, dgate and dx; h_last and dh0, floats, have it.
template <class T> __device__ __forceinline__ void sigmoid(float g, float& z, float& rest) {
  float t, e;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(t) : "f"(g), "f"(-87.f));
  if constexpr (sizeof(T) == 2) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t * -1.442695041f));
  else e = expf(-t);
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(z) : "f"(1.f + e));
  rest = e * z;
}

template <class T> __device__ __forceinline__ const T* at(const Rows& r, int k, int seq, int c) { return (const T*)r.data + k * r.step + seq * r.seq + c; }
template <class T> __device__ __forceinline__ T* to(const Rows& r, int k, int seq, int c) { return (T*)r.data + k * r.step + seq * r.seq + c; }

// ---- a thread's walk down the steps of W neighbouring channels -------------------------------------------------------------------------
// The loads of AHEAD steps are under way: a step that has been worked on makes room for the one AHEAD steps on.  They are kept in registers, or
// (RING) copied to the thread's own places in shared memory, [step][array][thread], which needs no registers and no barrier: a
// thread reads only what it has copied itself and waited for.

template <class T, int W, bool SIGMOID, bool BACK, bool APPLY, int AHEAD, bool RING> struct Walk {
  static constexpr bool X = !BACK || (SIGMOID && APPLY), H = BACK && APPLY;
  static constexpr int ARRAYS = 1 + X + H + BACK;
  struct Step { Pack<T, W> gate, x, h, dh; uint32_t cut; };
  const Args& a;
  const T *gate, *x, *h, *dh;        // of the next step to be loaded
  const uint8_t* flag;
  int k0, end;
  uint4* ring;                       // this thread's; the next array's place is `pitch` on
  int pitch;

  __device__ __forceinline__ Walk(const Args& args, int first, int last, int seq, int c, uint4* ring_, int pitch_)
      : a(args), k0(first), end(last), ring(ring_), pitch(pitch_) {
    gate = at<T>(a.gate, k0, seq, c);
    if (X) x = at<T>(a.x, k0, seq, c);
    if (BACK) dh = at<T>(a.dh, k0, seq, c);
    if (H) h = at<T>(a.h, k0 + 1, seq, c);             // the state before a step is that of the next one here
    flag = a.restart != nullptr ? a.restart + k0 * a.restart_step + seq * a.restart_seq : nullptr;
  }
  __device__ __forceinline__ void get(Pack<T, W>& p, const T* from, int place) {
    if constexpr (RING) paac::copy_to<16>(ring + place * pitch, from); else p.load(from);
  }
  // (the last step of all has no state before it in h)
  template <bool LAST> __device__ __forceinline__ void load(Step& s, int slot, int k) {
    int place = slot * ARRAYS;
    get(s.gate, gate, place++); gate += a.gate.step;
    if (X) { get(s.x, x, place++); x += a.x.step; }
    if (BACK) { get(s.dh, dh, place++); dh += a.dh.step; }
    if (H) { if (!LAST || k + 1 < a.t) get(s.h, h, place); h += a.h.step; }
    s.cut = 0;
    if (flag != nullptr) { s.cut = *flag; flag += a.restart_step; }
  }
  // what has been loaded for a step
  __device__ __forceinline__ void arrived(Step& s, int slot) {
    if constexpr (RING) {
      paac::copies_wait<AHEAD - 1>();
      const uint4* p = ring + slot * ARRAYS * pitch;
      s.gate.raw = *p; p += pitch;
      if (X) { s.x.raw = *p; p += pitch; }
      if (BACK) { s.dh.raw = *p; p += pitch; }
      if (H) s.h.raw = *p;
    }
  }
  // work(step, its number) for every step from the first to the last
  template <class F> __device__ __forceinline__ void run(F work) {
    Step s[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (k0 + u < end) load<true>(s[u], u, k0 + u);
      if (RING) paac::copies_end_step();
    }
    int k = k0;
    const int whole = H && end == a.t ? end - 1 : end;
    for (; whole - k >= 2 * AHEAD; k += AHEAD) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        arrived(s[u], u);
        work(s[u], k + u);
        load<false>(s[u], u, k + u + AHEAD);
        if (RING) paac::copies_end_step();
      }
    }
    for (; k < end; k += AHEAD) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
        if (k + u < end) {
          arrived(s[u], u);
          work(s[u], k + u);
          if (k + u + AHEAD < end) load<true>(s[u], u, k + u + AHEAD);
          if (RING) paac::copies_end_step();
        }
    }
  }
};

// one step backward of W channels: s = dh_t + r_{t+1}
template <class T, int W, bool SIGMOID>
__device__ __forceinline__ void step_back(const float (&g)[W], const float (&x)[W], const float (&before)[W], const float (&dh)[W], bool cut,
                                          float (&state)[W], float (&dgate)[W], float (&dx)[W]) {
#pragma unroll
  for (int j = 0; j < W; ++j) {
    const float s = dh[j] + state[j];
    float z = g[j], rest = 1.f;
    if (SIGMOID) {
      sigmoid<T>(g[j], z, rest);
      dgate[j] = s * ((cut ? 0.f : before[j]) - x[j]) * z * rest;
    } else {
      dgate[j] = cut ? 0.f : s * before[j];
    }
    dx[j] = s * rest;
    state[j] = cut ? 0.f : z * s;
  }
}

// steps [k0, end) from `state`, with all that is written for them
template <class T, int W, bool SIGMOID, bool BACK, int AHEAD, bool RING>
__device__ __forceinline__ void apply_steps(const Args& a, int k0, int end, int seq, int c, float (&state)[W], uint4* ring, int pitch) {
  typedef Walk<T, W, SIGMOID, BACK, true, AHEAD, RING> V;
  T* dgate_at = BACK ? to<T>(a.dgate, k0, seq, c) : nullptr;
  T* out_at = to<T>(a.out, k0, seq, c);
  const bool dgate_wanted = a.dgate.data != nullptr, out_wanted = a.out.data != nullptr;
  V(a, k0, end, seq, c, ring, pitch).run([&](const typename V::Step& s, int k) {
    float g[W], x[W], out[W];
    s.gate.widen(g);
    if (V::X) s.x.widen(x);
    const bool cut = s.cut != 0;
    Pack<T, W> p;
    if constexpr (!BACK) {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        float z = g[j], rest = 1.f;
        if (SIGMOID) sigmoid<T>(g[j], z, rest);
        const float b = rest * x[j];
        out[j] = state[j] = cut ? b : fmaf(z, state[j], b);
      }
    } else {
      float dh[W], before[W], dgate[W];
      s.dh.widen(dh);
      if (k + 1 < a.t) {
        s.h.widen(before);
      } else {
#pragma unroll
        for (int j = 0; j < W; ++j) before[j] = a.h0 != nullptr ? a.h0[(int64_t)seq * a.c + c + j] : 0.f;
      }
      step_back<T, W, SIGMOID>(g, x, before, dh, cut, state, dgate, out);
      if (dgate_wanted) {
        p.round(dgate);
        p.store(dgate_at);
        dgate_at += a.dgate.step;
      }
    }
    if (out_wanted) {
      p.round(out);
      p.store(out_at);
      out_at += a.out.step;
    }
  });
}

// ---- few steps or many columns: every thread walks from the first step to the last ---------------------------------------------------------------------
constexpr int COLUMN_THREADS = 128;
// Forward the steps under way are in registers, backward, with three or four arrays a step, in a ring.
template <class T, int W, bool SIGMOID, bool BACK> struct ColumnShape {
  static constexpr bool RING = W * sizeof(T) == 16 && BACK;
  static constexpr int AHEAD = RING ? 6 : (BACK ? 4 : 8), RING_BYTES = RING ? AHEAD * (SIGMOID ? 4 : 3) * COLUMN_THREADS * 16 : 0;
};

template <class T, int W, bool SIGMOID, bool BACK>
__global__ void __launch_bounds__(COLUMN_THREADS)
scan_columns_kernel(const __grid_constant__ Args a) {
  paac::pdl_entry();
  const int per = a.c / W, col = blockIdx.x * COLUMN_THREADS + threadIdx.x;
  if (col >= a.n * per) return;
  const int seq = col / per, c = (col - seq * per) * W;
  float state[W];
#pragma unroll
  for (int j = 0; j < W; ++j) state[j] = 0.f;
  if (a.first != nullptr) paac::load_floats(state, a.first + (int64_t)seq * a.c + c);
  typedef ColumnShape<T, W, SIGMOID, BACK> S;
  extern __shared__ uint4 ring[];
  apply_steps<T, W, SIGMOID, BACK, S::AHEAD, S::RING>(a, 0, a.t, seq, c, state, ring + threadIdx.x, COLUMN_THREADS);
  if (a.last != nullptr) paac::store_floats(a.last + (int64_t)seq * a.c + c, state);
}

// ---- few columns, many steps: a cluster of blocks takes the columns' steps in rounds --------------------------------------------------------
//
// Spans of steps are composed: span (A, B) takes a state h to A h + B, and one behind the other (A2, B2) makes (A2 A1, A2 B1 + B2).  A span with
// a restart in it takes nothing of the state: that is a flag of its own (A = 0 would still make a NaN of an infinity), passed between
// threads as A = -0.  A product of gates may be -0 too: exactly, or because a negative one is too small for a float.  So what is passed
// has +0 added to it once it has been rounded, which makes +0 of -0 and changes nothing else: a NaN times +0 stays a NaN.
//
// In a round a thread has a span of `each` steps of W channels, a warp CT columns of threads by 32 / CT spans, a block eight warps one behind
// the other, a cluster its blocks one behind the other.  Every thread first walks its span for (A, B); spans are joined by shuffles
// in a warp, through shared memory in a block and through the other blocks' shared memory in a cluster, always from the first
// to the last, so that results are the same bits in every run; then it walks the span again from the state it begins in, and writes.  Every block
// follows the state through the whole round by itself, so that one barrier of the cluster does for a round.  A round is no longer
// than L2 holds, so that the second walk reads from there: memory is read and written once.
constexpr int SPAN_THREADS = 256, SPAN_WARPS = SPAN_THREADS / 32, MAX_CLUSTER = 16;

// Whether steps under way are kept in a ring in shared memory (Walk): three blocks share a multiprocessor then instead of two.
template <class T, int W, bool BACK, bool RING> struct SpanShape {
  static constexpr int ROW = RING && sizeof(T) == 4 ? 128 : 64, WIDTH = W * (int)sizeof(T);
  static constexpr int CT = ROW / WIDTH < 32 ? ROW / WIDTH : 32;            // columns of threads: rows of 64 bytes, or 128
  static constexpr int COLS = CT * W, SPANS = SPAN_THREADS / CT;            // channels and spans of a block
  static constexpr int FOLD_AHEAD = WIDTH < 16 ? 8 : 4, APPLY_AHEAD = WIDTH < 16 ? (BACK && W > 1 ? 4 : 8) : (BACK ? (RING ? 3 : 2) : 4);
  static constexpr int RING_BYTES = RING ? (BACK ? 12 : 8) * SPAN_THREADS * 16 : 0;      // three steps of four arrays, or four of two
  static constexpr int BLOCKS = RING ? 3 : 2;
};

constexpr float CUT = -0.f;
__device__ __forceinline__ bool is_cut(float a) { return __float_as_uint(a) == 0x80000000u; }
// a product of gates as it is passed (added by itself: fma(a, b, +0) is still -0 where a b is a negative number that rounds to zero)
__device__ __forceinline__ float passed(float product) { return __fadd_rn(product, 0.f); }
__device__ __forceinline__ float2 joined(float2 first, float2 then) {       // as they are passed: A = -0 for a restart
  if (is_cut(then.x)) return then;
  return make_float2(is_cut(first.x) ? CUT : passed(__fmul_rn(then.x, first.x)), fmaf(then.x, first.y, then.y));
}
__device__ __forceinline__ float taken(float2 span, float h) { return is_cut(span.x) ? span.y : fmaf(span.x, h, span.y); }

// (A, B) of steps [k0, end), and whether a restart is among them (A then means nothing)
template <class T, int W, bool SIGMOID, bool BACK, int AHEAD, bool RING>
__device__ __forceinline__ void fold_steps(const Args& a, int k0, int end, int seq, int c, float (&A)[W], float (&B)[W], bool& D, uint4* ring, int pitch) {
  typedef Walk<T, W, SIGMOID, BACK, false, AHEAD, RING> V;
  V(a, k0, end, seq, c, ring, pitch).run([&](const typename V::Step& s, int) {
    float g[W], v[W];
    s.gate.widen(g);
    if constexpr (BACK) s.dh.widen(v); else s.x.widen(v);
    const bool cut = s.cut != 0;
#pragma unroll
    for (int j = 0; j < W; ++j) {
      float z = g[j], rest = 1.f;
      if (SIGMOID) sigmoid<T>(g[j], z, rest);
      if (BACK) {
        B[j] = cut ? 0.f : z * (v[j] + B[j]);
      } else {
        const float b = rest * v[j];
        B[j] = cut ? b : fmaf(z, B[j], b);
      }
      A[j] *= z;
    }
    D = D || cut;
  });
}

template <class T, int W, bool SIGMOID, bool BACK, bool RING>
__global__ void __launch_bounds__(SPAN_THREADS, SpanShape<T, W, BACK, RING>::BLOCKS)
scan_spans_kernel(const __grid_constant__ Args a, int cluster, int each) {
  typedef SpanShape<T, W, BACK, RING> S;
  constexpr int CT = S::CT, COLS = S::COLS;
  extern __shared__ uint4 ring[];
  __shared__ float2 of_warp[SPAN_WARPS][COLS];              // a warp's span; then that of all warps before it
  __shared__ float2 of_block[2][MAX_CLUSTER][COLS];         // every block's span, by the parity of the round
  __shared__ float at_warp[SPAN_WARPS][COLS];               // the state before a warp's first step

  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = paac::cluster_rank();
  const int cl = lane % CT, part = lane / CT;
  const int per = a.c / W, tile = blockIdx.x / cluster;
  const int64_t col = (int64_t)tile * CT + cl;
  const bool active = col < (int64_t)a.n * per;
  const int seq = active ? (int)(col / per) : 0, c = active ? (int)(col - (int64_t)seq * per) * W : 0;
  const int64_t round = (int64_t)cluster * S::SPANS * each;                 // steps of a round; this thread's first:
  const int64_t within = ((int64_t)rank * S::SPANS + warp * (32 / CT) + part) * each;

  paac::cluster_arrive();                                   // nobody stores into a block that has not begun
  paac::pdl_entry();
  // the thread that follows a channel's state through the rounds
  const int64_t channel = (int64_t)tile * COLS + threadIdx.x;
  const bool follows = threadIdx.x < COLS, holds = follows && channel < (int64_t)a.n * a.c;
  float state = holds && a.first != nullptr ? a.first[channel] : 0.f;

  int parity = 0;
  for (int64_t base = 0; base < a.t; base += round, parity ^= 1) {
    const int k0 = base + within < a.t ? (int)(base + within) : a.t, end = active ? (k0 + (int64_t)each < a.t ? k0 + each : a.t) : k0;
    float A[W], B[W];
    bool D = false;
#pragma unroll
    for (int j = 0; j < W; ++j) { A[j] = 1.f; B[j] = 0.f; }
    fold_steps<T, W, SIGMOID, BACK, S::FOLD_AHEAD, RING>(a, k0, end, seq, c, A, B, D, ring + threadIdx.x, SPAN_THREADS);
    // spans of the warp, up to and with this thread's
#pragma unroll
    for (int d = 1; d < 32 / CT; d *= 2) {
      const bool before = part >= d, DD = __shfl_up_sync(0xffffffffu, (int)D, d * CT) != 0;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float AA = __shfl_up_sync(0xffffffffu, A[j], d * CT), BB = __shfl_up_sync(0xffffffffu, B[j], d * CT);
        if (before) {
          B[j] = D ? B[j] : fmaf(A[j], BB, B[j]);
          A[j] *= AA;
        }
      }
      D = D || (before && DD);
    }
    if (part == 32 / CT - 1) {
#pragma unroll
      for (int j = 0; j < W; ++j) of_warp[warp][cl * W + j] = make_float2(D ? CUT : passed(A[j]), B[j]);
    }
    // those before this thread's
    if (32 / CT > 1) {
      D = __shfl_up_sync(0xffffffffu, (int)D, CT) != 0 && part > 0;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        A[j] = __shfl_up_sync(0xffffffffu, A[j], CT);
        B[j] = __shfl_up_sync(0xffffffffu, B[j], CT);
        if (part == 0) { A[j] = 1.f; B[j] = 0.f; }
      }
    } else {
      D = false;
#pragma unroll
      for (int j = 0; j < W; ++j) { A[j] = 1.f; B[j] = 0.f; }
    }
    __syncthreads();
    if (base == 0) paac::cluster_wait();
    if (follows) {
      float2 all = make_float2(1.f, 0.f);
#pragma unroll
      for (int w = 0; w < SPAN_WARPS; ++w) {
        const float2 mine = of_warp[w][threadIdx.x];
        of_warp[w][threadIdx.x] = all;
        all = joined(all, mine);
      }
      for (int r = 0; r < cluster; ++r) paac::store_in_block(&of_block[parity][rank][threadIdx.x], r, all);
    }
    paac::cluster_arrive();
    paac::cluster_wait();
    if (follows) {
      float mine = state;
      for (int r = 0; r < cluster; ++r) {
        if (r == rank) mine = state;
        state = taken(of_block[parity][r][threadIdx.x], state);
      }
#pragma unroll
      for (int w = 0; w < SPAN_WARPS; ++w) at_warp[w][threadIdx.x] = taken(of_warp[w][threadIdx.x], mine);
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < W; ++j) B[j] = D ? B[j] : fmaf(A[j], at_warp[warp][cl * W + j], B[j]);
    apply_steps<T, W, SIGMOID, BACK, S::APPLY_AHEAD, RING>(a, k0, end, seq, c, B, ring + threadIdx.x, SPAN_THREADS);
  }
  if (rank == 0 && holds && a.last != nullptr) a.last[channel] = state;
}

// What a round of all blocks together may read and write, so that the second walk finds in L2 what the first has read.
constexpr int64_t ROUND_BYTES = 110 << 20;
// From so many bytes on the ring is the better place for steps under way: 12 MB backward in bf16 6.6 us in registers and 8.3 in a ring, 49 MB
// 18.8 and 19.6, 147 MB 56 and 43; 240 MB in float 99 and 60, forward 49 MB 18.4 and 17.6, 144 MB 64 and 45.  Forward in bf16 never.
constexpr int64_t RING_FROM = 48 << 20;

// How many clusters of so many blocks are resident at once (more would wait for the others): depends on how the part's multiprocessors are
// grouped, so it is asked for, once on each device.
struct Resident { int clusters[MAX_CLUSTER + 1]; };
template <class K> bool ask_resident(K kernel, int ring_bytes, Resident& r) {
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ring_bytes) != cudaSuccess)
    return false;
  for (int i = 1; i <= MAX_CLUSTER; ++i) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(i); cfg.blockDim = dim3(SPAN_THREADS); cfg.dynamicSmemBytes = ring_bytes;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = i; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    r.clusters[i] = 0;
    if (cudaOccupancyMaxActiveClusters(&r.clusters[i], kernel, &cfg) != cudaSuccess) { cudaGetLastError(); r.clusters[i] = 0; }
  }
  return true;
}

template <class T, int W, bool SIGMOID, bool BACK, bool RING> cudaError_t launch_spans(const Args& a, int64_t columns, int64_t bytes, cudaStream_t s) {
  typedef SpanShape<T, W, BACK, RING> S;
  const auto kernel = scan_spans_kernel<T, W, SIGMOID, BACK, RING>;
  static paac::PerDevice<Resident> resident;
  int device = -1;
  const Resident* room = cudaGetDevice(&device) == cudaSuccess ? resident.get(device, [&](Resident& r) { return ask_resident(kernel, S::RING_BYTES, r); }) : nullptr;
  if (room == nullptr) return cudaErrorUnknown;
  const int64_t tiles = (columns + S::CT - 1) / S::CT;
  // the fewest steps a span for which all clusters find room, by the fewest blocks (8000 steps of 2048 channels in float: 64 tiles by 6
  // blocks 53 us, by 4 60; 1000 steps of 832 channels: 26 by 8 4.9 us, by 10, for which a span is as long, 6.9).  Sizes that are no power of
  // two with a twentieth to spare, since not all that are said to fit do: 40 by 10, where 41 should, 29 us, by 9 or 8 23.
  const int64_t rounds = (bytes + ROUND_BYTES - 1) / ROUND_BYTES;
  int cluster = 1;
  int64_t each = 0;
  for (int i = 1; i <= MAX_CLUSTER; ++i) {
    const bool odd = (i & (i - 1)) != 0;
    if (i > 1 && tiles * (odd ? 20 : 1) > (int64_t)room->clusters[i] * (odd ? 19 : 1)) continue;
    const int64_t spans = rounds * i * S::SPANS, steps = (a.t + spans - 1) / spans;
    if (i == 1 || steps < each) { cluster = i; each = steps; }
  }
  return paac::launch_clusters_on(s, kernel, dim3((unsigned)(tiles * cluster)), dim3(SPAN_THREADS), cluster, S::RING_BYTES, a, cluster, (int)each);
}

// Which of the two takes less time, by what was measured (us).  Columns: a step of a thread's walk is 0.14 forward (eight steps' loads under way),
// 0.22 or 0.4 backward, and the bytes pass at some 5.8 TB/s; 64 steps of 131,072 channels forward in bf16 17 (spans 69), of 524,288
// 35 (269), but 1000 steps of 13,312 127 (spans 32).  Spans: a wave of blocks needs 4.5 for its barriers and joins, and the bytes
// pass at some 2.9 TB/s; 200 steps of 65,536 channels backward in float 95 (columns 118).
bool by_columns(const Args& a, int64_t tiles, int64_t bytes, bool sigmoid, bool back) {
  const double walk = a.t * (back ? (sigmoid ? 0.4 : 0.22) : 0.14) + bytes / 5.8e6;
  const double spans = (double)((tiles + 148 * 2 - 1) / (148 * 2)) * 4.5 + bytes / 2.9e6;
  return walk <= spans;
}

template <class T, int W, bool SIGMOID, bool BACK> cudaError_t launch(const Args& a, cudaStream_t s) {
  const int64_t columns = (int64_t)a.n * (a.c / W), bytes = (BACK ? (SIGMOID ? 6 : 5) : 3) * (int64_t)sizeof(T) * a.n * a.c * a.t;
  constexpr int CT = SpanShape<T, W, BACK, false>::CT;
  if (by_columns(a, (columns + CT - 1) / CT, bytes, SIGMOID, BACK)) {
    typedef ColumnShape<T, W, SIGMOID, BACK> S;
    if (S::RING_BYTES > 48 << 10) {
      static paac::PerDevice<bool> ready;
      int device = -1;
      const bool ok = cudaGetDevice(&device) == cudaSuccess && ready.get(device, [](bool&) {
        return cudaFuncSetAttribute(scan_columns_kernel<T, W, SIGMOID, BACK>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::RING_BYTES) == cudaSuccess;
      }) != nullptr;
      if (!ok) return cudaErrorUnknown;
    }
    return paac::launch_overlapped_on(s, scan_columns_kernel<T, W, SIGMOID, BACK>, dim3((unsigned)((columns + COLUMN_THREADS - 1) / COLUMN_THREADS)),
                                      dim3(COLUMN_THREADS), S::RING_BYTES, a);
  }
  if constexpr (W * sizeof(T) == 16 && (BACK || sizeof(T) == 4))
    if (bytes >= RING_FROM) return launch_spans<T, W, SIGMOID, BACK, true>(a, columns, bytes, s);
  return launch_spans<T, W, SIGMOID, BACK, false>(a, columns, bytes, s);
}
template <class T, int W, bool BACK> cudaError_t launch_width(const Args& a, bool sig, cudaStream_t s) {
  return sig ? launch<T, W, true, BACK>(a, s) : launch<T, W, false, BACK>(a, s);
}
// accesses of W channels: as wide as the rows' places and the channels allow
template <bool BACK> cudaError_t launch_type(const Args& a, int type, int W, bool sig, cudaStream_t s) {
  if (type == PAAC_BF16)
    return W == 8 ? launch_width<bf16, 8, BACK>(a, sig, s) : W == 4 ? launch_width<bf16, 4, BACK>(a, sig, s)
         : W == 2 ? launch_width<bf16, 2, BACK>(a, sig, s) : launch_width<bf16, 1, BACK>(a, sig, s);
  return W == 4 ? launch_width<float, 4, BACK>(a, sig, s) : W == 2 ? launch_width<float, 2, BACK>(a, sig, s) : launch_width<float, 1, BACK>(a, sig, s);
}
cudaError_t dispatch(const Args& a, const paac_scan& s, bool back, int W, cudaStream_t st) {
  const bool sig = s.kind == PAAC_SCAN_SIGMOID;
  return back ? launch_type<true>(a, s.type, W, sig, st) : launch_type<false>(a, s.type, W, sig, st);
}

// ---- the host's part -------------------------------------------------------------------------------------------------------------------

int size_of(const paac_scan& s) { return s.type == PAAC_BF16 ? 2 : 4; }

// rows as the kernels walk them
Rows walked(const paac_rows& r, const paac_scan& s, bool from_the_end) {
  Rows w{r.data, s.t > 1 ? r.inner : 0, s.n > 1 ? r.outer : 0};
  if (from_the_end && r.data != nullptr) {
    w.data = (char*)r.data + (int64_t)(s.t - 1) * w.step * size_of(s);
    w.step = -w.step;
  }
  return w;
}
Args common_args(const paac_scan& s, bool from_the_end) {
  Args a{};
  a.t = s.t; a.n = s.n; a.c = s.c;
  a.restart = s.restart; a.restart_step = s.t > 1 ? s.restart_t : 0; a.restart_seq = s.n > 1 ? s.restart_n : 0;
  if (from_the_end && s.restart != nullptr) {
    a.restart = s.restart + (int64_t)(s.t - 1) * a.restart_step;
    a.restart_step = -a.restart_step;
  }
  return a;
}

bool shape_ok(const paac_scan* s) {
  return s != nullptr && s->t >= 1 && s->t <= (1 << 30) && s->n >= 1 && s->c >= 1 && (int64_t)s->n * s->c < ((int64_t)1 << 31) && (s->type == PAAC_FP32 || s->type == PAAC_BF16) &&
         (s->kind == PAAC_SCAN_LINEAR || s->kind == PAAC_SCAN_SIGMOID);
}

// Which arrays a call has, whether each is fit to be one, and whether what is written is apart from everything else.
struct Check {
  const paac_scan& s;
  bool ok = true;
  int align = 16;                    // bytes that all rows' places are multiples of
  paac::Arrays arrays;
  explicit Check(const paac_scan& s_) : s(s_) {
    if (s.restart == nullptr) return;
    const paac::RowSet flags(paac_rows{const_cast<uint8_t*>(s.restart), s.restart_n, s.restart_t}, s.n, s.t, 1, 1);
    ok = flags.sane();
    if (ok) arrays.keep(flags, false);
  }
  bool fit() const { return ok && arrays.apart; }
  void rows(const paac_rows& r, bool out, bool needed) {
    if (r.data == nullptr) { ok = ok && !needed; return; }
    const paac::RowSet set(r, s.n, s.t, s.c, size_of(s));
    if (!set.sane() || !set.aligned() || (out && !set.rows_apart())) { ok = false; return; }
    while (align > size_of(s) && !set.multiples_of(align)) align /= 2;
    arrays.keep(set, out);
  }
  // float [n][c]
  void state(const float* p, bool out) {
    if (p == nullptr) return;
    if ((uintptr_t)p & 3u) { ok = false; return; }
    if (((uintptr_t)p & 15u) != 0 && align > 2 * size_of(s)) align = 2 * size_of(s);      // four floats of a state are read at a time
    arrays.keep(p, (int64_t)s.n * s.c * 4, out);
  }
};

}  // namespace

extern "C" int paac_gated_scan(const paac_scan* s, paac_rows gate, paac_rows x, const float* h0, paac_rows h, float* h_last, void* stream) {
  if (!shape_ok(s)) return PAAC_ERR_ARG;
  Check check(*s);
  check.rows(gate, false, true);
  check.rows(x, false, true);
  check.rows(h, true, true);
  if (h0 != h_last) check.state(h0, false);
  check.state(h_last, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  const bool end = s->reverse != 0;
  Args a = common_args(*s, end);
  a.gate = walked(gate, *s, end); a.x = walked(x, *s, end); a.out = walked(h, *s, end);
  a.first = h0; a.last = h_last;
  return paac::launch_status(dispatch(a, *s, false, check.align / size_of(*s), static_cast<cudaStream_t>(stream)));
}

extern "C" int paac_gated_scan_backward(const paac_scan* s, paac_rows gate, paac_rows x, paac_rows h, paac_rows dh, const float* h0,
                                        const float* dh_last, paac_rows dgate, paac_rows dx, float* dh0, void* stream) {
  if (!shape_ok(s)) return PAAC_ERR_ARG;
  const bool sig = s->kind == PAAC_SCAN_SIGMOID;
  if (!sig) x.data = nullptr;                           // not read
  if (dgate.data == nullptr && dx.data == nullptr && dh0 == nullptr) return PAAC_ERR_ARG;
  Check check(*s);
  check.rows(gate, false, true);
  check.rows(x, false, sig);
  check.rows(h, false, true);
  check.rows(dh, false, true);
  check.state(h0, false);
  if (dh_last != dh0) check.state(dh_last, false);
  check.rows(dgate, true, false);
  check.rows(dx, true, false);
  check.state(dh0, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  const bool end = s->reverse == 0;
  Args a = common_args(*s, end);
  a.gate = walked(gate, *s, end); a.x = walked(x, *s, end); a.h = walked(h, *s, end); a.dh = walked(dh, *s, end);
  a.dgate = walked(dgate, *s, end); a.out = walked(dx, *s, end);
  a.h0 = h0; a.first = dh_last; a.last = dh0;
  return paac::launch_status(dispatch(a, *s, true, check.align / size_of(*s), static_cast<cudaStream_t>(stream)));
}
