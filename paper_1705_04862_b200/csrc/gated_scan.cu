// A gated linear recurrence over the steps of many sequences, and its gradient (paac_gated_scan, paac_gated_scan_backward).
//
// Every channel is a chain of its own, h_t = a_t h_{t-1} + b_t.  Backward, what step t passes on to the one before it is
// r_t = a_t (dh_t + r_{t+1}): the same chain in the state r, with the coefficients a_t and a_t dh_t, run the other way.
// A step that restarts takes nothing of the state: the state is left out there, not multiplied by 0.
//
// What bounds it: memory (three arrays forward, five or six backward, a few operations for each element), latency for few columns.
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

// z = 1 / (1 + e^-g) and 1 - z, each right to float rounding for any g: only e^-|g| is taken, which does not overflow.  The storage
// type's own rounding hides the faster exponential's error (some 2^-21) where it is bf16.
template <class T> __device__ __forceinline__ void sigmoid(float g, float& z, float& rest) {
  const float e = sizeof(T) == 2 ? __expf(-fabsf(g)) : expf(-fabsf(g)), s = __fdividef(1.f, 1.f + e), es = e * s;
  z = g < 0.f ? es : s;                // (a NaN is in both)
  rest = g < 0.f ? s : es;
}

template <class T> __device__ __forceinline__ const T* at(const Rows& r, int k, int seq, int c) { return (const T*)r.data + k * r.step + seq * r.seq + c; }
template <class T> __device__ __forceinline__ T* to(const Rows& r, int k, int seq, int c) { return (T*)r.data + k * r.step + seq * r.seq + c; }

// ---- many columns: a thread takes W neighbouring channels of a sequence and walks its steps ------------------------------------------
// Loads of the next AHEAD steps are under way while AHEAD are worked on.
constexpr int COLUMN_THREADS = 128;

template <class T, int W, bool SIGMOID, bool BACK, int AHEAD> struct Batch {
  Pack<T, W> gate[AHEAD], x[AHEAD], h[AHEAD], dh[AHEAD];
  bool cut[AHEAD];
  __device__ __forceinline__ void load(const Args& a, int k0, int seq, int c) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int k = k0 + u;
      if (k >= a.t) break;
      gate[u].load(at<T>(a.gate, k, seq, c));
      if (!BACK || SIGMOID) x[u].load(at<T>(a.x, k, seq, c));
      if (BACK) {
        dh[u].load(at<T>(a.dh, k, seq, c));
        if (k + 1 < a.t) h[u].load(at<T>(a.h, k + 1, seq, c));       // the state before this step
      }
      cut[u] = a.restart != nullptr && a.restart[k * a.restart_step + seq * a.restart_seq] != 0;
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

template <class T, int W, bool SIGMOID, bool BACK>
__global__ void __launch_bounds__(COLUMN_THREADS)
scan_columns_kernel(const __grid_constant__ Args a) {
  constexpr int AHEAD = W == 1 ? 8 : 4;
  paac::pdl_entry();
  const int per = a.c / W, col = blockIdx.x * COLUMN_THREADS + threadIdx.x;
  if (col >= a.n * per) return;
  const int seq = col / per, c = (col - seq * per) * W;
  float state[W], start[W];
#pragma unroll
  for (int j = 0; j < W; ++j) state[j] = start[j] = 0.f;
  if (a.first != nullptr) paac::load_floats(state, a.first + (int64_t)seq * a.c + c);
  if (BACK && a.h0 != nullptr) paac::load_floats(start, a.h0 + (int64_t)seq * a.c + c);
  Batch<T, W, SIGMOID, BACK, AHEAD> now, next;
  now.load(a, 0, seq, c);
  for (int k0 = 0; k0 < a.t; k0 += AHEAD) {
    next.load(a, k0 + AHEAD, seq, c);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int k = k0 + u;
      if (k >= a.t) break;
      float g[W], x[W], out[W];
      now.gate[u].widen(g);
      if (!BACK || SIGMOID) now.x[u].widen(x);
      if constexpr (!BACK) {
#pragma unroll
        for (int j = 0; j < W; ++j) {
          float z = g[j], rest = 1.f;
          if (SIGMOID) sigmoid<T>(g[j], z, rest);
          const float b = rest * x[j];
          out[j] = state[j] = now.cut[u] ? b : fmaf(z, state[j], b);
        }
      } else {
        float dh[W], before[W], dgate[W];
        now.dh[u].widen(dh);
        if (k + 1 < a.t) {
          now.h[u].widen(before);
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j) before[j] = start[j];
        }
        step_back<T, W, SIGMOID>(g, x, before, dh, now.cut[u], state, dgate, out);
        if (a.dgate.data != nullptr) {
          Pack<T, W> p;
          p.round(dgate);
          p.store(to<T>(a.dgate, k, seq, c));
        }
      }
      if (a.out.data != nullptr) {
        Pack<T, W> p;
        p.round(out);
        p.store(to<T>(a.out, k, seq, c));
      }
    }
    now = next;
  }
  if (a.last != nullptr) paac::store_floats(a.last + (int64_t)seq * a.c + c, state);
}

// ---- few columns, many steps: a cluster of blocks takes the columns' steps in rounds --------------------------------------------------------
//
// Spans of steps are composed: span (A, B) takes a state h to A h + B, and one behind the other (A2, B2) makes (A2 A1, A2 B1 + B2).  A span with
// a restart in it takes nothing of the state: that is a flag of its own (A = 0 would still make a NaN of an infinity), passed between
// threads as A = -0, which no product here gives: products are rounded as fma(A2, A1, +0).
//
// In a round a thread holds L steps of W channels in registers, a warp CT columns of threads by 32 / CT spans, a block eight warps one behind
// the other, a cluster its blocks one behind the other.  Spans are joined by shuffles in a warp, through shared memory in a block and
// through the other blocks' shared memory in a cluster, always from the first to the last, so that results are the same bits
// in every run; every block follows the state through the whole round by itself, so that one barrier of the cluster does for a
// round.  Each array is read and written once.  The loads of the next round are under way while this one is worked on.
constexpr int SPAN_THREADS = 256, SPAN_WARPS = SPAN_THREADS / 32, MAX_CLUSTER = 16;

template <class T, int W, bool BACK> struct SpanShape {
  static constexpr int CT = W == 1 ? 32 : 8;                                // columns of threads
  static constexpr int L = W == 1 ? 8 : (BACK && W == 8 ? 2 : 4);           // steps a thread
  static constexpr int COLS = CT * W, SPANS = SPAN_THREADS / CT, STEPS = SPANS * L;      // channels, spans and steps of a block
};

constexpr float CUT = -0.f;
__device__ __forceinline__ bool is_cut(float a) { return __float_as_uint(a) == 0x80000000u; }
__device__ __forceinline__ float2 joined(float2 first, float2 then) {       // as they are passed: A = -0 for a restart
  if (is_cut(then.x)) return then;
  return make_float2(is_cut(first.x) ? CUT : fmaf(then.x, first.x, 0.f), fmaf(then.x, first.y, then.y));
}
__device__ __forceinline__ float taken(float2 span, float h) { return is_cut(span.x) ? span.y : fmaf(span.x, h, span.y); }

template <class T, int W, bool SIGMOID, bool BACK>
__global__ void __launch_bounds__(SPAN_THREADS)
scan_spans_kernel(const __grid_constant__ Args a, int cluster) {
  typedef SpanShape<T, W, BACK> S;
  constexpr int CT = S::CT, L = S::L, COLS = S::COLS, STEPS = S::STEPS;
  __shared__ float2 of_warp[SPAN_WARPS][COLS];              // a warp's span; then that of all warps before it
  __shared__ float2 of_block[2][MAX_CLUSTER][COLS];         // every block's span, by the parity of the round
  __shared__ float at_warp[SPAN_WARPS][COLS];               // the state before a warp's first step

  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, rank = paac::cluster_rank();
  const int cl = lane % CT, part = lane / CT;
  const int per = a.c / W, tile = blockIdx.x / cluster;
  const int64_t col = (int64_t)tile * CT + cl;
  const bool active = col < (int64_t)a.n * per;
  const int seq = active ? (int)(col / per) : 0, c = active ? (int)(col - (int64_t)seq * per) * W : 0;
  const int within = rank * STEPS + (warp * (32 / CT) + part) * L;          // this thread's first step in a round

  paac::cluster_arrive();                                   // nobody stores into a block that has not begun
  paac::pdl_entry();
  // the thread that follows a channel's state through the rounds
  const int64_t channel = (int64_t)tile * COLS + threadIdx.x;
  const bool follows = threadIdx.x < COLS, holds = follows && channel < (int64_t)a.n * a.c;
  float state = holds && a.first != nullptr ? a.first[channel] : 0.f;

  Pack<T, W> gate[L], x[L], h[L], dh[L], next_gate[L], next_x[L];           // next_x: forward x, backward dh
  bool cut[L], next_cut[L];
  auto fetch = [&](int k0) {                                // what the spans are made of
#pragma unroll
    for (int u = 0; u < L; ++u) {
      const int k = k0 + u;
      if (active && k < a.t) {
        next_gate[u].load(at<T>(a.gate, k, seq, c));
        next_x[u].load(at<T>(BACK ? a.dh : a.x, k, seq, c));
        next_cut[u] = a.restart != nullptr && a.restart[k * a.restart_step + seq * a.restart_seq] != 0;
      } else {
        next_gate[u].zero(); next_x[u].zero();
        next_cut[u] = false;
      }
    }
  };
  fetch(within);
  paac::cluster_wait();

  int parity = 0;
  for (int64_t base = 0; base < a.t; base += (int64_t)cluster * STEPS, parity ^= 1) {
    const int k0 = base + within < a.t ? (int)base + within : a.t;          // (the sum may pass 32 bits)
    float fa[BACK ? 1 : L][W], fb[BACK ? 1 : L][W];         // forward: the steps themselves
    float A[W], B[W];
    bool D = false;
#pragma unroll
    for (int j = 0; j < W; ++j) { A[j] = 1.f; B[j] = 0.f; }
#pragma unroll
    for (int u = 0; u < L; ++u) {
      gate[u] = next_gate[u]; cut[u] = next_cut[u];
      if (BACK) dh[u] = next_x[u]; else x[u] = next_x[u];
      if (BACK && active && k0 + u < a.t) {                 // not needed before the state is known
        if (SIGMOID) x[u].load(at<T>(a.x, k0 + u, seq, c));
        if (k0 + u + 1 < a.t) h[u].load(at<T>(a.h, k0 + u + 1, seq, c));
      }
      const bool there = k0 + u < a.t;
      float g[W], v[W];
      gate[u].widen(g);
      (BACK ? dh[u] : x[u]).widen(v);
#pragma unroll
      for (int j = 0; j < W; ++j) {
        float z = g[j], rest = 1.f;
        if (SIGMOID) sigmoid<T>(g[j], z, rest);
        float b = BACK ? z * v[j] : rest * v[j];
        if (BACK && cut[u]) b = 0.f;
        if (!there) { z = 1.f; b = 0.f; }
        if (!BACK) { fa[u][j] = z; fb[u][j] = b; }
        B[j] = cut[u] ? b : fmaf(z, B[j], b);
        A[j] = fmaf(z, A[j], 0.f);
      }
      D = D || cut[u];
    }
    // spans of the warp, up to and with this thread's
#pragma unroll
    for (int d = 1; d < 32 / CT; d *= 2) {
      const bool before = part >= d, DD = __shfl_up_sync(0xffffffffu, (int)D, d * CT) != 0;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float AA = __shfl_up_sync(0xffffffffu, A[j], d * CT), BB = __shfl_up_sync(0xffffffffu, B[j], d * CT);
        if (before) {
          B[j] = D ? B[j] : fmaf(A[j], BB, B[j]);
          A[j] = fmaf(A[j], AA, 0.f);
        }
      }
      D = D || (before && DD);
    }
    if (part == 32 / CT - 1) {
#pragma unroll
      for (int j = 0; j < W; ++j) of_warp[warp][cl * W + j] = make_float2(D ? CUT : A[j], B[j]);
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
    {
      const int64_t ahead = base + (int64_t)cluster * STEPS + within;
      fetch(ahead < a.t ? (int)ahead : a.t);
    }
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
    float hs[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      hs[j] = at_warp[warp][cl * W + j];
      hs[j] = D ? B[j] : fmaf(A[j], hs[j], B[j]);
    }
#pragma unroll
    for (int u = 0; u < L; ++u) {
      const int k = k0 + u;
      if (!active || k >= a.t) break;
      Pack<T, W> p;
      if constexpr (!BACK) {
#pragma unroll
        for (int j = 0; j < W; ++j) hs[j] = cut[u] ? fb[u][j] : fmaf(fa[u][j], hs[j], fb[u][j]);
        p.round(hs);
        p.store(to<T>(a.out, k, seq, c));
      } else {
        float g[W], xv[W], before[W], dhv[W], dgate[W], dx[W];
        gate[u].widen(g);
        dh[u].widen(dhv);
        if (SIGMOID) x[u].widen(xv);
        if (k + 1 < a.t) {
          h[u].widen(before);
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j) before[j] = a.h0 != nullptr ? a.h0[(int64_t)seq * a.c + c + j] : 0.f;
        }
        step_back<T, W, SIGMOID>(g, xv, before, dhv, cut[u], hs, dgate, dx);
        if (a.dgate.data != nullptr) { p.round(dgate); p.store(to<T>(a.dgate, k, seq, c)); }
        if (a.out.data != nullptr) { p.round(dx); p.store(to<T>(a.out, k, seq, c)); }
      }
    }
  }
  if (rank == 0 && holds && a.last != nullptr) a.last[channel] = state;
}

// Blocks that are resident at once, two on a multiprocessor; clusters that do not fit in one go would wait for the others.
constexpr int SPAN_BLOCKS = 148 * 2;

template <class T, int W, bool SIGMOID, bool BACK> cudaError_t launch(const Args& a, cudaStream_t s) {
  typedef SpanShape<T, W, BACK> S;
  const int64_t columns = (int64_t)a.n * (a.c / W);
  if (a.t < 16 || columns >= 148 * 512)
    return paac::launch_overlapped_on(s, scan_columns_kernel<T, W, SIGMOID, BACK>, dim3((unsigned)((columns + COLUMN_THREADS - 1) / COLUMN_THREADS)),
                                      dim3(COLUMN_THREADS), 0, a);
  const int64_t tiles = (columns + S::CT - 1) / S::CT;
  int cluster = 1;
  while (cluster < MAX_CLUSTER && cluster * 2 * tiles <= SPAN_BLOCKS && cluster * S::STEPS < a.t) cluster *= 2;
  // a function's attributes belong to the current device, and this entry point works on any
  static paac::PerDevice<bool> ready;
  int device = -1;
  const bool ok = cudaGetDevice(&device) == cudaSuccess && ready.get(device, [](bool&) {
    return cudaFuncSetAttribute(scan_spans_kernel<T, W, SIGMOID, BACK>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
  }) != nullptr;
  if (!ok) return cudaErrorUnknown;
  return paac::launch_clusters_on(s, scan_spans_kernel<T, W, SIGMOID, BACK>, dim3((unsigned)(tiles * cluster)), dim3(SPAN_THREADS), cluster, a, cluster);
}
template <class T, bool BACK> cudaError_t launch_type(const Args& a, bool wide, bool sig, cudaStream_t s) {
  constexpr int W = 16 / sizeof(T);
  if (wide) return sig ? launch<T, W, true, BACK>(a, s) : launch<T, W, false, BACK>(a, s);
  return sig ? launch<T, 1, true, BACK>(a, s) : launch<T, 1, false, BACK>(a, s);
}
cudaError_t dispatch(const Args& a, const paac_scan& s, bool back, bool wide, cudaStream_t st) {
  const bool sig = s.kind == PAAC_SCAN_SIGMOID;
  if (s.type == PAAC_BF16) return back ? launch_type<bf16, true>(a, wide, sig, st) : launch_type<bf16, false>(a, wide, sig, st);
  return back ? launch_type<float, true>(a, wide, sig, st) : launch_type<float, false>(a, wide, sig, st);
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
  static constexpr int MOST = 10;
  const paac_scan& s;
  bool ok = true, wide = true;
  paac::RowSet kept[MOST] = {none(), none(), none(), none(), none(), none(), none(), none(), none(), none()};
  bool written[MOST] = {};
  int count = 0;
  static paac::RowSet none() { return paac::array_set(nullptr, 1); }
  explicit Check(const paac_scan& s_) : s(s_) {
    if (s.restart == nullptr) return;
    const paac::RowSet flags(paac_rows{const_cast<uint8_t*>(s.restart), s.restart_n, s.restart_t}, s.n, s.t, 1, 1);
    ok = flags.sane();
    if (ok) keep(flags, false);
  }
  void keep(const paac::RowSet& r, bool out) {
    for (int i = 0; i < count && ok; ++i)
      if ((out && !r.apart_from(kept[i])) || (written[i] && !kept[i].apart_from(r))) ok = false;
    kept[count] = r;
    written[count++] = out;
  }
  void rows(const paac_rows& r, bool out, bool needed) {
    if (r.data == nullptr) { ok = ok && !needed; return; }
    const paac::RowSet set(r, s.n, s.t, s.c, size_of(s));
    if (!set.sane() || !set.aligned() || (out && !set.rows_apart())) { ok = false; return; }
    wide = wide && set.multiples_of(16);
    keep(set, out);
  }
  // float [n][c]
  void state(const float* p, bool out) {
    if (p == nullptr) return;
    if ((uintptr_t)p & 3u) { ok = false; return; }
    wide = wide && ((uintptr_t)p & 15u) == 0;
    keep(paac::array_set(p, (int64_t)s.n * s.c * 4), out);
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
  if (!check.ok) return PAAC_ERR_ARG;
  const bool end = s->reverse != 0;
  Args a = common_args(*s, end);
  a.gate = walked(gate, *s, end); a.x = walked(x, *s, end); a.out = walked(h, *s, end);
  a.first = h0; a.last = h_last;
  return paac::launch_status(dispatch(a, *s, false, check.wide, static_cast<cudaStream_t>(stream)));
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
  if (!check.ok) return PAAC_ERR_ARG;
  const bool end = s->reverse == 0;
  Args a = common_args(*s, end);
  a.gate = walked(gate, *s, end); a.x = walked(x, *s, end); a.h = walked(h, *s, end); a.dh = walked(dh, *s, end);
  a.dgate = walked(dgate, *s, end); a.out = walked(dx, *s, end);
  a.h0 = h0; a.first = dh_last; a.last = dh0;
  return paac::launch_status(dispatch(a, *s, true, check.wide, static_cast<cudaStream_t>(stream)));
}
