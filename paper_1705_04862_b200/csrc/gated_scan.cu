// A gated linear recurrence over the steps of many sequences, and its gradient (paac_gated_scan, paac_gated_scan_backward).
//
// Every channel is a chain of its own, h_t = a_t h_{t-1} + b_t.  Backward, what step t passes on to the one before it is
// r_t = a_t (dh_t + r_{t+1}): the same chain in the state r, with the coefficients a_t and a_t dh_t, run the other way.
// A step that restarts takes nothing of the state: the state is left out there, not multiplied by 0.
//
// What bounds it: memory (three arrays forward, five or six backward, a few operations for each element), latency for few columns.
#include "common.cuh"
#include "pack.cuh"
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

template <class T, int W, bool SIGMOID, bool BACK> cudaError_t launch(const Args& a, cudaStream_t s) {
  const int64_t columns = (int64_t)a.n * (a.c / W);
  return paac::launch_overlapped_on(s, scan_columns_kernel<T, W, SIGMOID, BACK>, dim3((unsigned)((columns + COLUMN_THREADS - 1) / COLUMN_THREADS)),
                                    dim3(COLUMN_THREADS), 0, a);
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
  return s != nullptr && s->t >= 1 && s->n >= 1 && s->c >= 1 && (int64_t)s->n * s->c < ((int64_t)1 << 31) && (s->type == PAAC_FP32 || s->type == PAAC_BF16) &&
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
