// A short causal convolution of every channel by itself over the steps of many sequences, and its gradient (paac_causal_conv,
// paac_causal_conv_backward).
//
// v_t = bias + sum_k w_k x_{t-K+1+k}, y_t = act(v_t).  A thread walks a part of the steps of W neighbouring channels with the K - 1 inputs
// before the present one in registers, so every input is loaded once but for the K - 1 in front of a part.  A restart makes those 0.
// Backward it walks the same way, works v_t out again, dv_t = dy_t act'(v_t), and hands dv_t w_k to the K inputs of the step: the
// gradient of an input is complete K - 1 steps later.  So a part walks K - 1 steps beyond its end, whose shares it needs, and what
// is left of inputs before its begin belongs to the part before.  Sums over steps (dw, dbias) are kept by the thread, added up in a block, and a
// second kernel adds up the blocks' sums in a fixed order.
//
// What bounds it: the latency of loads with 20 warps a multiprocessor forward (96 registers) and 16 backward (128), beside memory and issue slots, of which
// neither is full.  Accesses of four channels: eight take so many registers for weights and inputs that fewer threads are resident (71 us instead of 42).
// Measured in a graph, SiLU, inputs in turn that L2 does not hold together: 8192 steps of 2 sequences with 2048 channels in bf16 33 us (134 MB at 4.0 TB/s; issue
// slots 58 %; without an activation 30), in float 58 (269 MB at 4.7 TB/s); the gradient of 2048 steps of 8 with 1024 in bf16 39 us (101 MB at 2.6 TB/s), in float 64 (201 MB
// at 3.2); a step of 32 with 1024 2.8; that call through the binding 8.9.
#include "sequence.cuh"

namespace {
using paac::bf16;
using paac::Pack;
using paac::StepRows;

struct Args {
  StepRows x, y, dy, dx;
  paac::StepFlags restart;
  const float *weight, *bias;
  const void *before, *dafter;
  void *after, *dbefore;
  float* partial;                      // backward: [row][c][K + 1] sums over a block's steps: dw, then dbias
  int t, n, c;
  int part;                            // steps of a thread
};

// Steps whose loads are under way.
constexpr int THREADS = 128, AHEAD = 8;
constexpr int BACK_THREADS = 128, BACK_AHEAD = 4;

template <int W, int K> __device__ __forceinline__ void load_weights(const Args& a, int c, float (&w)[K][W], float (&bias)[W]) {
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int k = 0; k < K; ++k) w[k][j] = a.weight[(int64_t)(c + j) * K + k];
#pragma unroll
  for (int j = 0; j < W; ++j) bias[j] = a.bias != nullptr ? a.bias[c + j] : 0.f;
}

// the K - 1 inputs before the present step, oldest first
template <class T, int W, int K> struct History {
  float v[K - 1][W];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int k = 0; k < K - 1; ++k)
#pragma unroll
      for (int j = 0; j < W; ++j) v[k][j] = 0.f;
  }
  __device__ __forceinline__ void push(const float (&x)[W]) {
#pragma unroll
    for (int k = 0; k + 1 < K - 1; ++k)
#pragma unroll
      for (int j = 0; j < W; ++j) v[k][j] = v[k + 1][j];
#pragma unroll
    for (int j = 0; j < W; ++j) v[K - 2][j] = x[j];
  }
  // [K - 1][c] of a sequence
  __device__ __forceinline__ void load(const T* p, int c) {
#pragma unroll
    for (int k = 0; k < K - 1; ++k) { Pack<T, W> q; q.load(p + (int64_t)k * c); q.widen(v[k]); }
  }
  __device__ __forceinline__ void store(T* p, int c) const {
#pragma unroll
    for (int k = 0; k < K - 1; ++k) { Pack<T, W> q; q.round(v[k]); q.store(p + (int64_t)k * c); }
  }
};

template <class T, int W, int K> __device__ __forceinline__ void argument(const float (&w)[K][W], const float (&bias)[W], const History<T, W, K>& h, const float (&x)[W], float (&v)[W]) {
#pragma unroll
  for (int j = 0; j < W; ++j) v[j] = bias[j];
#pragma unroll
  for (int k = 0; k < K - 1; ++k) paac::fma_all(v, w[k], h.v[k]);
  paac::fma_all(v, w[K - 1], x);
}
template <class T, int W, int KIND> __device__ __forceinline__ void activate(const float (&v)[W], float (&y)[W]) {
#pragma unroll
  for (int j = 0; j < W; ++j) {
    if (KIND == PAAC_ACT_SILU) y[j] = paac::silu<T>(v[j]);
    else if (KIND == PAAC_ACT_RELU) asm("max.NaN.f32 %0, %1, %2;" : "=f"(y[j]) : "f"(v[j]), "f"(0.f));
    else y[j] = v[j];
  }
}

// The state in front of step k0, and how many of the inputs in it belong to the same episode as that step (restarts at k0 itself not counted).
template <class T, int W, int K> __device__ __forceinline__ void enter(const Args& a, int k0, int seq, int c, History<T, W, K>& h, int& live) {
  h.clear();
  live = K - 1;
  int k = k0 - (K - 1);
  if (k < 0) {
    if (a.before != nullptr) h.load((const T*)a.before + (int64_t)seq * (K - 1) * a.c + c, a.c);
    k = 0;
  }
  for (; k < k0; ++k) {
    if (a.restart.data != nullptr && a.restart.data[k * a.restart.step + seq * a.restart.seq] != 0) { h.clear(); live = 0; }
    Pack<T, W> p;
    float x[W];
    p.load(paac::row_at<T>(a.x, k, seq) + c);
    p.widen(x);
    h.push(x);
    live = live < K - 1 ? live + 1 : live;
  }
}

// The loads of COUNT steps are under way: a step that has been worked on makes room for the one COUNT steps on.  work(place of the step, its number) for
// every step from the first to the last, load(place, number) in order.
template <int COUNT, class Load, class Work> __device__ __forceinline__ void walk(int first, int end, Load load, Work work) {
#pragma unroll
  for (int u = 0; u < COUNT; ++u)
    if (first + u < end) load(u, first + u);
  int k = first;
  for (; end - k >= 2 * COUNT; k += COUNT) {
#pragma unroll
    for (int u = 0; u < COUNT; ++u) {
      work(u, k + u);
      load(u, k + u + COUNT);
    }
  }
  for (; k < end; k += COUNT) {
#pragma unroll
    for (int u = 0; u < COUNT; ++u)
      if (k + u < end) {
        work(u, k + u);
        if (k + u + COUNT < end) load(u, k + u + COUNT);
      }
  }
}

template <class T, int W, int K, int KIND>
__global__ void __launch_bounds__(THREADS)
conv_kernel(const __grid_constant__ Args a) {
  paac::pdl_entry();
  const uint32_t per = a.c / W, col = blockIdx.x * THREADS + threadIdx.x;
  if (col >= (uint32_t)a.n * per) return;
  const int seq = (int)(col / per), c = (int)(col - seq * per) * W;
  const int k0 = blockIdx.y * a.part, end = a.t - k0 < a.part ? a.t : k0 + a.part;
  float w[K][W], bias[W];
  History<T, W, K> h;
  int live;
  load_weights<W, K>(a, c, w, bias);
  enter<T, W, K>(a, k0, seq, c, h, live);
  if (a.after != nullptr && blockIdx.y == 0) {
    // the state behind the last step, by the threads that read the one before the first, which it may replace
    History<T, W, K> last = h;
    for (int k = a.t > K - 1 ? a.t - (K - 1) : 0; k < a.t; ++k) {
      if (a.restart.data != nullptr && a.restart.data[k * a.restart.step + seq * a.restart.seq] != 0) last.clear();
      Pack<T, W> p;
      float x[W];
      p.load(paac::row_at<T>(a.x, k, seq) + c);
      p.widen(x);
      last.push(x);
    }
    last.store((T*)a.after + (int64_t)seq * (K - 1) * a.c + c, a.c);
  }
  const T* from = paac::row_at<T>(a.x, k0, seq) + c;
  const uint8_t* flag = a.restart.data != nullptr ? a.restart.data + k0 * a.restart.step + seq * a.restart.seq : nullptr;
  T* to = paac::row_to<T>(a.y, k0, seq) + c;
  struct { Pack<T, W> x; uint32_t cut; } s[AHEAD];
  walk<AHEAD>(k0, end, [&](int u, int) {
    s[u].x.load(from);
    from += a.x.step;
    s[u].cut = 0;
    if (flag != nullptr) { s[u].cut = *flag; flag += a.restart.step; }
  }, [&](int u, int) {
    float x[W], v[W], y[W];
    s[u].x.widen(x);
    if (s[u].cut != 0) h.clear();
    argument<T, W, K>(w, bias, h, x, v);
    activate<T, W, KIND>(v, y);
    h.push(x);
    Pack<T, W> p;
    p.round(y);
    p.store(to);
    to += a.y.step;
  });
}

// dL/dv from dL/dy
template <class T, int W, int KIND> __device__ __forceinline__ void slope(const float (&v)[W], float (&d)[W]) {
#pragma unroll
  for (int j = 0; j < W; ++j) {
    if (KIND == PAAC_ACT_SILU) {
      float s, rest;
      paac::logistic<T>(v[j], s, rest);
      d[j] *= fmaf(v[j] * s, rest, s);
    } else if (KIND == PAAC_ACT_RELU) {
      d[j] = v[j] > 0.f ? d[j] : (v[j] == v[j] ? 0.f : v[j]);
    }
  }
}

// A block: CT columns of threads, side by side in the channels, by BACK_THREADS / CT parts of the steps.  `ct` a power of two up to 32.
template <class T, int W, int K, int KIND>
__global__ void __launch_bounds__(BACK_THREADS, 4)
conv_back_kernel(const __grid_constant__ Args a, int ct, int tiles) {
  paac::pdl_entry();
  constexpr int SUMS = W * (K + 1);
  __shared__ float of_warp[BACK_THREADS / 32][32][SUMS + 1];
  const int per = a.c / W, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row = blockIdx.x / tiles, tile = blockIdx.x - row * tiles;
  const int col = tile * ct + threadIdx.x % ct, c = col * W;
  const int parts = (a.t + a.part - 1) / a.part;
  const int64_t which = (int64_t)row * (BACK_THREADS / ct) + threadIdx.x / ct;
  const bool active = col < per && which < (int64_t)parts * a.n;
  float dw[K][W], dbias[W];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    dbias[j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) dw[k][j] = 0.f;
  }
  if (active) {
    const int seq = (int)(which / parts), k0 = (int)(which - (int64_t)seq * parts) * a.part;
    const int end = a.t - k0 < a.part ? a.t : k0 + a.part, beyond = a.t - end < K - 1 ? a.t : end + K - 1;
    float w[K][W], bias[W], due[K - 1][W];      // due: the gradients of the inputs in h, as far as they have come
    History<T, W, K> h;
    int live;
    load_weights<W, K>(a, c, w, bias);
    enter<T, W, K>(a, k0, seq, c, h, live);
#pragma unroll
    for (int k = 0; k < K - 1; ++k)
#pragma unroll
      for (int j = 0; j < W; ++j) due[k][j] = 0.f;
    // what has come of the oldest input when it leaves
    T* dx_at = paac::row_to<T>(a.dx, k0, seq) + c;
    auto leave = [&](int k, const float (&v)[W]) {
      Pack<T, W> p;
      p.round(v);
      if (k >= k0 && k < end) {
        if (a.dx.data != nullptr) p.store(dx_at);
        dx_at += a.dx.step;
      } else if (k < 0 && a.dbefore != nullptr) {
        p.store((T*)a.dbefore + ((int64_t)seq * (K - 1) + k + K - 1) * a.c + c);
      }
    };
    const T *from = paac::row_at<T>(a.x, k0, seq) + c, *dfrom = paac::row_at<T>(a.dy, k0, seq) + c;
    const uint8_t* flag = a.restart.data != nullptr ? a.restart.data + k0 * a.restart.step + seq * a.restart.seq : nullptr;
    struct { Pack<T, W> x, dy; uint32_t cut; } s[BACK_AHEAD];
    walk<BACK_AHEAD>(k0, beyond, [&](int u, int) {
      s[u].x.load(from);
      s[u].dy.load(dfrom);
      from += a.x.step;
      dfrom += a.dy.step;
      s[u].cut = 0;
      if (flag != nullptr) { s[u].cut = *flag; flag += a.restart.step; }
    }, [&](int u, int k) {
      float x[W], v[W], d[W];
      s[u].x.widen(x);
      s[u].dy.widen(d);
      if (s[u].cut != 0) { h.clear(); live = 0; }
      argument<T, W, K>(w, bias, h, x, v);
      slope<T, W, KIND>(v, d);
      if (k < end) {
        paac::add_all(dbias, d);
#pragma unroll
        for (int q = 0; q < K - 1; ++q) paac::fma_all(dw[q], d, h.v[q]);
        paac::fma_all(dw[K - 1], d, x);
      }
      if (live == K - 1) {
#pragma unroll
        for (int q = 0; q < K - 1; ++q) paac::fma_all(due[q], w[q], d);
      } else {
#pragma unroll
        for (int q = 0; q < K - 1; ++q)
          if (K - 1 - q <= live) paac::fma_all(due[q], w[q], d);
        ++live;
      }
      leave(k - (K - 1), due[0]);
#pragma unroll
      for (int q = 0; q + 1 < K - 1; ++q)
#pragma unroll
        for (int j = 0; j < W; ++j) due[q][j] = due[q + 1][j];
#pragma unroll
      for (int j = 0; j < W; ++j) due[K - 2][j] = w[K - 1][j] * d[j];
      h.push(x);
    });
    if (beyond == a.t) {
      // behind the last step: what the following call took of these inputs (a part that ends before the last step leaves those to the last part,
      // but for the ones that are its own)
      if (a.dafter != nullptr) {
        History<T, W, K> more;
        more.load((const T*)a.dafter + (int64_t)seq * (K - 1) * a.c + c, a.c);
#pragma unroll
        for (int q = 0; q < K - 1; ++q)
          if (K - 1 - q <= live) paac::add_all(due[q], more.v[q]);
      }
#pragma unroll
      for (int q = 0; q < K - 1; ++q) leave(a.t - (K - 1) + q, due[q]);
    }
  }
  if (a.partial == nullptr) return;
  // sums of the threads of a column: in the warp, then over the warps
  float all[SUMS];
#pragma unroll
  for (int j = 0; j < W; ++j) {
#pragma unroll
    for (int k = 0; k < K; ++k) all[j * (K + 1) + k] = dw[k][j];
    all[j * (K + 1) + K] = dbias[j];
  }
  for (int d = 16; d >= ct; d >>= 1)
#pragma unroll
    for (int i = 0; i < SUMS; ++i) all[i] += __shfl_xor_sync(0xffffffffu, all[i], d);
  if (lane < ct)
#pragma unroll
    for (int i = 0; i < SUMS; ++i) of_warp[warp][lane][i] = all[i];
  __syncthreads();
  for (int i = threadIdx.x; i < ct * SUMS; i += BACK_THREADS) {
    const int l = i / SUMS, q = i - l * SUMS;
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < BACK_THREADS / 32; ++u) sum += of_warp[u][l][q];
    const int64_t at = ((int64_t)tile * ct + l) * SUMS + q;
    if (at < (int64_t)a.c * (K + 1)) a.partial[(int64_t)row * a.c * (K + 1) + at] = sum;
  }
}

// The blocks' sums, [rows][c][K + 1], added up in 64 bits: 32 sums a block, every eighth row by each of its warps.
__global__ void __launch_bounds__(256)
conv_sums_kernel(const float* partial, int rows, int c, int width, float* dweight, float* dbias) {
  paac::pdl_entry();
  const int64_t count = (int64_t)c * (width + 1), i = (int64_t)blockIdx.x * 32 + (threadIdx.x & 31);
  __shared__ double of_warp[8][32];
  double sum = 0.0;
  if (i < count)
    for (int r = threadIdx.x >> 5; r < rows; r += 8) sum += partial[r * count + i];
  of_warp[threadIdx.x >> 5][threadIdx.x & 31] = sum;
  __syncthreads();
  if (threadIdx.x < 32 && i < count) {
    sum = 0.0;
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += of_warp[u][threadIdx.x];
    const int64_t ch = i / (width + 1);
    const int k = (int)(i - ch * (width + 1));
    if (k < width) { if (dweight != nullptr) dweight[ch * width + k] = (float)sum; }
    else if (dbias != nullptr) dbias[ch] = (float)sum;
  }
}

// ---- the host's part -------------------------------------------------------------------------------------------------------------------

// Steps of a thread forward: what comes to some 640 threads a multiprocessor, as many as are resident with four taps in bf16 (in float 384 are, with two or three taps up to 1024), but so
// many that the inputs in front of a part weigh little.  Measured, 8192 steps of 2 x 2048 channels: the 89 of this rule, 744 blocks for 740 places, 33.6 us; 90 to 92, with which all are
// resident at once, 34.7 to 35.3, 16 to 80 40 to 50, 96 to 180 34.5 to 49.  In float this rule's 57.7, 150 (440 blocks for 444 places) 51.3, other ones 55 to 74.
int forward_part(const paac_conv& s, int64_t columns) {
  const int64_t steps = ((int64_t)s.t * columns + 148 * 640 - 1) / (148 * 640);
  return (int)(steps < 16 ? 16 : steps > 4096 ? 4096 : steps);
}
int lanes_of(int64_t per) {
  int ct = 1;
  while (ct < 32 && ct < per) ct *= 2;
  return ct;
}
// Backward the same for accesses of four channels, whatever they are: what the scratch goes by.
int back_part(const paac_conv& s) {
  const int64_t steps = ((int64_t)s.t * s.n * s.c / 4 + 148 * 512 - 1) / (148 * 512);
  return (int)(steps < 16 ? 16 : steps > 4096 ? 4096 : steps);
}
int64_t back_rows(const paac_conv& s, int ct) {
  const int part = back_part(s), each = BACK_THREADS / ct;
  const int64_t parts = (int64_t)((s.t + (int64_t)part - 1) / part) * s.n;
  return (parts + each - 1) / each;
}

bool shape_ok(const paac_conv* s) {
  return s != nullptr && s->t >= 1 && s->t <= (1 << 30) && s->n >= 1 && s->c >= 1 && (int64_t)s->n * s->c < ((int64_t)1 << 31) && s->width >= 2 && s->width <= 4 &&
         (s->type == PAAC_FP32 || s->type == PAAC_BF16) && s->activation >= PAAC_ACT_NONE && s->activation <= PAAC_ACT_SILU;
}
int size_of(const paac_conv& s) { return s.type == PAAC_BF16 ? 2 : 4; }

template <class T, int W, int K, int KIND> cudaError_t forward(Args a, const paac_conv& s, cudaStream_t st) {
  const int64_t columns = (int64_t)a.n * (a.c / W);
  a.part = forward_part(s, columns);
  const int64_t parts = (a.t + (int64_t)a.part - 1) / a.part;
  if (parts > 65535) a.part = (int)((a.t + (int64_t)65534) / 65535);
  return paac::launch_overlapped_on(st, conv_kernel<T, W, K, KIND>, dim3((unsigned)((columns + THREADS - 1) / THREADS), (unsigned)((a.t + (int64_t)a.part - 1) / a.part)),
                                    dim3(THREADS), 0, a);
}
template <class T, int W, int K, int KIND> cudaError_t backward(Args a, const paac_conv& s, float* dweight, float* dbias, cudaStream_t st) {
  const int per = a.c / W, ct = lanes_of(per), tiles = (per + ct - 1) / ct;
  a.part = back_part(s);
  const int64_t rows = back_rows(s, ct);
  const cudaError_t e = paac::launch_overlapped_on(st, conv_back_kernel<T, W, K, KIND>, dim3((unsigned)(rows * tiles)), dim3(BACK_THREADS), 0, a, ct, tiles);
  if (e != cudaSuccess || a.partial == nullptr) return e;
  return paac::launch_overlapped_on(st, conv_sums_kernel, dim3((unsigned)(((int64_t)a.c * (K + 1) + 31) / 32)), dim3(256), 0, (const float*)a.partial, (int)rows, a.c, K,
                                    dweight, dbias);
}
template <int KIND, class F> cudaError_t by_width(int width, F f) {
  typedef std::integral_constant<int, KIND> Kind;
  if (width == 4) return f(std::integral_constant<int, 4>(), Kind());
  if (width == 3) return f(std::integral_constant<int, 3>(), Kind());
  return f(std::integral_constant<int, 2>(), Kind());
}
// f(width, activation) with both as constants
template <class F> cudaError_t by_form(const paac_conv& s, F f) {
  if (s.activation == PAAC_ACT_SILU) return by_width<PAAC_ACT_SILU>(s.width, f);
  return s.activation == PAAC_ACT_RELU ? by_width<PAAC_ACT_RELU>(s.width, f) : by_width<PAAC_ACT_NONE>(s.width, f);
}

}  // namespace

extern "C" int paac_causal_conv(const paac_conv* s, const paac_conv_out* out, void* stream) {
  if (!shape_ok(s) || out == nullptr) return PAAC_ERR_ARG;
  const paac_rows x = s->x, y = out->y;
  const float *weight = s->weight, *bias = s->bias;
  const void* before = s->before;
  void* after = out->after;
  paac::StepCheck check(s->t, s->n, size_of(*s), s->restart, s->restart_n, s->restart_t);
  const int64_t reach = s->width - 1;
  check.steps(x, s->c, false, true);
  check.steps(y, s->c, true, true);
  check.floats(weight, (int64_t)s->c * s->width, false, true);
  check.floats(bias, s->c, false);
  if (before != after) check.rows(paac_rows{const_cast<void*>(before), reach * s->c, s->c}, s->n, reach, s->c, false, false);
  check.rows(paac_rows{after, reach * s->c, s->c}, s->n, reach, s->c, true, false);
  if (!check.fit()) return PAAC_ERR_ARG;
  Args a{};
  a.x = paac::step_rows(x, s->t, s->n); a.y = paac::step_rows(y, s->t, s->n);
  a.restart = {s->restart, s->t > 1 ? s->restart_t : 0, s->n > 1 ? s->restart_n : 0};
  a.weight = weight; a.bias = bias; a.before = before; a.after = after;
  a.t = s->t; a.n = s->n; a.c = s->c;
  const int most = check.align / size_of(*s), W = most > 4 ? 4 : most;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return paac::launch_status(by_form(*s, [&](auto k, auto kind) {
    constexpr int K = decltype(k)::value, ACT = decltype(kind)::value;
    if (s->type == PAAC_BF16)
      return W == 4 ? forward<bf16, 4, K, ACT>(a, *s, st) : W == 2 ? forward<bf16, 2, K, ACT>(a, *s, st) : forward<bf16, 1, K, ACT>(a, *s, st);
    return W == 4 ? forward<float, 4, K, ACT>(a, *s, st) : W == 2 ? forward<float, 2, K, ACT>(a, *s, st) : forward<float, 1, K, ACT>(a, *s, st);
  }));
}

extern "C" size_t paac_causal_conv_workspace_bytes(const paac_conv* s) {
  if (!shape_ok(s)) return 0;
  int64_t rows = 0;
  for (int W = 1; W <= 4; W *= 2)
    if (s->c % W == 0) { const int64_t r = back_rows(*s, lanes_of(s->c / W)); rows = r > rows ? r : rows; }
  return (size_t)rows * s->c * (s->width + 1) * 4;
}

extern "C" int paac_causal_conv_backward(const paac_conv* s, const paac_conv_grads* g, void* stream) {
  if (!shape_ok(s) || g == nullptr) return PAAC_ERR_ARG;
  const paac_rows x = s->x, dy = g->dy, dx = g->dx;
  const float *weight = s->weight, *bias = s->bias;
  const void *before = s->before, *dafter = g->dafter;
  float *dweight = g->dweight, *dbias = g->dbias;
  void *dbefore = g->dbefore, *workspace = g->workspace;
  if (dx.data == nullptr && dweight == nullptr && dbias == nullptr && dbefore == nullptr) return PAAC_ERR_ARG;
  paac::StepCheck check(s->t, s->n, size_of(*s), s->restart, s->restart_n, s->restart_t);
  const int64_t reach = s->width - 1;
  check.steps(x, s->c, false, true);
  check.steps(dy, s->c, false, true);
  check.steps(dx, s->c, true, false);
  check.floats(weight, (int64_t)s->c * s->width, false, true);
  check.floats(bias, s->c, false);
  check.rows(paac_rows{const_cast<void*>(before), reach * s->c, s->c}, s->n, reach, s->c, false, false);
  check.rows(paac_rows{const_cast<void*>(dafter), reach * s->c, s->c}, s->n, reach, s->c, false, false);
  check.rows(paac_rows{dbefore, reach * s->c, s->c}, s->n, reach, s->c, true, false);
  check.floats(dweight, (int64_t)s->c * s->width, true);
  check.floats(dbias, s->c, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  const size_t need = paac_causal_conv_workspace_bytes(s);
  if (workspace == nullptr || ((uintptr_t)workspace & 15u) != 0 || g->workspace_bytes < need) return PAAC_ERR_WORKSPACE;
  check.arrays.keep(workspace, (int64_t)need, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  Args a{};
  a.x = paac::step_rows(x, s->t, s->n); a.dy = paac::step_rows(dy, s->t, s->n); a.dx = paac::step_rows(dx, s->t, s->n);
  a.restart = {s->restart, s->t > 1 ? s->restart_t : 0, s->n > 1 ? s->restart_n : 0};
  a.weight = weight; a.bias = bias; a.before = before; a.dafter = dafter; a.dbefore = dbefore;
  a.partial = dweight != nullptr || dbias != nullptr ? (float*)workspace : nullptr;
  a.t = s->t; a.n = s->n; a.c = s->c;
  const int most = check.align / size_of(*s), W = most > 4 ? 4 : most;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  return paac::launch_status(by_form(*s, [&](auto k, auto kind) {
    constexpr int K = decltype(k)::value, ACT = decltype(kind)::value;
    if (s->type == PAAC_BF16)
      return W == 4 ? backward<bf16, 4, K, ACT>(a, *s, dweight, dbias, st) : W == 2 ? backward<bf16, 2, K, ACT>(a, *s, dweight, dbias, st) : backward<bf16, 1, K, ACT>(a, *s, dweight, dbias, st);
    return W == 4 ? backward<float, 4, K, ACT>(a, *s, dweight, dbias, st) : W == 2 ? backward<float, 2, K, ACT>(a, *s, dweight, dbias, st) : backward<float, 1, K, ACT>(a, *s, dweight, dbias, st);
  }));
}
