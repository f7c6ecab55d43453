// Group normalisation with scale, shift and activation, channels last, and its gradient (paac_group_norm, paac_group_norm_backward).
//
//   y = act(v), v = gamma (x - mean) rstd + beta;   mean and rstd over a run of channels and all pixels of a sample
//   dv = dy act'(v);  dbeta = sum dv;  dgamma = sum dv xhat;  xhat = (x - mean) rstd
//   dx = rstd (gamma dv - S1 / m - xhat S2 / m),  S1 = sum gamma dv, S2 = sum gamma dv xhat over the group's m elements
//
// What bounds it: memory, two arrays forward and three backward, if a sample is read once.  Measured (the kernels back to back in a graph,
// inputs in turn that L2 does not hold together): 5120 samples of 400 pixels with 32 channels in bf16 with ReLU 50 us (262 MB at 5.2
// TB/s); backward 5120 of 81 with 64 43 us (160 MB at 3.7 TB/s: half of all issue slots, 25 instructions an element) and 37 of 7056
// with 48, float, SiLU 51 us (150 MB at 2.9 TB/s: a sample fills clusters of blocks, whose waits for one another are not covered);
// forward 66 of those 50 us (179 MB at 3.6 TB/s); 32 samples of 400 with 32 3.3 us (a call through the binding 10).
//
// A block works on a slice of channels, whole groups or a part of one large group, and a slab of pixels; a thread keeps to W neighbouring
// channels of it and goes down the rows, so that gamma, beta and the statistics stay in registers.  Means and sums of squared
// deviations are merged in pairs of parts (Chan, Golub and LeVeque's update), never taken as a difference of large sums.
#include <algorithm>

#include "cluster.cuh"
#include "pack.cuh"
#include "per_device.h"
#include "rows.h"

namespace {
using paac::bf16;
using paac::Pack;

constexpr int TB = 256, WARPS = TB / 32;
constexpr int GRID = 148 * 8;

// How samples are cut up.  parts == 1: a slice is `gps` whole groups; else a slice is one of the `parts` pieces of a group, `cap` channels each.
struct Geo {
  int n, pixels, c, groups, cg;
  int gps, parts, cap, slices;
  int slab_rows, slabs;
};
struct Slice { int c0, width, g0, groups; };         // first channel, channels, first group, groups
__device__ __forceinline__ Slice slice_of(const Geo& q, int i) {
  if (q.parts == 1) {
    const int g0 = i * q.gps, gs = min(q.gps, q.groups - g0);
    return Slice{g0 * q.cg, gs * q.cg, g0, gs};
  }
  const int g = i / q.parts, p = i - g * q.parts;
  return Slice{g * q.cg + p * q.cap, min(q.cap, q.cg - p * q.cap), g, 1};
}

struct View { void* data; int64_t sample, pixel; };
template <class T> __device__ __forceinline__ T* at(const View& v, int64_t n, int64_t p, int c) { return (T*)v.data + n * v.sample + p * v.pixel + c; }

struct Args {
  Geo q;
  View x, dy, out;                    // out: y or dx
  const float *gamma, *beta;
  const float *mean, *rstd;           // [n][groups]
  float *mean_out, *rstd_out;
  int activation;
  float eps;
};

// s = sigma(v) = 1 / (1 + e^-v); e^-v may become infinite, s is 0 then.  bf16 storage takes the faster exponential, whose argument is a
// rounded product with log2(e): off by up to (2 + 1.2 |v|) 2^-23 of its value.  The storage's rounding hides that in y and dx; dgamma
// and dbeta, floats, have it.
template <class T, int W> __device__ __forceinline__ void logistic_all(float (&s)[W], const float (&v)[W]) {
  float one[W], scale[W];
#pragma unroll
  for (int j = 0; j < W; ++j) { one[j] = 1.f; scale[j] = -1.442695041f; s[j] = v[j]; }
  if constexpr (sizeof(T) == 2) {
    paac::mul_all(s, scale);
#pragma unroll
    for (int j = 0; j < W; ++j) asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(s[j]) : "f"(s[j]));
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) s[j] = expf(-s[j]);
  }
  paac::add_all(s, one);
#pragma unroll
  for (int j = 0; j < W; ++j) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s[j]) : "f"(s[j]));
}
// v <- act(v)
template <class T, int W> __device__ __forceinline__ void act_all(float (&v)[W], int kind) {
  if (kind == PAAC_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = v[j] < 0.f ? 0.f : v[j];              // a NaN stays one
  } else if (kind == PAAC_ACT_SILU) {
    float s[W];
    logistic_all<T, W>(s, v);
    paac::mul_all(v, s);
  }
}
// d <- d act'(v)
template <class T, int W> __device__ __forceinline__ void slope_all(float (&d)[W], const float (&v)[W], int kind) {
  if (kind == PAAC_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < W; ++j) d[j] = v[j] > 0.f ? d[j] : 0.f;              // whatever comes in where it is off
  } else if (kind == PAAC_ACT_SILU) {                                        // s (1 + v (1 - s))
    float s[W], t[W], one[W], less[W];
    logistic_all<T, W>(s, v);
#pragma unroll
    for (int j = 0; j < W; ++j) { one[j] = 1.f; less[j] = -1.f; }
    paac::fma_all_to(t, s, less, one);
    paac::fma_all_to(t, t, v, one);
    paac::mul_all(d, s);
    paac::mul_all(d, t);
  }
}

// rows that row lane r of R takes of a slab
__device__ __forceinline__ int rows_of(int rows, int r, int R) { return rows > r ? (rows - r + R - 1) / R : 0; }

// Statistics of one of the block's groups from those of its threads: entry (r, q) of `mean` and `m2` (q < cols) stands for one
// channel of rows_of(rows, r, R) rows.  A warp takes a group; the result is in every lane.
struct Stats { float n, mean, m2; };
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ Stats merge_group(const float* mean, const float* m2, int R, int cols, int first, int width, int rows, int lane) {
  float s = 0.f, k = 0.f;
  for (int i = lane; i < R * width; i += 32) {
    const int r = i / width, q = first + i - r * width;
    const float cnt = (float)rows_of(rows, r, R);
    s = fmaf(cnt, mean[r * cols + q], s);
    k += cnt;
  }
  const float n = warp_sum(k), m = n > 0.f ? warp_sum(s) / n : 0.f;
  float d2 = 0.f;
  for (int i = lane; i < R * width; i += 32) {
    const int r = i / width, q = first + i - r * width;
    const float cnt = (float)rows_of(rows, r, R), d = mean[r * cols + q] - m;
    d2 += fmaf(cnt * d, d, m2[r * cols + q]);
  }
  return Stats{n, m, warp_sum(d2)};
}

// ---- samples that stay on chip: one read ---------------------------------------------------------------------------------------------------
//
// A block, or a cluster of up to MAX_CLUSTER blocks with neighbouring slabs of pixels, holds a slice of a sample in shared memory (of x,
// and of dy) between the read and the write: first the mean, then the squared deviations from it, then the result.  Every thread
// copies its own accesses there and reads no others, and copies those of its next sample into their places as it writes; what it
// has of dgamma and dbeta stays in registers until the end.  (In registers throughout, up to 13 accesses a thread: 50 us for the
// gradient of the update batch behind the second convolution, since 168 registers leave three small blocks to a multiprocessor.)
//
// Sums over a group: where accesses and groups are powers of two (ALIGNED) the lanes that share a group are joined by shuffles and every thread
// adds up what the warps have; else the threads' values go to shared memory and a warp adds up a group.  Blocks of a cluster hand one another
// their (mean, squared deviations), merged as parts, or sums.
enum Mode { ALIGNED, BY_ACCESS, BY_CHANNEL };       // sums of an access's channels, or (groups begin within accesses) of each
constexpr int MAX_CLUSTER = 16, MAX_GROUPS = 32, MAX_WIDTH = 512;           // groups and channels of a slice
constexpr int REGISTER_BLOCKS = 2;          // blocks of TB threads that the registers are cut for
// rows of the slab of block `rank`
__device__ __forceinline__ int slab_of(int pixels, int slab, int rank) { const int left = pixels - rank * slab; return left < 0 ? 0 : (left < slab ? left : slab); }


// What a thread knows of its place: slice, row lane r of R, access v of cv, and of the cluster.
template <int W> struct Place {
  Slice s;
  int cv, R, r, v, c, wide, rank, rows, cnt, warp, lane, warps;      // c: its first channel; wide: accesses of a group; cnt: its rows
  __device__ __forceinline__ Place(const Geo& q, int id, int slab, int rank_) : s(slice_of(q, id % q.slices)), rank(rank_) {
    cv = s.width / W; R = blockDim.x / cv; r = threadIdx.x / cv; v = threadIdx.x - r * cv; c = s.c0 + v * W; wide = q.cg / W;
    rows = slab_of(q.pixels, slab, rank);
    cnt = r < R ? rows_of(rows, r, R) : 0;
    warp = threadIdx.x >> 5; lane = threadIdx.x & 31; warps = blockDim.x >> 5;
  }
};

__device__ __forceinline__ float plus(float a, float b) { return a + b; }
__device__ __forceinline__ float2 plus(float2 a, float2 b) { return make_float2(a.x + b.x, a.y + b.y); }
__device__ __forceinline__ float from_lane(float v, int o) { return __shfl_xor_sync(0xffffffffu, v, o); }
__device__ __forceinline__ float2 from_lane(float2 v, int o) { return make_float2(from_lane(v.x, o), from_lane(v.y, o)); }

// Sums over groups of a value V of each thread (BY_CHANNEL: of each of its channels).
template <int W, Mode M, class V> struct GroupSum {
  static constexpr int NV = M == BY_CHANNEL ? W : 1, ENTRIES = M == ALIGNED ? 2 * TB : TB * NV;
  V entry[ENTRIES];                  // ALIGNED: two turns of [warp][lane]
  V total[MAX_GROUPS];
  // group[j]: of value[j], within the slice
  __device__ __forceinline__ void run(const Geo& q, const Place<W>& at, int turn, const int (&group)[NV], V (&value)[NV]) {
    if constexpr (M == ALIGNED) {
      V t = value[0];
#pragma unroll
      for (int o = 1; o < 32; o *= 2)
        if (o < at.wide || o >= at.cv) t = plus(t, from_lane(t, o));
      V* mine = entry + (turn & 1) * TB;
      mine[threadIdx.x] = t;
      __syncthreads();
      const int step = at.cv > 32 ? at.cv >> 5 : 1;                         // warps that have the same accesses
      int w = at.warp & (step - 1);
      t = mine[w * 32 + at.lane];
      for (w += step; w < at.warps; w += step) t = plus(t, mine[w * 32 + at.lane]);
      value[0] = t;
    } else {
      const int cols = at.cv * NV, each = M == BY_CHANNEL ? q.cg : at.wide;
      if (at.r < at.R) {
#pragma unroll
        for (int j = 0; j < NV; ++j) entry[at.r * cols + at.v * NV + j] = value[j];
      }
      __syncthreads();
      for (int g = at.warp; g < at.s.groups; g += at.warps) {
        V t{};
        for (int i = at.lane; i < at.R * each; i += 32) {
          const int row = i / each;
          t = plus(t, entry[row * cols + g * each + i - row * each]);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) t = plus(t, from_lane(t, o));
        if (at.lane == 0) total[g] = t;
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NV; ++j) value[j] = total[group[j]];
    }
  }
};

// A thread's accesses of a sample, ARRAYS tensors each.  Those of the next take their places one by one as they are done with.
template <class T, int W, int ARRAYS> struct Held {
  typedef typename Pack<T, W>::Raw Raw;
  Raw* mine;
  __device__ __forceinline__ explicit Held(void* shared) : mine((Raw*)shared + threadIdx.x) {}
  __device__ __forceinline__ Raw* place(int k, int array) const { return mine + (k * ARRAYS + array) * (int)blockDim.x; }
  __device__ __forceinline__ Pack<T, W> get(int k, int array) const { Pack<T, W> p; p.raw = *place(k, array); return p; }
  __device__ __forceinline__ void put(int k, int array, const Pack<T, W>& p) const { *place(k, array) = p.raw; }
  // there when all copies have been waited for
  __device__ __forceinline__ void fetch(int k, int array, const T* from) const {
    if constexpr (sizeof(Raw) >= 4) paac::copy_to<(int)sizeof(Raw)>(place(k, array), from);
    else *place(k, array) = *reinterpret_cast<const Raw*>(from);             // two bytes cannot be copied asynchronously
  }
};

struct Exchange { float2 of_block[2][MAX_CLUSTER][MAX_GROUPS]; };           // by the parity of the sample

// What both kernels begin with: the groups of a thread's values, whether it is the one that speaks for them, gamma and beta.
template <int W, Mode M, int NV>
__device__ __forceinline__ void channels_of(const Args& a, const Place<W>& me, float (&gamma)[W], float (&beta)[W], int (&group)[NV], bool (&speaks)[NV]) {
#pragma unroll
  for (int j = 0; j < W; ++j) {
    gamma[j] = a.gamma != nullptr && me.cnt > 0 ? a.gamma[me.c + j] : 1.f;
    beta[j] = a.beta != nullptr && me.cnt > 0 ? a.beta[me.c + j] : 0.f;
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    group[j] = min((me.v * W + j) / a.q.cg, me.s.groups - 1);               // (idle threads have one too)
    speaks[j] = me.r == 0 && (me.v * W + j) % a.q.cg == 0;
  }
}
// sums by channel as those of a thread's values
template <int W, Mode M, int NV> __device__ __forceinline__ void joined(const float (&acc)[W], float (&value)[NV]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) value[j] = acc[j];
  if constexpr (NV == 1) {
#pragma unroll
    for (int j = 1; j < W; ++j) value[0] += acc[j];
  }
}

template <class T, int W, Mode M>
__global__ void __launch_bounds__(TB, REGISTER_BLOCKS) resident_kernel(const __grid_constant__ Args a, int cluster, int slab, int stride) {
  typedef GroupSum<W, M, float> Sums;
  constexpr int NV = Sums::NV;
  extern __shared__ uint4 room[];
  __shared__ Sums sums;
  __shared__ Exchange ex;
  const Geo& q = a.q;
  const int id = blockIdx.x / cluster;
  const Place<W> me(q, id, slab, paac::cluster_rank());
  if (cluster > 1) paac::cluster_arrive();                  // nobody stores into a block that has not begun
  paac::pdl_entry();
  float gamma[W], beta[W];
  int group[NV];
  bool speaks[NV];                                          // for the group, at its first access or channel
  channels_of<W, M>(a, me, gamma, beta, group, speaks);
  const float mine = (float)max(me.rows, 1) * (float)q.cg, all = 1.f / ((float)q.pixels * (float)q.cg);       // a group's elements here; 1 / all of them
  const int64_t in_step = (int64_t)me.R * a.x.pixel, out_step = (int64_t)me.R * a.out.pixel;
  int64_t n = id / q.slices;
  const T* from = at<const T>(a.x, n, (int64_t)me.rank * slab + me.r, me.c);
  T* to = at<T>(a.out, n, (int64_t)me.rank * slab + me.r, me.c);
  const Held<T, W, 1> held(room);
  if (n < q.n) {
    const T* p = from;
    for (int k = 0; k < me.cnt; ++k, p += in_step) held.fetch(k, 0, p);
  }
  paac::copies_end_step();
  if (cluster > 1) paac::cluster_wait();
  for (int turn = 0; n < q.n; turn ^= 1) {
    const int64_t now = n;
    n += stride;
    from += stride * a.x.sample;
    paac::copies_wait<0>();
    float acc[W], mean[NV], d2[NV];
#pragma unroll
    for (int j = 0; j < W; ++j) acc[j] = 0.f;
#pragma unroll 4
    for (int k = 0; k < me.cnt; ++k) { float f[W]; held.get(k, 0).widen(f); paac::add_all(acc, f); }
    joined<W, M>(acc, mean);
    sums.run(q, me, 0, group, mean);
    float less[W];
#pragma unroll
    for (int j = 0; j < NV; ++j) mean[j] = __fdiv_rn(mean[j], mine);         // (a group of one value has exactly that mean)
#pragma unroll
    for (int j = 0; j < W; ++j) { less[j] = -mean[j % NV]; acc[j] = 0.f; }
#pragma unroll 4
    for (int k = 0; k < me.cnt; ++k) { float f[W]; held.get(k, 0).widen(f); paac::add_all(f, less); paac::fma_all(acc, f, f); }
    joined<W, M>(acc, d2);
    sums.run(q, me, 1, group, d2);
    if (cluster > 1) {
#pragma unroll
      for (int j = 0; j < NV; ++j)
        if (speaks[j])
          for (int b = 0; b < cluster; ++b) paac::store_in_block(&ex.of_block[turn][me.rank][group[j]], b, make_float2(mean[j], d2[j]));
      paac::cluster_arrive();
      paac::cluster_wait();
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        float m = 0.f, d = 0.f;
        for (int b = 0; b < cluster; ++b) m = fmaf((float)slab_of(q.pixels, slab, b), ex.of_block[turn][b][group[j]].x, m);
        m /= (float)q.pixels;
        for (int b = 0; b < cluster; ++b) {
          const float2 e = ex.of_block[turn][b][group[j]];
          const float off = e.x - m;
          d += fmaf((float)slab_of(q.pixels, slab, b) * (float)q.cg * off, off, e.y);
        }
        mean[j] = m; d2[j] = d;
      }
    }
    float scale[W];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      d2[j] = rsqrtf(fmaf(d2[j], all, a.eps));
      if (speaks[j] && me.rank == 0) {
        const int64_t g = now * q.groups + me.s.g0 + group[j];
        a.mean_out[g] = mean[j]; a.rstd_out[g] = d2[j];
      }
    }
#pragma unroll
    for (int j = 0; j < W; ++j) { less[j] = -mean[j % NV]; scale[j] = d2[j % NV] * gamma[j]; }
    T* p_out = to;
    to += stride * a.out.sample;
    const T* p_in = from;
    const bool more = n < q.n;
#pragma unroll 2
    for (int k = 0; k < me.cnt; ++k, p_out += out_step, p_in += in_step) {
      float f[W], y[W];
      held.get(k, 0).widen(f);
      paac::add_all(f, less);
      paac::fma_all_to(y, f, scale, beta);
      Pack<T, W> p;
      if (a.activation == PAAC_ACT_RELU) p.round_positive(y);
      else { act_all<T, W>(y, a.activation); p.round(y); }
      p.store(p_out);
      if (more) held.fetch(k, 0, p_in);
    }
    paac::copies_end_step();
  }
}

template <class T, int W, Mode M>
__global__ void __launch_bounds__(TB, REGISTER_BLOCKS) resident_back_kernel(const __grid_constant__ Args a, int cluster, int slab, int stride,
                                                                            float* sums_to /* [rows][2][c] */) {
  typedef GroupSum<W, M, float2> Sums;
  constexpr int NV = Sums::NV;
  extern __shared__ uint4 room[];
  __shared__ Sums sums;
  __shared__ Exchange ex;
  const Geo& q = a.q;
  const int id = blockIdx.x / cluster;
  const Place<W> me(q, id, slab, paac::cluster_rank());
  if (cluster > 1) paac::cluster_arrive();
  paac::pdl_entry();
  float gamma[W], beta[W], all_b[W], all_g[W];
  int group[NV];
  bool speaks[NV];
  channels_of<W, M>(a, me, gamma, beta, group, speaks);
#pragma unroll
  for (int j = 0; j < W; ++j) all_b[j] = all_g[j] = 0.f;
  const float each = -1.f / ((float)q.pixels * (float)q.cg);
  const int64_t row = (int64_t)me.rank * slab + me.r;
  const int64_t x_step = (int64_t)me.R * a.x.pixel, d_step = (int64_t)me.R * a.dy.pixel, out_step = (int64_t)me.R * a.out.pixel;
  int64_t n = id / q.slices;
  const T *x_at = at<const T>(a.x, n, row, me.c), *d_at = at<const T>(a.dy, n, row, me.c);
  T* out_at = at<T>(a.out, n, row, me.c);
  const float *mean_at = a.mean + n * q.groups + me.s.g0, *rstd_at = a.rstd + n * q.groups + me.s.g0;
  const Held<T, W, 2> held(room);
  float next_mean[NV], next_rstd[NV];
  auto fetch_stats = [&]() {
#pragma unroll
    for (int j = 0; j < NV; ++j) { next_mean[j] = mean_at[group[j]]; next_rstd[j] = rstd_at[group[j]]; }
  };
  if (n < q.n) {
    fetch_stats();
    const T *p = x_at, *e = d_at;
    for (int k = 0; k < me.cnt; ++k, p += x_step, e += d_step) { held.fetch(k, 0, p); held.fetch(k, 1, e); }
  }
  paac::copies_end_step();
  if (cluster > 1) paac::cluster_wait();
  for (int turn = 0; n < q.n; turn ^= 1) {
    float less[W], rstd[W], db[W], dg[W];
#pragma unroll
    for (int j = 0; j < W; ++j) { less[j] = -next_mean[j % NV]; rstd[j] = next_rstd[j % NV]; db[j] = dg[j] = 0.f; }
    n += stride;
    x_at += stride * a.x.sample; d_at += stride * a.dy.sample;
    mean_at += (int64_t)stride * q.groups; rstd_at += (int64_t)stride * q.groups;
    const bool more = n < q.n;
    if (more) fetch_stats();
    paac::copies_wait<0>();
    // xhat and dv of access k
    auto derive = [&](int k, float (&xh)[W], float (&dv)[W]) {
      held.get(k, 0).widen(xh);
      held.get(k, 1).widen(dv);
      paac::add_all(xh, less);
      paac::mul_all(xh, rstd);
      if (a.activation != PAAC_ACT_NONE) {
        float arg[W];
        paac::fma_all_to(arg, xh, gamma, beta);
        slope_all<T, W>(dv, arg, a.activation);
      }
    };
    // dv is a value of the storage type, and is kept in the place of dy from the first use on; likewise xhat, if float
    const bool kept = sizeof(T) == 4 || a.activation != PAAC_ACT_SILU;
#pragma unroll 2
    for (int k = 0; k < me.cnt; ++k) {
      float xh[W], dv[W];
      derive(k, xh, dv);
      paac::add_all(db, dv);
      paac::fma_all(dg, dv, xh);
      Pack<T, W> p;
      if (sizeof(T) == 4) { p.round(xh); held.put(k, 0, p); }
      if (kept) { p.round(dv); held.put(k, 1, p); }
    }
    paac::add_all(all_b, db);
    paac::add_all(all_g, dg);
    float2 value[NV];
    const bool wanted = a.out.data != nullptr;
    if (wanted) {
      float v1[NV], v2[NV];
      paac::mul_all(db, gamma);
      paac::mul_all(dg, gamma);
      joined<W, M>(db, v1);
      joined<W, M>(dg, v2);
#pragma unroll
      for (int j = 0; j < NV; ++j) value[j] = make_float2(v1[j], v2[j]);
      sums.run(q, me, turn, group, value);
      if (cluster > 1) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
          if (speaks[j])
            for (int b = 0; b < cluster; ++b) paac::store_in_block(&ex.of_block[turn][me.rank][group[j]], b, value[j]);
        paac::cluster_arrive();
        paac::cluster_wait();
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          value[j] = make_float2(0.f, 0.f);
          for (int b = 0; b < cluster; ++b) value[j] = plus(value[j], ex.of_block[turn][b][group[j]]);
        }
      }
    }
    T* o_at = out_at;
    out_at += stride * a.out.sample;
    const T *p_x = x_at, *p_d = d_at;
    if (!wanted) {
      for (int k = 0; k < me.cnt && more; ++k, p_x += x_step, p_d += d_step) { held.fetch(k, 0, p_x); held.fetch(k, 1, p_d); }
      paac::copies_end_step();
      continue;
    }
    float s1[W], s2[W];
#pragma unroll
    for (int j = 0; j < W; ++j) { s1[j] = value[j % NV].x * each; s2[j] = value[j % NV].y * each; }
#pragma unroll 2
    for (int k = 0; k < me.cnt; ++k, o_at += out_step, p_x += x_step, p_d += d_step) {
      float xh[W], dv[W], o[W];
      if (kept) {
        held.get(k, 0).widen(xh);
        held.get(k, 1).widen(dv);
        if (sizeof(T) != 4) { paac::add_all(xh, less); paac::mul_all(xh, rstd); }
      } else {
        derive(k, xh, dv);
      }
      paac::fma_all_to(o, gamma, dv, s1);
      paac::fma_all(o, xh, s2);
      paac::mul_all(o, rstd);
      Pack<T, W> p;
      p.round(o);
      p.store(o_at);
      if (more) { held.fetch(k, 0, p_x); held.fetch(k, 1, p_d); }
    }
    paac::copies_end_step();
  }
  if (sums_to == nullptr) return;
  // dbeta and dgamma of the block's own samples and pixels, the row lanes one after the other; what was held is done with
  float* of_row = reinterpret_cast<float*>(room);           // [row lane][channel]
  float* to = sums_to + ((int64_t)(id / q.slices) * cluster + me.rank) * 2 * q.c + me.s.c0;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    __syncthreads();
    if (me.r < me.R) {
#pragma unroll
      for (int j = 0; j < W; ++j) of_row[me.r * me.s.width + me.v * W + j] = which ? all_g[j] : all_b[j];
    }
    __syncthreads();
    // `parts` threads a channel, each leaving its sum in the first row that it has added up
    const int width = me.s.width, most = min((int)blockDim.x / width, me.R), parts = most < 1 ? 1 : (most > 16 ? 16 : most);
    for (int i = threadIdx.x; i < width * parts; i += blockDim.x) {
      const int part = i / width, ch = i - part * width;
      float t = 0.f;
      for (int k = part; k < me.R; k += parts) t += of_row[k * width + ch];
      of_row[i] = t;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < width; i += blockDim.x) {
      float t = 0.f;
      for (int k = 0; k < parts; ++k) t += of_row[k * width + i];
      to[which * q.c + i] = t;
    }
  }
}

// ---- samples too large for that: statistics, then the result, each reading x ---------------------------------------------------------------

template <class T, int W>
__global__ void __launch_bounds__(TB) stats_kernel(const __grid_constant__ Args a, float2* partial /* [n][groups][slabs * parts] */) {
  __shared__ float sm[TB * W], sq[TB * W];
  paac::pdl_entry();
  const Geo& q = a.q;
  const int64_t units = (int64_t)q.n * q.slabs * q.slices;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int i = (int)(u % q.slices), slab = (int)(u / q.slices % q.slabs);
    const int64_t n = u / q.slices / q.slabs;
    const Slice s = slice_of(q, i);
    const int cv = s.width / W, R = TB / cv, r = threadIdx.x / cv, v = threadIdx.x - r * cv;
    const int p0 = slab * q.slab_rows, rows = min(q.slab_rows, q.pixels - p0);
    if (r < R) {
      float shift[W], d1[W], d2[W];
      const int cnt = rows_of(rows, r, R);
#pragma unroll
      for (int j = 0; j < W; ++j) shift[j] = d1[j] = d2[j] = 0.f;
#pragma unroll 4
      for (int k = 0; k < cnt; ++k) {
        Pack<T, W> p;
        float x[W];
        p.load(at<T>(a.x, n, p0 + r + k * R, s.c0 + v * W));
        p.widen(x);
#pragma unroll
        for (int j = 0; j < W; ++j) {
          if (k == 0) shift[j] = x[j];
          const float d = x[j] - shift[j];
          d1[j] += d;
          d2[j] = fmaf(d, d, d2[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float m = cnt > 0 ? d1[j] / (float)cnt : 0.f;
        sm[r * s.width + v * W + j] = shift[j] + m;
        sq[r * s.width + v * W + j] = fmaxf(d2[j] - d1[j] * m, 0.f) + (d2[j] - d2[j]);      // (the larger of NaN and 0 is 0)
      }
    }
    __syncthreads();
    for (int g = threadIdx.x >> 5; g < s.groups; g += WARPS) {
      const int width = q.parts == 1 ? q.cg : s.width;
      const Stats t = merge_group(sm, sq, R, s.width, g * width, width, rows, threadIdx.x & 31);
      if ((threadIdx.x & 31) == 0)
        partial[(n * q.groups + s.g0 + g) * (q.slabs * q.parts) + slab * q.parts + (q.parts == 1 ? 0 : i % q.parts)] = make_float2(t.mean, t.m2);
    }
    __syncthreads();
  }
}

__global__ void __launch_bounds__(TB) finish_stats_kernel(const __grid_constant__ Geo q, const float2* partial, float eps, float* mean, float* rstd) {
  paac::pdl_entry();
  const int64_t units = (int64_t)q.n * q.groups;
  const int lane = threadIdx.x & 31, each = q.slabs * q.parts;
  for (int64_t u = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * WARPS) {
    const float2* p = partial + u * each;
    auto count = [&](int e) {
      const int slab = e / q.parts, part = e - slab * q.parts;
      return (float)min(q.slab_rows, q.pixels - slab * q.slab_rows) * (float)(q.parts == 1 ? q.cg : min(q.cap, q.cg - part * q.cap));
    };
    float s = 0.f;
    for (int e = lane; e < each; e += 32) s = fmaf(count(e), p[e].x, s);
    const float total = (float)q.pixels * (float)q.cg, m = warp_sum(s) / total;
    float d2 = 0.f;
    for (int e = lane; e < each; e += 32) { const float d = p[e].x - m; d2 += fmaf(count(e) * d, d, p[e].y); }
    d2 = warp_sum(d2);
    if (lane == 0) { mean[u] = m; rstd[u] = 1.f / sqrtf(d2 / total + eps); }
  }
}

// what a thread keeps of its W channels
template <int W> struct Channels {
  float gamma[W], beta[W], mean[W], rstd[W];
  __device__ __forceinline__ void load(const Args& a, const float* mean_at, const float* rstd_at, int c) {
#pragma unroll
    for (int j = 0; j < W; ++j) {
      gamma[j] = a.gamma != nullptr ? a.gamma[c + j] : 1.f;
      beta[j] = a.beta != nullptr ? a.beta[c + j] : 0.f;
      const int g = (c + j) / a.q.cg;
      mean[j] = mean_at[g];
      rstd[j] = rstd_at[g];
    }
  }
  __device__ __forceinline__ float argument(int j, float x) const { return fmaf((x - mean[j]) * rstd[j], gamma[j], beta[j]); }
};

template <class T, int W>
__global__ void __launch_bounds__(TB) apply_kernel(const __grid_constant__ Args a) {
  paac::pdl_entry();
  const Geo& q = a.q;
  const int64_t units = (int64_t)q.n * q.slabs * q.slices;
  for (int64_t u = units - 1 - blockIdx.x; u >= 0; u -= gridDim.x) {          // from the end, where the statistics have just been
    const int i = (int)(u % q.slices), slab = (int)(u / q.slices % q.slabs);
    const int64_t n = u / q.slices / q.slabs;
    const Slice s = slice_of(q, i);
    const int cv = s.width / W, R = TB / cv, r = threadIdx.x / cv, v = threadIdx.x - r * cv;
    const int p0 = slab * q.slab_rows, rows = min(q.slab_rows, q.pixels - p0);
    if (r >= R) continue;
    Channels<W> ch;
    ch.load(a, a.mean + n * q.groups, a.rstd + n * q.groups, s.c0 + v * W);
#pragma unroll 4
    for (int k = r; k < rows; k += R) {
      Pack<T, W> p;
      float x[W];
      p.load(at<T>(a.x, n, p0 + k, s.c0 + v * W));
      p.widen(x);
#pragma unroll
      for (int j = 0; j < W; ++j) x[j] = ch.argument(j, x[j]);
      act_all<T, W>(x, a.activation);
      p.round(x);
      p.store(at<T>(a.out, n, p0 + k, s.c0 + v * W));
    }
  }
}

// per channel of a slab: sum dv and sum dv xhat
template <class T, int W>
__global__ void __launch_bounds__(TB) sums_kernel(const __grid_constant__ Args a, float* sums /* [n * slabs][2][c] */) {
  __shared__ float sb[TB * W], sg[TB * W];
  paac::pdl_entry();
  const Geo& q = a.q;
  const int64_t units = (int64_t)q.n * q.slabs * q.slices;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int i = (int)(u % q.slices), slab = (int)(u / q.slices % q.slabs);
    const int64_t n = u / q.slices / q.slabs;
    const Slice s = slice_of(q, i);
    const int cv = s.width / W, R = TB / cv, r = threadIdx.x / cv, v = threadIdx.x - r * cv;
    const int p0 = slab * q.slab_rows, rows = min(q.slab_rows, q.pixels - p0);
    if (r < R) {
      Channels<W> ch;
      ch.load(a, a.mean + n * q.groups, a.rstd + n * q.groups, s.c0 + v * W);
      float db[W], dg[W];
#pragma unroll
      for (int j = 0; j < W; ++j) db[j] = dg[j] = 0.f;
#pragma unroll 2
      for (int k = r; k < rows; k += R) {
        Pack<T, W> px, pd;
        float x[W], d[W];
        px.load(at<T>(a.x, n, p0 + k, s.c0 + v * W));
        pd.load(at<T>(a.dy, n, p0 + k, s.c0 + v * W));
        px.widen(x);
        pd.widen(d);
        float arg[W];
#pragma unroll
        for (int j = 0; j < W; ++j) arg[j] = ch.argument(j, x[j]);
        slope_all<T, W>(d, arg, a.activation);
#pragma unroll
        for (int j = 0; j < W; ++j) { db[j] += d[j]; dg[j] = fmaf(d[j], (x[j] - ch.mean[j]) * ch.rstd[j], dg[j]); }
      }
#pragma unroll
      for (int j = 0; j < W; ++j) { sb[r * s.width + v * W + j] = db[j]; sg[r * s.width + v * W + j] = dg[j]; }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < s.width; c += TB) {
      float b = 0.f, g = 0.f;
      for (int k = 0; k < R; ++k) { b += sb[k * s.width + c]; g += sg[k * s.width + c]; }
      float* to = sums + (n * q.slabs + slab) * 2 * (int64_t)q.c + s.c0 + c;
      to[0] = b;
      to[q.c] = g;
    }
    __syncthreads();
  }
}

// per group of a sample: S1 / m and S2 / m
__global__ void __launch_bounds__(TB) group_sums_kernel(const __grid_constant__ Geo q, const float* sums, const float* gamma, float2* out /* [n][groups] */) {
  paac::pdl_entry();
  const int64_t units = (int64_t)q.n * q.groups;
  const int lane = threadIdx.x & 31;
  for (int64_t u = (int64_t)blockIdx.x * WARPS + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * WARPS) {
    const int64_t n = u / q.groups;
    const int c0 = (int)(u - n * q.groups) * q.cg;
    float s1 = 0.f, s2 = 0.f;
    for (int k = 0; k < q.slabs; ++k)
      for (int c = c0 + lane; c < c0 + q.cg; c += 32) {
        const float* p = sums + (n * q.slabs + k) * 2 * (int64_t)q.c + c;
        const float g = gamma != nullptr ? gamma[c] : 1.f;
        s1 = fmaf(g, p[0], s1);
        s2 = fmaf(g, p[q.c], s2);
      }
    s1 = warp_sum(s1);
    s2 = warp_sum(s2);
    const float m = (float)q.pixels * (float)q.cg;
    if (lane == 0) out[u] = make_float2(s1 / m, s2 / m);
  }
}

template <class T, int W>
__global__ void __launch_bounds__(TB) apply_back_kernel(const __grid_constant__ Args a, const float2* group_sums) {
  paac::pdl_entry();
  const Geo& q = a.q;
  const int64_t units = (int64_t)q.n * q.slabs * q.slices;
  for (int64_t u = units - 1 - blockIdx.x; u >= 0; u -= gridDim.x) {
    const int i = (int)(u % q.slices), slab = (int)(u / q.slices % q.slabs);
    const int64_t n = u / q.slices / q.slabs;
    const Slice s = slice_of(q, i);
    const int cv = s.width / W, R = TB / cv, r = threadIdx.x / cv, v = threadIdx.x - r * cv;
    const int p0 = slab * q.slab_rows, rows = min(q.slab_rows, q.pixels - p0);
    if (r >= R) continue;
    Channels<W> ch;
    ch.load(a, a.mean + n * q.groups, a.rstd + n * q.groups, s.c0 + v * W);
    float s1[W], s2[W];
#pragma unroll
    for (int j = 0; j < W; ++j) { const float2 g = group_sums[n * q.groups + (s.c0 + v * W + j) / q.cg]; s1[j] = g.x; s2[j] = g.y; }
#pragma unroll 2
    for (int k = r; k < rows; k += R) {
      Pack<T, W> px, pd;
      float x[W], d[W];
      px.load(at<T>(a.x, n, p0 + k, s.c0 + v * W));
      pd.load(at<T>(a.dy, n, p0 + k, s.c0 + v * W));
      px.widen(x);
      pd.widen(d);
      float arg[W];
#pragma unroll
      for (int j = 0; j < W; ++j) arg[j] = ch.argument(j, x[j]);
      slope_all<T, W>(d, arg, a.activation);
#pragma unroll
      for (int j = 0; j < W; ++j) x[j] = ch.rstd[j] * (fmaf(ch.gamma[j], d[j], -s1[j]) - (x[j] - ch.mean[j]) * ch.rstd[j] * s2[j]);
      px.round(x);
      px.store(at<T>(a.out, n, p0 + k, s.c0 + v * W));
    }
  }
}

// dgamma and dbeta: the rows of `sums` added up, eight columns (a sector) a block, so that a thread has few loads one after the other
constexpr int CHANNEL_LANES = 8, ROW_LANES = 128;
__global__ void __launch_bounds__(CHANNEL_LANES * ROW_LANES)
channel_sums_kernel(const float* sums /* [rows][2][c] */, int64_t rows, int c, float* dgamma, float* dbeta) {
  constexpr int OF_WARP = 32 / CHANNEL_LANES, ROW_WARPS = ROW_LANES / OF_WARP;
  __shared__ float sh[ROW_WARPS][CHANNEL_LANES];
  paac::pdl_entry();
  const int lane = threadIdx.x % CHANNEL_LANES, r = threadIdx.x / CHANNEL_LANES;
  const int64_t col = (int64_t)blockIdx.x * CHANNEL_LANES + lane;           // of 2 c: dbeta, then dgamma
  float s = 0.f;
  if (col < 2 * (int64_t)c) {
#pragma unroll 8
    for (int64_t k = r; k < rows; k += ROW_LANES) s += sums[k * 2 * c + col];
  }
#pragma unroll
  for (int o = CHANNEL_LANES; o < 32; o *= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (r % OF_WARP == 0) sh[r / OF_WARP][lane] = s;
  __syncthreads();
  if (r == 0 && col < 2 * (int64_t)c) {
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < ROW_WARPS; ++k) t += sh[k][lane];
    if (col < c) { if (dbeta != nullptr) dbeta[col] = t; }
    else if (dgamma != nullptr) dgamma[col - c] = t;
  }
}

// ---- the host's part -------------------------------------------------------------------------------------------------------------------

int gcd(int a, int b) { while (b) { const int t = a % b; a = b; b = t; } return a; }

// slices for accesses of W channels; false where whole groups and whole accesses do not go together
bool cut(Geo& q, int W) {
  q.cap = TB * W;
  if (q.c % W != 0) return false;
  if (q.c <= q.cap) { q.gps = q.groups; q.parts = 1; q.slices = 1; return true; }
  const int unit = W / gcd(q.cg, W);                    // groups between two slices' beginnings
  if (q.cg <= q.cap) {
    q.gps = q.cap / q.cg / unit * unit;
    if (q.gps == 0) return false;
    q.parts = 1;
    q.slices = (q.groups + q.gps - 1) / q.gps;
    return true;
  }
  if (q.cg % W != 0) return false;
  q.gps = 1;
  q.parts = (q.cg + q.cap - 1) / q.cap;
  q.slices = q.groups * q.parts;
  return true;
}
void cut_rows(Geo& q, int W) {
  const int width = q.parts == 1 ? (q.gps < q.groups ? q.gps : q.groups) * q.cg : q.cap, R = TB / (width / W);
  q.slab_rows = R * 16;
  if (q.slab_rows > q.pixels) q.slab_rows = q.pixels;
  q.slabs = (q.pixels - 1) / q.slab_rows + 1;           // (pixels + rows may not fit 32 bits)
}

// How the resident kernels take a shape, if they do: `q` with slices of whole groups, blocks of `threads` with `slab` pixels each,
// `smem` bytes for a sample, `share` blocks to a multiprocessor, clusters of `cluster` blocks.
struct Resident { Geo q; int cluster, slab, threads, smem, share; Mode mode; };
bool power_of_two(int v) { return v > 0 && (v & (v - 1)) == 0; }
constexpr int MAX_DEPTH = 64;         // terms that a thread adds up one after the other in float
constexpr int SM_BYTES = 227 << 10, OWN_BYTES = 26 << 10;    // shared memory of a multiprocessor; what a block has besides, at most
// Of the ways to cut a shape up the one that should take least time.  A thread's work on a sample is its rows and what it does once, about
// eight rows' work, more the more threads wait for one another and six or so more if a cluster has to meet; there is the work of all
// threads, for 512 of them to a multiprocessor, and the time that one turn takes by itself, half of a row's work being waits, times the
// turns of those that are resident.  Channels one by one are more work a row, so that the rest counts for less (2000 samples of 400
// pixels with 24 channels in 8 groups backward: 64 threads 122 us, 128 82; 1000 of 96 in 32: 128 threads 118, now 94).  Rows of less
// than 32 bytes would be read twice; those of less than 128 cost a little.
bool resident_mode(Geo q, int W, int size, bool back, Mode mode, Resident& out) {
  const int unit = W / gcd(q.cg, W), wide = q.cg / W;                       // unit: groups between two slices' beginnings
  if (q.c % W != 0 || (mode == ALIGNED && (q.cg % W != 0 || !power_of_two(wide) || wide > 32))) return false;
  auto fits = [&](int g) {
    if (g > MAX_GROUPS || g * q.cg > MAX_WIDTH || g * q.cg / W > TB || (g < q.groups && g % unit != 0)) return false;
    return mode != ALIGNED || (power_of_two(g) && (q.groups % g == 0 || power_of_two(q.groups % g)));
  };
  double best = 0.0;
  int first = 1;                                            // the largest power of two
  while (first * 2 <= q.groups && first < MAX_GROUPS) first *= 2;
  for (int g = q.groups; g >= 1; g = g > first ? first : g / 2) {           // all groups, then powers of two
    if (!fits(g) || (g < q.groups && g * q.cg * size < 32)) continue;
    const int cv = g * q.cg / W, slices = (q.groups + g - 1) / g, bytes = g * q.cg * size;
    for (int cluster = 1; cluster <= MAX_CLUSTER && cluster <= q.pixels; cluster *= 2) {
      const int slab = (q.pixels - 1) / cluster + 1;
      for (int threads = 64; threads <= TB; threads *= 2) {
        if (threads < cv) continue;
        const int depth = (slab - 1) / (threads / cv) + 1;
        if (depth > MAX_DEPTH) continue;
        // (the backward pass adds up its sums by channel in the same place in the end)
        const int64_t held = (int64_t)depth * (back ? 2 : 1) * threads * W * size, sums = back ? (int64_t)threads * W * 4 : 0, smem = held > sums ? held : sums;
        if (smem > SM_BYTES - OWN_BYTES) continue;
        int share = (int)(SM_BYTES / (smem + OWN_BYTES / 2)), most = REGISTER_BLOCKS * TB / threads;
        if (share > most) share = most;
        if (share < 1) share = 1;
        const double total = (double)q.n * slices * cluster * threads, turns = total / (148 * share * threads), all = total / (148 * 512);
        const double once = 8 + threads / 128.0 + (cluster > 1 ? 4 + threads / 64.0 + cluster / 4.0 : 0.0);
        const double waits = (turns < 1.0 ? 1.0 : turns) * (depth * 0.5 + once), works = all * (depth + (mode == BY_CHANNEL ? 3 : once));
        const double cost = (waits > works ? waits : works) * (g < q.groups && bytes < 128 ? (bytes < 64 ? 1.12 : 1.03) : 1.0);
        if (best != 0.0 && cost >= best) continue;
        best = cost;
        q.gps = g; q.parts = 1; q.cap = TB * W; q.slices = slices;
        out = Resident{q, cluster, slab, threads, (int)smem, share, mode};
      }
    }
  }
  return best != 0.0;
}
bool resident(const Geo& q, int W, int size, bool back, Resident& out) {
  return resident_mode(q, W, size, back, ALIGNED, out) || resident_mode(q, W, size, back, q.cg % W == 0 ? BY_ACCESS : BY_CHANNEL, out);
}
// clusters that a slice's samples may be dealt out to: the backward pass has room for the sums of so many
int dealt(const Resident& r) {
  const int most = GRID / (r.q.slices * r.cluster);
  return r.q.n < most ? r.q.n : (most < 1 ? 1 : most);
}
// blocks of a slice that may leave sums, whatever way a shape is cut up: a cluster's a sample, GRID in all unless one cluster is more; there
// are no fewer slices than their widest ones make
int64_t most_dealt(const paac_norm& s) {
  const int slices = (s.c + MAX_WIDTH - 1) / MAX_WIDTH, all = GRID / slices;
  const int64_t by_sample = (int64_t)s.n * (s.pixels < MAX_CLUSTER ? s.pixels : MAX_CLUSTER);
  return std::min<int64_t>(by_sample, all > MAX_CLUSTER ? all : MAX_CLUSTER);
}

bool shape_ok(const paac_norm* s) {
  return s != nullptr && s->n >= 1 && s->pixels >= 1 && s->c >= 1 && s->groups >= 1 && s->c <= 65536 && s->c % s->groups == 0 &&
         (int64_t)s->n * s->groups < ((int64_t)1 << 31) && (int64_t)s->n * s->pixels < ((int64_t)1 << 31) &&
         (s->type == PAAC_FP32 || s->type == PAAC_BF16) && s->activation >= PAAC_ACT_NONE && s->activation <= PAAC_ACT_SILU && s->eps > 0.f;
}
// The widest accesses that the rows' places (multiples of `align` bytes) and the channels allow; of those the widest that no group begins
// within, if that is more than one element: a group's sums are then those of accesses.  Else up to four elements, whose sums are kept one by
// one (eight: 82 us instead of 44 for the gradient of 669 samples of 441 pixels with 32 channels in as many groups, for want of registers).
Geo geometry(const paac_norm& s, int align, int& W) {
  Geo q{};
  q.n = s.n; q.pixels = s.pixels; q.c = s.c; q.groups = s.groups; q.cg = s.c / s.groups;
  const int size = s.type == PAAC_BF16 ? 2 : 4;
  W = align / size < 1 ? 1 : align / size;
  while (W > 1 && !cut(q, W)) W /= 2;
  int whole = W;
  while (whole > 1 && (q.cg % whole != 0 || !cut(q, whole))) whole /= 2;
  if (whole > 1) W = whole;
  else if (W > 4) W = 4;
  cut(q, W);
  cut_rows(q, W);
  return q;
}
size_t round_up(size_t v) { return (v + 255) / 256 * 256; }
struct Scratch { size_t first, second, total; };
// first: partial statistics or sums of a slab, or of a resident block; second: statistics or sums of a group.  Enough for accesses of any
// width.
Scratch scratch(const paac_norm& s) {
  const size_t row = (size_t)2 * s.c * sizeof(float);
  Scratch r;
  r.first = (size_t)most_dealt(s) * row;
  for (int W = s.type == PAAC_BF16 ? 8 : 4; W >= 1; W /= 2) {
    Geo q{};
    q.n = s.n; q.pixels = s.pixels; q.c = s.c; q.groups = s.groups; q.cg = s.c / s.groups;
    if (!cut(q, W)) continue;
    cut_rows(q, W);
    const size_t stats = (size_t)q.n * q.groups * q.slabs * q.parts * sizeof(float2), sums = (size_t)q.n * q.slabs * row;
    if (stats > r.first) r.first = stats;
    if (sums > r.first) r.first = sums;
  }
  r.first = round_up(r.first);
  r.second = round_up((size_t)s.n * s.groups * sizeof(float2));
  r.total = r.first + r.second;
  return r;
}

View view(const paac_rows& r, const paac_norm& s) { return View{r.data, s.n > 1 ? r.outer : 0, s.pixels > 1 ? r.inner : 0}; }
unsigned blocks(int64_t units, int most) { return (unsigned)(units < most ? units : most); }

struct Check {
  const paac_norm& s;
  int size, align = 16;              // align: bytes that all rows' places are multiples of
  bool ok = true;
  paac::Arrays arrays;
  explicit Check(const paac_norm& s_) : s(s_), size(s_.type == PAAC_BF16 ? 2 : 4) {}
  paac::RowSet rows(const paac_rows& r, bool out) {
    const paac::RowSet set(r, s.n, s.pixels, s.c, size);
    if (r.data == nullptr || !set.sane() || !set.aligned() || (out && !set.rows_apart())) ok = false;
    else while (align > size && !set.multiples_of(align)) align /= 2;
    return set;
  }
  // `count` floats, or none
  void floats(const float* p, int64_t count, bool out) {
    if ((uintptr_t)p & 3u) ok = false;
    arrays.keep(p, count * 4, out);
  }
  bool fit() const { return ok && arrays.apart; }
};

// How many clusters of 1, 2, 4, 8, 16 blocks are resident at once with one block to a multiprocessor: depends on how the part's
// multiprocessors are grouped, so it is asked for, once on each device (a function's attributes belong to the current one, and these
// entry points work on any).
struct Room { int clusters[5]; };
template <class Kernel> bool ask_room(Kernel kernel, Room& room) {
  cudaFuncAttributes own;
  if (cudaFuncGetAttributes(&own, kernel) != cudaSuccess) return false;
  const int most = SM_BYTES - (int)own.sharedSizeBytes;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess)
    return false;
  for (int i = 0; i < 5; ++i) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1 << i); cfg.blockDim = dim3(TB); cfg.dynamicSmemBytes = most;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1 << i; attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&room.clusters[i], kernel, &cfg) != cudaSuccess) { cudaGetLastError(); room.clusters[i] = 1; }
  }
  return true;
}
int log2_of(int v) { int i = 0; while ((1 << i) < v) ++i; return i; }
// launches as many clusters as are resident, `most` a slice at most, with the samples dealt out evenly; *deal: clusters a slice
template <class Kernel, class... Args_> cudaError_t launch_resident(paac::PerDevice<Room>& rooms, Kernel kernel, const Resident& r, int most, int* deal, cudaStream_t s,
                                                                    const Args& a, Args_... rest) {
  int device = -1;
  const Room* room = cudaGetDevice(&device) == cudaSuccess ? rooms.get(device, [&](Room& made) { return ask_room(kernel, made); }) : nullptr;
  if (room == nullptr) return cudaErrorUnknown;
  int each = room->clusters[log2_of(r.cluster)] * r.share / r.q.slices;
  if (each > most) each = most;
  if (each < 1) each = 1;
  const int turns = (r.q.n + each - 1) / each;
  *deal = (r.q.n + turns - 1) / turns;
  return paac::launch_clusters_on(s, kernel, dim3((unsigned)(*deal * r.q.slices * r.cluster)), dim3(r.threads), r.cluster, r.smem, a, r.cluster, r.slab, *deal,
                                  rest...);
}

template <class T, int W, Mode M> cudaError_t forward_mode(const Args& a, const Resident& r, cudaStream_t s) {
  static paac::PerDevice<Room> rooms;
  int deal = 0;
  return launch_resident(rooms, resident_kernel<T, W, M>, r, r.q.n, &deal, s, a);
}
// *rows: rows of sums that are there afterwards
template <class T, int W, Mode M> cudaError_t backward_mode(const Args& a, const Resident& r, float* sums, int64_t* rows, cudaStream_t s) {
  static paac::PerDevice<Room> rooms;
  int deal = 0;
  const cudaError_t e = launch_resident(rooms, resident_back_kernel<T, W, M>, r, dealt(r), &deal, s, a, sums);
  *rows = (int64_t)deal * r.cluster;
  return e;
}
// (accesses of one element have no group beginning within them, those of eight are not taken then)
template <class T, int W> cudaError_t forward_resident(Args a, const Resident& r, cudaStream_t s) {
  a.q = r.q;
  if (r.mode == ALIGNED) return forward_mode<T, W, ALIGNED>(a, r, s);
  if (r.mode == BY_CHANNEL) return forward_mode<T, W, W == 1 || W == 8 ? BY_ACCESS : BY_CHANNEL>(a, r, s);
  return forward_mode<T, W, BY_ACCESS>(a, r, s);
}
template <class T, int W> cudaError_t backward_resident(Args a, const Resident& r, float* sums, int64_t* rows, cudaStream_t s) {
  a.q = r.q;
  if (r.mode == ALIGNED) return backward_mode<T, W, ALIGNED>(a, r, sums, rows, s);
  if (r.mode == BY_CHANNEL) return backward_mode<T, W, W == 1 || W == 8 ? BY_ACCESS : BY_CHANNEL>(a, r, sums, rows, s);
  return backward_mode<T, W, BY_ACCESS>(a, r, sums, rows, s);
}

template <class T, int W> cudaError_t forward(const Args& a, float2* partial, cudaStream_t s) {
  Resident r;
  if (resident(a.q, W, sizeof(T), false, r)) return forward_resident<T, W>(a, r, s);
  const Geo& q = a.q;
  const int64_t units = (int64_t)q.n * q.slabs * q.slices, groups = (int64_t)q.n * q.groups;
  cudaError_t e = paac::launch_overlapped_on(s, stats_kernel<T, W>, dim3(blocks(units, GRID)), dim3(TB), 0, a, partial);
  if (e != cudaSuccess) return e;
  e = paac::launch_overlapped_on(s, finish_stats_kernel, dim3(blocks((groups + WARPS - 1) / WARPS, GRID)), dim3(TB), 0, q, (const float2*)partial, a.eps,
                                 a.mean_out, a.rstd_out);
  if (e != cudaSuccess) return e;
  return paac::launch_overlapped_on(s, apply_kernel<T, W>, dim3(blocks(units, GRID)), dim3(TB), 0, a);
}
template <class T, int W> cudaError_t backward(const Args& a, float* sums, float2* group_sums, float* dgamma, float* dbeta, cudaStream_t s) {
  Resident r;
  const bool wanted = dgamma != nullptr || dbeta != nullptr;
  int64_t rows;
  cudaError_t e;
  if (resident(a.q, W, sizeof(T), true, r)) {
    e = backward_resident<T, W>(a, r, wanted ? sums : nullptr, &rows, s);
  } else {
    const Geo& q = a.q;
    const int64_t units = (int64_t)q.n * q.slabs * q.slices, groups = (int64_t)q.n * q.groups;
    rows = (int64_t)q.n * q.slabs;
    e = paac::launch_overlapped_on(s, sums_kernel<T, W>, dim3(blocks(units, GRID)), dim3(TB), 0, a, sums);
    if (e == cudaSuccess && a.out.data != nullptr) {
      e = paac::launch_overlapped_on(s, group_sums_kernel, dim3(blocks((groups + WARPS - 1) / WARPS, GRID)), dim3(TB), 0, q, (const float*)sums, a.gamma, group_sums);
      if (e == cudaSuccess) e = paac::launch_overlapped_on(s, apply_back_kernel<T, W>, dim3(blocks(units, GRID)), dim3(TB), 0, a, (const float2*)group_sums);
    }
  }
  if (e != cudaSuccess || !wanted) return e;
  return paac::launch_overlapped_on(s, channel_sums_kernel, dim3((unsigned)((2 * (int64_t)a.q.c + CHANNEL_LANES - 1) / CHANNEL_LANES)), dim3(CHANNEL_LANES * ROW_LANES), 0,
                                    (const float*)sums, rows, a.q.c, dgamma, dbeta);
}

}  // namespace

extern "C" size_t paac_group_norm_workspace_bytes(const paac_norm* s) { return shape_ok(s) ? scratch(*s).total : 0; }

extern "C" int paac_group_norm(const paac_norm* s, paac_rows x, const float* gamma, const float* beta, paac_rows y, float* mean, float* rstd,
                               void* workspace, size_t workspace_bytes, void* stream) {
  if (!shape_ok(s)) return PAAC_ERR_ARG;
  Check check(*s);
  const paac::RowSet xs = check.rows(x, false), ys = check.rows(y, true);
  if (!check.ok) return PAAC_ERR_ARG;
  const int64_t of_groups = (int64_t)s->n * s->groups;
  check.arrays.keep(ys, true);
  if (!ys.same_as(xs)) check.arrays.keep(xs, false);
  check.floats(gamma, s->c, false); check.floats(beta, s->c, false); check.floats(mean, of_groups, true); check.floats(rstd, of_groups, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  const Scratch room = scratch(*s);
  if (workspace == nullptr || ((uintptr_t)workspace & 15u) != 0 || workspace_bytes < room.total) return PAAC_ERR_WORKSPACE;
  check.arrays.keep(workspace, (int64_t)room.total, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  int W;
  Args a{};
  a.q = geometry(*s, check.align, W);
  a.x = view(x, *s); a.out = view(y, *s);
  a.gamma = gamma; a.beta = beta; a.activation = s->activation; a.eps = s->eps;
  float* own = reinterpret_cast<float*>((char*)workspace + room.first);
  a.mean_out = mean != nullptr ? mean : own;
  a.rstd_out = rstd != nullptr ? rstd : own + (int64_t)s->n * s->groups;
  a.mean = a.mean_out; a.rstd = a.rstd_out;
  float2* partial = static_cast<float2*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (s->type == PAAC_BF16) e = W == 8 ? forward<bf16, 8>(a, partial, st) : W == 4 ? forward<bf16, 4>(a, partial, st)
                                : W == 2 ? forward<bf16, 2>(a, partial, st) : forward<bf16, 1>(a, partial, st);
  else e = W == 4 ? forward<float, 4>(a, partial, st) : W == 2 ? forward<float, 2>(a, partial, st) : forward<float, 1>(a, partial, st);
  return paac::launch_status(e);
}

extern "C" int paac_group_norm_backward(const paac_norm* s, paac_rows x, paac_rows dy, const float* gamma, const float* beta, const float* mean,
                                        const float* rstd, paac_rows dx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                                        void* stream) {
  if (!shape_ok(s) || mean == nullptr || rstd == nullptr) return PAAC_ERR_ARG;
  if (dx.data == nullptr && dgamma == nullptr && dbeta == nullptr) return PAAC_ERR_ARG;
  Check check(*s);
  const paac::RowSet xs = check.rows(x, false), ds = check.rows(dy, false);
  const paac::RowSet os = dx.data != nullptr ? check.rows(dx, true) : paac::RowSet();
  if (!check.ok) return PAAC_ERR_ARG;
  const int64_t of_groups = (int64_t)s->n * s->groups;
  if (dx.data != nullptr) check.arrays.keep(os, true);
  check.arrays.keep(xs, false);
  if (!os.same_as(ds)) check.arrays.keep(ds, false);
  check.floats(gamma, s->c, false); check.floats(beta, s->c, false); check.floats(mean, of_groups, false); check.floats(rstd, of_groups, false);
  check.floats(dgamma, s->c, true); check.floats(dbeta, s->c, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  const Scratch room = scratch(*s);
  if (workspace == nullptr || ((uintptr_t)workspace & 15u) != 0 || workspace_bytes < room.total) return PAAC_ERR_WORKSPACE;
  check.arrays.keep(workspace, (int64_t)room.total, true);
  if (!check.fit()) return PAAC_ERR_ARG;
  int W;
  Args a{};
  a.q = geometry(*s, check.align, W);
  a.x = view(x, *s); a.dy = view(dy, *s); a.out = view(dx, *s);
  a.gamma = gamma; a.beta = beta; a.mean = mean; a.rstd = rstd; a.activation = s->activation; a.eps = s->eps;
  float* sums = static_cast<float*>(workspace);
  float2* group_sums = reinterpret_cast<float2*>((char*)workspace + room.first);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (s->type == PAAC_BF16) e = W == 8 ? backward<bf16, 8>(a, sums, group_sums, dgamma, dbeta, st) : W == 4 ? backward<bf16, 4>(a, sums, group_sums, dgamma, dbeta, st)
                                : W == 2 ? backward<bf16, 2>(a, sums, group_sums, dgamma, dbeta, st) : backward<bf16, 1>(a, sums, group_sums, dgamma, dbeta, st);
  else e = W == 4 ? backward<float, 4>(a, sums, group_sums, dgamma, dbeta, st) : W == 2 ? backward<float, 2>(a, sums, group_sums, dgamma, dbeta, st)
                                                                                        : backward<float, 1>(a, sums, group_sums, dgamma, dbeta, st);
  return paac::launch_status(e);
}
