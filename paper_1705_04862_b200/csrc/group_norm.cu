// Group normalisation with scale, shift and activation, channels last, and its gradient (paac_group_norm, paac_group_norm_backward).
//
//   y = act(v), v = gamma (x - mean) rstd + beta;   mean and rstd over a run of channels and all pixels of a sample
//   dv = dy act'(v);  dbeta = sum dv;  dgamma = sum dv xhat;  xhat = (x - mean) rstd
//   dx = rstd (gamma dv - S1 / m - xhat S2 / m),  S1 = sum gamma dv, S2 = sum gamma dv xhat over the group's m elements
//
// What bounds it: memory, two arrays forward and three backward, if a sample is read once.
//
// A block works on a slice of channels, whole groups or a part of one large group, and a slab of pixels; a thread keeps to W neighbouring
// channels of it and goes down the rows, so that gamma, beta and the statistics stay in registers.  Means and sums of squared
// deviations are merged in pairs of parts (Chan, Golub and LeVeque's update), never taken as a difference of large sums.
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

// sigma(v) for the activation and its derivative; storage in bf16 hides the faster exponential's error
template <class T> __device__ __forceinline__ float logistic(float v) { return __fdividef(1.f, 1.f + (sizeof(T) == 2 ? __expf(-v) : expf(-v))); }
template <class T> __device__ __forceinline__ float act(float v, int kind) {
  if (kind == PAAC_ACT_RELU) return v < 0.f ? 0.f : v;                       // a NaN stays one
  if (kind == PAAC_ACT_SILU) return v * logistic<T>(v);
  return v;
}
template <class T> __device__ __forceinline__ float act_slope(float v, int kind) {
  if (kind == PAAC_ACT_RELU) return v > 0.f ? 1.f : 0.f;
  if (kind == PAAC_ACT_SILU) { const float s = logistic<T>(v); return s * fmaf(v, 1.f - s, 1.f); }
  return 1.f;
}

template <class T, int W> __device__ __forceinline__ void act_all(float (&v)[W], int kind) {
  if (kind == PAAC_ACT_NONE) return;
#pragma unroll
  for (int j = 0; j < W; ++j) v[j] = act<T>(v[j], kind);
}
// d <- d act'(v)
template <class T, int W> __device__ __forceinline__ void slope_all(float (&d)[W], const float (&v)[W], int kind) {
  if (kind == PAAC_ACT_NONE) return;
#pragma unroll
  for (int j = 0; j < W; ++j) d[j] *= act_slope<T>(v[j], kind);
}

// rows that row lane r of R takes of a slab
__device__ __forceinline__ int rows_of(int rows, int r, int R) { return rows > r ? (rows - r + R - 1) / R : 0; }

// Statistics of one of the block's groups from those of its threads: entry (r, q) of `mean` and `m2` (q < cols) stands for `each`
// elements of each of rows_of(rows, r, R) rows.  A warp takes a group; the result is in every lane.
struct Stats { float n, mean, m2; };
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ Stats merge_group(const float* mean, const float* m2, int R, int cols, int first, int width, int rows, int each, int lane) {
  float s = 0.f, k = 0.f;
  for (int i = lane; i < R * width; i += 32) {
    const int r = i / width, q = first + i - r * width;
    const float cnt = (float)(rows_of(rows, r, R) * each);
    s = fmaf(cnt, mean[r * cols + q], s);
    k += cnt;
  }
  const float n = warp_sum(k), m = n > 0.f ? warp_sum(s) / n : 0.f;
  float d2 = 0.f;
  for (int i = lane; i < R * width; i += 32) {
    const int r = i / width, q = first + i - r * width;
    const float cnt = (float)(rows_of(rows, r, R) * each), d = mean[r * cols + q] - m;
    d2 += fmaf(cnt * d, d, m2[r * cols + q]);
  }
  return Stats{n, m, warp_sum(d2)};
}

// ---- samples that stay on chip: one read ---------------------------------------------------------------------------------------------------
//
// A block, or a cluster of up to MAX_CLUSTER blocks with neighbouring slabs of pixels, holds a slice of a sample in registers, K accesses a
// thread (of x, and of dy), between the read and the write.  Statistics are merged through shared memory, and through that of the
// other blocks in a cluster.  A block goes on to the next sample that is its own; what it has of dgamma and dbeta stays with it until the
// end.  Several blocks share a multiprocessor, so that one reads while another writes.
constexpr int MAX_CLUSTER = 16, MAX_GROUPS = 32, MAX_WIDTH = 512;           // groups and channels of a slice
// rows of the slab of block `rank`
__device__ __forceinline__ int slab_of(int pixels, int slab, int rank) { const int left = pixels - rank * slab; return left < 0 ? 0 : (left < slab ? left : slab); }

// A value pair per group from every block of the cluster; the barrier lies between put() and get().
struct Exchange {
  float2 of_block[2][MAX_CLUSTER][MAX_GROUPS];
  __device__ __forceinline__ void put(int parity, int rank, int cluster, int g, float2 v, int lane) {
    if (lane < cluster) paac::store_in_block(&of_block[parity][rank][g], lane, v);
  }
};

// PER_CHANNEL: an access lies across groups, and statistics are kept by channel; else by access.
template <class T, int W, int K, bool PER_CHANNEL>
__global__ void __launch_bounds__(TB, 2) resident_kernel(const __grid_constant__ Args a, int cluster, int slab, int stride) {
  constexpr int NV = PER_CHANNEL ? W : 1, EACH = W / NV;
  __shared__ float sm[TB * NV], sq[TB * NV];
  __shared__ float2 stat[MAX_GROUPS];
  __shared__ Exchange ex;
  const Geo& q = a.q;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int rank = paac::cluster_rank(), id = blockIdx.x / cluster, slice = id % q.slices;
  const Slice s = slice_of(q, slice);
  const int cv = s.width / W, R = blockDim.x / cv, r = threadIdx.x / cv, v = threadIdx.x - r * cv, cols = cv * NV, wide = q.cg / EACH;
  const int rows = slab_of(q.pixels, slab, rank), cnt = r < R ? rows_of(rows, r, R) : 0, c = s.c0 + v * W;
  if (cluster > 1) paac::cluster_arrive();                  // nobody stores into a block that has not begun
  paac::pdl_entry();
  bool begun = cluster == 1;
  int parity = 0;
  for (int64_t n = id / q.slices; n < q.n; n += stride, parity ^= 1) {
    Pack<T, W> x[K];
    const T* p = at<const T>(a.x, n, (int64_t)rank * slab + r, c);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (k < cnt) x[k].load(p + (int64_t)k * R * a.x.pixel); else x[k].zero();
    }
    float m[NV], d2[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) m[j] = d2[j] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {                           // (what is not there is 0)
      float f[W];
      x[k].widen(f);
#pragma unroll
      for (int j = 0; j < W; ++j) m[j % NV] += f[j];
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) m[j] = cnt > 0 ? m[j] / (float)(cnt * EACH) : 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float f[W];
      x[k].widen(f);
      if (k < cnt) {
#pragma unroll
        for (int j = 0; j < W; ++j) { const float d = f[j] - m[j % NV]; d2[j % NV] = fmaf(d, d, d2[j % NV]); }
      }
    }
    if (r < R) {
#pragma unroll
      for (int j = 0; j < NV; ++j) { sm[r * cols + v * NV + j] = m[j]; sq[r * cols + v * NV + j] = d2[j]; }
    }
    __syncthreads();
    if (!begun) { paac::cluster_wait(); begun = true; }
    for (int g = warp; g < s.groups; g += warps) {
      const Stats t = merge_group(sm, sq, R, cols, g * wide, wide, rows, EACH, lane);
      if (cluster > 1) ex.put(parity, rank, cluster, g, make_float2(t.mean, t.m2), lane);
      else if (lane == 0) {
        const float rs = 1.f / sqrtf(t.m2 / t.n + a.eps);
        stat[g] = make_float2(t.mean, rs);
        if (a.mean_out != nullptr) a.mean_out[n * q.groups + s.g0 + g] = t.mean;
        if (a.rstd_out != nullptr) a.rstd_out[n * q.groups + s.g0 + g] = rs;
      }
    }
    if (cluster > 1) {
      paac::cluster_arrive();
      paac::cluster_wait();
      if (threadIdx.x < s.groups) {
        const int g = threadIdx.x;
        float sum = 0.f, d = 0.f;
        for (int b = 0; b < cluster; ++b) sum = fmaf((float)slab_of(q.pixels, slab, b), ex.of_block[parity][b][g].x, sum);
        const float mean = sum / (float)q.pixels;
        for (int b = 0; b < cluster; ++b) {
          const float2 e = ex.of_block[parity][b][g];
          const float off = e.x - mean;
          d += fmaf((float)slab_of(q.pixels, slab, b) * (float)q.cg * off, off, e.y);
        }
        const float rs = 1.f / sqrtf(d / ((float)q.pixels * (float)q.cg) + a.eps);
        stat[g] = make_float2(mean, rs);
        if (rank == 0 && a.mean_out != nullptr) a.mean_out[n * q.groups + s.g0 + g] = mean;
        if (rank == 0 && a.rstd_out != nullptr) a.rstd_out[n * q.groups + s.g0 + g] = rs;
      }
    }
    __syncthreads();
    float gamma[W], beta[W], mean[NV], rstd[NV];
    if (cnt > 0) {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        gamma[j] = a.gamma != nullptr ? a.gamma[c + j] : 1.f;
        beta[j] = a.beta != nullptr ? a.beta[c + j] : 0.f;
      }
#pragma unroll
      for (int j = 0; j < NV; ++j) { const float2 t = stat[(v * W + j) / q.cg]; mean[j] = t.x; rstd[j] = t.y; }
    }
    T* to = at<T>(a.out, n, (int64_t)rank * slab + r, c);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (k < cnt) {
        float f[W];
        x[k].widen(f);
#pragma unroll
        for (int j = 0; j < W; ++j) f[j] = fmaf((f[j] - mean[j % NV]) * rstd[j % NV], gamma[j], beta[j]);
        act_all<T, W>(f, a.activation);
        x[k].round(f);
        x[k].store(to + (int64_t)k * R * a.out.pixel);
      }
    }
  }
  if (!begun) paac::cluster_wait();
}

template <class T, int W, int K, bool PER_CHANNEL>
__global__ void __launch_bounds__(TB, 2) resident_back_kernel(const __grid_constant__ Args a, int cluster, int slab, int stride, float* sums /* [rows][2][c] */) {
  constexpr int NV = PER_CHANNEL ? W : 1;
  __shared__ __align__(16) float sb[TB * W], sg[TB * W];    // by row lane and channel
  __shared__ float tb[MAX_WIDTH], tg[MAX_WIDTH], all_b[MAX_WIDTH], all_g[MAX_WIDTH];      // by channel: of this sample, of all samples
  __shared__ float2 stat[MAX_GROUPS];
  __shared__ Exchange ex;
  const Geo& q = a.q;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int rank = paac::cluster_rank(), id = blockIdx.x / cluster, slice = id % q.slices;
  const Slice s = slice_of(q, slice);
  const int cv = s.width / W, R = blockDim.x / cv, r = threadIdx.x / cv, v = threadIdx.x - r * cv;
  const int rows = slab_of(q.pixels, slab, rank), cnt = r < R ? rows_of(rows, r, R) : 0, c = s.c0 + v * W;
  const int P = blockDim.x / s.width > 1 ? (blockDim.x / s.width < R ? blockDim.x / s.width : R) : 1;      // threads a channel is added up by
  const float count = (float)q.pixels * (float)q.cg;
  if (cluster > 1) paac::cluster_arrive();
  paac::pdl_entry();
  for (int i = threadIdx.x; i < s.width; i += blockDim.x) all_b[i] = all_g[i] = 0.f;
  float gamma[W], beta[W];
  if (cnt > 0) {
#pragma unroll
    for (int j = 0; j < W; ++j) {
      gamma[j] = a.gamma != nullptr ? a.gamma[c + j] : 1.f;
      beta[j] = a.beta != nullptr ? a.beta[c + j] : 0.f;
    }
  }
  bool begun = cluster == 1;
  int parity = 0;
  for (int64_t n = id / q.slices; n < q.n; n += stride, parity ^= 1) {
    Pack<T, W> x[K], d[K];
    float mean[NV], rstd[NV], db[W], dg[W];
    const int64_t row = (int64_t)rank * slab + r;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (k < cnt) {
        x[k].load(at<const T>(a.x, n, row + (int64_t)k * R, c));
        d[k].load(at<const T>(a.dy, n, row + (int64_t)k * R, c));
      }
    }
    if (cnt > 0) {
#pragma unroll
      for (int j = 0; j < NV; ++j) { const int64_t g = n * q.groups + (c + j) / q.cg; mean[j] = a.mean[g]; rstd[j] = a.rstd[g]; }
    }
#pragma unroll
    for (int j = 0; j < W; ++j) db[j] = dg[j] = 0.f;
    // xhat and dv of access k
    auto derive = [&](int k, float (&xh)[W], float (&dv)[W]) {
      float arg[W];
      x[k].widen(xh);
      d[k].widen(dv);
#pragma unroll
      for (int j = 0; j < W; ++j) { xh[j] = (xh[j] - mean[j % NV]) * rstd[j % NV]; arg[j] = fmaf(xh[j], gamma[j], beta[j]); }
      slope_all<T, W>(dv, arg, a.activation);
    };
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (k < cnt) {
        float xh[W], dv[W];
        derive(k, xh, dv);
#pragma unroll
        for (int j = 0; j < W; ++j) { db[j] += dv[j]; dg[j] = fmaf(dv[j], xh[j], dg[j]); }
      }
    }
    if (r < R) {
      paac::store_floats(&sb[r * s.width + v * W], db);
      paac::store_floats(&sg[r * s.width + v * W], dg);
    }
    __syncthreads();
    // over the row lanes: P threads a channel, each leaving its sum where it began
    for (int i = threadIdx.x; i < s.width * P; i += blockDim.x) {
      const int part = i / s.width, ch = i - part * s.width;
      float b = 0.f, g = 0.f;
      for (int k = part; k < R; k += P) { b += sb[k * s.width + ch]; g += sg[k * s.width + ch]; }
      sb[i] = b;
      sg[i] = g;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < s.width; i += blockDim.x) {
      float b = 0.f, g = 0.f;
      for (int k = 0; k < P; ++k) { b += sb[k * s.width + i]; g += sg[k * s.width + i]; }
      tb[i] = b; tg[i] = g;
      all_b[i] += b; all_g[i] += g;
    }
    if (a.out.data == nullptr) { __syncthreads(); continue; }
    __syncthreads();
    if (!begun) { paac::cluster_wait(); begun = true; }
    for (int g = warp; g < s.groups; g += warps) {
      float s1 = 0.f, s2 = 0.f;
      for (int i = lane; i < q.cg; i += 32) {
        const int ch = g * q.cg + i;
        const float w = a.gamma != nullptr ? a.gamma[s.c0 + ch] : 1.f;
        s1 = fmaf(w, tb[ch], s1);
        s2 = fmaf(w, tg[ch], s2);
      }
      s1 = warp_sum(s1);
      s2 = warp_sum(s2);
      if (cluster > 1) ex.put(parity, rank, cluster, g, make_float2(s1, s2), lane);
      else if (lane == 0) stat[g] = make_float2(s1 / count, s2 / count);
    }
    if (cluster > 1) {
      paac::cluster_arrive();
      paac::cluster_wait();
      if (threadIdx.x < s.groups) {
        float s1 = 0.f, s2 = 0.f;
        for (int b = 0; b < cluster; ++b) { const float2 e = ex.of_block[parity][b][threadIdx.x]; s1 += e.x; s2 += e.y; }
        stat[threadIdx.x] = make_float2(s1 / count, s2 / count);
      }
    }
    __syncthreads();
    if (cnt > 0) {
      float s1[NV], s2[NV];
#pragma unroll
      for (int j = 0; j < NV; ++j) { const float2 t = stat[(v * W + j) / q.cg]; s1[j] = t.x; s2[j] = t.y; }
#pragma unroll
      for (int k = 0; k < K; ++k) {
        if (k < cnt) {
          float xh[W], dv[W];
          derive(k, xh, dv);
#pragma unroll
          for (int j = 0; j < W; ++j) dv[j] = rstd[j % NV] * (fmaf(gamma[j], dv[j], -s1[j % NV]) - xh[j] * s2[j % NV]);
          x[k].round(dv);
          x[k].store(at<T>(a.out, n, row + (int64_t)k * R, c));
        }
      }
    }
  }
  if (!begun) paac::cluster_wait();
  if (sums == nullptr) return;
  float* to = sums + ((int64_t)(id / q.slices) * cluster + rank) * 2 * q.c + s.c0;
  for (int i = threadIdx.x; i < s.width; i += blockDim.x) { to[i] = all_b[i]; to[q.c + i] = all_g[i]; }
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
      const Stats t = merge_group(sm, sq, R, s.width, g * width, width, rows, 1, threadIdx.x & 31);
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
      for (int j = 0; j < W; ++j) x[j] = act<T>(ch.argument(j, x[j]), a.activation);
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
#pragma unroll
        for (int j = 0; j < W; ++j) {
          const float dv = d[j] * act_slope<T>(ch.argument(j, x[j]), a.activation);
          db[j] += dv;
          dg[j] = fmaf(dv, (x[j] - ch.mean[j]) * ch.rstd[j], dg[j]);
        }
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
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float dv = d[j] * act_slope<T>(ch.argument(j, x[j]), a.activation), xhat = (x[j] - ch.mean[j]) * ch.rstd[j];
        x[j] = ch.rstd[j] * (fmaf(ch.gamma[j], dv, -s1[j]) - xhat * s2[j]);
      }
      px.round(x);
      px.store(at<T>(a.out, n, p0 + k, s.c0 + v * W));
    }
  }
}

// dgamma and dbeta: the rows of `sums` added up, 32 channels a block
constexpr int CHANNEL_LANES = 32, ROW_LANES = 32;
__global__ void __launch_bounds__(CHANNEL_LANES * ROW_LANES)
channel_sums_kernel(const float* sums /* [rows][2][c] */, int64_t rows, int c, float* dgamma, float* dbeta) {
  __shared__ float sh[ROW_LANES][CHANNEL_LANES + 1];
  paac::pdl_entry();
  const int lane = threadIdx.x % CHANNEL_LANES, r = threadIdx.x / CHANNEL_LANES;
  const int64_t col = (int64_t)blockIdx.x * CHANNEL_LANES + lane;           // of 2 c: dbeta, then dgamma
  float s = 0.f;
  if (col < 2 * (int64_t)c) {
#pragma unroll 4
    for (int64_t k = r; k < rows; k += ROW_LANES) s += sums[k * 2 * c + col];
  }
  sh[r][lane] = s;
  __syncthreads();
  if (r == 0 && col < 2 * (int64_t)c) {
    float t = 0.f;
    for (int k = 0; k < ROW_LANES; ++k) t += sh[k][lane];
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
  q.slabs = (q.pixels + q.slab_rows - 1) / q.slab_rows;
}

// How the resident kernels take a shape, if they do: `q` with slices of whole groups, blocks of `threads` with `rows` pixels each, K accesses a
// thread, clusters of `cluster` blocks.
struct Resident { Geo q; int cluster, slab, threads, K; };
bool resident(const Geo& whole, int W, Resident& out) {
  Geo q = whole;
  const int unit = W / gcd(q.cg, W), size = W == 1 ? 1 : 16 / W;            // groups between two slices' beginnings; (bytes of an element, if wide)
  int gps = q.groups;
  auto fits = [&](int groups) { return groups <= MAX_GROUPS && groups * q.cg <= MAX_WIDTH && groups * q.cg / W <= TB; };
  auto narrower = [&](int groups) { const int half = (groups / 2 + unit - 1) / unit * unit; return half >= 1 && half < groups ? half : 0; };
  if (q.c % W != 0) return false;
  while (gps != 0 && !fits(gps)) gps = narrower(gps);
  // the widest slice that up to 8 blocks hold; then the widest that 16 do; rows of less than 32 bytes would be read twice
  for (int most = 8; most <= MAX_CLUSTER; most *= 2)
    for (int g = gps; g != 0 && (g == gps || g * q.cg * size >= 32); g = narrower(g)) {
      const int cv = g * q.cg / W, R = TB / cv;
      int cluster = 1;
      while (cluster < most && (int64_t)R * 8 * cluster < q.pixels) cluster *= 2;
      if ((int64_t)R * 8 * cluster < q.pixels) continue;
      q.gps = g; q.parts = 1; q.cap = TB * W;
      q.slices = (q.groups + g - 1) / g;
      // few samples: more blocks each, down to two rows a thread
      while (cluster < 8 && (int64_t)q.n * q.slices * cluster * 2 <= 148 && q.pixels >= (int64_t)R * 2 * cluster) cluster *= 2;
      const int slab = (q.pixels + cluster - 1) / cluster;
      // small slabs: fewer threads, so that each has some rows
      int threads = TB;
      while (threads > 64 && threads / 2 >= cv && (slab + threads / 2 / cv - 1) / (threads / 2 / cv) <= 4) threads /= 2;
      const int per = (slab + threads / cv - 1) / (threads / cv);
      out = Resident{q, cluster, slab, threads, per <= 2 ? 2 : (per <= 4 ? 4 : 8)};
      return true;
    }
  return false;
}
// clusters that a slice's samples are dealt out to in the backward pass
int dealt(const Resident& r) {
  const int most = 148 * 4 / (r.q.slices * r.cluster);
  return r.q.n < most ? r.q.n : (most < 1 ? 1 : most);
}

bool shape_ok(const paac_norm* s) {
  return s != nullptr && s->n >= 1 && s->pixels >= 1 && s->c >= 1 && s->groups >= 1 && s->c <= 65536 && s->c % s->groups == 0 &&
         (int64_t)s->n * s->groups < ((int64_t)1 << 31) && (int64_t)s->n * s->pixels < ((int64_t)1 << 31) &&
         (s->type == PAAC_FP32 || s->type == PAAC_BF16) && s->activation >= PAAC_ACT_NONE && s->activation <= PAAC_ACT_SILU && s->eps > 0.f;
}
// accesses of 16 bytes where rows and groups allow them, else of one element
Geo geometry(const paac_norm& s, bool wide, int& W) {
  Geo q{};
  q.n = s.n; q.pixels = s.pixels; q.c = s.c; q.groups = s.groups; q.cg = s.c / s.groups;
  W = s.type == PAAC_BF16 ? 8 : 4;
  if (!wide || !cut(q, W)) { W = 1; cut(q, 1); }
  cut_rows(q, W);
  return q;
}
size_t round_up(size_t v) { return (v + 255) / 256 * 256; }
struct Scratch { size_t first, second, total; };
// first: partial statistics or sums of a slab; second: statistics or sums of a group
Scratch scratch(const Geo& q, int W) {
  const size_t stats = (size_t)q.n * q.groups * q.slabs * q.parts * sizeof(float2), sums = (size_t)q.n * q.slabs * 2 * q.c * sizeof(float);
  Scratch s;
  s.first = round_up(stats > sums ? stats : sums);
  Resident r;
  if (resident(q, W, r)) {
    const size_t dealt_sums = round_up((size_t)dealt(r) * r.cluster * 2 * q.c * sizeof(float));
    if (dealt_sums > s.first) s.first = dealt_sums;
  }
  s.second = round_up((size_t)q.n * q.groups * sizeof(float2));
  s.total = s.first + s.second;
  return s;
}

size_t scratch_bytes(const paac_norm& s, bool wide) {
  int W;
  const Geo q = geometry(s, wide, W);
  return scratch(q, W).total;
}

View view(const paac_rows& r, const paac_norm& s) { return View{r.data, s.n > 1 ? r.outer : 0, s.pixels > 1 ? r.inner : 0}; }
unsigned blocks(int64_t units, int most) { return (unsigned)(units < most ? units : most); }

struct Check {
  const paac_norm& s;
  int size;
  bool ok = true, wide = true;
  explicit Check(const paac_norm& s_) : s(s_), size(s_.type == PAAC_BF16 ? 2 : 4) {}
  paac::RowSet rows(const paac_rows& r, bool out) {
    const paac::RowSet set(r, s.n, s.pixels, s.c, size);
    if (r.data == nullptr || !set.sane() || !set.aligned() || (out && !set.rows_apart())) ok = false;
    else wide = wide && set.multiples_of(16);
    return set;
  }
  void floats(const float* p) { if ((uintptr_t)p & 3u) ok = false; }
};

template <class K> bool allow_clusters(K kernel, bool& done) {
  return done = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
}
// a function's attributes belong to the current device, and these entry points work on any
template <class... KArgs, class... Args> cudaError_t launch_resident(paac::PerDevice<bool>& ready, void (*kernel)(KArgs...), const Resident& r, int64_t clusters,
                                                                     cudaStream_t s, Args... args) {
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess || ready.get(device, [&](bool& done) { return allow_clusters(kernel, done); }) == nullptr) return cudaErrorUnknown;
  return paac::launch_clusters_on(s, kernel, dim3((unsigned)(clusters * r.cluster)), dim3(r.threads), r.cluster, args...);
}

constexpr int64_t MOST_CLUSTERS = 1 << 16;
template <class T, int W, int K, bool PER_CHANNEL> cudaError_t forward_k(const Args& a, const Resident& r, cudaStream_t s) {
  static paac::PerDevice<bool> ready;
  const int64_t most = MOST_CLUSTERS / r.q.slices + 1, deal = r.q.n < most ? r.q.n : most;
  return launch_resident(ready, resident_kernel<T, W, K, PER_CHANNEL>, r, deal * r.q.slices, s, a, r.cluster, r.slab, (int)deal);
}
template <class T, int W, int K, bool PER_CHANNEL> cudaError_t backward_k(const Args& a, const Resident& r, float* sums, cudaStream_t s) {
  static paac::PerDevice<bool> ready;
  const int deal = dealt(r);
  return launch_resident(ready, resident_back_kernel<T, W, K, PER_CHANNEL>, r, (int64_t)deal * r.q.slices, s, a, r.cluster, r.slab, deal, sums);
}
template <class T, int W, bool PER_CHANNEL> cudaError_t forward_resident(const Args& a, const Resident& r, cudaStream_t s) {
  return r.K == 2 ? forward_k<T, W, 2, PER_CHANNEL>(a, r, s) : r.K == 4 ? forward_k<T, W, 4, PER_CHANNEL>(a, r, s) : forward_k<T, W, 8, PER_CHANNEL>(a, r, s);
}
template <class T, int W, bool PER_CHANNEL> cudaError_t backward_resident(const Args& a, const Resident& r, float* sums, cudaStream_t s) {
  return r.K == 2 ? backward_k<T, W, 2, PER_CHANNEL>(a, r, sums, s)
                  : r.K == 4 ? backward_k<T, W, 4, PER_CHANNEL>(a, r, sums, s) : backward_k<T, W, 8, PER_CHANNEL>(a, r, sums, s);
}

template <class T, int W> cudaError_t forward(Args a, float2* partial, cudaStream_t s) {
  Resident r;
  if (resident(a.q, W, r)) {
    a.q = r.q;
    if (W > 1 && a.q.cg % W != 0) return forward_resident<T, W, (W > 1)>(a, r, s);
    return forward_resident<T, W, false>(a, r, s);
  }
  const Geo& q = a.q;
  const int64_t units = (int64_t)q.n * q.slabs * q.slices, groups = (int64_t)q.n * q.groups;
  cudaError_t e = paac::launch_overlapped_on(s, stats_kernel<T, W>, dim3(blocks(units, GRID)), dim3(TB), 0, a, partial);
  if (e != cudaSuccess) return e;
  e = paac::launch_overlapped_on(s, finish_stats_kernel, dim3(blocks((groups + WARPS - 1) / WARPS, GRID)), dim3(TB), 0, q, (const float2*)partial, a.eps,
                                 a.mean_out, a.rstd_out);
  if (e != cudaSuccess) return e;
  return paac::launch_overlapped_on(s, apply_kernel<T, W>, dim3(blocks(units, GRID)), dim3(TB), 0, a);
}
template <class T, int W> cudaError_t backward(Args a, float* sums, float2* group_sums, float* dgamma, float* dbeta, cudaStream_t s) {
  Resident r;
  const bool wanted = dgamma != nullptr || dbeta != nullptr;
  int64_t rows;
  cudaError_t e;
  if (resident(a.q, W, r)) {
    a.q = r.q;
    rows = (int64_t)dealt(r) * r.cluster;
    float* to = wanted ? sums : nullptr;
    e = W > 1 && a.q.cg % W != 0 ? backward_resident<T, W, (W > 1)>(a, r, to, s) : backward_resident<T, W, false>(a, r, to, s);
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

extern "C" size_t paac_group_norm_workspace_bytes(const paac_norm* s) {
  if (!shape_ok(s)) return 0;
  const size_t a = scratch_bytes(*s, true), b = scratch_bytes(*s, false);
  return a > b ? a : b;
}

extern "C" int paac_group_norm(const paac_norm* s, paac_rows x, const float* gamma, const float* beta, paac_rows y, float* mean, float* rstd,
                               void* workspace, size_t workspace_bytes, void* stream) {
  if (!shape_ok(s)) return PAAC_ERR_ARG;
  Check check(*s);
  const paac::RowSet xs = check.rows(x, false), ys = check.rows(y, true);
  check.floats(gamma); check.floats(beta); check.floats(mean); check.floats(rstd);
  if (!check.ok || (!ys.same_as(xs) && !ys.apart_from(xs))) return PAAC_ERR_ARG;
  if (workspace == nullptr || ((uintptr_t)workspace & 15u) != 0 || workspace_bytes < paac_group_norm_workspace_bytes(s)) return PAAC_ERR_WORKSPACE;
  int W;
  Args a{};
  a.q = geometry(*s, check.wide, W);
  const Scratch room = scratch(a.q, W);
  a.x = view(x, *s); a.out = view(y, *s);
  a.gamma = gamma; a.beta = beta; a.activation = s->activation; a.eps = s->eps;
  float* own = reinterpret_cast<float*>((char*)workspace + room.first);
  a.mean_out = mean != nullptr ? mean : own;
  a.rstd_out = rstd != nullptr ? rstd : own + (int64_t)s->n * s->groups;
  a.mean = a.mean_out; a.rstd = a.rstd_out;
  float2* partial = static_cast<float2*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (s->type == PAAC_BF16) e = W == 8 ? forward<bf16, 8>(a, partial, st) : forward<bf16, 1>(a, partial, st);
  else e = W == 4 ? forward<float, 4>(a, partial, st) : forward<float, 1>(a, partial, st);
  return paac::launch_status(e);
}

extern "C" int paac_group_norm_backward(const paac_norm* s, paac_rows x, paac_rows dy, const float* gamma, const float* beta, const float* mean,
                                        const float* rstd, paac_rows dx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                                        void* stream) {
  if (!shape_ok(s) || mean == nullptr || rstd == nullptr) return PAAC_ERR_ARG;
  if (dx.data == nullptr && dgamma == nullptr && dbeta == nullptr) return PAAC_ERR_ARG;
  Check check(*s);
  const paac::RowSet xs = check.rows(x, false), ds = check.rows(dy, false);
  check.floats(gamma); check.floats(beta); check.floats(mean); check.floats(rstd); check.floats(dgamma); check.floats(dbeta);
  if (dx.data != nullptr) {
    const paac::RowSet os = check.rows(dx, true);
    if (check.ok && (!os.apart_from(xs) || (!os.same_as(ds) && !os.apart_from(ds)))) check.ok = false;
  }
  if (!check.ok) return PAAC_ERR_ARG;
  if (workspace == nullptr || ((uintptr_t)workspace & 15u) != 0 || workspace_bytes < paac_group_norm_workspace_bytes(s)) return PAAC_ERR_WORKSPACE;
  int W;
  Args a{};
  a.q = geometry(*s, check.wide, W);
  const Scratch room = scratch(a.q, W);
  a.x = view(x, *s); a.dy = view(dy, *s); a.out = view(dx, *s);
  a.gamma = gamma; a.beta = beta; a.mean = mean; a.rstd = rstd; a.activation = s->activation; a.eps = s->eps;
  float* sums = static_cast<float*>(workspace);
  float2* group_sums = reinterpret_cast<float2*>((char*)workspace + room.first);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (s->type == PAAC_BF16) e = W == 8 ? backward<bf16, 8>(a, sums, group_sums, dgamma, dbeta, st) : backward<bf16, 1>(a, sums, group_sums, dgamma, dbeta, st);
  else e = W == 4 ? backward<float, 4>(a, sums, group_sums, dgamma, dbeta, st) : backward<float, 1>(a, sums, group_sums, dgamma, dbeta, st);
  return paac::launch_status(e);
}
