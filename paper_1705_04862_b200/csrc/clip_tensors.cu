// The global L2 norm over many tensors, and their clipping (paac_clip_tensors).
//
//   norm = sqrt(sum src^2), factor = min(1, clip / norm), dst = factor * src
//
// What bounds it: memory for large lists, launches for small ones.  The factor is known only when everything has been read, so there are
// two passes: the first reads every src and leaves one partial sum a block; the second reads it again, from L2 as far as that
// reaches, and writes.  Blocks of the second pass go through the list from its end, where the first pass has just been, and one
// whose tensors are in place has nothing to do where the factor is 1.
//
// The list goes to the kernels as their argument (no copy to the device, nothing to keep alive for a captured graph), a table of
// up to MAX_TABLE tensors a launch.  Work is cut into tiles of 16 KB of src, counted through the whole table; a block takes a run of
// neighbouring tiles and finds the tensor of its first one by bisection.  Tiles begin on 16-byte boundaries of src wherever the
// tensor does: the first one is short by what is missing.
//
// Accuracy and range: 16 or 32 neighbouring squares of a thread are added up in float, those sums in double, in an order that does not change from
// run to run.  Where the largest of them is beyond 1e15 or below 1e-15 the squares themselves could leave the range of float, and
// are taken in double.
#include <algorithm>
#include <new>

#include "common.cuh"

namespace {
using paac::bf16;

constexpr int TILE_BYTES = 16384, THREADS = 256;
constexpr int MAX_COUNT = 65536, MAX_TABLE = 1024, SMALL_TABLE = 96;
constexpr uint64_t MAX_BYTES = (uint64_t)1 << 45;
constexpr int SUM_BLOCKS = 148 * 8, WRITE_BLOCKS = 148 * 8;

// A table's tensors: first_tile[i] counts the tiles before tensor i; entry `count` is the total.
template <int CAP> struct Table {
  const void* src[CAP];
  void* dst[CAP];
  uint64_t n[CAP];
  uint32_t first_tile[CAP + 1];
  uint8_t types[CAP];            // bit 0: src is bf16, bit 1: dst is bf16
  int count;
};

template <class Tab> __device__ __forceinline__ int tensor_of(const Tab& tab, uint32_t tile) {
  int lo = 0, hi = tab.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (tab.first_tile[mid] <= tile) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// elements [first, end) of a tensor that tile `k` of it covers; whole 16-byte words but for the two ends of the tensor
struct Span { int64_t first, end; };
__device__ __forceinline__ Span span_of(const void* src, uint64_t n, int size, uint32_t k) {
  const int64_t per = TILE_BYTES / size, missing = ((uintptr_t)src & 15u) / size;
  Span s{(int64_t)k * per - missing, ((int64_t)k + 1) * per - missing};
  if (s.first < 0) s.first = 0;
  if (s.end > (int64_t)n) s.end = (int64_t)n;
  return s;
}

// 16 bytes as floats
__device__ __forceinline__ void widen(const uint4& w, float (&v)[4]) {
  v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ void widen(const uint4& w, float (&v)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(u[i] << 16); v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u); }
}

constexpr float LARGE = 1e15f, SMALL = 1e-15f;

template <class T> __device__ __forceinline__ double square(T v) { const double d = (double)paac::to_f(v); return d * d; }

// sum of squares of the thread's share of a span
template <class T> __device__ double span_squares(const T* src, Span s) {
  constexpr int W = 16 / (int)sizeof(T), AHEAD = TILE_BYTES / 16 / THREADS;
  double acc = 0.0;
  // the ends that are not whole words
  const int64_t head = ((16 - ((uintptr_t)(src + s.first) & 15u)) & 15u) / sizeof(T);
  const int64_t a = s.first + head < s.end ? s.first + head : s.end, words = (s.end - a) / W;
  if (threadIdx.x < a - s.first) acc += square(src[s.first + threadIdx.x]);
  if (threadIdx.x < s.end - (a + words * W)) acc += square(src[a + words * W + threadIdx.x]);
  const uint4* p = reinterpret_cast<const uint4*>(src + a);
  uint4 w[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    const int i = threadIdx.x + u * THREADS;
    w[u] = i < words ? __ldg(p + i) : make_uint4(0, 0, 0, 0);
  }
  float sum = 0.f, most = 0.f;
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    float v[W];
    widen(w[u], v);
#pragma unroll
    for (int j = 0; j < W; ++j) { sum = fmaf(v[j], v[j], sum); most = fmaxf(most, fabsf(v[j])); }
  }
  // most is no NaN; a NaN among the values is in sum, and stays
  if (most < LARGE && (most > SMALL || most == 0.f)) return acc + (double)sum;
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    float v[W];
    widen(w[u], v);
#pragma unroll
    for (int j = 0; j < W; ++j) acc += (double)v[j] * (double)v[j];
  }
  return acc;
}

// the same sum in every thread, added up in the same order
__device__ __forceinline__ double block_total(double v, double* sh /* [THREADS / 32] */) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) t += sh[w];
  return t;
}

template <class Tab>
__global__ void __launch_bounds__(THREADS)
squares_kernel(const __grid_constant__ Tab tab, double* partials) {
  __shared__ double sh[THREADS / 32];
  paac::pdl_entry();
  const uint32_t tiles = tab.first_tile[tab.count];
  uint32_t k = (uint32_t)((uint64_t)tiles * blockIdx.x / gridDim.x);
  const uint32_t end = (uint32_t)((uint64_t)tiles * (blockIdx.x + 1) / gridDim.x);
  double acc = 0.0;
  if (k < end) {
    int i = tensor_of(tab, k);
    for (; k < end; ++k) {
      while (k >= tab.first_tile[i + 1]) ++i;
      const uint32_t own = k - tab.first_tile[i];
      if (tab.types[i] & 1) acc += span_squares((const bf16*)tab.src[i], span_of(tab.src[i], tab.n[i], 2, own));
      else acc += span_squares((const float*)tab.src[i], span_of(tab.src[i], tab.n[i], 4, own));
    }
  }
  const double t = block_total(acc, sh);
  if (threadIdx.x == 0) partials[blockIdx.x] = t;
}

// (plain loads: in place, what is read here is written here)
template <class S, class D> __device__ __forceinline__ void write_span(const S* src, D* dst, Span s, float factor) {
  constexpr int W = 8;                                  // elements a step: one or two words on either side
  const int64_t head = ((16 - ((uintptr_t)(src + s.first) & 15u)) & 15u) / sizeof(S);
  const int64_t a = s.first + head < s.end ? s.first + head : s.end;
  const bool wide = ((uintptr_t)(dst + a) & 15u) == 0;
  const int64_t steps = wide ? (s.end - a) / W : 0, rest = a + steps * W;
  if (threadIdx.x < a - s.first) dst[s.first + threadIdx.x] = paac::from_f<D>(factor * paac::to_f(src[s.first + threadIdx.x]));
  for (int64_t i = threadIdx.x; i < steps; i += THREADS) {
    float v[W];
    if constexpr (sizeof(S) == 2) {
      widen(reinterpret_cast<const uint4*>(src + a)[i], v);
    } else {
      const float4 x = reinterpret_cast<const float4*>(src + a)[2 * i], y = reinterpret_cast<const float4*>(src + a)[2 * i + 1];
      v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
    }
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] *= factor;
    if constexpr (sizeof(D) == 2) {
      __nv_bfloat162 h[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
      reinterpret_cast<uint4*>(dst + a)[i] = *reinterpret_cast<const uint4*>(h);
    } else {
      reinterpret_cast<float4*>(dst + a)[2 * i] = make_float4(v[0], v[1], v[2], v[3]);
      reinterpret_cast<float4*>(dst + a)[2 * i + 1] = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
  for (int64_t i = rest + threadIdx.x; i < s.end; i += THREADS) dst[i] = paac::from_f<D>(factor * paac::to_f(src[i]));
}

template <class Tab>
__global__ void __launch_bounds__(THREADS)
write_kernel(const __grid_constant__ Tab tab, const double* partials, int n_partials, float clip, float* norm_and_scale, int tell) {
  __shared__ double sh[THREADS / 32];
  paac::pdl_entry();
  double acc = 0.0;
  for (int i = threadIdx.x; i < n_partials; i += THREADS) acc += partials[i];
  const float norm = (float)sqrt(block_total(acc, sh));
  const bool ok = isfinite(norm);
  float factor = 1.f;
  if (ok && clip > 0.f && norm > clip) factor = clip / norm;
  if (tell && blockIdx.x == 0 && threadIdx.x == 0 && norm_and_scale != nullptr) { norm_and_scale[0] = norm; norm_and_scale[1] = ok ? factor : 0.f; }
  if (!ok) return;
  // runs of tiles from the end of the list, the last tile of a run first
  const uint32_t tiles = tab.first_tile[tab.count], b = gridDim.x - 1 - blockIdx.x;
  const uint32_t begin = (uint32_t)((uint64_t)tiles * b / gridDim.x);
  uint32_t k = (uint32_t)((uint64_t)tiles * (b + 1) / gridDim.x);
  if (k <= begin) return;
  int i = tensor_of(tab, k - 1);
  while (k-- > begin) {
    while (k < tab.first_tile[i]) --i;
    const uint32_t own = k - tab.first_tile[i];
    const void* src = tab.src[i];
    void* dst = tab.dst[i];
    if (dst == nullptr || (factor == 1.f && dst == src)) continue;
    const int types = tab.types[i];
    const Span s = span_of(src, tab.n[i], types & 1 ? 2 : 4, own);
    if (types == 0) write_span((const float*)src, (float*)dst, s, factor);
    else if (types == 1) write_span((const bf16*)src, (float*)dst, s, factor);
    else if (types == 2) write_span((const float*)src, (bf16*)dst, s, factor);
    else write_span((const bf16*)src, (bf16*)dst, s, factor);
  }
}

int element_size(int type) { return type == PAAC_BF16 ? 2 : 4; }

struct Extent { uintptr_t begin, end; bool written; };

// Whether no dst overlaps another tensor.  Lists mostly come in the order of their addresses; others are sorted first.
bool apart(Extent* e, size_t count) {
  const auto before = [](const Extent& a, const Extent& b) { return a.begin < b.begin; };
  if (!std::is_sorted(e, e + count, before)) std::sort(e, e + count, before);
  uintptr_t end = 0, written_end = 0;                   // of all before, and of the written ones among them
  for (size_t i = 0; i < count; ++i) {
    if (e[i].begin < (e[i].written ? end : written_end)) return false;
    if (e[i].end > end) end = e[i].end;
    if (e[i].written && e[i].end > written_end) written_end = e[i].end;
  }
  return true;
}

int check(const paac_tensor* t, size_t count) {
  if (count == 0) return PAAC_OK;
  Extent* e = new (std::nothrow) Extent[2 * count];
  if (e == nullptr) return PAAC_ERR_LIMIT;
  size_t k = 0;
  int status = PAAC_OK;
  uint64_t total = 0;                                   // bytes; up to MAX_BYTES the tiles of a list can be counted in 32 bits
  for (size_t i = 0; i < count; ++i) {
    const paac_tensor& x = t[i];
    if ((x.src_type != PAAC_FP32 && x.src_type != PAAC_BF16) || (x.dst_type != PAAC_FP32 && x.dst_type != PAAC_BF16)) { status = PAAC_ERR_ARG; break; }
    if (x.n == 0) continue;
    const uintptr_t src = (uintptr_t)x.src, dst = (uintptr_t)x.dst;
    const int ss = element_size(x.src_type), ds = element_size(x.dst_type);
    if (src == 0 || src % ss != 0 || dst % ds != 0 || x.n > MAX_BYTES / 4 || (total += x.n * ss) > MAX_BYTES) { status = PAAC_ERR_ARG; break; }
    if (dst == src && ds != ss) { status = PAAC_ERR_ARG; break; }
    e[k++] = Extent{src, src + x.n * ss, dst == src};
    if (dst != 0 && dst != src) e[k++] = Extent{dst, dst + x.n * ds, true};
  }
  if (status == PAAC_OK && !apart(e, k)) status = PAAC_ERR_ARG;
  delete[] e;
  return status;
}

// fills a table from tensor `at` on; returns the first tensor that found no room
template <int CAP> size_t fill(Table<CAP>& tab, const paac_tensor* t, size_t at, size_t count) {
  tab.count = 0;
  uint64_t tiles = 0;
  for (; at < count && tab.count < CAP; ++at) {
    const paac_tensor& x = t[at];
    if (x.n == 0) continue;
    const int size = element_size(x.src_type), i = tab.count++;
    tab.src[i] = x.src; tab.dst[i] = x.dst; tab.n[i] = x.n;
    tab.types[i] = (uint8_t)((x.src_type == PAAC_BF16 ? 1 : 0) | (x.dst_type == PAAC_BF16 ? 2 : 0));
    tab.first_tile[i] = (uint32_t)tiles;
    tiles += (x.n * size + ((uintptr_t)x.src & 15u) + TILE_BYTES - 1) / TILE_BYTES;
  }
  tab.first_tile[tab.count] = (uint32_t)tiles;
  return at;
}
int blocks_for(uint32_t tiles, int most) { return tiles == 0 ? 1 : tiles < (uint32_t)most ? (int)tiles : most; }

template <int CAP>
cudaError_t launch_all(const paac_tensor* t, size_t count, float clip, float* norm_and_scale, double* partials, cudaStream_t s) {
  Table<CAP> tab;
  int n_partials = 0;
  size_t at = 0;
  do {
    at = fill(tab, t, at, count);
    const int blocks = blocks_for(tab.first_tile[tab.count], SUM_BLOCKS);
    const cudaError_t e = paac::launch_overlapped_on(s, squares_kernel<Table<CAP>>, dim3(blocks), dim3(THREADS), 0, tab, partials + n_partials);
    if (e != cudaSuccess) return e;
    n_partials += blocks;
  } while (at < count);
  at = 0;
  int tell = 1;
  do {
    if (count > (size_t)CAP) at = fill(tab, t, at, count);
    else at = count;                                    // the one table is still there
    const cudaError_t e = paac::launch_overlapped_on(s, write_kernel<Table<CAP>>, dim3(blocks_for(tab.first_tile[tab.count], WRITE_BLOCKS)), dim3(THREADS), 0, tab,
                                                     (const double*)partials, n_partials, clip, norm_and_scale, tell);
    if (e != cudaSuccess) return e;
    tell = 0;
  } while (at < count);
  return cudaSuccess;
}

}  // namespace

extern "C" size_t paac_clip_tensors_workspace_bytes(size_t count) {
  if (count > (size_t)MAX_COUNT) return 0;
  return (count / MAX_TABLE + 1) * SUM_BLOCKS * sizeof(double);
}

extern "C" int paac_clip_tensors(const paac_tensor* tensors, size_t count, float clip_norm, float* norm_and_scale, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  if (tensors == nullptr && count != 0) return PAAC_ERR_ARG;
  if (count > (size_t)MAX_COUNT) return PAAC_ERR_LIMIT;
  if (clip_norm != clip_norm || ((uintptr_t)norm_and_scale & 3u) != 0) return PAAC_ERR_ARG;
  const int bad = check(tensors, count);
  if (bad != PAAC_OK) return bad;
  if (workspace == nullptr || ((uintptr_t)workspace & 15u) != 0 || workspace_bytes < paac_clip_tensors_workspace_bytes(count)) return PAAC_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  double* partials = static_cast<double*>(workspace);
  const cudaError_t e = count <= (size_t)SMALL_TABLE ? launch_all<SMALL_TABLE>(tensors, count, clip_norm, norm_and_scale, partials, s)
                                                      : launch_all<MAX_TABLE>(tensors, count, clip_norm, norm_and_scale, partials, s);
  return paac::launch_status(e);
}
