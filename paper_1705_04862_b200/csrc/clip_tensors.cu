// The global L2 norm over many tensors, and their clipping (paac_clip_tensors).
//
//   norm = sqrt(sum src^2), factor = min(1, clip / norm), dst = factor * src
//
// What bounds it: memory for large lists, launches for small ones.  The factor is known only when everything has been read, so there are
// two passes: the first reads every src and leaves one partial sum a block; the second reads it again, from L2 as far as that
// reaches, and writes.  Blocks of the second pass go through their part from its end, which the first pass has read last, and one
// whose tensors are in place has nothing to do where the factor is 1.  Where there is no more than a tile for each block of a
// cluster, one cluster does both in one launch.
//
// Measured (the kernels back to back in a graph, inputs in turn that L2 does not hold together; a copy passes at 6.5 TB/s): 1,000 floats
// 2.9 us in one cluster (4.1 in two launches); the larger network's twelve tensors, 1.7 M in bf16 into float, 8.3 us (7.5 where L2
// holds them, a call through the binding 9.2); 300 tensors of 12 M floats in place with the factor 1 15.4 us (48 MB at 3.1 TB/s: two
// launches and filling the memory's queue), scaled 34 (96 MB); 60 of 120 M in bf16 125 us, the first pass 46 of them (5.2
// TB/s) and the second 79 (433 MB at 5.4 TB/s), in place 49 with the factor 1 and 124 scaled.  Tried there: a tile's loads under way
// while the one before is written, 133 us with three blocks a multiprocessor and 188 with four (registers); five to eight blocks 148 to
// 153 (they no longer begin where L2 ends).
//
// The list goes to the kernels as their argument (no copy to the device, nothing to keep alive for a captured graph), a table of
// up to MAX_TABLE tensors a launch, which is what 32 KB of arguments hold.  Each launch copies its whole table, so there are smaller ones, each
// some four times the one before; a call on 64 tensors of 4000 floats takes 7.9 us, on 65 9.1, on 320 14.4, on 321 20.6, on 1024 34.  Work is cut into tiles of 16 KB of src, AHEAD accesses of 16 bytes for each thread, counted
// through the whole table; a block takes a run of neighbouring tiles and finds the tensor of its first one by bisection.  Tiles
// begin on 16-byte boundaries of src wherever the tensor does: the first one is short by what is missing.
//
// Accuracy and range: 16 or 32 squares of a thread are added up in float, those sums in double, in an order that does not change from
// run to run.  Where such a sum is not finite or below 1e-35 squares may have left the range of float, and are taken in double
// (what float loses of a sum above that is 32 times 2^-150 at most).
#include <algorithm>
#include <new>

#include "cluster.cuh"
#include "pack.cuh"
#include "per_device.h"

namespace {
using paac::bf16;
using paac::Pack;

constexpr int THREADS = 256, AHEAD = 4, TILE = THREADS * 16 * AHEAD, WARPS = THREADS / 32;
constexpr int MAX_COUNT = 65536, MAX_TABLE = 1024, MIDDLE_TABLE = 320, SMALL_TABLE = 64;
constexpr uint64_t MAX_BYTES = (uint64_t)1 << 43;
constexpr int PER_SM = 4, BLOCKS = 148 * PER_SM;       // blocks that are resident at once
constexpr int CLUSTER = 16;

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
  const int64_t per = TILE / size, missing = ((uintptr_t)src & 15u) / size;
  Span s{(int64_t)k * per - missing, ((int64_t)k + 1) * per - missing};
  if (s.first < 0) s.first = 0;
  if (s.end > (int64_t)n) s.end = (int64_t)n;
  return s;
}
// the words of a span: where they begin, how many there are
template <class T> struct WordsOf {
  int64_t at;
  int count;
  __device__ __forceinline__ WordsOf(const T* src, Span s) {
    const int64_t head = ((16 - ((uintptr_t)(src + s.first) & 15u)) & 15u) / sizeof(T);
    at = s.first + head < s.end ? s.first + head : s.end;
    count = (int)((s.end - at) / (int64_t)(16 / sizeof(T)));
  }
};

constexpr float MOST = 3e38f, LEAST = 1e-35f;

template <class T> __device__ __forceinline__ double square(T v) { const double d = (double)paac::to_f(v); return d * d; }

// The thread's words of a tile, whatever their type, on their way while the tile before is added up.
struct Words { uint4 w[AHEAD]; };
struct Tile {
  const void* src;
  Span s;
  int64_t at;                        // first element of the words
  int count, type;
};
template <class Tab> __device__ __forceinline__ Tile tile_of(const Tab& tab, int i, uint32_t k) {
  Tile t;
  t.src = tab.src[i];
  t.type = tab.types[i] & 1;
  t.s = span_of(t.src, tab.n[i], t.type ? 2 : 4, k - tab.first_tile[i]);
  if (t.type) { const WordsOf<bf16> words((const bf16*)t.src, t.s); t.at = words.at; t.count = words.count; }
  else { const WordsOf<float> words((const float*)t.src, t.s); t.at = words.at; t.count = words.count; }
  return t;
}
__device__ __forceinline__ void fetch(const Tile& t, Words& to) {
  const uint4* p = reinterpret_cast<const uint4*>((const char*)t.src + t.at * (t.type ? 2 : 4)) + threadIdx.x;
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) to.w[u] = threadIdx.x + u * THREADS < t.count ? p[u * THREADS] : make_uint4(0, 0, 0, 0);
}

// sum of squares of the thread's share of a tile
template <class T> __device__ __forceinline__ double squares_of(const Tile& t, const Words& words) {
  constexpr int W = 16 / (int)sizeof(T);
  const T* src = (const T*)t.src;
  double acc = 0.0;
  // the ends that are not whole words
  const int64_t rest = t.at + (int64_t)t.count * W;
  if (threadIdx.x < t.at - t.s.first) acc += square(src[t.s.first + threadIdx.x]);
  if (threadIdx.x < t.s.end - rest) acc += square(src[rest + threadIdx.x]);
  float even = 0.f, odd = 0.f;
  uint32_t bits = 0;
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    Pack<T, W> p;
    float v[W];
    p.raw = words.w[u];
    p.widen(v);
    bits |= p.raw.x | p.raw.y | p.raw.z | p.raw.w;
#pragma unroll
    for (int j = 0; j < W; j += 2) paac::fma2(even, odd, v[j], v[j + 1], v[j], v[j + 1]);
  }
  const float sum = even + odd;                         // (a NaN is in no range)
  if ((sum > LEAST && sum < MOST) || (bits & (sizeof(T) == 2 ? 0x7FFF7FFFu : 0x7FFFFFFFu)) == 0) return acc + (double)sum;
#pragma unroll
  for (int u = 0; u < AHEAD; ++u) {
    Pack<T, W> p;
    float v[W];
    p.raw = words.w[u];
    p.widen(v);
#pragma unroll
    for (int j = 0; j < W; ++j) acc += (double)v[j] * (double)v[j];
  }
  return acc;
}

// the same sum in every thread, added up in the same order
__device__ __forceinline__ double block_total(double v, double* sh /* [WARPS] */) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) t += sh[w];
  return t;
}

// tiles [begin, end) of the table: run `part` of `parts`
struct Run { uint32_t begin, end; };
template <class Tab> __device__ __forceinline__ Run run_of(const Tab& tab, uint32_t part, uint32_t parts) {
  const uint64_t all = tab.first_tile[tab.count];
  return Run{(uint32_t)(all * part / parts), (uint32_t)(all * (part + 1) / parts)};
}

template <class Tab> __device__ __forceinline__ double run_squares(const Tab& tab, Run run) {
  double acc = 0.0;
  uint32_t k = run.begin;
  if (k >= run.end) return acc;
  int i = tensor_of(tab, k);
  Tile next = tile_of(tab, i, k);
  Words coming;
  fetch(next, coming);
  while (k < run.end) {
    const Tile now = next;
    const Words here = coming;
    if (++k < run.end) {
      while (k >= tab.first_tile[i + 1]) ++i;
      next = tile_of(tab, i, k);
      fetch(next, coming);
    }
    acc += now.type ? squares_of<bf16>(now, here) : squares_of<float>(now, here);
  }
  return acc;
}

// Words of src whose place in dst is no whole word: a thread rounds E elements, takes the end of its neighbour's by shuffles and stores whole words
// of dst made of both.  What a warp's first and last words lack goes element by element, from src again.  (Through shared memory
// instead, 16 KB a block: 2 to 4 us more for any list, since the two kernels then want the multiprocessor's memory split differently.)
template <class S, class D> __device__ __noinline__ void shift_words(const S* src, int words, D* q, float factor) {
  constexpr int W = 16 / (int)sizeof(S), E = sizeof(S) == 4 && sizeof(D) == 4 ? 4 : 8, R = E * (int)sizeof(D) / 4;
  const int total = words * W, bytes = (int)((uintptr_t)q & 15u), off = bytes / (int)sizeof(D), back = 16 - bytes, lane = threadIdx.x & 31;
  constexpr int TURNS = AHEAD * W / E;
  Pack<S, W> w[TURNS][E / W];
#pragma unroll
  for (int t = 0; t < TURNS; ++t)
#pragma unroll
    for (int j = 0; j < E; j += W) {
      const int e = (t * THREADS + (int)threadIdx.x) * E + j;
      if (e < total) w[t][j / W].load(src + e); else w[t][j / W].zero();
    }
#pragma unroll
  for (int t = 0; t < TURNS; ++t) {
    const int e0 = (t * THREADS + (int)threadIdx.x) * E, count = max(0, min(E, total - e0));
    if (t * THREADS * E >= total) break;
    float v[E];
#pragma unroll
    for (int j = 0; j < E; j += W) {
      float part[W];
      w[t][j / W].widen(part);
#pragma unroll
      for (int e = 0; e < W; ++e) v[j + e] = factor * part[e];
    }
    uint32_t c[4 + R];                                      // the end of the neighbour's, then this thread's
    if constexpr (sizeof(D) == 4) {
#pragma unroll
      for (int i = 0; i < R; ++i) c[4 + i] = __float_as_uint(v[i]);
    } else {
      Pack<D, E> out;
      out.round(v);
      const uint32_t r[4] = {out.raw.x, out.raw.y, out.raw.z, out.raw.w};
#pragma unroll
      for (int i = 0; i < R; ++i) c[4 + i] = r[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = __shfl_up_sync(0xffffffffu, c[R + i], 1);
    if (back & 8) {
#pragma unroll
      for (int i = 0; i < 2 + R; ++i) c[i] = c[i + 2];
    }
    if (back & 4) {
#pragma unroll
      for (int i = 0; i < 3 + R; ++i) c[i] = c[i + 1];
    }
    if (back & 2) {
#pragma unroll
      for (int i = 0; i < R; ++i) c[i] = __funnelshift_r(c[i], c[i + 1], 16);
    }
    const auto one_by_one = [&](int from, int end) {
      for (int e = from; e < end; ++e) q[e] = paac::from_f<D>(factor * paac::to_f(src[e]));
    };
    if (lane > 0 && count >= E - off) {
#pragma unroll
      for (int i = 0; i < R; i += 4) reinterpret_cast<uint4*>(q + e0 - off)[i / 4] = make_uint4(c[i], c[i + 1], c[i + 2], c[i + 3]);
    } else if (count > 0) {
      one_by_one(lane > 0 ? e0 - off : e0, e0 + min(count, E - off));
    }
    if (lane == 31 || e0 + E >= total) one_by_one(e0 + E - off, e0 + count);
  }
}

template <class S, class D> __device__ __noinline__ void write_span(const S* src, D* dst, Span s, float factor) {
  constexpr int W = 16 / (int)sizeof(S);
  const WordsOf<S> words(src, s);
  const S* p = src + words.at;
  D* q = dst + words.at;
  const int64_t rest = words.at + (int64_t)words.count * W;
  if (threadIdx.x < words.at - s.first) dst[s.first + threadIdx.x] = paac::from_f<D>(factor * paac::to_f(src[s.first + threadIdx.x]));
  if (threadIdx.x < s.end - rest) dst[rest + threadIdx.x] = paac::from_f<D>(factor * paac::to_f(src[rest + threadIdx.x]));
  constexpr int STORE = W * sizeof(D) < 16 ? W * (int)sizeof(D) : 16, PER = STORE / (int)sizeof(D);      // bytes and elements of a store
  if (((uintptr_t)q & (STORE - 1)) != 0) return shift_words(p, words.count, q, factor);
  Pack<S, W> w[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (threadIdx.x + u * THREADS < words.count) w[u].load(p + (threadIdx.x + u * THREADS) * W);
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (threadIdx.x + u * THREADS < words.count) {
      float v[W];
      w[u].widen(v);
#pragma unroll
      for (int j = 0; j < W; j += PER) {
        float part[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) part[e] = factor * v[j + e];
        Pack<D, PER> out;
        out.round(part);
        out.store(q + (threadIdx.x + u * THREADS) * W + j);
      }
    }
}

// from the end of the run to its beginning
template <class Tab> __device__ __forceinline__ void write_run(const Tab& tab, Run run, float factor) {
  uint32_t k = run.end;
  if (k <= run.begin) return;
  int i = tensor_of(tab, k - 1);
  while (k-- > run.begin) {
    while (k < tab.first_tile[i]) --i;
    const void* src = tab.src[i];
    void* dst = tab.dst[i];
    if (dst == nullptr || (factor == 1.f && dst == src)) continue;
    const int types = tab.types[i];
    const Span s = span_of(src, tab.n[i], types & 1 ? 2 : 4, k - tab.first_tile[i]);
    if (types == 0) write_span((const float*)src, (float*)dst, s, factor);
    else if (types == 1) write_span((const bf16*)src, (float*)dst, s, factor);
    else if (types == 2) write_span((const float*)src, (bf16*)dst, s, factor);
    else write_span((const bf16*)src, (bf16*)dst, s, factor);
  }
}

// the factor; -1 where the norm is not finite and nothing may be written.  One thread tells.
__device__ __forceinline__ float factor_of(double total, float clip, float* norm_and_scale, bool tells) {
  const float norm = (float)sqrt(total);
  const float factor = !isfinite(norm) ? -1.f : (clip > 0.f && norm > clip ? clip / norm : 1.f);
  if (tells && norm_and_scale != nullptr) { norm_and_scale[0] = norm; norm_and_scale[1] = fmaxf(factor, 0.f); }
  return factor;
}

template <class Tab>
__global__ void __launch_bounds__(THREADS, PER_SM)
squares_kernel(const __grid_constant__ Tab tab, double* partials) {
  __shared__ double sh[WARPS];
  paac::pdl_entry();
  const double t = block_total(run_squares(tab, run_of(tab, blockIdx.x, gridDim.x)), sh);
  if (threadIdx.x == 0) partials[blockIdx.x] = t;
}

template <class Tab>
__global__ void __launch_bounds__(THREADS, PER_SM)
write_kernel(const __grid_constant__ Tab tab, const double* partials, int n_partials, float clip, float* norm_and_scale, int tells) {
  __shared__ double sh[WARPS];
  paac::pdl_entry();
  double acc = 0.0;
  for (int i = threadIdx.x; i < n_partials; i += THREADS) acc += partials[i];
  const float factor = factor_of(block_total(acc, sh), clip, norm_and_scale, tells != 0 && blockIdx.x == 0 && threadIdx.x == 0);
  if (factor >= 0.f) write_run(tab, run_of(tab, gridDim.x - 1 - blockIdx.x, gridDim.x), factor);
}

template <class Tab>
__global__ void __launch_bounds__(THREADS, 2)
one_cluster_kernel(const __grid_constant__ Tab tab, float clip, float* norm_and_scale) {
  __shared__ double sh[WARPS];
  __shared__ double of_block[CLUSTER];
  paac::cluster_arrive();                                                   // nobody stores into a block that has not begun
  paac::pdl_entry();
  const int rank = paac::cluster_rank();
  const Run run = run_of(tab, rank, CLUSTER);
  const double t = block_total(run_squares(tab, run), sh);
  paac::cluster_wait();
  if (threadIdx.x < CLUSTER) paac::store_in_block(&of_block[rank], threadIdx.x, t);
  paac::cluster_arrive();
  paac::cluster_wait();
  double total = 0.0;
#pragma unroll
  for (int b = 0; b < CLUSTER; ++b) total += of_block[b];
  const float factor = factor_of(total, clip, norm_and_scale, rank == 0 && threadIdx.x == 0);
  if (factor >= 0.f) write_run(tab, run, factor);
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

// `also`: what else is written
int check(const paac_tensor* t, size_t count, const Extent (&also)[2]) {
  if (also[0].begin < also[1].end && also[1].begin < also[0].end) return PAAC_ERR_ARG;
  if (count == 0) return PAAC_OK;
  const auto clear = [&](const Extent& e) {
    return (e.end <= also[0].begin || also[0].end <= e.begin) && (e.end <= also[1].begin || also[1].end <= e.begin);
  };
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
    if (!clear(e[k - 1]) || !clear(e[k > 1 ? k - 2 : 0])) { status = PAAC_ERR_ARG; break; }
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
    tiles += (x.n * size + ((uintptr_t)x.src & 15u) + TILE - 1) / TILE;
  }
  tab.first_tile[tab.count] = (uint32_t)tiles;
  return at;
}
template <int CAP> int blocks_for(const Table<CAP>& tab) {
  const uint32_t tiles = tab.first_tile[tab.count];
  return tiles == 0 ? 1 : tiles < (uint32_t)BLOCKS ? (int)tiles : BLOCKS;
}

template <int CAP>
cudaError_t launch_all(const paac_tensor* t, size_t count, float clip, float* norm_and_scale, double* partials, cudaStream_t s) {
  Table<CAP> tab;
  size_t at = fill(tab, t, 0, count);
  if (at == count && tab.first_tile[tab.count] <= CLUSTER) {
    // a function's attributes belong to the current device, and this entry point works on any
    static paac::PerDevice<bool> ready;
    int device = -1;
    const bool ok = cudaGetDevice(&device) == cudaSuccess && ready.get(device, [](bool&) {
      return cudaFuncSetAttribute(one_cluster_kernel<Table<CAP>>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
    }) != nullptr;
    if (!ok) return cudaErrorUnknown;
    return paac::launch_clusters_on(s, one_cluster_kernel<Table<CAP>>, dim3(CLUSTER), dim3(THREADS), CLUSTER, 0, tab, clip, norm_and_scale);
  }
  int n_partials = 0;
  for (;;) {
    const int blocks = blocks_for(tab);
    const cudaError_t e = paac::launch_overlapped_on(s, squares_kernel<Table<CAP>>, dim3(blocks), dim3(THREADS), 0, tab, partials + n_partials);
    if (e != cudaSuccess) return e;
    n_partials += blocks;
    if (at == count) break;
    at = fill(tab, t, at, count);
  }
  // (a single table is still there)
  if (count > (size_t)CAP) at = fill(tab, t, 0, count);
  for (int tells = 1;; tells = 0) {
    const cudaError_t e = paac::launch_overlapped_on(s, write_kernel<Table<CAP>>, dim3(blocks_for(tab)), dim3(THREADS), 0, tab, (const double*)partials, n_partials, clip,
                                                     norm_and_scale, tells);
    if (e != cudaSuccess || at == count) return e;
    at = fill(tab, t, at, count);
  }
}

}  // namespace

extern "C" size_t paac_clip_tensors_workspace_bytes(size_t count) {
  if (count > (size_t)MAX_COUNT) return 0;
  return (count / MAX_TABLE + 1) * BLOCKS * sizeof(double);
}

extern "C" int paac_clip_tensors(const paac_tensor* tensors, size_t count, float clip_norm, float* norm_and_scale, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  if (tensors == nullptr && count != 0) return PAAC_ERR_ARG;
  if (count > (size_t)MAX_COUNT) return PAAC_ERR_LIMIT;
  if (clip_norm != clip_norm || ((uintptr_t)norm_and_scale & 3u) != 0) return PAAC_ERR_ARG;
  const size_t need = paac_clip_tensors_workspace_bytes(count);
  const bool room = workspace != nullptr && ((uintptr_t)workspace & 15u) == 0 && workspace_bytes >= need;
  const uintptr_t told = (uintptr_t)norm_and_scale, scratch = room ? (uintptr_t)workspace : 0;
  const int bad = check(tensors, count, {Extent{told, told == 0 ? 0 : told + 8, true}, Extent{scratch, room ? scratch + need : 0, true}});
  if (bad != PAAC_OK) return bad;
  if (!room) return PAAC_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  double* partials = static_cast<double*>(workspace);
  const cudaError_t e = count <= (size_t)SMALL_TABLE    ? launch_all<SMALL_TABLE>(tensors, count, clip_norm, norm_and_scale, partials, s)
                        : count <= (size_t)MIDDLE_TABLE ? launch_all<MIDDLE_TABLE>(tensors, count, clip_norm, norm_and_scale, partials, s)
                                                        : launch_all<MAX_TABLE>(tensors, count, clip_norm, norm_and_scale, partials, s);
  return paac::launch_status(e);
}
