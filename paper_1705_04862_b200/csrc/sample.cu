// An action out of many for each row of logits (paac_sample): temperature, top-k, top-p, min-p, then the inverse of the running sum.
//
// Every filter keeps a beginning of the order (largest logit first, of equal ones the lower index), so what stays is: keys above a threshold, and
// of those equal to it the ones below an index.  The key is the logit as a whole number of the same order.  A threshold is found digit by digit
// of the key: how many actions (top-k), or how much of the whole (top-p), each digit holds, from the largest on.  Nothing is sorted.
// Shares of the whole are whole numbers of 64 bits, so that sums do not depend on their order; the exponential under them is in 64 bits, since
// the draw has to be right next to a border of the running sum.
//
// A cluster of blocks has a row: each block a run of neighbouring chunks of CHUNK actions, kept in shared memory from the first read on where it
// fits.
#include "cluster.cuh"
#include "per_device.h"
#include "pack.cuh"
#include "rows.h"

namespace {
using paac::bf16;

constexpr int THREADS = 512, WARPS = THREADS / 32, CHUNK = 256, EACH = CHUNK / 32, MOST_CLUSTER = 8, MOST_CHUNKS = 4096, BINS = 2048;
constexpr int MOST_ACTIONS = MOST_CLUSTER * MOST_CHUNKS * CHUNK;
typedef unsigned long long u64;

struct Args {
  const void* logits;
  const uint8_t* allowed;
  int64_t logits_row, allowed_row;
  const float *uniforms, *temperature, *top_p, *min_p;
  const int32_t* top_k;
  int32_t* actions;
  float* logprobs;
  int v, bits;                         // bits: of the likeliest action's share
  int cluster, chunks, staged;           // blocks of a row, chunks of a block; whether a block keeps its logits
};

constexpr uint32_t NOTHING = 0x007FFFFFu;          // the key of -inf: what has it or a smaller one is left out
constexpr uint32_t INFINITE = 0xFF800000u, BAD = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l + 0.f);      // -0 is 0
  return l != l ? BAD : (b >> 31 ? ~b : b | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7FFFFFFFu : ~key); }

__device__ __forceinline__ void put(uint32_t* p, int rank, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(paac::in_block(p, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void put(u64* p, int rank, u64 v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(paac::in_block(p, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ uint32_t get(const uint32_t* p, int rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(paac::in_block(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ u64 get(const u64* p, int rank) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(paac::in_block(p, rank)) : "memory");
  return v;
}
__device__ __forceinline__ void together() { paac::cluster_arrive(); paac::cluster_wait(); }
__device__ __forceinline__ u64 warp_sum(u64 v) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
  return v;
}
__device__ __forceinline__ u64 warp_before(u64 v) {          // the sum of the lanes before this one
  u64 all = v;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const u64 o = __shfl_up_sync(0xffffffffu, all, d);
    if ((int)(threadIdx.x & 31) >= d) all += o;
  }
  return all - v;
}

struct alignas(16) Shared {
  uint32_t count[BINS], all_count[BINS];
  u64 mass[BINS], all_mass[BINS];
  u64 chunk[MOST_CHUNKS];
  u64 of_warp[WARPS], of_block[2][MOST_CLUSTER];
  u64 found_above, found_mass;
  uint32_t found_count, found_at;
  int found;
};

// the sum over the block of v, and of the threads before this one
__device__ __forceinline__ u64 block_before(Shared& s, u64 v, u64& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  u64 before = warp_before(v);
  if (lane == 31) s.of_warp[warp] = before + v;
  __syncthreads();
  all = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    if (w == warp) before += all;
    all += s.of_warp[w];
  }
  __syncthreads();
  return before;
}

template <class T, bool WIDE> struct Row {
  const Args& a;
  Shared& s;
  T* kept;                             // the block's logits, or none
  int rank, row, lane, warp, chunks, begin;      // chunks and first action of this block
  int parity = 0;
  float largest = 0.f;
  double inverse = 1.0;                // of the temperature
  double scale = 1.0;                  // the likeliest action's share
  // what stays: keys above `above`, and those that equal it with an index below `until`
  uint32_t above = NOTHING;
  int until = 0;

  __device__ __forceinline__ int index(int chunk, int j) const { return begin + chunk * CHUNK + (WIDE ? lane * EACH + j : j * 32 + lane); }
  __device__ __forceinline__ void keys(int chunk, uint32_t (&k)[EACH], bool first) const {
    const int i0 = index(chunk, 0), step = WIDE ? 1 : 32;
    const bool from_kept = kept != nullptr && !first;
    const T* p = from_kept ? kept + (i0 - begin) : (const T*)a.logits + row * a.logits_row + i0;
    const uint8_t* allowed = a.allowed != nullptr && !from_kept ? a.allowed + row * a.allowed_row + i0 : nullptr;
    float l[EACH];
    if (WIDE) {
      if (i0 < a.v) {                  // (a whole number of eights)
        constexpr int W = 16 / sizeof(T);
#pragma unroll
        for (int j = 0; j < EACH; j += W) {
          paac::Pack<T, W> q;
          float v[W];
          q.load(p + j);
          q.widen(v);
#pragma unroll
          for (int i = 0; i < W; ++i) l[j + i] = v[i];
        }
        if (allowed != nullptr) {
          const uint2 m = *reinterpret_cast<const uint2*>(allowed);
#pragma unroll
          for (int j = 0; j < EACH; ++j)
            if (((j < 4 ? m.x : m.y) >> (j % 4 * 8) & 0xFFu) == 0) l[j] = -INFINITY;
        }
      } else {
#pragma unroll
        for (int j = 0; j < EACH; ++j) l[j] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const bool there = i0 + j * step < a.v && (allowed == nullptr || allowed[j * step] != 0);
        l[j] = there ? paac::to_f(p[j * step]) : -INFINITY;
      }
    }
    if (first && kept != nullptr) {
#pragma unroll
      for (int j = 0; j < EACH; ++j) kept[i0 - begin + j * step] = paac::from_f<T>(l[j]);
    }
#pragma unroll
    for (int j = 0; j < EACH; ++j) k[j] = key_of(l[j]);
  }
  template <class F> __device__ __forceinline__ void for_chunks(F f, bool first = false) const {
    for (int c = warp; c < chunks; c += WARPS) {
      uint32_t k[EACH];
      keys(c, k, first);
      f(c, k);
    }
  }
  __device__ __forceinline__ bool stays(uint32_t key, int i) const { return key > above || (key == above && i < until); }
  __device__ __forceinline__ double exponent(uint32_t key) const { return ((double)value_of(key) - (double)largest) * inverse; }
  __device__ __forceinline__ u64 share(double e) const { return (u64)__double2ll_rn(e * scale); }

  // the largest key and the first action with it
  __device__ __forceinline__ u64 first_of_all() {
    u64 best = 0;
    for_chunks([&](int c, const uint32_t (&k)[EACH]) {
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const u64 v = (u64)k[j] << 32 | (uint32_t)~index(c, j);
        best = v > best ? v : best;
      }
    }, true);
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
      const u64 o = __shfl_xor_sync(0xffffffffu, best, d);
      best = o > best ? o : best;
    }
    if (lane == 0) s.of_warp[warp] = best;
    __syncthreads();
    if (threadIdx.x < a.cluster) {
      for (int w = 0; w < WARPS; ++w) best = s.of_warp[w] > best ? s.of_warp[w] : best;
      put(&s.of_block[parity][rank], threadIdx.x, best);
    }
    together();
    for (int r = 0; r < a.cluster; ++r) best = s.of_block[parity][r] > best ? s.of_block[parity][r] : best;
    parity ^= 1;
    return best;
  }

  // The last key of the order before which less than `limit` actions, or (MASS) less than `part` of the whole, lie among what stays; what stays from
  // then on ends with it.
  template <bool MASS> __device__ __forceinline__ void cut(u64 limit, double part) {
    uint32_t prefix = 0, known = 0;
    u64 before = 0;
    constexpr int LEVELS = sizeof(T) == 4 ? 3 : 2;      // a bf16's lower 16 bits say nothing
#pragma unroll
    for (int level = 0; level < LEVELS; ++level) {
      const int shift = level == 0 ? 21 : level == 1 ? 10 : 0;
      for (int i = threadIdx.x; i < BINS; i += THREADS) { s.count[i] = 0; if (MASS) s.mass[i] = 0; }
      if (threadIdx.x == 0) s.found = -1;
      __syncthreads();
      for_chunks([&](int c, const uint32_t (&k)[EACH]) {
#pragma unroll
        for (int j = 0; j < EACH; ++j)
          if (k[j] > NOTHING && (k[j] & known) == prefix && stays(k[j], index(c, j))) {
            const int bin = k[j] >> shift & (BINS - 1);
            atomicAdd(&s.count[bin], 1u);
            if (MASS) atomicAdd(&s.mass[bin], share(exp(exponent(k[j]))));
          }
      });
      together();
      // every block adds up a part of the bins and tells the others
      const int part_of = BINS / a.cluster;
      for (int i = threadIdx.x; i < part_of; i += THREADS) {
        const int bin = rank * part_of + i;
        uint32_t n = 0;
        u64 m = 0;
        for (int r = 0; r < a.cluster; ++r) { n += get(&s.count[bin], r); if (MASS) m += get(&s.mass[bin], r); }
        for (int r = 0; r < a.cluster; ++r) { put(&s.all_count[bin], r, n); if (MASS) put(&s.all_mass[bin], r, m); }
      }
      together();
      // from the largest on
      constexpr int PER = BINS / THREADS;
      u64 mine = 0, all, lies[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int bin = BINS - 1 - (threadIdx.x * PER + i);
        lies[i] = mine;
        mine += MASS ? s.all_mass[bin] : s.all_count[bin];
      }
      const u64 ahead = before + block_before(s, mine, all);
      if (MASS && level == 0) {
        limit = (u64)__double2ll_ru(part * (double)all);
        limit = limit < 1 ? 1 : limit;
      }
#pragma unroll
      for (int i = PER - 1; i >= 0; --i) {
        const int at = threadIdx.x * PER + i;
        if (s.all_count[BINS - 1 - at] != 0 && ahead + lies[i] < limit) { atomicMax(&s.found, at); break; }
      }
      __syncthreads();
      const int at = s.found;
      if (at / PER == (int)threadIdx.x) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (at % PER == i) s.found_above = ahead + lies[i];
        s.found_count = s.all_count[BINS - 1 - at];
        if (MASS) s.found_mass = s.all_mass[BINS - 1 - at];
      }
      __syncthreads();
      before = s.found_above;
      prefix |= (uint32_t)(BINS - 1 - at) << shift;
      known = 0xFFFFFFFFu << shift;
    }
    // of the actions with that key the first few
    const u64 ties = s.found_count;
    u64 few = limit - before;
    if (MASS) {
      const u64 one = s.found_mass / ties;
      few = one == 0 ? ties : (few + one - 1) / one;
    }
    uint32_t key = prefix;
    if (sizeof(T) == 2 && !(prefix >> 31)) key |= 0x3FFu;       // (a negative one's lower bits are ones)
    const uint32_t was = above;
    const int was_until = until;
    __syncthreads();
    int stop = key == was ? was_until : a.v;
    if (few < ties) {
      u64 whole;
      const int last = locate([&](uint32_t k, int i) -> u64 { return k == key && stays(k, i) ? 1 : 0; }, [&](u64) { return few - 1; }, whole);
      stop = last + 1;
    }
    above = key;
    until = stop;
  }

  // The first action, by index, at which the running sum of f(key, index) is more than target(the whole).
  template <class F, class G> __device__ __forceinline__ int locate(F f, G target, u64& whole) {
    for_chunks([&](int c, const uint32_t (&k)[EACH]) {
      u64 sum = 0;
#pragma unroll
      for (int j = 0; j < EACH; ++j) sum += f(k[j], index(c, j));
      sum = warp_sum(sum);
      if (lane == 0) s.chunk[c] = sum;
    });
    __syncthreads();
    const int per = (chunks + THREADS - 1) / THREADS, c0 = threadIdx.x * per;
    u64 mine = 0, all;
    for (int i = 0; i < per; ++i)
      if (c0 + i < chunks) mine += s.chunk[c0 + i];
    u64 ahead = block_before(s, mine, all);
    if (threadIdx.x < a.cluster) put(&s.of_block[parity][rank], threadIdx.x, all);
    together();
    u64 before = 0;
    whole = 0;
    for (int r = 0; r < a.cluster; ++r) {
      if (r == rank) before = whole;
      whole += s.of_block[parity][r];
    }
    parity ^= 1;
    const u64 aim = target(whole);
    if (aim >= before && aim < before + all) {
      ahead += before;
      if (aim >= ahead && aim < ahead + mine) {
        int c = c0;
        while (aim >= ahead + s.chunk[c]) ahead += s.chunk[c++];
        s.found = c;
        s.found_above = ahead;
      }
      __syncthreads();
      if (warp == 0) {
        const int c = s.found;
        uint32_t k[EACH];
        keys(c, k, false);
        u64 run = s.found_above;
        int at = -1;
        if (WIDE) {
          u64 m[EACH], sum = 0;
#pragma unroll
          for (int j = 0; j < EACH; ++j) { m[j] = f(k[j], index(c, j)); sum += m[j]; }
          run += warp_before(sum);
#pragma unroll
          for (int j = 0; j < EACH; ++j) {
            if (aim >= run && aim < run + m[j]) at = index(c, j);
            run += m[j];
          }
        } else {
#pragma unroll
          for (int j = 0; j < EACH; ++j) {
            const u64 m = f(k[j], index(c, j)), ahead_here = run + warp_before(m);
            if (aim >= ahead_here && aim < ahead_here + m) at = index(c, j);
            run += warp_sum(m);
          }
        }
        if (at >= 0)
          for (int r = 0; r < a.cluster; ++r) put(&s.found_at, r, (uint32_t)at);
      }
    }
    together();
    return (int)s.found_at;
  }
};

template <class T, bool WIDE>
__global__ void __launch_bounds__(THREADS)
sample_kernel(const __grid_constant__ Args a) {
  paac::pdl_entry();
  extern __shared__ uint4 raw[];
  Shared& s = *reinterpret_cast<Shared*>(raw);
  const int total = (a.v + CHUNK - 1) / CHUNK, rank = paac::cluster_rank(), row = blockIdx.x / a.cluster;
  const int left = total - rank * a.chunks;
  Row<T, WIDE> r{a, s, a.staged ? reinterpret_cast<T*>(&s + 1) : nullptr, rank, row, (int)(threadIdx.x & 31), (int)(threadIdx.x >> 5),
                 left < 0 ? 0 : left < a.chunks ? left : a.chunks, rank * a.chunks * CHUNK};
  together();                          // nobody stores into a block that has not begun
  const u64 first = r.first_of_all();
  const uint32_t largest = (uint32_t)(first >> 32);
  const float temperature = a.temperature != nullptr ? a.temperature[row] : 1.f;
  int action = -1;
  float logprob = -INFINITY;
  if (largest <= NOTHING) {
  } else if (largest >= INFINITE || temperature != temperature) {
    logprob = __uint_as_float(0x7FFFFFFFu);
  } else if (temperature <= 0.f) {
    action = (int)~(uint32_t)first;
    logprob = 0.f;
  } else {
    r.largest = value_of(largest);
    r.inverse = 1.0 / (double)temperature;
    r.scale = (double)((u64)1 << a.bits);
    const int k = a.top_k != nullptr ? a.top_k[row] : 0;
    if (k > 0 && k < a.v) r.template cut<false>((u64)k, 0.0);
    const float p = a.top_p != nullptr ? a.top_p[row] : 1.f;
    if (p < 1.f) r.template cut<true>(0, p > 0.f ? (double)p : 0.0);
    float least = a.min_p != nullptr ? a.min_p[row] : 0.f;
    least = least > 1.f ? 1.f : least;
    float u = a.uniforms[row];
    u = u > 0.f ? (u < 1.f ? u : 0.99999994f) : 0.f;
    u64 whole;
    action = r.locate([&](uint32_t key, int i) -> u64 {
      if (key <= NOTHING || !r.stays(key, i)) return 0;
      const double e = exp(r.exponent(key));
      return least > 0.f && e < (double)least ? 0 : r.share(e);
    }, [&](u64 all) { return (u64)__double2ll_rd((double)u * (double)all); }, whole);
    if (rank == 0 && threadIdx.x == 0) {
      float l = paac::to_f(((const T*)a.logits)[row * a.logits_row + action]);
      logprob = (float)(r.exponent(key_of(l)) - log((double)whole / r.scale));
    }
  }
  if (rank == 0 && threadIdx.x == 0) {
    a.actions[row] = action;
    if (a.logprobs != nullptr) a.logprobs[row] = logprob;
  }
}

// ---- the host's part -------------------------------------------------------------------------------------------------------------------

// Bytes of logits a block may keep: two blocks share a multiprocessor up to the first, one has it up to the second.
constexpr int64_t KEPT = 32 << 10, MOST_KEPT = 128 << 10;

template <class T, bool WIDE> cudaError_t launch(Args a, int64_t n, cudaStream_t st) {
  const int total = (a.v + CHUNK - 1) / CHUNK;
  const auto bytes = [&](int cluster) { return (int64_t)((total + cluster - 1) / cluster) * CHUNK * sizeof(T); };
  int cluster = 1;
  // as many blocks for a row as it takes to keep it, and while multiprocessors are left and every warp has a chunk
  while (cluster < MOST_CLUSTER && (bytes(cluster) > KEPT || (n * cluster * 2 <= 148 && total >= cluster * 2 * WARPS))) cluster *= 2;
  a.cluster = cluster;
  a.chunks = (total + cluster - 1) / cluster;
  a.staged = bytes(cluster) <= MOST_KEPT;
  const size_t smem = sizeof(Shared) + (a.staged ? (size_t)bytes(cluster) : 0);
  static paac::PerDevice<bool> ready;
  int device = -1;
  const bool ok = cudaGetDevice(&device) == cudaSuccess && ready.get(device, [](bool&) {
    return cudaFuncSetAttribute(sample_kernel<T, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(Shared) + MOST_KEPT)) == cudaSuccess;
  }) != nullptr;
  if (!ok) return cudaErrorUnknown;
  return paac::launch_clusters_on(st, sample_kernel<T, WIDE>, dim3((unsigned)(n * cluster)), dim3(THREADS), cluster, smem, a);
}

}  // namespace

extern "C" int paac_sample(const paac_draw* s, const void* logits, const float* uniforms, int32_t* actions, float* logprobs, void* stream) {
  if (s == nullptr || s->n < 1 || s->v < 1 || s->v > MOST_ACTIONS || (s->type != PAAC_FP32 && s->type != PAAC_BF16) || s->n > (1 << 28)) return PAAC_ERR_ARG;
  if (logits == nullptr || uniforms == nullptr || actions == nullptr) return PAAC_ERR_ARG;
  const int size = s->type == PAAC_BF16 ? 2 : 4;
  for (const void* p : {(const void*)uniforms, (const void*)s->temperature, (const void*)s->top_k, (const void*)s->top_p, (const void*)s->min_p, (const void*)actions, (const void*)logprobs})
    if ((uintptr_t)p & 3u) return PAAC_ERR_ARG;
  const paac::RowSet rows(paac_rows{const_cast<void*>(logits), s->logits_row, 0}, s->n, 1, s->v, size);
  if (!rows.sane() || !rows.aligned()) return PAAC_ERR_ARG;
  paac::Arrays arrays;
  arrays.keep(rows, false);
  if (s->allowed != nullptr) {
    const paac::RowSet mask(paac_rows{const_cast<uint8_t*>(s->allowed), s->allowed_row, 0}, s->n, 1, s->v, 1);
    if (!mask.sane()) return PAAC_ERR_ARG;
    arrays.keep(mask, false);
  }
  const int64_t each = (int64_t)s->n * 4;
  arrays.keep(uniforms, each, false);
  arrays.keep(s->temperature, each, false);
  arrays.keep(s->top_k, each, false);
  arrays.keep(s->top_p, each, false);
  arrays.keep(s->min_p, each, false);
  arrays.keep(actions, each, true);
  arrays.keep(logprobs, each, true);
  if (!arrays.apart) return PAAC_ERR_ARG;
  Args a{};
  a.logits = logits; a.allowed = s->allowed; a.logits_row = s->n > 1 ? s->logits_row : 0; a.allowed_row = s->n > 1 ? s->allowed_row : 0;
  a.uniforms = uniforms; a.temperature = s->temperature; a.top_k = s->top_k; a.top_p = s->top_p; a.min_p = s->min_p;
  a.actions = actions; a.logprobs = logprobs; a.v = s->v;
  int log2 = 0;
  while (((int64_t)1 << log2) < s->v) ++log2;
  a.bits = 62 - log2;
  const bool wide = s->v % EACH == 0 && rows.multiples_of(16) && (s->allowed == nullptr || ((uintptr_t)s->allowed % 8 == 0 && a.allowed_row % 8 == 0));
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (s->type == PAAC_BF16) return paac::launch_status(wide ? launch<bf16, true>(a, s->n, st) : launch<bf16, false>(a, s->n, st));
  return paac::launch_status(wide ? launch<float, true>(a, s->n, st) : launch<float, false>(a, s->n, st));
}
