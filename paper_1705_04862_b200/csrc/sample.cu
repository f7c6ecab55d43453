// An action out of many for each row of logits (paac_sample): temperature, top-k, top-p, min-p, then the inverse of the running sum.
//
// Every filter keeps a beginning of the order (largest logit first, of equal ones the lower index), so what stays is: logits above one, and
// of those equal to it the ones below an index.  That border is found by the first digit of the logits as whole numbers of the same order: how many
// actions (top-k), or how much of the whole (top-p), each digit holds, from the largest on; the actions with the digit at the border are put in
// order in one block (or told apart by the next digit, if they are many).  Nothing else is sorted.
// Shares of the whole are whole numbers of 64 bits, so that sums do not depend on their order; the exponential under them is in 64 bits, since
// the draw has to be right next to a border of the running sum.
//
// A cluster of blocks has a row: each block a run of neighbouring chunks of CHUNK actions, kept in shared memory from the first read on where it
// fits.  What bounds it: passes over a row in shared memory, barriers of the cluster, and where the whole row is needed (top-p without top-k, no filter) 64-bit
// arithmetic, ten operations an action.  Measured in a graph, bf16: 256 rows of 131,072 with no filter 88 us (read alone 10), the likeliest 42, top-k 50 77, top-p 0.9
// 333, both 83, every row with settings of its own 139 to 156; one row of 50,001 floats 9.8, top-k 18, top-p 35; 32 rows of 1000 6.1.  Before: sums of top-p in shared
// memory digit by digit 798 us, lists put together by one counter of the cluster (20 ns an action) 647, sorted with a barrier a step 421.
#include "cluster.cuh"
#include "per_device.h"
#include "pack.cuh"
#include "rows.h"

namespace {
using paac::bf16;

constexpr int THREADS = 512, WARPS = THREADS / 32, CHUNK = 256, EACH = CHUNK / 32, MOST_CLUSTER = 8, MOST_CHUNKS = 4096, BINS = 4096, DIGITS = 1024, LIST = 4096;
constexpr int MOST_ACTIONS = MOST_CLUSTER * MOST_CHUNKS * CHUNK, MOST_BITS = 50, TABLE = 64;
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

// Logits as whole numbers of the same order (-0 as 0, a NaN as the largest).
constexpr uint32_t NOTHING = 0x007FFFFFu, INFINITE = 0xFF800000u, BAD = 0xFFFFFFFFu;         // -inf, +inf, NaN
__device__ __forceinline__ uint32_t key_of(float l) {
  const uint32_t b = __float_as_uint(l + 0.f);
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
__device__ __forceinline__ void together(int cluster) {
  if (cluster == 1) { __syncthreads(); return; }
  paac::cluster_arrive();
  paac::cluster_wait();
}
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
__device__ __forceinline__ float larger(float a, float b) {
  float v;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(v) : "f"(a), "f"(b));
  return v;
}

// 2^(i / TABLE)
__constant__ double TABLE_VALUES[TABLE] = {
    1, 1.0108892860517005, 1.0218971486541166, 1.0330248790212284, 1.0442737824274138, 1.0556451783605572, 1.0671404006768237, 1.0787607977571199,
    1.0905077326652577, 1.1023825833078409, 1.1143867425958924, 1.1265216186082418, 1.1387886347566916, 1.1511892299529827, 1.1637248587775775, 1.1763969916502812,
    1.189207115002721, 1.2021567314527031, 1.215247359980469, 1.22848053610687, 1.241857812073484, 1.2553807570246911, 1.2690509571917332, 1.2828700160787783,
    1.2968395546510096, 1.3109612115247644, 1.3252366431597413, 1.3396675240533029, 1.3542555469368927, 1.3690024229745905, 1.383909881963832, 1.3989796725383112,
    1.4142135623730951, 1.42961333839197, 1.4451808069770467, 1.460917794180647, 1.4768261459394993, 1.4929077282912648, 1.5091644275934228, 1.5255981507445384,
    1.5422108254079407, 1.5590044002378369, 1.5759808451078865, 1.593142151342267, 1.6104903319492543, 1.6280274218573478, 1.6457554781539649, 1.6636765803267364,
    1.681792830507429, 1.7001063537185235, 1.7186192981224779, 1.7373338352737062, 1.7562521603732995, 1.7753764925265212, 1.7947090750031072, 1.8142521755003989,
    1.8340080864093424, 1.8539791250833855, 1.8741676341103, 1.8945759815869656, 1.9152065613971474, 1.9360617934922943, 1.9571441241754002, 1.9784560263879509,
};

struct alignas(16) Shared {
  union {                              // one after the other, a barrier of the cluster between them
    struct { uint32_t far[BINS], all_far[BINS]; };
    struct { uint32_t count[DIGITS], all_count[DIGITS]; u64 mass[DIGITS], all_mass[DIGITS]; };
    u64 list[LIST];                    // keys and, inverted, indexes
  };
  double table[TABLE];
  u64 of_warp[WARPS], of_block[2][MOST_CLUSTER], of_above[MOST_CLUSTER], of_more[MOST_CLUSTER];
  u64 found_above, found_mass;
  uint32_t found_count, found_at, border_key, border_index, listed, settled;
  int found, found_low;
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
  u64* chunk_sums;                     // [chunks]
  T* kept;                             // the block's logits, or none
  int rank, row, lane, warp, chunks, begin;      // chunks and first action of this block
  int parity = 0;
  // what the share of a logit takes: 2^(bits + (l - largest) rate / TABLE)
  double largest = 0.0, inverse = 1.0, rate = 0.0, step = 0.0;
  // what stays: logits above `border`, and those that equal it with an index below `until`
  float border = -INFINITY, bound = -INFINITY;      // bound: what is below it is beyond the first top_k, certainly
  int until = 0;

  __device__ __forceinline__ int index(int chunk, int j) const { return begin + chunk * CHUNK + (WIDE ? lane * EACH + j : j * 32 + lane); }
  // a chunk's logits of this lane, -inf where there is nothing or it is not allowed
  __device__ __forceinline__ void load(int chunk, float (&l)[EACH], bool first) const {
    const int i0 = index(chunk, 0), step = WIDE ? 1 : 32;
    const bool from_kept = kept != nullptr && !first;
    const T* p = from_kept ? kept + (i0 - begin) : (const T*)a.logits + row * a.logits_row + i0;
    const uint8_t* allowed = a.allowed != nullptr && !from_kept ? a.allowed + row * a.allowed_row + i0 : nullptr;
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
      if (WIDE) {
        constexpr int W = 16 / sizeof(T);
#pragma unroll
        for (int j = 0; j < EACH; j += W) {
          paac::Pack<T, W> q;
          float v[W];
#pragma unroll
          for (int i = 0; i < W; ++i) v[i] = l[j + i];
          q.round(v);
          q.store(kept + (i0 - begin) + j);
        }
      } else {
#pragma unroll
        for (int j = 0; j < EACH; ++j) kept[i0 - begin + j * step] = paac::from_f<T>(l[j]);
      }
    }
  }
  // f(chunk, logits) for the warp's chunks, two loaded at a time
  template <class F> __device__ __forceinline__ void for_chunks(F f, bool first = false) const {
    int c = warp;
    for (; c + WARPS < chunks; c += 2 * WARPS) {
      float l[EACH], m[EACH];
      load(c, l, first);
      load(c + WARPS, m, first);
      f(c, l);
      f(c + WARPS, m);
    }
    if (c < chunks) {
      float l[EACH];
      load(c, l, first);
      f(c, l);
    }
  }
  __device__ __forceinline__ bool stays(float l, int i) const { return l > border || (l == border && i < until); }
  // 2^((l - largest) rate / TABLE) for l <= largest, by the nearest of the table's steps and the first terms of the exponential's series in what is left,
  // |f| <= 1/2 steps: off by less than (ln 2 / 128)^5 / 120 = 4e-14 of it.  Below 2^-1000 0.
  __device__ __forceinline__ double weight(float l) const {
    constexpr double MAGIC = 6755399441055744.0, K = 0.010830424696249145;      // 1.5 2^52: a sum's lower bits are a whole number; ln 2 / 64
    const double d = (double)l - largest, t = fma(d, rate, MAGIC), f = fma(d, rate, -(t - MAGIC));
    const int i = __double2loint(t);
    double p = K * K * K * K / 24;
    p = fma(p, f, K * K * K / 6);
    p = fma(p, f, K * K / 2);
    p = fma(p, f, K);
    p = fma(p, f, 1.0);
    const double e = s.table[i & (TABLE - 1)];
    const double w = p * __hiloint2double(__double2hiint(e) + (i >> 6 << 20), __double2loint(e));
    return d * rate > -64000.0 ? w : 0.0;      // (no branch, so that several are worked on at a time)
  }
  // to the nearest by the sum with 2^52, whose lower bits then are the number
  __device__ __forceinline__ u64 share_of(double weight) const { return (u64)__double_as_longlong(fma(weight, step, 4503599627370496.0)) & 0xFFFFFFFFFFFFFull; }
  __device__ __forceinline__ u64 share(float l) const { return share_of(weight(l)); }

  // The largest of the block's logits that this lane has seen, all of them read for the first time.
  __device__ __forceinline__ float first_look() const {
    float most = -INFINITY;
    if constexpr (WIDE) {
      if (kept != nullptr && a.allowed == nullptr) {
        // as they are, four chunks under way
        constexpr int W = 16 / sizeof(T), PACKS = EACH / W;
        const T* from = (const T*)a.logits + row * a.logits_row;
        for (int c = warp; c < chunks; c += 4 * WARPS) {
          paac::Pack<T, W> q[4][PACKS];
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int i0 = index(c + u * WARPS, 0);
#pragma unroll
            for (int j = 0; j < PACKS; ++j)
              if (c + u * WARPS < chunks && i0 < a.v) q[u][j].load(from + i0 + j * W);
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int i0 = index(c + u * WARPS, 0);
            if (c + u * WARPS >= chunks) continue;
#pragma unroll
            for (int j = 0; j < PACKS; ++j) {
              float v[W];
#pragma unroll
              for (int i = 0; i < W; ++i) v[i] = -INFINITY;
              if (i0 < a.v) q[u][j].widen(v); else q[u][j].round(v);
              q[u][j].store(kept + (i0 - begin) + j * W);
#pragma unroll
              for (int i = 0; i < W; ++i) most = larger(most, v[i]);
            }
          }
        }
        return most;
      }
    }
    for_chunks([&](int, const float (&l)[EACH]) {
#pragma unroll
      for (int j = 0; j < EACH; ++j) most = larger(most, l[j]);
    }, true);
    return most;
  }

  // The largest logit's key, and a bound that at least k logits reach: the smallest of the largest ones of k groups of lanes or more.
  __device__ __forceinline__ uint32_t look(int k) {
    const float most = first_look();
    int group = 32;
    while (group > 1 && a.cluster * (THREADS / group) < k) group /= 2;
    float of_group = most;
    for (int d = 1; d < group; d *= 2) of_group = larger(of_group, __shfl_xor_sync(0xffffffffu, of_group, d));
    if (a.cluster * (THREADS / group) < k) of_group = -INFINITY;
    uint32_t high = key_of(of_group), low = high;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t h = __shfl_xor_sync(0xffffffffu, high, d), w = __shfl_xor_sync(0xffffffffu, low, d);
      high = h > high ? h : high;
      low = w < low ? w : low;
    }
    const uint32_t top = key_of(most);
    uint32_t top_all = top;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const uint32_t h = __shfl_xor_sync(0xffffffffu, top_all, d);
      top_all = h > top_all ? h : top_all;
    }
    if (lane == 0) s.of_warp[warp] = (u64)top_all << 32 | low;
    __syncthreads();
    high = 0;
    low = BAD;
    if (a.cluster > 1) paac::cluster_wait();      // (nobody stores into a block that has not begun)
    if (threadIdx.x < a.cluster) {
      for (int w = 0; w < WARPS; ++w) {
        const uint32_t h = (uint32_t)(s.of_warp[w] >> 32), l = (uint32_t)s.of_warp[w];
        high = h > high ? h : high;
        low = l < low ? l : low;
      }
      put(&s.of_block[parity][rank], threadIdx.x, (u64)high << 32 | low);
    }
    together(a.cluster);
    high = 0;
    low = BAD;
    for (int r = 0; r < a.cluster; ++r) {
      const uint32_t h = (uint32_t)(s.of_block[parity][r] >> 32), l = (uint32_t)s.of_block[parity][r];
      high = h > high ? h : high;
      low = l < low ? l : low;
    }
    parity ^= 1;
    bound = low > NOTHING && low < INFINITE ? value_of(low) : -INFINITY;
    return high;
  }

  // The last action of the order before which less than `limit` actions, or (MASS) less than `part` of the whole, lie among what stays: what stays from
  // then on ends with it.
  template <bool MASS> __device__ __forceinline__ void cut(u64 limit, double part) {
    uint32_t prefix = 0, known = 0;
    u64 before = 0;
    constexpr int LEVELS = sizeof(T) == 4 ? 4 : 2;      // a bf16's lower 16 bits say nothing
    constexpr int PER = DIGITS / THREADS;
    const float low = bound;
    for (int level = 0; level < LEVELS; ++level) {
      const int shift = level == 0 ? 22 : level == 1 ? 12 : level == 2 ? 2 : 0;
      const uint32_t digits = level == 3 ? 3 : DIGITS - 1;
      together(a.cluster);
      for (int i = threadIdx.x; i < DIGITS; i += THREADS) { s.count[i] = 0; if (MASS) s.mass[i] = 0; }
      if (threadIdx.x == 0) { s.found = -1; s.listed = 0; }
      __syncthreads();
      for_chunks([&](int c, const float (&l)[EACH]) {
#pragma unroll
        for (int j = 0; j < EACH; ++j)
          if (l[j] >= low && stays(l[j], index(c, j))) {
            const uint32_t k = key_of(l[j]);
            if ((k & known) != prefix) continue;
            const int bin = k >> shift & digits;
            if (MASS) {
              const u64 m = share(l[j]);
              if (m != 0) atomicAdd(&s.mass[bin], m);
            }
            atomicAdd(&s.count[bin], 1u);
          }
      });
      together(a.cluster);
      // every block adds up a part of the bins and tells the others
      if (a.cluster > 1) {
        const int part_of = DIGITS / a.cluster;
        for (int i = threadIdx.x; i < part_of; i += THREADS) {
          const int bin = rank * part_of + i;
          uint32_t n[MOST_CLUSTER];
          u64 m[MOST_CLUSTER];
#pragma unroll
          for (int r = 0; r < MOST_CLUSTER; ++r) {
            n[r] = r < a.cluster ? get(&s.count[bin], r) : 0;
            m[r] = MASS && r < a.cluster ? get(&s.mass[bin], r) : 0;
          }
#pragma unroll
          for (int r = 1; r < MOST_CLUSTER; ++r) { n[0] += n[r]; m[0] += m[r]; }
#pragma unroll
          for (int r = 0; r < MOST_CLUSTER; ++r)
            if (r < a.cluster) { put(&s.all_count[bin], r, n[0]); if (MASS) put(&s.all_mass[bin], r, m[0]); }
        }
        together(a.cluster);
      } else {
        for (int i = threadIdx.x; i < DIGITS; i += THREADS) { s.all_count[i] = s.count[i]; if (MASS) s.all_mass[i] = s.mass[i]; }
        __syncthreads();
      }
      // from the largest on
      u64 mine = 0, all, lies[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        const int bin = DIGITS - 1 - (threadIdx.x * PER + i);
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
        if (s.all_count[DIGITS - 1 - at] != 0 && ahead + lies[i] < limit) { atomicMax(&s.found, at); break; }
      }
      __syncthreads();
      const int at = s.found;
      if (at / PER == (int)threadIdx.x) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (at % PER == i) s.found_above = ahead + lies[i];
        s.found_count = s.all_count[DIGITS - 1 - at];
        if (MASS) s.found_mass = s.all_mass[DIGITS - 1 - at];
      }
      __syncthreads();
      before = s.found_above;
      prefix |= (uint32_t)(DIGITS - 1 - at) << shift;
      known = 0xFFFFFFFFu << shift;
      if (s.found_count <= LIST) {
        in_order<MASS>(prefix, known, before, limit, low);
        return;
      }
    }
    // more than are put in order, of the same key: of them the first few
    const u64 ties = s.found_count;
    u64 few = limit - before;
    if (MASS) {
      const u64 one = s.found_mass / ties;
      few = one == 0 ? ties : (few + one - 1) / one;
    }
    uint32_t key = prefix;
    if (sizeof(T) == 2 && !(prefix >> 31)) key |= 0xFFFu;       // (a negative one's lower bits are ones)
    const float value = value_of(key);
    __syncthreads();
    int stop = value == border ? until : a.v;
    if (few < ties) {
      u64 whole;
      stop = 1 + locate([&](float l) { return l == value; }, [&](float l, int i) -> u64 { return l == value && stays(l, i) ? 1 : 0; }, [&](u64) { return few - 1; }, whole);
    }
    border = value;
    until = stop;
  }

  // The border among the actions whose keys begin with `prefix`, at most LIST of them: gathered in the first block and sorted there.
  template <bool MASS> __device__ __forceinline__ void in_order(uint32_t prefix, uint32_t known, u64 before, u64 limit, float low) {
    together(a.cluster);                 // nobody reads the sums in its place any more
    for_chunks([&](int c, const float (&l)[EACH]) {
#pragma unroll
      for (int j = 0; j < EACH; ++j)
        if (l[j] >= low && (key_of(l[j]) & known) == prefix && stays(l[j], index(c, j))) list(l[j], index(c, j));
    });
    const uint32_t count = bring();
    if (rank == 0) {
      sort(count);
      u64 whole;
      const int last = MASS ? last_before(count, before, limit, whole) : (int)(limit - before) - 1;
      tell(last < (int)count - 1 ? last : (int)count - 1);
    }
    together(a.cluster);
    told();
  }
  // (by the first block) the list from the largest on.  A warp puts 64 neighbours in order in registers, two to a lane, and does every merge's steps among them
  // there; steps further than that go through shared memory.
  __device__ __forceinline__ void sort(uint32_t count) {
    int room = 64;
    while (room < (int)count) room *= 2;
    for (int i = count + threadIdx.x; i < room; i += THREADS) s.list[i] = 0;
    __syncthreads();
    for (int run = 64; run <= room; run *= 2) {
      for (int d = run / 2; d >= 64; d /= 2) {
        for (int i = threadIdx.x; i < room / 2; i += THREADS) {
          const int x = (i & ~(d - 1)) * 2 + (i & (d - 1)), y = x + d;      // (d is a power of two)
          const u64 p = s.list[x], q = s.list[y];
          if ((p < q) == ((x & run) == 0)) { s.list[x] = q; s.list[y] = p; }
        }
        __syncthreads();
      }
      for (int base = warp * 64; base < room; base += WARPS * 64) {
        u64 v[2] = {s.list[base + lane], s.list[base + 32 + lane]};
        for (int r = run == 64 ? 2 : run; r <= run; r *= 2)
          for (int d = r / 2 < 32 ? r / 2 : 32; d > 0; d /= 2) {
            if (d == 32) {
              const bool down = (base & r) == 0;
              if ((v[0] < v[1]) == down) { const u64 w = v[0]; v[0] = v[1]; v[1] = w; }
            } else {
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const u64 o = __shfl_xor_sync(0xffffffffu, v[u], d);
                const bool down = ((base + u * 32 + lane) & r) == 0, first = (lane & d) == 0;
                const bool larger_here = first == down;           // whether this place takes the larger one
                v[u] = (o > v[u]) == larger_here ? o : v[u];
              }
            }
          }
        s.list[base + lane] = v[0];
        s.list[base + 32 + lane] = v[1];
      }
      __syncthreads();
    }
  }
  // The last of the list's first `count` before which less than `limit` lies, `before` being ahead of all of them (0 where there is none).
  __device__ __forceinline__ int last_before(uint32_t count, u64 before, u64 limit, u64& all) {
    constexpr int PER = LIST / THREADS;
    const int per = ((int)count + THREADS - 1) / THREADS;
    u64 lies[PER], mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = threadIdx.x * per + i;
      lies[i] = mine;
      if (i < per && at < (int)count) mine += share(value_of((uint32_t)(s.list[at] >> 32)));
    }
    if (threadIdx.x == 0) s.found = 0;
    const u64 ahead = before + block_before(s, mine, all);
#pragma unroll
    for (int i = PER - 1; i >= 0; --i) {
      const int at = threadIdx.x * per + i;
      if (i < per && at < (int)count && ahead + lies[i] < limit) { atomicMax(&s.found, at); break; }
    }
    __syncthreads();
    return s.found;
  }
  // the border from the first block to all
  __device__ __forceinline__ void tell(int last) {
    if (threadIdx.x < a.cluster) {
      put(&s.border_key, threadIdx.x, (uint32_t)(s.list[last] >> 32));
      put(&s.border_index, threadIdx.x, ~(uint32_t)s.list[last]);
    }
  }
  __device__ __forceinline__ void told() {
    border = value_of(s.border_key);
    until = (int)s.border_index + 1;
  }

  // one more of the block's list, which `listed` counts on beyond its end
  __device__ __forceinline__ void list(float l, int i) const {
    const uint32_t at = atomicAdd(&s.listed, 1u);
    if (at < LIST) s.list[at] = (u64)key_of(l) << 32 | (uint32_t)~i;
  }
  // The blocks' lists in the first one's, and how many that is; more than LIST: they are not.
  __device__ __forceinline__ uint32_t bring() {
    together(a.cluster);
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int r = 0; r < MOST_CLUSTER; ++r)
      if (r < a.cluster) {
        const uint32_t n = get(&s.listed, r);
        before += r < rank ? n : 0;
        all += n;
      }
    if (rank > 0 && all <= LIST)
      for (uint32_t i = threadIdx.x; before + i < all && i < s.listed; i += THREADS) put(&s.list[before + i], 0, s.list[i]);
    together(a.cluster);
    return all;
  }

  // The draw among the first k of the order, which are all from `bound` on: in the first block, by a list of what is.  False (in all blocks): the
  // list does not hold them, nothing has been done.
  __device__ __forceinline__ bool draw_of_few(int k, float p, float least, float u, int& action, float& logprob) {
    if (threadIdx.x == 0) s.listed = 0;
    together(a.cluster);
    const float low = bound;
    for_chunks([&](int c, const float (&l)[EACH]) {
#pragma unroll
      for (int j = 0; j < EACH; ++j)
        if (l[j] >= low && l[j] > -INFINITY) list(l[j], index(c, j));
    });
    const uint32_t listed = bring();
    if (listed > LIST) return false;
    if (rank != 0) return true;
    int count = (int)listed;
    sort(count);
    count = count < k ? count : k;
    u64 whole;
    if (p < 1.f) {
      last_before(count, 0, 0, whole);
      u64 limit = (u64)__double2ll_ru((p > 0.f ? (double)p : 0.0) * (double)whole);
      limit = limit < 1 ? 1 : limit;
      __syncthreads();
      count = last_before(count, 0, limit, whole) + 1;
    }
    // by index: inverted, so that the order is the same
    __syncthreads();
    int stay = 0;
    for (int i = threadIdx.x; i < count; i += THREADS) {
      const u64 e = s.list[i];
      const float l = value_of((uint32_t)(e >> 32));
      const bool in = !(least > 0.f) || weight(l) >= (double)least;
      s.list[i] = in ? e << 32 | e >> 32 : 0;      // (0: beyond the last, whatever its index)
      stay += in;
    }
    u64 all;
    block_before(s, (u64)stay, all);
    sort(count);
    count = (int)all;
    constexpr int PER = LIST / THREADS;
    const int per = (count + THREADS - 1) / THREADS;
    u64 m[PER], mine = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int at = threadIdx.x * per + i;
      m[i] = i < per && at < count ? share(value_of((uint32_t)s.list[at])) : 0;
      mine += m[i];
    }
    u64 run = block_before(s, mine, whole);
    const u64 aim = (u64)__double2ll_rd((double)u * (double)whole);
    if (threadIdx.x == 0) s.found = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (aim >= run && aim < run + m[i]) s.found = threadIdx.x * per + i;
      run += m[i];
    }
    __syncthreads();
    const u64 e = s.list[s.found];
    action = (int)~(uint32_t)(e >> 32);
    logprob = (float)(((double)value_of((uint32_t)e) - largest) * inverse - log((double)whole / step));
    return true;
  }

  // The blocks' counts `far` added up in everybody's `all_far`.
  __device__ __forceinline__ void add_far() {
    together(a.cluster);
    const int part_of = BINS / a.cluster;
    for (int i = threadIdx.x; i < part_of; i += THREADS) {
      const int bin = rank * part_of + i;
      uint32_t n[MOST_CLUSTER];
#pragma unroll
      for (int r = 0; r < MOST_CLUSTER; ++r) n[r] = r < a.cluster ? get(&s.far[bin], r) : 0;
#pragma unroll
      for (int r = 1; r < MOST_CLUSTER; ++r) n[0] += n[r];
#pragma unroll
      for (int r = 0; r < MOST_CLUSTER; ++r)
        if (r < a.cluster) put(&s.all_far[bin], r, n[0]);
    }
    together(a.cluster);
  }
  // The bins [first, last] between which the border certainly lies, by their counts, and how many actions that is.  A bin's share lies between its count times
  // the weights at its ends, which are `each` of the exponent apart from `top` on; in units of 2^-38 of the likeliest.  The border is where `ahead` and the
  // bins up to it make part of the whole, or (whole < 0) of what all bins make.  (What rounding of the distances moves is found out by the exact sums.)
  __device__ __forceinline__ u64 between(float top, float each, double ahead, double whole, double part, int& first, int& last) {
    constexpr int PER = BINS / THREADS;
    u64 low = 0, high = 0, all_low, all_high, mine = 0, all;
    for (int i = 0; i < PER; ++i) {
      const int bin = threadIdx.x * PER + i;
      const u64 n = s.all_far[bin];
      high += n * (u64)(exp2f(top + bin * each) * 274877906944.f * 1.0001f);
      low += n * (u64)(exp2f(top + (bin + 1) * each) * 274877906944.f * 0.9999f);
    }
    if (threadIdx.x == 0) s.found = s.found_low = BINS - 1;
    u64 low_ahead = block_before(s, low, all_low), high_ahead = block_before(s, high, all_high);
    const double from = whole < 0.0 ? part * (double)all_low : (part * whole - ahead) * 274877906944.0, to = whole < 0.0 ? part * (double)all_high : from;
    for (int i = 0; i < PER; ++i) {
      const int bin = threadIdx.x * PER + i;
      const u64 n = s.all_far[bin];
      high_ahead += n * (u64)(exp2f(top + bin * each) * 274877906944.f * 1.0001f);
      low_ahead += n * (u64)(exp2f(top + (bin + 1) * each) * 274877906944.f * 0.9999f);
      if ((double)high_ahead >= from) atomicMin(&s.found_low, bin);
      if ((double)low_ahead >= to) atomicMin(&s.found, bin);
    }
    __syncthreads();
    first = s.found_low;
    last = s.found;
    for (int i = 0; i < PER; ++i) {
      const int bin = threadIdx.x * PER + i;
      if (bin >= first && bin <= last) mine += s.all_far[bin];
    }
    block_before(s, mine, all);
    return all;
  }

  // cut<true> by far less sums: actions are counted by their distance from the largest logit, which says between which distances the border
  // lies; then everything is summed once, exactly, and what lies between them gathered and sorted (or, if that is too much, counted by finer distances
  // first).  False (in all blocks): it has not been found that way (too many lie as near to the border), nothing has been cut.
  __device__ __forceinline__ bool cut_by_distance(double part) {
    const float top = (float)largest, width = (float)(rate * BINS / (TABLE * (double)(a.bits + 1))), fall = -(float)(a.bits + 1) / BINS;      // bins a unit of the logits
    const auto distance = [&](float l) { const float d = (top - l) * width; return d < BINS - 1 ? d : (float)(BINS - 1); };
    const auto clear = [&] {
      together(a.cluster);
      for (int i = threadIdx.x; i < BINS; i += THREADS) s.far[i] = 0;
      if (threadIdx.x == 0) s.listed = 0;
      __syncthreads();
    };
    clear();
    for_chunks([&](int c, const float (&l)[EACH]) {
#pragma unroll
      for (int j = 0; j < EACH; ++j)
        if (stays(l[j], index(c, j))) atomicAdd(&s.far[(int)distance(l[j])], 1u);
    });
    add_far();
    int first, last, first2 = 0, last2 = BINS - 1;
    const bool at_once = between(0.f, fall, 0.0, -1.0, part, first, last) <= LIST;
    const float zoom = (float)BINS / (last + 1 - first);
    const auto fine = [&](float d) { const float f = (d - first) * zoom; return f < BINS - 1 ? (int)f : BINS - 1; };
    // the exact sums, and the list, or the finer counts
    if (at_once) together(a.cluster); else clear();
    u64 total = 0, above = 0;
    for_chunks([&](int c, const float (&l)[EACH]) {
#pragma unroll
      for (int j = 0; j < EACH; ++j) {
        const int i = index(c, j);
        const float d = distance(l[j]);
        const bool in = stays(l[j], i);
        const u64 m = in ? share(l[j]) : 0;
        total += m;
        above += (int)d < first ? m : 0;
        if (in && (int)d >= first && (int)d <= last) {
          if (at_once) list(l[j], i); else atomicAdd(&s.far[fine(d)], 1u);
        }
      }
    });
    block_before(s, total, total);
    block_before(s, above, above);
    if (threadIdx.x < a.cluster) { put(&s.of_block[parity][rank], threadIdx.x, total); put(&s.of_above[rank], threadIdx.x, above); }
    if (!at_once) {
      add_far();
      total = above = 0;
      for (int r = 0; r < a.cluster; ++r) { total += s.of_block[parity][r]; above += s.of_above[r]; }
      if (between(first * fall, fall / zoom, (double)above / step, (double)total / step, part, first2, last2) > LIST) {
        parity ^= 1;
        together(a.cluster);
        return false;
      }
      together(a.cluster);
      u64 more = 0;
      for_chunks([&](int c, const float (&l)[EACH]) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) {
          const int i = index(c, j);
          const float d = distance(l[j]);
          if ((int)d < first || (int)d > last || !stays(l[j], i)) continue;
          const int bin = fine(d);
          if (bin < first2) more += share(l[j]);
          else if (bin <= last2) list(l[j], i);
        }
      });
      block_before(s, more, more);
      if (threadIdx.x == 0) put(&s.of_more[rank], 0, more);
    }
    const uint32_t count = bring();
    if (rank == 0) {
      total = above = 0;
      for (int r = 0; r < a.cluster; ++r) { total += s.of_block[parity][r]; above += s.of_above[r] + (at_once ? 0 : s.of_more[r]); }
      u64 limit = (u64)__double2ll_ru(part * (double)total), listed = 0;
      limit = limit < 1 ? 1 : limit;
      int at = 0;
      if (count > 0 && count <= LIST) {
        sort(count);
        at = last_before(count, above, limit, listed);
      }
      // the border is in the list if less than the limit is ahead of it, and nothing less likely than the list's has to stay
      const bool settled = count > 0 && count <= LIST && above < limit && (above + listed >= limit || above + listed == total);
      if (settled) tell(at);
      if (threadIdx.x < a.cluster) put(&s.settled, threadIdx.x, settled ? 1u : 0u);
    }
    parity ^= 1;
    together(a.cluster);
    if (s.settled == 0) return false;
    told();
    return true;
  }

  // The first action, by index, at which the running sum of f(logit, index) is more than target(the whole); f is 0 but where may(logit).
  // Told to all blocks, or (DRAW) known to the one that has it alone; -1 elsewhere.
  template <bool DRAW = false, class M, class F, class G> __device__ __forceinline__ int locate(M may, F f, G target, u64& whole) {
    for_chunks([&](int c, const float (&l)[EACH]) {
      bool any = false;
#pragma unroll
      for (int j = 0; j < EACH; ++j) any = any || may(l[j]);
      u64 sum = 0;
      if (__any_sync(0xffffffffu, any)) {
#pragma unroll
        for (int j = 0; j < EACH; ++j) sum += f(l[j], index(c, j));
        sum = warp_sum(sum);
      }
      if (lane == 0) chunk_sums[c] = sum;
    });
    __syncthreads();
    const int per = (chunks + THREADS - 1) / THREADS, c0 = threadIdx.x * per;
    u64 mine = 0, all;
    for (int i = 0; i < per; ++i)
      if (c0 + i < chunks) mine += chunk_sums[c0 + i];
    u64 ahead = block_before(s, mine, all);
    if (threadIdx.x < a.cluster) put(&s.of_block[parity][rank], threadIdx.x, all);
    together(a.cluster);
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
        while (aim >= ahead + chunk_sums[c]) ahead += chunk_sums[c++];
        s.found = c;
        s.found_above = ahead;
      }
      __syncthreads();
      if (warp == 0) {
        const int c = s.found;
        float l[EACH];
        load(c, l, false);
        u64 run = s.found_above;
        int at = -1;
        if (WIDE) {
          u64 m[EACH], sum = 0;
#pragma unroll
          for (int j = 0; j < EACH; ++j) { m[j] = f(l[j], index(c, j)); sum += m[j]; }
          run += warp_before(sum);
#pragma unroll
          for (int j = 0; j < EACH; ++j) {
            if (aim >= run && aim < run + m[j]) at = index(c, j);
            run += m[j];
          }
        } else {
#pragma unroll
          for (int j = 0; j < EACH; ++j) {
            const u64 m = f(l[j], index(c, j)), here = run + warp_before(m);
            if (aim >= here && aim < here + m) at = index(c, j);
            run += warp_sum(m);
          }
        }
        if (DRAW) {
          const uint32_t has = __ballot_sync(0xffffffffu, at >= 0);
          return __shfl_sync(0xffffffffu, at, __ffs(has) - 1);
        }
        if (at >= 0)
          for (int r = 0; r < a.cluster; ++r) put(&s.found_at, r, (uint32_t)at);
      }
    }
    if (DRAW) return -1;
    together(a.cluster);
    return (int)s.found_at;
  }
};

template <class T, bool WIDE>
__global__ void __launch_bounds__(THREADS, 2)
sample_kernel(const __grid_constant__ Args a) {
  extern __shared__ uint4 raw[];
  Shared& s = *reinterpret_cast<Shared*>(raw);
  if (a.cluster > 1) paac::cluster_arrive();
  if (threadIdx.x < TABLE) s.table[threadIdx.x] = TABLE_VALUES[threadIdx.x];
  paac::pdl_entry();
  const int total = (a.v + CHUNK - 1) / CHUNK, rank = a.cluster > 1 ? paac::cluster_rank() : 0, row = blockIdx.x / a.cluster;
  const int left = total - rank * a.chunks;
  u64* chunk_sums = reinterpret_cast<u64*>(&s + 1);
  Row<T, WIDE> r{a, s, chunk_sums, a.staged ? reinterpret_cast<T*>(chunk_sums + (a.chunks + 1) / 2 * 2) : nullptr, rank, row, (int)(threadIdx.x & 31), (int)(threadIdx.x >> 5),
                 left < 0 ? 0 : left < a.chunks ? left : a.chunks, rank * a.chunks * CHUNK};
  const float temperature = a.temperature != nullptr ? a.temperature[row] : 1.f, p = a.top_p != nullptr ? a.top_p[row] : 1.f;
  const int k = a.top_k != nullptr ? a.top_k[row] : 0;
  const float least = a.min_p != nullptr ? a.min_p[row] : 0.f;
  float u = a.uniforms[row];
  u = u > 0.f ? (u < 1.f ? u : 0.99999994f) : 0.f;
  const bool some = k > 0 && k < a.v;
  const uint32_t largest = r.look(some ? k : a.v);

  int action = -1;
  float logprob = -INFINITY;
  bool mine = rank == 0 && threadIdx.x == 0;      // who writes
  if (largest <= NOTHING) {
  } else if (largest >= INFINITE || temperature != temperature) {
    logprob = __uint_as_float(0x7FFFFFFFu);
  } else if (temperature <= 0.f || least > 1.f) {          // (min_p above 1: not even the first's equals are likely enough)
    const float top = value_of(largest);
    u64 whole;
    action = r.template locate<true>([&](float l) { return l == top; }, [&](float l, int) -> u64 { return l == top ? 1 : 0; }, [&](u64) { return (u64)0; }, whole);
    logprob = 0.f;
    mine = action >= 0 && threadIdx.x == 0;
  } else {
    r.largest = (double)value_of(largest);
    r.inverse = 1.0 / (double)temperature;
    r.rate = r.inverse * (1.4426950408889634 * TABLE);
    r.step = (double)((u64)1 << a.bits);
    const bool listed = some ? r.bound > -INFINITY || a.v <= LIST : p < 1.f && a.v <= LIST;
    if (!listed || !r.draw_of_few(some ? k : a.v, p, least, u, action, logprob)) {
      if (some) r.template cut<false>((u64)k, 0.0);
      if (p < 1.f) {
        const double part = p > 0.f ? (double)p : 0.0;
        if (!r.cut_by_distance(part)) r.template cut<true>(0, part);
      }
      u64 whole;
      const float low = r.border;
      const double smallest = least > 0.f ? (double)least : 0.0;
      action = r.template locate<true>([&](float l) { return l >= low && l > -INFINITY; }, [&](float l, int i) -> u64 {
        const double w = r.weight(l);
        const u64 m = r.share_of(w);
        return r.stays(l, i) && w >= smallest ? m : 0;
      }, [&](u64 all) { return (u64)__double2ll_rd((double)u * (double)all); }, whole);
      mine = action >= 0 && threadIdx.x == 0;
      if (mine) logprob = (float)(((double)paac::to_f(((const T*)a.logits)[row * a.logits_row + action]) - r.largest) * r.inverse - log((double)whole / r.step));
    }
  }
  if (mine) {
    a.actions[row] = action;
    if (a.logprobs != nullptr) a.logprobs[row] = logprob;
  }
}

// ---- the host's part -------------------------------------------------------------------------------------------------------------------

// Bytes of logits a block may keep: two blocks share a multiprocessor up to the first, one has it up to the second.
constexpr int64_t KEPT = 64 << 10, MOST_KEPT = 128 << 10;

int64_t block_bytes(int v, int size, int cluster) { return (((int64_t)v + CHUNK - 1) / CHUNK + cluster - 1) / cluster * CHUNK * size; }
// as many blocks for a row as it takes to keep it, and while multiprocessors are left and every warp has a chunk
int blocks_of_row(int64_t n, int v, int size) {
  const int total = (v + CHUNK - 1) / CHUNK;
  int cluster = 1;
  while (cluster < MOST_CLUSTER && (block_bytes(v, size, cluster) > KEPT || (n * cluster * 2 <= 148 && total >= cluster * 2 * WARPS))) cluster *= 2;
  return cluster;
}

template <class T, bool WIDE> cudaError_t launch(Args a, int64_t n, cudaStream_t st) {
  const int total = (a.v + CHUNK - 1) / CHUNK, cluster = blocks_of_row(n, a.v, sizeof(T));
  const int64_t bytes = block_bytes(a.v, sizeof(T), cluster);
  a.cluster = cluster;
  a.chunks = (total + cluster - 1) / cluster;
  a.staged = bytes <= MOST_KEPT;
  const size_t smem = sizeof(Shared) + (size_t)((a.chunks + 1) / 2 * 2) * 8 + (a.staged ? (size_t)bytes : 0);
  static paac::PerDevice<bool> ready;
  int device = -1;
  const bool ok = cudaGetDevice(&device) == cudaSuccess && ready.get(device, [](bool&) {
    return cudaFuncSetAttribute(sample_kernel<T, WIDE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(sizeof(Shared) + MOST_CHUNKS * 8 + MOST_KEPT)) == cudaSuccess;
  }) != nullptr;
  if (!ok) return cudaErrorUnknown;
  return paac::launch_clusters_on(st, sample_kernel<T, WIDE>, dim3((unsigned)(n * cluster)), dim3(THREADS), cluster, smem, a);
}

}  // namespace

extern "C" int paac_sample(const paac_draw* s, void* stream) {
  if (s == nullptr || s->n < 1 || s->v < 1 || s->v > MOST_ACTIONS || (s->type != PAAC_FP32 && s->type != PAAC_BF16) || s->n > (1 << 28)) return PAAC_ERR_ARG;
  const void* logits = s->logits;
  const float* uniforms = s->uniforms;
  int32_t* actions = s->actions;
  float* logprobs = s->logprobs;
  if (logits == nullptr || uniforms == nullptr || actions == nullptr) return PAAC_ERR_ARG;
  const int size = s->type == PAAC_BF16 ? 2 : 4;
  if (s->n * (int64_t)blocks_of_row(s->n, s->v, size) > INT32_MAX) return PAAC_ERR_ARG;      // (what a grid holds)
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
  a.bits = 62 - log2 < MOST_BITS ? 62 - log2 : MOST_BITS;
  const bool wide = s->v % EACH == 0 && rows.multiples_of(16) && (s->allowed == nullptr || ((uintptr_t)s->allowed % 8 == 0 && a.allowed_row % 8 == 0));
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (s->type == PAAC_BF16) return paac::launch_status(wide ? launch<bf16, true>(a, s->n, st) : launch<bf16, false>(a, s->n, st));
  return paac::launch_status(wide ? launch<float, true>(a, s->n, st) : launch<float, false>(a, s->n, st));
}
