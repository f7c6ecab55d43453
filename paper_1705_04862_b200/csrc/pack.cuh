// W neighbouring elements of storage type T as one access, and as floats.
#pragma once
#include "common.cuh"

namespace paac {

template <int BYTES> struct Word;
template <> struct Word<16> { typedef uint4 type; };
template <> struct Word<8> { typedef uint2 type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<2> { typedef uint16_t type; };

template <class T, int W> struct Pack {
  typedef typename Word<W * sizeof(T)>::type Raw;
  Raw raw;
  __device__ __forceinline__ void load(const T* p) { raw = *reinterpret_cast<const Raw*>(p); }
  __device__ __forceinline__ void zero() { raw = Raw{}; }
  __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<Raw*>(p) = raw; }
  __device__ __forceinline__ void widen(float (&v)[W]) const {
    if constexpr (sizeof(T) == 4) {
      const float* f = reinterpret_cast<const float*>(&raw);
#pragma unroll
      for (int j = 0; j < W; ++j) v[j] = f[j];
    } else if constexpr (W == 1) {
      v[0] = __uint_as_float((uint32_t)raw << 16);           // a bf16 is the upper half of a float
    } else {
      const uint32_t* u = reinterpret_cast<const uint32_t*>(&raw);
#pragma unroll
      for (int j = 0; j < W / 2; ++j) { v[2 * j] = __uint_as_float(u[j] << 16); v[2 * j + 1] = __uint_as_float(u[j] & 0xFFFF0000u); }
    }
  }
  // what is below 0 as 0, a NaN as one
  __device__ __forceinline__ void round_positive(float (&v)[W]) {
    if constexpr (sizeof(T) == 2 && W > 1) {
      uint32_t* u = reinterpret_cast<uint32_t*>(&raw);
#pragma unroll
      for (int j = 0; j < W / 2; ++j) asm("cvt.rn.relu.bf16x2.f32 %0, %1, %2;" : "=r"(u[j]) : "f"(v[2 * j + 1]), "f"(v[2 * j]));
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j) asm("max.NaN.f32 %0, %1, %2;" : "=f"(v[j]) : "f"(v[j]), "f"(0.f));
      round(v);
    }
  }
  __device__ __forceinline__ void round(const float (&v)[W]) {
    if constexpr (sizeof(T) == 4) {
      float* f = reinterpret_cast<float*>(&raw);
#pragma unroll
      for (int j = 0; j < W; ++j) f[j] = v[j];
    } else if constexpr (W == 1) {
      raw = __bfloat16_as_ushort(__float2bfloat16_rn(v[0]));
    } else {
      __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&raw);
#pragma unroll
      for (int j = 0; j < W / 2; ++j) h[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
    }
  }
};

// Asynchronous copies of one access to shared memory; a thread that reads only what it has copied itself waits for no other.
template <int BYTES> __device__ __forceinline__ void copy_to(void* shared, const void* from) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(shared)), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((uint32_t)__cvta_generic_to_shared(shared)), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_end_step() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// until all but the last N steps' copies are there
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Two floats a register pair and an instruction: each result is rounded once, as by the operation on one float.
__device__ __forceinline__ void add2(float& x, float& y, float a, float b) {             // (x, y) + (a, b)
  asm("{ .reg .b64 p, q; mov.b64 p, {%0, %1}; mov.b64 q, {%2, %3}; add.rn.f32x2 p, p, q; mov.b64 {%0, %1}, p; }" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
__device__ __forceinline__ void mul2(float& x, float& y, float a, float b) {             // (x, y) (a, b)
  asm("{ .reg .b64 p, q; mov.b64 p, {%0, %1}; mov.b64 q, {%2, %3}; mul.rn.f32x2 p, p, q; mov.b64 {%0, %1}, p; }" : "+f"(x), "+f"(y) : "f"(a), "f"(b));
}
__device__ __forceinline__ void fma2(float& x, float& y, float a, float b, float c, float d) {      // (a, b) (c, d) + (x, y)
  asm("{ .reg .b64 p, q, r; mov.b64 p, {%0, %1}; mov.b64 q, {%2, %3}; mov.b64 r, {%4, %5}; fma.rn.f32x2 p, q, r, p; mov.b64 {%0, %1}, p; }"
      : "+f"(x), "+f"(y) : "f"(a), "f"(b), "f"(c), "f"(d));
}
__device__ __forceinline__ void fma2_to(float& x, float& y, float a, float b, float c, float d, float e, float f) {      // (a, b) (c, d) + (e, f)
  asm("{ .reg .b64 q, r, s; mov.b64 q, {%2, %3}; mov.b64 r, {%4, %5}; mov.b64 s, {%6, %7}; fma.rn.f32x2 q, q, r, s; mov.b64 {%0, %1}, q; }"
      : "=f"(x), "=f"(y) : "f"(a), "f"(b), "f"(c), "f"(d), "f"(e), "f"(f));
}
// element by element: v += a, v *= a, v += a b, v = a b + c
template <int W> __device__ __forceinline__ void fma_all_to(float (&v)[W], const float (&a)[W], const float (&b)[W], const float (&c)[W]) {
  if constexpr (W == 1) { v[0] = fmaf(a[0], b[0], c[0]); } else {
#pragma unroll
    for (int j = 0; j < W; j += 2) fma2_to(v[j], v[j + 1], a[j], a[j + 1], b[j], b[j + 1], c[j], c[j + 1]);
  }
}
template <int W> __device__ __forceinline__ void add_all(float (&v)[W], const float (&a)[W]) {
  if constexpr (W == 1) { v[0] += a[0]; } else {
#pragma unroll
    for (int j = 0; j < W; j += 2) add2(v[j], v[j + 1], a[j], a[j + 1]);
  }
}
template <int W> __device__ __forceinline__ void mul_all(float (&v)[W], const float (&a)[W]) {
  if constexpr (W == 1) { v[0] *= a[0]; } else {
#pragma unroll
    for (int j = 0; j < W; j += 2) mul2(v[j], v[j + 1], a[j], a[j + 1]);
  }
}
template <int W> __device__ __forceinline__ void fma_all(float (&v)[W], const float (&a)[W], const float (&b)[W]) {
  if constexpr (W == 1) { v[0] = fmaf(a[0], b[0], v[0]); } else {
#pragma unroll
    for (int j = 0; j < W; j += 2) fma2(v[j], v[j + 1], a[j], a[j + 1], b[j], b[j + 1]);
  }
}

// W floats; from 4 on at a multiple of 16 bytes
template <int W> __device__ __forceinline__ void load_floats(float (&v)[W], const float* p) {
  if constexpr (W >= 4) {
#pragma unroll
    for (int j = 0; j < W; j += 4) {
      const float4 x = *reinterpret_cast<const float4*>(p + j);
      v[j] = x.x; v[j + 1] = x.y; v[j + 2] = x.z; v[j + 3] = x.w;
    }
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = p[j];
  }
}
template <int W> __device__ __forceinline__ void store_floats(float* p, const float (&v)[W]) {
  if constexpr (W >= 4) {
#pragma unroll
    for (int j = 0; j < W; j += 4) *reinterpret_cast<float4*>(p + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) p[j] = v[j];
  }
}

}  // namespace paac
