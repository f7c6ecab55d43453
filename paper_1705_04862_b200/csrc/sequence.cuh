// What the operators over the steps of sequences share: rows as their kernels walk them, what a call's arguments have to be, and the activations.
#pragma once
#include "pack.cuh"
#include "rows.h"

namespace paac {

// Rows (sequence, step) in elements; a stride that is never taken is 0.
struct StepRows { void* data; int64_t step, seq; };
struct StepFlags { const uint8_t* data; int64_t step, seq; };

template <class T> __device__ __forceinline__ const T* row_at(const StepRows& r, int64_t k, int64_t seq) { return (const T*)r.data + k * r.step + seq * r.seq; }
template <class T> __device__ __forceinline__ T* row_to(const StepRows& r, int64_t k, int64_t seq) { return (T*)r.data + k * r.step + seq * r.seq; }

// e^-v for v >= 0.  Beside bf16 storage the faster one, whose argument is a rounded product with log2(e): off by up to (2 + 1.2 v) 2^-23.
template <class T> __device__ __forceinline__ float exp_minus(float v) {
  if constexpr (sizeof(T) == 4) return expf(-v);
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v * -1.442695041f));
  return e;
}
__device__ __forceinline__ float reciprocal(float v) {        // within two steps of a float
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
// s = 1 / (1 + e^-v) and 1 - s, neither as a difference from 1
template <class T> __device__ __forceinline__ void logistic(float v, float& s, float& rest) {
  if constexpr (sizeof(T) == 2) {            // (the difference is off by 2^-24, of an s that is next to 1 where that weighs)
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v * -1.442695041f));
    s = reciprocal(1.f + e);
    rest = 1.f - s;
    return;
  }
  const float e = exp_minus<T>(fabsf(v)), large = reciprocal(1.f + e), small = e * large;
  s = v >= 0.f ? large : small;
  rest = v >= 0.f ? small : large;
  if (v != v) s = rest = v;
}
// log(1 + e^v) = max(v, 0) + log(1 + e), e = e^-|v|, and log(1 + e) = 2 artanh(q), q = e / (2 + e) <= 1 / 3: artanh(q) / q - 1 = p (1 / 3 + p / 5 + ...) in
// p = q^2 <= 1 / 9, whose factor of p is interpolated at four Chebyshev points: off by less than 2^-25 of the whole.
template <class T> __device__ __forceinline__ float softplus(float v) {
  const float e = exp_minus<T>(fabsf(v)), q = e * reciprocal(2.f + e), p = q * q;
  const float s = fmaf(fmaf(fmaf(0.13425749f, p, 0.1411831f), p, 0.2000378f), p, 0.3333332f) * p;
  float top;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(top) : "f"(v), "f"(0.f));
  return fmaf(2.f, fmaf(s, q, q), top);
}
// v / (1 + e^-v); far below zero 0
template <class T> __device__ __forceinline__ float silu(float v) {
  float e;
  if constexpr (sizeof(T) == 4) e = expf(-v);
  else asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v * -1.442695041f));
  return v * reciprocal(1.f + e);
}

// ---- the host's part -------------------------------------------------------------------------------------------------------------------

inline StepRows step_rows(const paac_rows& r, int t, int n) { return StepRows{r.data, t > 1 ? r.inner : 0, n > 1 ? r.outer : 0}; }

// Which arrays a call has, whether each is fit to be one, and whether what is written is apart from everything else.
struct StepCheck {
  int t, n, size;                    // of the storage type
  bool ok = true;
  int align = 16;                    // bytes that all rows' places are multiples of
  Arrays arrays;
  StepCheck(int t_, int n_, int size_, const uint8_t* restart, int64_t by_sequence, int64_t by_step) : t(t_), n(n_), size(size_) {
    if (restart == nullptr) return;
    const RowSet flags(paac_rows{const_cast<uint8_t*>(restart), by_sequence, by_step}, n, t, 1, 1);
    ok = flags.sane();
    if (ok) arrays.keep(flags, false);
  }
  bool fit() const { return ok && arrays.apart; }
  // rows of c elements for each of `outer` sequences and `inner` steps; `wide`: they are accessed several elements at a time
  void rows(const paac_rows& r, int64_t outer, int64_t inner, int64_t c, bool out, bool needed, bool wide = true) {
    if (r.data == nullptr) { ok = ok && !needed; return; }
    const RowSet set(r, outer, inner, c, size);
    if (!set.sane() || !set.aligned() || (out && !set.rows_apart())) { ok = false; return; }
    while (wide && align > size && !set.multiples_of(align)) align /= 2;
    arrays.keep(set, out);
  }
  void steps(const paac_rows& r, int64_t c, bool out, bool needed, bool wide = true) { rows(r, n, t, c, out, needed, wide); }
  void floats(const float* p, int64_t count, bool out, bool needed = false) {
    if (p == nullptr) { ok = ok && !needed; return; }
    if ((uintptr_t)p & 3u) { ok = false; return; }
    arrays.keep(p, count * 4, out);
  }
};

}  // namespace paac
