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
  const float e = exp_minus<T>(fabsf(v)), large = reciprocal(1.f + e), small = e * large;
  s = v >= 0.f ? large : small;
  rest = v >= 0.f ? small : large;
  if (v != v) s = rest = v;
}
// log(1 + e^v) = max(v, 0) + log(1 + e), e = e^-|v|, and log(1 + e) = 2 artanh(q), q = e / (2 + e) <= 1 / 3, by its series: what is left out
// of q^17 / 17 on is below 2^-31 of the sum.
template <class T> __device__ __forceinline__ float softplus(float v) {
  const float e = exp_minus<T>(fabsf(v)), q = e * reciprocal(2.f + e), p = q * q;
  float s = 1.f / 15;
  s = fmaf(s, p, 1.f / 13); s = fmaf(s, p, 1.f / 11); s = fmaf(s, p, 1.f / 9); s = fmaf(s, p, 1.f / 7); s = fmaf(s, p, 1.f / 5); s = fmaf(s, p, 1.f / 3);
  s = fmaf(s * p, q, q);
  float top;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(top) : "f"(v), "f"(0.f));
  return fmaf(2.f, s, top);
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
