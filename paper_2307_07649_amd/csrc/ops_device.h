// Shared by the sequence-layer operators (k_scan.hip, k_conv.hip, k_layernorm.hip, k_clip.hip): the types of row arrays,
// sums over many partial rows, and where the rows of a sequence are.
#pragma once
#include <hip/hip_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "tgnn_internal.h"

namespace tgnn {

// ---- types of row arrays: TGNN_F32, TGNN_BF16, TGNN_F16.  Arithmetic is in float; a conversion back rounds once, to nearest even.
using bf16 = __bf16;
using f16 = _Float16;
inline int type_size(int dtype) { return dtype == TGNN_F32 ? 4 : 2; }
inline bool type_known(int dtype) { return dtype == TGNN_F32 || dtype == TGNN_BF16 || dtype == TGNN_F16; }
template <class F> inline void with_type(int dtype, F f) {   // f(T()) for the type's T
  if (dtype == TGNN_F32) f(float());
  else if (dtype == TGNN_BF16) f(bf16());
  else f(f16());
}

// V values of T as one access; the address has to be a multiple of V * sizeof(T)
template <class T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };
template <class T, int V> __device__ __forceinline__ void load_pack(const T* p, float (&x)[V]) {
  const Pack<T, V> q = *reinterpret_cast<const Pack<T, V>*>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = (float)q.v[i];
}
template <class T, int V> __device__ __forceinline__ void store_pack(T* p, const float (&x)[V]) {
  Pack<T, V> q;
#pragma unroll
  for (int i = 0; i < V; ++i) q.v[i] = (T)x[i];
  *reinterpret_cast<Pack<T, V>*>(p) = q;
}

// N values that are next to each other, at any address of one
template <class T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Run { T v[N]; };
template <int N> using FloatRun = Run<float, N>;

inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool spans_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a != nullptr && b != nullptr && na > 0 && nb > 0 && x < y + nb && y < x + na;
}
// from the first value of a row array to behind its last one, in bytes
inline size_t rows_span(int64_t rows, int64_t cols, int64_t ld, int size) {
  return rows > 0 && cols > 0 ? ((size_t)(rows - 1) * ld + cols) * size : 0;
}

// ---- out[m] (+)= sum over p of part[p, m], for gradients of weights that many workgroups have parts of.  Columns
// [0, c0) go to o0, [c0, c0 + c1) to o1, the next c2 to o2; the sums are taken in double and in one order.
struct ColumnSum {
  const float* part;
  int n_part;
  int64_t cols;             // c0 + c1 + c2 = the row pitch of part
  float* out[3];            // NULL: these columns are not wanted
  int64_t c[3];
  int accumulate;           // add to what is there
};
void column_sum(const ColumnSum& a, hipStream_t s);

}  // namespace tgnn
