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

// Sixteen bytes that this call will not read again, past the caches (STREAM): what is there stays for what is read again.
template <class Q> __device__ __forceinline__ Q stream_load(const Q* p) {
  typedef unsigned U __attribute__((ext_vector_type(sizeof(Q) / 4), aligned(alignof(Q) < 4 ? 4 : alignof(Q))));
  const U u = __builtin_nontemporal_load(reinterpret_cast<const U*>(p));
  Q q;
  __builtin_memcpy(&q, &u, sizeof(q));
  return q;
}
template <class Q> __device__ __forceinline__ void stream_store(Q* p, const Q& q) {
  typedef unsigned U __attribute__((ext_vector_type(sizeof(Q) / 4), aligned(alignof(Q) < 4 ? 4 : alignof(Q))));
  U u;
  __builtin_memcpy(&u, &q, sizeof(q));
  __builtin_nontemporal_store(u, reinterpret_cast<U*>(p));
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

// V values of a row from p on, of which `left` are the row's own (the others: zeros, not written).  ANY: the row's values may begin
// at any address of one and their number be no multiple of V; a pack that is all there is one access all the same, which the
// hardware takes at any address.
template <class T, int V, bool ANY, bool STREAM = false> __device__ __forceinline__ Pack<T, V> take(const T* p, int left) {
  Pack<T, V> q;
  if constexpr (!ANY && STREAM) {
    q = stream_load(reinterpret_cast<const Pack<T, V>*>(p));
  } else if constexpr (!ANY) {
    q = *reinterpret_cast<const Pack<T, V>*>(p);
  } else if (left >= V) {
    const Run<T, V> r = *reinterpret_cast<const Run<T, V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) q.v[i] = r.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) q.v[i] = i < left ? p[i] : (T)0.0f;
  }
  return q;
}
template <class T, int V> __device__ __forceinline__ void unpack(const Pack<T, V>& q, float (&x)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = (float)q.v[i];
}
template <class T, int V, bool ANY, bool STREAM = false> __device__ __forceinline__ void put(T* p, const float (&x)[V], int left) {
  if constexpr (!ANY && STREAM) {
    Pack<T, V> q;
#pragma unroll
    for (int i = 0; i < V; ++i) q.v[i] = (T)x[i];
    stream_store(reinterpret_cast<Pack<T, V>*>(p), q);
  } else if constexpr (!ANY) {
    store_pack<T, V>(p, x);
  } else if (left >= V) {
    Run<T, V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.v[i] = (T)x[i];
    *reinterpret_cast<Run<T, V>*>(p) = r;
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < left) p[i] = (T)x[i];
  }
}
// the same of floats, with `other` beyond the row or without a row
template <int V> __device__ __forceinline__ void take_floats(const float* p, int left, float other, float (&w)[V]) {
  if (p != nullptr && left >= V) {
    const FloatRun<V> r = *reinterpret_cast<const FloatRun<V>*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = r.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) w[i] = p != nullptr && i < left ? p[i] : other;
  }
}

inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool spans_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a != nullptr && b != nullptr && na > 0 && nb > 0 && x < y + nb && y < x + na;
}
// whether packs of `pack` values fit all rows of n arrays: the columns and, from row to row, the addresses
inline bool packs_fit(int dtype, int pack, int cols, int64_t rows, const void* const* p, const int64_t* ld, int n) {
  bool ok = cols % pack == 0;
  for (int i = 0; i < n; ++i) ok = ok && aligned_to(p[i], (size_t)pack * type_size(dtype)) && (rows <= 1 || ld[i] % pack == 0);
  return ok;
}
// from the first value of a row array to behind its last one, in bytes
inline size_t rows_span(int64_t rows, int64_t cols, int64_t ld, int size) {
  return rows > 0 && cols > 0 ? ((size_t)(rows - 1) * ld + cols) * size : 0;
}

// Whether two row arrays of the same rows share memory; columns of one buffer that lie next to each other do not.
struct RowArray { const void* p; int64_t cols, ld; };
inline bool rows_overlap(int64_t rows, int size, const RowArray& a, const RowArray& b) {
  if (!spans_overlap(a.p, rows_span(rows, a.cols, a.ld, size), b.p, rows_span(rows, b.cols, b.ld, size))) return false;
  if (a.ld != b.ld) return true;
  const uintptr_t pitch = (uintptr_t)a.ld * size, x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  const uintptr_t from = y >= x ? (y - x) % pitch : (pitch - (x - y) % pitch) % pitch;   // where b's columns begin in a's rows
  return from < (uintptr_t)a.cols * size || from + (uintptr_t)b.cols * size > pitch;
}

// A launch of n <= INT_MAX workgroups of at most `threads` threads: a grid has fewer than 2^32 threads along x, so that the workgroups of a
// larger one are spread over y as well.  Some may lie behind the last one: a kernel has to look at its number.
inline dim3 group_grid(int64_t n, int threads = 256) {
  const int64_t row = (int64_t(1) << 31) / threads;
  return n <= row ? dim3((unsigned)n) : dim3((unsigned)row, (unsigned)((n + row - 1) / row));
}
__device__ __forceinline__ unsigned group_number() { return blockIdx.y * gridDim.x + blockIdx.x; }

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
