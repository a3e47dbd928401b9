// Global gradient norm and clipping (tgnn_grad_norm, tgnn_clip_grads): norm = sqrt(sum of all g^2) over a list of tensors,
// and g * max_norm / norm where norm > max_norm.
//
// Two launches per 128 tensors: partial sums of squares, then the scaled copy, whose workgroups each add up all partial sums (at most
// 1,024 doubles per first launch) for themselves: no counter to clear, no last workgroup to wait for, the same sum in the same
// order whenever it is taken.  Squares are taken and added in double: exact for a float's square, no overflow for any float.
// Bound by memory: a gradient is read for its norm, read again and written.  200M elements, a third of them in 16 bits, in 300 tensors: 444
// us, 4.6 TB/s; nineteen tensors of one model, 0.3M elements: 12 us of two launches.
#include <math.h>

#include <algorithm>
#include <new>

#include "ops_device.h"
#include "writeback_device.h"

namespace tgnn {

constexpr int CLIP_TENSORS = 128;          // per launch: the table of a launch is part of its arguments (4 KB)
constexpr int CLIP_BLOCKS = CLIP_PARTS;    // partial sums per launch: four workgroups for every compute unit
constexpr int CLIP_CHUNK = 4096;           // elements a workgroup takes at a time

struct ClipArgs {
  const void* src[CLIP_TENSORS];
  void* dst[CLIP_TENSORS];
  int64_t n[CLIP_TENSORS];                 // elements; bits 60-61: the type
  int32_t first[CLIP_TENSORS + 1];         // first chunk of a tensor
  int32_t tensors;
  int32_t n_part;                          // partial sums of all launches
  float max_norm;
  double* part;                            // where this launch's (norm) or all launches' (clip) partial sums are
  float* out_norm;
  int32_t write_norm;
};

// f(tensor, first element, elements) for every chunk of the workgroup's share, a run of neighbouring ones
template <class F> __device__ __forceinline__ void clip_chunks(const ClipArgs& a, F f) {
  const int64_t total = a.first[a.tensors];
  const int c0 = (int)(total * blockIdx.x / gridDim.x), c1 = (int)(total * (blockIdx.x + 1) / gridDim.x);
  if (c0 >= c1) return;
  int lo = 0, hi = a.tensors - 1;          // the last tensor that begins at or before chunk c0
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.first[mid] <= c0) lo = mid; else hi = mid - 1;
  }
  for (int c = c0, t = lo; c < c1; ++c) {
    while (a.first[t + 1] <= c) ++t;       // (an empty tensor has no chunk)
    const int64_t n = a.n[t] & ((int64_t(1) << 60) - 1), at = (int64_t)(c - a.first[t]) * CLIP_CHUNK;
    f(t, (int)(a.n[t] >> 60), at, (int)(n - at < CLIP_CHUNK ? n - at : CLIP_CHUNK));
  }
}

template <class T> __device__ __forceinline__ double chunk_squares(const T* p, int n) {
  constexpr int V = 16 / sizeof(T);
  double sum = 0.0;
  if (n == CLIP_CHUNK && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    float x[CLIP_CHUNK / 256 / V][V];
#pragma unroll
    for (int i = 0; i < CLIP_CHUNK / 256 / V; ++i) load_pack<T, V>(p + (i * 256 + threadIdx.x) * V, x[i]);
#pragma unroll
    for (int i = 0; i < CLIP_CHUNK / 256 / V; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) sum = fma((double)x[i][j], (double)x[i][j], sum);
  } else {
    for (int i = threadIdx.x; i < n; i += 256) {
      const double v = (double)(float)p[i];
      sum = fma(v, v, sum);
    }
  }
  return sum;
}

// sum over the 256 threads of a workgroup, in all of them
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double parts[4];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
  __syncthreads();
  return (parts[0] + parts[1]) + (parts[2] + parts[3]);
}

__global__ __launch_bounds__(256) void clip_squares_kernel(ClipArgs a) {
  double sum = 0.0;
  clip_chunks(a, [&](int t, int type, int64_t at, int n) {
    if (type == TGNN_F32) sum += chunk_squares(static_cast<const float*>(a.src[t]) + at, n);
    else if (type == TGNN_BF16) sum += chunk_squares(static_cast<const bf16*>(a.src[t]) + at, n);
    else sum += chunk_squares(static_cast<const f16*>(a.src[t]) + at, n);
  });
  sum = block_sum(sum);
  if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

__device__ __forceinline__ double norm_of_parts(const double* part, int n) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) sum += part[i];
  return sqrt(block_sum(sum));
}

__global__ __launch_bounds__(256) void clip_norm_kernel(const double* part, int n, float* out) {
  const double norm = norm_of_parts(part, n);
  if (threadIdx.x == 0) *out = (float)norm;
}

// (The last read of a gradient and the write go past the caches: with 200M elements in 300 tensors this launch and the next call's squares
// take 97 and 51 us per 128 tensors, through the caches 102 and 62.)
template <class T> __device__ __forceinline__ void chunk_scale(const T* p, T* o, int n, double scale) {
  constexpr int V = 16 / sizeof(T);
  if (n == CLIP_CHUNK && ((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(o)) & 15) == 0) {
    float x[CLIP_CHUNK / 256 / V][V];
#pragma unroll
    for (int i = 0; i < CLIP_CHUNK / 256 / V; ++i) unpack(take<T, V, false, true>(p + (i * 256 + threadIdx.x) * V, V), x[i]);
#pragma unroll
    for (int i = 0; i < CLIP_CHUNK / 256 / V; ++i) {
#pragma unroll
      for (int j = 0; j < V; ++j) x[i][j] = (float)((double)x[i][j] * scale);
      put<T, V, false, true>(o + (i * 256 + threadIdx.x) * V, x[i], V);
    }
  } else {
    for (int i = threadIdx.x; i < n; i += 256) o[i] = (T)(float)((double)(float)p[i] * scale);
  }
}

// A norm that is no finite number scales nothing: the gradients stay (or are copied) as they are, and the norm says so.  The factor is
// held in double, and so are its products: with gradients of 1e38 it is smaller than a float holds, and they are not.
__device__ __forceinline__ double clip_scale(double norm, float max_norm) {
  return norm > (double)max_norm && norm < HUGE_VAL ? (double)max_norm / norm : 1.0;
}

__global__ __launch_bounds__(256) void clip_scale_kernel(ClipArgs a) {
  const double norm = norm_of_parts(a.part, a.n_part);
  if (a.write_norm && blockIdx.x == 0 && threadIdx.x == 0) *a.out_norm = (float)norm;
  const double scale = clip_scale(norm, a.max_norm);
  clip_chunks(a, [&](int t, int type, int64_t at, int n) {
    if (scale == 1.0 && a.dst[t] == a.src[t]) return;
    if (type == TGNN_F32) chunk_scale(static_cast<const float*>(a.src[t]) + at, static_cast<float*>(a.dst[t]) + at, n, scale);
    else if (type == TGNN_BF16) chunk_scale(static_cast<const bf16*>(a.src[t]) + at, static_cast<bf16*>(a.dst[t]) + at, n, scale);
    else chunk_scale(static_cast<const f16*>(a.src[t]) + at, static_cast<f16*>(a.dst[t]) + at, n, scale);
  });
}

// The update of a training step with clipped gradients: as in the scaled copy, every workgroup adds up the partial sums.
__global__ __launch_bounds__(256) void clipped_update_kernel(const SgdSet* set, const AdamSet* adam, const double* part, int n_part,
                                                             float max_norm, float lr, float* out_norm) {
  const double norm = norm_of_parts(part, n_part);
  if (out_norm != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *out_norm = (float)norm;
  param_update_block(*set, adam, blockIdx.x >> 6, blockIdx.x & 63, lr, clip_scale(norm, max_norm));
}

static int check_tensors(int32_t n, const void* const* g, const int64_t* numel, const int32_t* dtype) {
  if (n < 0) return set_error(TGNN_E_INVALID_ARG, "n_tensors = %d is negative", n);
  if (n == 0) return TGNN_OK;
  if (g == nullptr || numel == nullptr || dtype == nullptr) return set_error(TGNN_E_NULL_PTR, "a list of the tensors is NULL");
  for (int i = 0; i < n; ++i) {
    if (!type_known(dtype[i])) return set_error(TGNN_E_INVALID_ARG, "dtype[%d] = %d is none of TGNN_F32, TGNN_BF16, TGNN_F16", i, dtype[i]);
    // 2^42 elements: what the card holds many times over, and a chunk count that fits 31 bits
    if (numel[i] < 0 || numel[i] > (int64_t(1) << 42)) return set_error(TGNN_E_OUT_OF_RANGE, "numel[%d] = %lld", i, (long long)numel[i]);
    if (numel[i] > 0 && g[i] == nullptr) return set_error(TGNN_E_NULL_PTR, "tensor %d is NULL", i);
    if (!aligned_to(g[i], type_size(dtype[i]))) return set_error(TGNN_E_MISALIGNED, "tensor %d is not aligned to its type", i);
  }
  return TGNN_OK;
}

// Launches of the list: up to CLIP_TENSORS tensors each, and as many as their chunks fit 31 bits
template <class F> static int clip_launches(int32_t n, const void* const* g, void* const* out, const int64_t* numel,
                                            const int32_t* dtype, ClipArgs& a, F launch) {
  for (int i = 0; i < n;) {
    int64_t chunks = 0;
    a.tensors = 0;
    for (; i < n && a.tensors < CLIP_TENSORS; ++i) {
      const int64_t c = (numel[i] + CLIP_CHUNK - 1) / CLIP_CHUNK;
      if (chunks + c > INT_MAX) break;
      a.src[a.tensors] = g[i];
      a.dst[a.tensors] = out ? out[i] : const_cast<void*>(g[i]);
      a.n[a.tensors] = numel[i] | ((int64_t)dtype[i] << 60);
      a.first[a.tensors++] = (int32_t)chunks;
      chunks += c;
    }
    a.first[a.tensors] = (int32_t)chunks;
    if (chunks == 0) continue;
    launch((int)(chunks < CLIP_BLOCKS ? chunks : CLIP_BLOCKS));
    TGNN_LAUNCH_CHECK();
  }
  return TGNN_OK;
}

static int64_t clip_bytes(int32_t n) { return ((int64_t)(n > 0 ? n : 1) + CLIP_TENSORS - 1) / CLIP_TENSORS * CLIP_BLOCKS * sizeof(double); }

// No written tensor may share memory with another tensor of the call: it would be scaled twice, or read half scaled.
static int check_apart(int32_t n, void* const* g, void* const* out, const int64_t* numel, const int32_t* dtype) {
  struct Span { uintptr_t at, end; bool written; };
  Span* v = new (std::nothrow) Span[2 * (size_t)(n > 0 ? n : 1)];
  if (v == nullptr) return set_error(TGNN_E_WORKSPACE, "no host memory for the list of %d tensors", n);
  int m = 0;
  for (int i = 0; i < n; ++i) {
    const size_t bytes = (size_t)numel[i] * type_size(dtype[i]);
    if (bytes == 0) continue;
    const uintptr_t at = reinterpret_cast<uintptr_t>(g[i]), to = reinterpret_cast<uintptr_t>(out ? out[i] : g[i]);
    v[m++] = Span{to, to + bytes, true};
    if (to != at) v[m++] = Span{at, at + bytes, false};
  }
  std::sort(v, v + m, [](const Span& a, const Span& b) { return a.at < b.at; });
  uintptr_t end = 0, end_written = 0;
  bool apart = true;
  for (int i = 0; i < m && apart; ++i) {
    apart = v[i].at >= end_written && (!v[i].written || v[i].at >= end);
    end = std::max(end, v[i].end);
    if (v[i].written) end_written = std::max(end_written, v[i].end);
  }
  delete[] v;
  return apart ? TGNN_OK : set_error(TGNN_E_INVALID_ARG, "a tensor to be written shares memory with another one of the call");
}

static int norm_launches(int32_t n, const void* const* g, const int64_t* numel, const int32_t* dtype, ClipArgs& a, double* ws,
                         int64_t ws_bytes, hipStream_t s, int& n_part) {
  n_part = 0;
  const int64_t room = ws_bytes / (int64_t)sizeof(double);
  bool fits = true;
  const int rc = clip_launches(n, g, nullptr, numel, dtype, a, [&](int blocks) {
    if (n_part + blocks > room) { fits = false; return; }
    a.part = ws + n_part;
    hipLaunchKernelGGL(clip_squares_kernel, dim3(blocks), dim3(256), 0, s, a);
    n_part += blocks;
  });
  if (rc == TGNN_OK && !fits) return set_error(TGNN_E_WORKSPACE, "the workspace is too small for the list's partial sums");
  return rc;
}

int clipped_update(const SgdSet& host, const SgdSet* set, const AdamSet* adam, double* part, float max_norm, float lr, float* out_norm,
                   hipStream_t s) {
  static_assert(sizeof(SgdSet::p) / sizeof(float*) <= CLIP_TENSORS, "one launch has all tensors of a training step");
  int64_t numel[CLIP_TENSORS];
  int32_t dtype[CLIP_TENSORS];
  for (int i = 0; i < host.cnt; ++i) { numel[i] = host.n[i]; dtype[i] = TGNN_F32; }
  ClipArgs a = {};
  int n_part = 0;
  if (int rc = norm_launches(host.cnt, reinterpret_cast<const void* const*>(host.g), numel, dtype, a, part,
                             CLIP_PARTS * (int64_t)sizeof(double), s, n_part))
    return rc;
  hipLaunchKernelGGL(clipped_update_kernel, dim3(64 * host.cnt), dim3(256), 0, s, set, adam, part, n_part, max_norm, lr, out_norm);
  TGNN_LAUNCH_CHECK();
  return TGNN_OK;
}

}  // namespace tgnn

using namespace tgnn;

extern "C" int64_t tgnn_clip_workspace_bytes(int32_t n_tensors) { return clip_bytes(n_tensors); }

static int check_norm_call(int32_t n, const void* const* g, const int64_t* numel, const int32_t* dtype, const float* out_norm,
                           const void* ws, int64_t ws_bytes) {
  if (int rc = check_tensors(n, g, numel, dtype)) return rc;
  if (out_norm == nullptr) return set_error(TGNN_E_NULL_PTR, "out_norm is NULL");
  if (!aligned_to(out_norm, 4)) return set_error(TGNN_E_MISALIGNED, "out_norm is not aligned to its type");
  if (ws == nullptr) return set_error(TGNN_E_NULL_PTR, "workspace is NULL");
  if (!aligned_to(ws, 16)) return set_error(TGNN_E_MISALIGNED, "workspace is not 16-byte aligned");
  if (ws_bytes < clip_bytes(n))
    return set_error(TGNN_E_WORKSPACE, "workspace of %lld bytes, %lld are needed", (long long)ws_bytes, (long long)clip_bytes(n));
  return TGNN_OK;
}

extern "C" int32_t tgnn_grad_norm(int32_t n_tensors, const void* const* g, const int64_t* numel, const int32_t* dtype, float* out_norm,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
  if (int rc = check_norm_call(n_tensors, g, numel, dtype, out_norm, workspace, workspace_bytes)) return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  ClipArgs a = {};
  int n_part = 0;
  if (int rc = norm_launches(n_tensors, g, numel, dtype, a, static_cast<double*>(workspace), workspace_bytes, s, n_part)) return rc;
  hipLaunchKernelGGL(clip_norm_kernel, dim3(1), dim3(256), 0, s, static_cast<const double*>(workspace), n_part, out_norm);
  TGNN_LAUNCH_CHECK();
  return TGNN_OK;
}

extern "C" int32_t tgnn_clip_grads(int32_t n_tensors, void* const* g, const int64_t* numel, const int32_t* dtype, float max_norm,
                                   void* const* out, float* out_norm, void* workspace, int64_t workspace_bytes, void* stream) {
  if (int rc = check_norm_call(n_tensors, const_cast<const void* const*>(g), numel, dtype, out_norm, workspace, workspace_bytes)) return rc;
  if (!(max_norm > 0.0f)) return set_error(TGNN_E_INVALID_ARG, "max_norm = %g: a positive number is needed", (double)max_norm);
  for (int i = 0; out != nullptr && i < n_tensors; ++i) {
    if (numel[i] > 0 && out[i] == nullptr) return set_error(TGNN_E_NULL_PTR, "out[%d] is NULL", i);
    if (!aligned_to(out[i], type_size(dtype[i]))) return set_error(TGNN_E_MISALIGNED, "out[%d] is not aligned to its type", i);
  }
  if (int rc = check_apart(n_tensors, g, out, numel, dtype)) return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  ClipArgs a = {};
  int n_part = 0;
  double* part = static_cast<double*>(workspace);
  if (int rc = norm_launches(n_tensors, const_cast<const void* const*>(g), numel, dtype, a, part, workspace_bytes, s, n_part)) return rc;
  if (n_part == 0) {   // nothing to clip
    hipLaunchKernelGGL(clip_norm_kernel, dim3(1), dim3(256), 0, s, part, 0, out_norm);
    TGNN_LAUNCH_CHECK();
    return TGNN_OK;
  }
  a.part = part; a.n_part = n_part; a.max_norm = max_norm; a.out_norm = out_norm; a.write_norm = 1;
  return clip_launches(n_tensors, const_cast<const void* const*>(g), out, numel, dtype, a, [&](int blocks) {
    hipLaunchKernelGGL(clip_scale_kernel, dim3(blocks), dim3(256), 0, s, a);
    a.write_norm = 0;
  });
}
