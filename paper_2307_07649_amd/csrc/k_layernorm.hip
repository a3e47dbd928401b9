// Layer norm over the columns of a row, forward and backward (tgnn_layer_norm_fwd, tgnn_layer_norm_bwd).
//
//   forward   mean = sum x / C, var = sum (x - mean)^2 / C, rstd = 1 / sqrt(var + eps), xh = (x - mean) rstd, y = xh w + b
//   backward  g = dy w:  dx = rstd (g - mean(g) - xh mean(g xh));  dw = sum over the rows of dy xh, db = sum of dy
//
// Bound by memory (132,000 rows of 100 columns of float: forward 22 us, 4.7 TB/s, backward 28 us, 5.7, some of it out of the caches; 8,191
// rows of 4,096 in bfloat16: 28 us, 4.8 TB/s, and 38, 5.3): a row is read once (twice where it is wider than the registers of a workgroup hold) and written once.
// G threads have a row between them, K packs of V values each, so that the second pass of the variance, and the second use of x
// and dy in the backward pass, come from registers: 16 threads for up to 128 columns of float (a wavefront has four rows),
// a wavefront up to 1,024, a workgroup up to 8,192.  The backward pass walks over the rows with a fixed grid; a thread has the
// same columns in every row and adds up its part of dw and db in registers, a workgroup adds up its threads' parts in LDS
// and leaves one partial row.
#include <math.h>

#include <algorithm>

#include "ops_device.h"

namespace tgnn {

constexpr int norm_threads(int g) { return g > 256 ? g : 256; }   // of a workgroup

// sum over the G neighbouring threads that have a row
template <int G, class S> __device__ __forceinline__ S row_sum(S v, S* parts) {
#pragma unroll
  for (int o = (G < 64 ? G : 64) / 2; o > 0; o >>= 1) v += __shfl_xor(v, o);
  if constexpr (G > 64) {
    __syncthreads();   // the parts of the sum before this one have been read
    if ((threadIdx.x & 63) == 0) parts[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < G / 64; ++w) v += parts[w];
  }
  return v;
}

struct NormArgs {
  const void *x, *dy;
  const float *weight, *bias, *mean, *rstd;   // weight, bias: NULL for ones and zeros
  void* y;                                    // y, or dx
  float *out_mean, *out_rstd;                 // may be NULL
  float* part;                                // [grid, 2 C] partial sums of dw and db; NULL: not wanted
  int64_t rows, ld_x, ld_dy, ld_y;
  int cols;
  float eps;
};

// A group of threads walks over rows with the weights of its columns in registers and the next row on its way.
// ANY: rows at any address, of any number of columns (rows that packs fit taken that way: 28 for 22 and 40 for 28 us).
template <class T, int V, int G, int K, bool ANY>
__global__ __launch_bounds__(norm_threads(G)) void norm_fwd_kernel(NormArgs a) {
  __shared__ float parts[8];
  constexpr int GROUPS = norm_threads(G) / G;
  const int c0 = (threadIdx.x % G) * V;
  const float inv = 1.0f / (float)a.cols;
  float w[K][V], b[K][V];
#pragma unroll
  for (int k = 0; k < K; ++k)
    if (c0 + k * G * V < a.cols) {
      take_floats<V>(a.weight ? a.weight + c0 + k * G * V : nullptr, a.cols - c0 - k * G * V, 1.0f, w[k]);
      take_floats<V>(a.bias ? a.bias + c0 + k * G * V : nullptr, a.cols - c0 - k * G * V, 0.0f, b[k]);
    }
  const T* x = static_cast<const T*>(a.x) + c0;
  T* y = static_cast<T*>(a.y) + c0;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G;
  Pack<T, V> next[K];
  auto ask = [&](int64_t r) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (c0 + k * G * V < a.cols) next[k] = take<T, V, ANY>(x + r * a.ld_x + k * G * V, a.cols - c0 - k * G * V);
  };
  if (row < a.rows) ask(row);
  for (; row < a.rows; row += step) {
    float v[K][V], sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[k][i] = c0 + k * G * V < a.cols ? (float)next[k].v[i] : 0.0f;
        sum += v[k][i];
      }
    if (row + step < a.rows) ask(row + step);
    const float mean = row_sum<G>(sum, parts) * inv;
    sum = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (c0 + k * G * V < a.cols)
#pragma unroll
        for (int i = 0; i < V; ++i) sum += !ANY || c0 + k * G * V + i < a.cols ? (v[k][i] - mean) * (v[k][i] - mean) : 0.0f;
    const float rstd = 1.0f / sqrtf(row_sum<G>(sum, parts) * inv + a.eps);
    if (threadIdx.x % G == 0) {
      if (a.out_mean) a.out_mean[row] = mean;
      if (a.out_rstd) a.out_rstd[row] = rstd;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (c0 + k * G * V >= a.cols) continue;
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = (v[k][i] - mean) * rstd * w[k][i] + b[k][i];
      put<T, V, ANY>(y + row * a.ld_y + k * G * V, o, a.cols - c0 - k * G * V);
    }
  }
}

// Rows wider than the registers: three passes, the second and third out of the L2.  A thread has a 256th of a row: its sums are held in
// double, so that errors do not grow with the columns (2,048 rows of 16,384 in bfloat16: 67 us, 2.0 TB/s, and 94 backward; with float
// sums 64 and 92).
template <class T>
__global__ __launch_bounds__(256) void norm_fwd_wide_kernel(NormArgs a) {
  __shared__ double parts[4];
  const int64_t row = group_number();
  if (row >= a.rows) return;
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  double sum = 0.0;
  for (int c = threadIdx.x; c < a.cols; c += 256) sum += (double)(float)x[c];
  const double exact = row_sum<256>(sum, parts) / a.cols;
  sum = 0.0;
  for (int c = threadIdx.x; c < a.cols; c += 256) {
    const double d = (double)(float)x[c] - exact;
    sum = fma(d, d, sum);
  }
  const float mean = (float)exact, rstd = (float)(1.0 / sqrt(row_sum<256>(sum, parts) / a.cols + (double)a.eps));
  if (threadIdx.x == 0) {
    if (a.out_mean) a.out_mean[row] = mean;
    if (a.out_rstd) a.out_rstd[row] = rstd;
  }
  T* y = static_cast<T*>(a.y) + row * a.ld_y;
  for (int c = threadIdx.x; c < a.cols; c += 256)
    y[c] = (T)(((float)x[c] - mean) * rstd * (a.weight ? a.weight[c] : 1.0f) + (a.bias ? a.bias[c] : 0.0f));
}

template <class T, int V, int G, int K, bool ANY>
__global__ __launch_bounds__(norm_threads(G)) void norm_bwd_kernel(NormArgs a) {
  __shared__ float parts[8];
  constexpr int GROUPS = norm_threads(G) / G, W = G * K * V;   // row groups of a workgroup; columns its threads cover
  __shared__ float acc[GROUPS > 1 ? GROUPS : 1][GROUPS > 1 ? W : 1];
  const int c0 = (threadIdx.x % G) * V, group = threadIdx.x / G;
  float w[K][V], dw[K][V], db[K][V];
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int i = 0; i < V; ++i) w[k][i] = dw[k][i] = db[k][i] = 0.0f;   // (columns beyond the row weigh nothing)
    if (c0 + k * G * V < a.cols) take_floats<V>(a.weight ? a.weight + c0 + k * G * V : nullptr, a.cols - c0 - k * G * V, 1.0f, w[k]);
  }
  const float inv = 1.0f / (float)a.cols;
  const T* x = static_cast<const T*>(a.x) + c0;
  const T* dy = static_cast<const T*>(a.dy) + c0;
  T* dx = static_cast<T*>(a.y) + c0;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  int64_t row = (int64_t)blockIdx.x * GROUPS + group;
  Pack<T, V> nx[K], ndy[K];
  float next_mean = 0.0f, next_rstd = 0.0f;
  auto ask = [&](int64_t r) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (c0 + k * G * V < a.cols) {
        nx[k] = take<T, V, ANY>(x + r * a.ld_x + k * G * V, a.cols - c0 - k * G * V);
        ndy[k] = take<T, V, ANY>(dy + r * a.ld_dy + k * G * V, a.cols - c0 - k * G * V);
      }
    next_mean = a.mean[r];
    next_rstd = a.rstd[r];
  };
  if (row < a.rows) ask(row);
  for (; row < a.rows; row += step) {
    const float mean = next_mean, rstd = next_rstd;
    float xh[K][V], g[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) { xh[k][i] = (float)nx[k].v[i]; g[k][i] = (float)ndy[k].v[i]; }
    if (row + step < a.rows) ask(row + step);
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const bool in = c0 + k * G * V + (ANY ? i : 0) < a.cols;
        const float h = in ? (xh[k][i] - mean) * rstd : 0.0f, d = in ? g[k][i] : 0.0f;
        xh[k][i] = h;
        dw[k][i] += d * h;
        db[k][i] += d;
        g[k][i] = d * w[k][i];
        s1 += g[k][i];
        s2 += g[k][i] * h;
      }
    }
    s1 = row_sum<G>(s1, parts) * inv;
    s2 = row_sum<G>(s2, parts) * inv;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (c0 + k * G * V >= a.cols) continue;
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = rstd * (g[k][i] - s1 - xh[k][i] * s2);
      put<T, V, ANY>(dx + row * a.ld_y + k * G * V, o, a.cols - c0 - k * G * V);
    }
  }
  if (a.part == nullptr) return;
  float* part = a.part + (int64_t)blockIdx.x * 2 * a.cols;
#pragma unroll
  for (int q = 0; q < 2; ++q) {   // dw, then db
    if constexpr (GROUPS > 1) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[group][c0 + k * G * V + i] = q ? db[k][i] : dw[k][i];
      __syncthreads();
      for (int c = threadIdx.x; c < a.cols; c += norm_threads(G)) {
        float sum = 0.0f;
#pragma unroll
        for (int r = 0; r < GROUPS; ++r) sum += acc[r][c];
        part[q * a.cols + c] = sum;
      }
    } else {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (c0 + k * G * V < a.cols)
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (!ANY || c0 + k * G * V + i < a.cols) part[q * a.cols + c0 + k * G * V + i] = q ? db[k][i] : dw[k][i];
    }
  }
}

// Rows wider than the registers: the rows' gradients (x and dy twice, the second time out of the L2), after ...
template <class T>
__global__ __launch_bounds__(256) void norm_bwd_wide_kernel(NormArgs a) {
  __shared__ double parts[4];
  const int64_t row = group_number();
  if (row >= a.rows) return;
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
  const float mean = a.mean[row], rstd = a.rstd[row];
  double sum1 = 0.0, sum2 = 0.0;
  for (int c = threadIdx.x; c < a.cols; c += 256) {
    const float g = (float)dy[c] * (a.weight ? a.weight[c] : 1.0f);
    sum1 += (double)g;
    sum2 += (double)(g * (((float)x[c] - mean) * rstd));
  }
  const float s1 = (float)(row_sum<256>(sum1, parts) / a.cols), s2 = (float)(row_sum<256>(sum2, parts) / a.cols);
  T* dx = static_cast<T*>(a.y) + row * a.ld_y;
  for (int c = threadIdx.x; c < a.cols; c += 256) {
    const float g = (float)dy[c] * (a.weight ? a.weight[c] : 1.0f);
    dx[c] = (T)(rstd * (g - s1 - ((float)x[c] - mean) * rstd * s2));
  }
}
// ... the weights', a column per thread over the rows blockIdx.y, + gridDim.y, ...
template <class T>
__global__ __launch_bounds__(256) void norm_bwd_wide_weights_kernel(NormArgs a) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.cols) return;
  double dw = 0.0, db = 0.0;
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float d = (float)static_cast<const T*>(a.dy)[row * a.ld_dy + c];
    dw += (double)(d * (((float)static_cast<const T*>(a.x)[row * a.ld_x + c] - a.mean[row]) * a.rstd[row]));
    db += (double)d;
  }
  float* part = a.part + (int64_t)blockIdx.y * 2 * a.cols;
  part[c] = (float)dw;
  part[a.cols + c] = (float)db;
}

constexpr int NORM_FWD_GRID = 2048;   // workgroups of the forward pass: eight to a compute unit
constexpr int NORM_GRID = 1024;       // workgroups of the backward pass (partial rows of dw and db), 768 where rows are
                                      // so wide that the partial rows' way counts and registers allow three to a compute unit
constexpr int NORM_WIDE_PARTS = 64;   // the same where rows are wider than the registers

// f(G, K) for the smallest group of threads that covers `packs` packs of V values of a row; false: none does.  (Four packs of eight
// values and their sums are more than a thread's registers; 4,810 rows of 1,468 columns in bfloat16 forward and backward with three packs
// a thread in a wavefront 53 us, with one in four wavefronts 43.)
template <int V, class F> static bool norm_shape(int64_t packs, F f) {
  using std::integral_constant;
#define TGNN_NORM_SHAPE(G, K) \
  if (packs <= (G) * (K)) { f(integral_constant<int, G>(), integral_constant<int, K>()); return true; }
  TGNN_NORM_SHAPE(16, 1)
  TGNN_NORM_SHAPE(16, 2)
  TGNN_NORM_SHAPE(64, 1)
  TGNN_NORM_SHAPE(64, 2)
  if constexpr (V == 4) {
    TGNN_NORM_SHAPE(64, 4)
  } else {
    TGNN_NORM_SHAPE(256, 1)
  }
  TGNN_NORM_SHAPE(256, 2)
  TGNN_NORM_SHAPE(512, 2)
  if constexpr (V == 4) {
    TGNN_NORM_SHAPE(512, 4)
  }
#undef TGNN_NORM_SHAPE
  return false;
}
static int64_t norm_grid(int64_t rows, int cols) {
  const int64_t most = cols > 1024 ? 768 : NORM_GRID;
  return rows < most ? (rows > 0 ? rows : 1) : most;
}

static int check_rows(const char* name, const void* p, int64_t ld, int64_t rows, int cols, int dtype) {
  if (rows > 0 && p == nullptr) return set_error(TGNN_E_NULL_PTR, "%s is NULL", name);
  if (!aligned_to(p, type_size(dtype))) return set_error(TGNN_E_MISALIGNED, "%s is not aligned to its type", name);
  if (ld < cols) return set_error(TGNN_E_INVALID_ARG, "the rows of %s are %lld apart and %d long", name, (long long)ld, cols);
  return TGNN_OK;
}
static int check_floats(const char* name, const float* p, bool needed) {
  if (needed && p == nullptr) return set_error(TGNN_E_NULL_PTR, "%s is NULL", name);
  if (!aligned_to(p, 4)) return set_error(TGNN_E_MISALIGNED, "%s is not aligned to its type", name);
  return TGNN_OK;
}
static int check_norm(int32_t dtype, int64_t n_rows, int32_t n_cols) {
  if (!type_known(dtype)) return set_error(TGNN_E_INVALID_ARG, "dtype = %d is none of TGNN_F32, TGNN_BF16, TGNN_F16", dtype);
  if (n_cols < 1 || n_cols > 1 << 28) return set_error(TGNN_E_UNSUPPORTED_DIM, "n_cols = %d outside [1, 2^28]", n_cols);   // (2 n_cols fits an int)
  if (n_rows < 0 || n_rows > INT_MAX) return set_error(TGNN_E_OUT_OF_RANGE, "n_rows = %lld outside [0, 2^31)", (long long)n_rows);
  return TGNN_OK;
}

}  // namespace tgnn

using namespace tgnn;

extern "C" int32_t tgnn_layer_norm_fwd(int32_t dtype, int64_t n_rows, int32_t n_cols, const void* x, int64_t ld_x, const float* weight,
                                       const float* bias, float eps, void* y, int64_t ld_y, float* out_mean, float* out_rstd,
                                       void* stream) {
  if (int rc = check_norm(dtype, n_rows, n_cols)) return rc;
  if (int rc = check_rows("x", x, ld_x, n_rows, n_cols, dtype)) return rc;
  if (int rc = check_rows("y", y, ld_y, n_rows, n_cols, dtype)) return rc;
  if (int rc = check_floats("weight", weight, false)) return rc;
  if (int rc = check_floats("bias", bias, false)) return rc;
  if (int rc = check_floats("out_mean", out_mean, false)) return rc;
  if (int rc = check_floats("out_rstd", out_rstd, false)) return rc;
  if (!(eps >= 0.0f)) return set_error(TGNN_E_INVALID_ARG, "eps = %g: a number that is not negative is needed", (double)eps);
  const int size = type_size(dtype);
  if (!(x == y && ld_x == ld_y) && rows_overlap(n_rows, size, {x, n_cols, ld_x}, {y, n_cols, ld_y}))
    return set_error(TGNN_E_INVALID_ARG, "y overlaps x without being it");
  if (n_rows == 0) return TGNN_OK;
  NormArgs a = {};
  a.x = x; a.weight = weight; a.bias = bias; a.y = y; a.out_mean = out_mean; a.out_rstd = out_rstd;
  a.rows = n_rows; a.ld_x = ld_x; a.ld_y = ld_y; a.cols = n_cols; a.eps = eps;
  const void* p[] = {x, y};
  const int64_t ld[] = {ld_x, ld_y};
  const bool fit = packs_fit(dtype, 16 / type_size(dtype), n_cols, n_rows, p, ld, 2);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  with_type(dtype, [&](auto t) {
    using T = decltype(t);
    constexpr int V = 16 / sizeof(T);
    const bool fits = norm_shape<V>((n_cols + V - 1) / V, [&](auto g, auto k) {
      constexpr int G = decltype(g)::value, K = decltype(k)::value, THREADS = norm_threads(G), PER = THREADS / G;
      const dim3 grid((unsigned)std::min<int64_t>((n_rows + PER - 1) / PER, NORM_FWD_GRID));
      if (fit) hipLaunchKernelGGL((norm_fwd_kernel<T, V, G, K, false>), grid, dim3(THREADS), 0, s, a);
      else hipLaunchKernelGGL((norm_fwd_kernel<T, V, G, K, true>), grid, dim3(THREADS), 0, s, a);
    });
    if (!fits) hipLaunchKernelGGL((norm_fwd_wide_kernel<T>), group_grid(n_rows), dim3(256), 0, s, a);
  });
  TGNN_LAUNCH_CHECK();
  return TGNN_OK;
}

extern "C" int64_t tgnn_layer_norm_workspace_bytes(int64_t n_rows, int32_t n_cols) {
  const int64_t parts = norm_grid(n_rows, n_cols);
  return (parts > NORM_WIDE_PARTS ? parts : NORM_WIDE_PARTS) * 2 * (int64_t)(n_cols > 0 ? n_cols : 1) * (int64_t)sizeof(float);
}

extern "C" int32_t tgnn_layer_norm_bwd(int32_t dtype, int64_t n_rows, int32_t n_cols, const void* dy, int64_t ld_dy, const void* x,
                                       int64_t ld_x, const float* mean, const float* rstd, const float* weight, void* dx,
                                       int64_t ld_dx, float* d_weight, float* d_bias, int32_t accumulate, void* workspace,
                                       int64_t workspace_bytes, void* stream) {
  if (int rc = check_norm(dtype, n_rows, n_cols)) return rc;
  if (int rc = check_rows("dy", dy, ld_dy, n_rows, n_cols, dtype)) return rc;
  if (int rc = check_rows("x", x, ld_x, n_rows, n_cols, dtype)) return rc;
  if (int rc = check_rows("dx", dx, ld_dx, n_rows, n_cols, dtype)) return rc;
  if (int rc = check_floats("mean", mean, n_rows > 0)) return rc;
  if (int rc = check_floats("rstd", rstd, n_rows > 0)) return rc;
  if (int rc = check_floats("weight", weight, false)) return rc;
  if (int rc = check_floats("d_weight", d_weight, false)) return rc;
  if (int rc = check_floats("d_bias", d_bias, false)) return rc;
  const int size = type_size(dtype);
  if (!(dy == dx && ld_dy == ld_dx) && rows_overlap(n_rows, size, {dy, n_cols, ld_dy}, {dx, n_cols, ld_dx}))
    return set_error(TGNN_E_INVALID_ARG, "dx overlaps dy without being it");
  if (rows_overlap(n_rows, size, {x, n_cols, ld_x}, {dx, n_cols, ld_dx})) return set_error(TGNN_E_INVALID_ARG, "dx overlaps x");
  const bool weights = d_weight != nullptr || d_bias != nullptr;
  if (weights) {
    if (workspace == nullptr) return set_error(TGNN_E_NULL_PTR, "workspace is NULL");
    if (!aligned_to(workspace, 16)) return set_error(TGNN_E_MISALIGNED, "workspace is not 16-byte aligned");
    if (workspace_bytes < tgnn_layer_norm_workspace_bytes(n_rows, n_cols))
      return set_error(TGNN_E_WORKSPACE, "workspace of %lld bytes, %lld are needed", (long long)workspace_bytes,
                       (long long)tgnn_layer_norm_workspace_bytes(n_rows, n_cols));
  }
  NormArgs a = {};
  a.x = x; a.dy = dy; a.weight = weight; a.mean = mean; a.rstd = rstd; a.y = dx; a.part = weights ? static_cast<float*>(workspace) : nullptr;
  a.rows = n_rows; a.ld_x = ld_x; a.ld_dy = ld_dy; a.ld_y = ld_dx; a.cols = n_cols;
  const void* p[] = {x, dy, dx};
  const int64_t ld[] = {ld_x, ld_dy, ld_dx};
  const bool fit = packs_fit(dtype, 16 / type_size(dtype), n_cols, n_rows, p, ld, 3);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  int n_part = 0;
  if (n_rows > 0) {
    with_type(dtype, [&](auto t) {
      using T = decltype(t);
      constexpr int V = 16 / sizeof(T);
      const bool fits = norm_shape<V>((n_cols + V - 1) / V, [&](auto g, auto k) {
        constexpr int G = decltype(g)::value, K = decltype(k)::value, THREADS = norm_threads(G), PER = THREADS / G;
        n_part = (int)norm_grid((n_rows + PER - 1) / PER, n_cols);
        if (fit) hipLaunchKernelGGL((norm_bwd_kernel<T, V, G, K, false>), dim3(n_part), dim3(THREADS), 0, s, a);
        else hipLaunchKernelGGL((norm_bwd_kernel<T, V, G, K, true>), dim3(n_part), dim3(THREADS), 0, s, a);
      });
      if (fits) return;
      if (weights) {   // (first: dx may be written over dy)
        n_part = (int)(n_rows < NORM_WIDE_PARTS ? n_rows : NORM_WIDE_PARTS);
        hipLaunchKernelGGL((norm_bwd_wide_weights_kernel<T>), dim3((n_cols + 255) / 256, n_part), dim3(256), 0, s, a);
      }
      hipLaunchKernelGGL((norm_bwd_wide_kernel<T>), group_grid(n_rows), dim3(256), 0, s, a);
    });
    TGNN_LAUNCH_CHECK();
  }
  if (weights) {
    column_sum(ColumnSum{a.part, n_part, 2 * (int64_t)n_cols, {d_weight, d_bias, nullptr}, {n_cols, n_cols, 0}, accumulate}, s);
    TGNN_LAUNCH_CHECK();
  }
  return TGNN_OK;
}
