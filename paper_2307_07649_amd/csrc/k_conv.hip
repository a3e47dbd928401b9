// Short causal convolution over the events of a sequence, one filter per column (tgnn_causal_conv_fwd, _bwd, _step):
//
//   pre[t, c] = b[c] + sum over j < W of w[c, j] x[t - (W - 1) + j, c],  y = pre or silu(pre) = pre / (1 + exp(-pre))
//   g = dy silu'(pre);  dx[t] = sum over j of w[j] g[t + (W - 1) - j];  dw[j] = sum over t of g[t] x[t - (W - 1) + j];  db = sum of g
//
// What lies before a sequence's first event is its state, the W - 1 inputs before it, or zero.
//
// Bound by memory: a thread has one pack of columns and walks along a segment of a sequence with the last W inputs (and, on the way
// back, the last W values of g, from which a row of dx is complete) in registers, so that a row is read once; what two
// neighbouring segments both need (W - 1 rows on either side) is read twice.  Threads of a workgroup that no column is
// left for take another segment.  29,000 rows of 1,024 columns in bfloat16, four taps: forward 30 us, 4.0 TB/s; backward 62 us, 2.9
// TB/s, the vector units busy in 53 per cent of the cycles of three wavefronts each; 4,000 single events 18.7 us, 3.5 TB/s.
#include <algorithm>

#include "seq_device.h"

namespace tgnn {

constexpr int CONV_GRID = 768;    // workgroups of the backward pass (partial rows of dw and db): three to a compute unit
constexpr int AHEAD = 4;          // rows on their way
constexpr int CONV_ANY = TGNN_MAX_CONV_WIDTH;

struct ConvArgs {
  tgnn_seqs q;
  const void *x, *dy;
  const float *w, *bias;
  const void* state_in;
  void* state_out;
  const int32_t* state_idx;
  void* y;                        // y, or dx
  float* part;                    // [grid, d W + d]
  int64_t ld_x, ld_dy, ld_y, items;
  int d, width, n_states, silu, per_x, bits;   // per_x: threads of a workgroup along the columns; segments of 2^bits rows
};

__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }

// Taps of V columns, `left` of which there are; W == CONV_ANY: any number of them up to that, in the places behind.  (V * W values
// next to each other: as vector loads, for which four bytes are aligned enough.)
template <int V, int W> __device__ __forceinline__ void conv_taps(const ConvArgs& a, int c, int left, float (&w)[W][V], float (&b)[V]) {
  if constexpr (W != CONV_ANY) {
    float r[V * W];
    take_floats<V * W>(a.w + (int64_t)c * W, left * W, 0.0f, r);
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) w[j][i] = r[i * W + j];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const int k = j - (W - a.width);
        w[j][i] = k >= 0 && i < left ? a.w[(int64_t)(c + i) * a.width + k] : 0.0f;
      }
  }
  take_floats<V>(a.bias ? a.bias + c : nullptr, left, 0.0f, b);
}
// the input at place t of the sequence: a row, a row of the state, or zero
template <class T, int V, bool ANY>
__device__ __forceinline__ void conv_input(const ConvArgs& a, const Seq& r, int64_t state, int t, int c, float (&v)[V]) {
  const T* p = nullptr;
  if (t >= 0) p = static_cast<const T*>(a.x) + seq_row(a.q, r, t) * a.ld_x + c;
  else if (state >= 0 && a.state_in != nullptr) p = static_cast<const T*>(a.state_in) + (state * (a.width - 1) + (a.width - 1) + t) * a.d + c;
  if (p != nullptr) unpack(take<T, V, ANY>(p, a.d - c), v);
  else
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = 0.0f;
}
template <int V, int W> __device__ __forceinline__ void conv_sum(const ConvArgs& a, const float (&win)[W][V], const float (&w)[W][V],
                                                                const float (&b)[V], float (&pre)[V]) {
#pragma unroll
  for (int i = 0; i < V; ++i) pre[i] = b[i];
#pragma unroll
  for (int j = 0; j < W; ++j)
    if (W != CONV_ANY || j >= W - a.width)   // (a place without a tap may hold an infinity)
#pragma unroll
      for (int i = 0; i < V; ++i) pre[i] = fmaf(w[j][i], win[j][i], pre[i]);
}
template <int V, int W> __device__ __forceinline__ void shift_in(float (&win)[W][V], const float (&v)[V]) {
#pragma unroll
  for (int j = 0; j + 1 < W; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) win[j][i] = win[j + 1][i];
#pragma unroll
  for (int i = 0; i < V; ++i) win[W - 1][i] = v[i];
}
__device__ __forceinline__ int64_t state_of(const int32_t* idx, int n_states, int s) {
  const int64_t i = idx != nullptr ? idx[s] : s;
  return i >= 0 && i < n_states ? i : -1;
}

// WIDE: a wavefront's threads are all at one segment, whose numbers are then scalars (backward 63 us, and 74 without).  ANY: rows at any
// address, of any number of columns (rows that packs fit taken that way: forward 47 us for 30, backward 109 for 63).
template <class T, int V, int W, bool WIDE, bool ANY>
__global__ __launch_bounds__(256) void conv_fwd_kernel(ConvArgs a) {
  const int per_y = 256 / a.per_x, col_tiles = (a.d + a.per_x * V - 1) / (a.per_x * V);
  const unsigned number = group_number();
  const int c = ((int)(number % col_tiles) * a.per_x + (int)threadIdx.x % a.per_x) * V;
  const int64_t first = (int64_t)(number / col_tiles) * per_y;
  if (first >= a.items) return;
  const int item0 = (int)first, item = item0 + (int)threadIdx.x / a.per_x;
  const int s0 = seg_find(a.q, item0, a.bits);
  if (c >= a.d || item >= a.items) return;
  const int at = WIDE ? __builtin_amdgcn_readfirstlane(item) : item;
  const Piece p = piece_of(a.q, at, a.bits, seg_find_from(a.q, at, a.bits, s0));
  if (p.none) return;
  const int64_t state = state_of(a.state_idx, a.n_states, p.s);
  float w[W][V], b[V], win[W][V];
  conv_taps<V, W>(a, c, a.d - c, w, b);
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int i = 0; i < V; ++i) win[j][i] = 0.0f;
#pragma unroll
  for (int j = 0; j + 1 < W; ++j)
    if (j + 1 < a.width) {   // the places t0 - (width - 1) .. t0 - 1
      float v[V];
      conv_input<T, V, ANY>(a, p.r, state, p.t0 - (a.width - 1) + j, c, v);
      shift_in<V, W>(win, v);
    }
  // rows are asked for AHEAD before their use, past the caches: 29,000 rows of 1,024 columns in bfloat16 30 us, through them 40 (what
  // reads x next is the backward pass; there, and for y, it gains nothing)
  const int64_t step = a.q.newest_first ? -1 : 1;
  const T* x = static_cast<const T*>(a.x) + seq_row(a.q, p.r, p.t0) * a.ld_x + c;
  T* y = static_cast<T*>(a.y) + seq_row(a.q, p.r, p.t0) * a.ld_y + c;
  Pack<T, V> next[AHEAD];
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (p.t0 + u < p.t1) next[u] = take<T, V, ANY, true>(x + u * step * a.ld_x, a.d - c);
  const bool silu = a.silu != 0;
  auto row = [&](int u) {
    float v[V], pre[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)next[u].v[i];
    shift_in<V, W>(win, v);
    conv_sum<V, W>(a, win, w, b, pre);
#pragma unroll
    for (int i = 0; i < V; ++i) pre[i] *= silu ? sigmoid(pre[i]) : 1.0f;
    put<T, V, ANY>(y + u * step * a.ld_y, pre, a.d - c);
  };
  int t = p.t0;
  for (; t + AHEAD <= p.t1; t += AHEAD) {   // whole groups
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      row(u);
      const int ahead = min(u + AHEAD, p.t1 - 1 - t);   // (past the end: a row that is there)
      next[u] = take<T, V, ANY, true>(x + ahead * step * a.ld_x, a.d - c);
    }
    x += AHEAD * step * a.ld_x;
    y += AHEAD * step * a.ld_y;
  }
#pragma unroll
  for (int u = 0; u < AHEAD; ++u)
    if (t + u < p.t1) row(u);
  if (!p.last) return;
  float zero[V] = {};
  for (int t = p.r.len; t < p.r.slot; ++t) put<T, V, ANY>(static_cast<T*>(a.y) + (p.r.begin + t) * a.ld_y + c, zero, a.d - c);
  if (state >= 0 && a.state_out != nullptr)
#pragma unroll
    for (int j = 1; j < W; ++j)
      if (j >= W - (a.width - 1))
        put<T, V, ANY>(static_cast<T*>(a.state_out) + (state * (a.width - 1) + j - (W - (a.width - 1))) * a.d + c, win[j], a.d - c);
}

// One event of each of `items` nodes.
template <class T, int V, int W, bool ANY>
__global__ __launch_bounds__(256) void conv_step_kernel(ConvArgs a) {
  const int packs = (a.d + V - 1) / V;
  const int64_t i = (int64_t)group_number() * 256 + threadIdx.x;
  if (i >= a.items * packs) return;
  const int64_t row = i / packs;
  const int c = (int)(i - row * packs) * V;
  const int64_t state = state_of(a.state_idx, a.n_states, (int)row);
  float w[W][V], b[V], win[W][V], pre[V];
#pragma unroll
  for (int j = 0; j < W; ++j)
#pragma unroll
    for (int k = 0; k < V; ++k) win[j][k] = 0.0f;
#pragma unroll
  for (int j = 0; j + 1 < W; ++j) {
    const int k = j - (W - a.width);
    if (k >= 0 && state >= 0 && a.state_in != nullptr)
      unpack(take<T, V, ANY>(static_cast<const T*>(a.state_in) + (state * (a.width - 1) + k) * a.d + c, a.d - c), win[j]);
  }
  unpack(take<T, V, ANY>(static_cast<const T*>(a.x) + row * a.ld_x + c, a.d - c), win[W - 1]);
  conv_taps<V, W>(a, c, a.d - c, w, b);
  conv_sum<V, W>(a, win, w, b, pre);
  if (a.silu)
#pragma unroll
    for (int k = 0; k < V; ++k) pre[k] *= sigmoid(pre[k]);
  put<T, V, ANY>(static_cast<T*>(a.y) + row * a.ld_y + c, pre, a.d - c);
  if (state >= 0 && a.state_out != nullptr)
#pragma unroll
    for (int j = 1; j < W; ++j) {
      const int k = j - 1 - (W - a.width);
      // (past the caches: 4,000 rows of 1,024 columns in float16 18.9 us, through them 20.5)
      if (k >= 0) put<T, V, ANY, true>(static_cast<T*>(a.state_out) + (state * (a.width - 1) + k) * a.d + c, win[j], a.d - c);
    }
}

template <class T, int V, int W, bool WIDE, bool ANY>
__global__ __launch_bounds__(256) void conv_bwd_kernel(ConvArgs a) {
  __shared__ float acc[256 * V];
  const int per_y = 256 / a.per_x, col_tiles = (a.d + a.per_x * V - 1) / (a.per_x * V);
  const int tx = (int)threadIdx.x % a.per_x, ty = (int)threadIdx.x / a.per_x;
  const int c = ((int)(blockIdx.x % col_tiles) * a.per_x + tx) * V;
  const int worker = blockIdx.x / col_tiles, workers = gridDim.x / col_tiles;
  const bool on = c < a.d;
  float w[W][V], b[V], dw[W][V], db[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    b[i] = db[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < W; ++j) w[j][i] = dw[j][i] = 0.0f;
  }
  if (on) conv_taps<V, W>(a, c, a.d - c, w, b);
  const int halo = a.width - 1;
  for (int64_t item0 = (int64_t)worker * per_y; item0 < a.items; item0 += (int64_t)workers * per_y) {
    const int s0 = seg_find(a.q, (int)item0, a.bits), item = (int)item0 + ty;
    if (!on || item >= a.items) continue;
    const int at = WIDE ? __builtin_amdgcn_readfirstlane(item) : item;
    const Piece p = piece_of(a.q, at, a.bits, seg_find_from(a.q, at, a.bits, s0));
    if (p.none) continue;
    const int64_t state = state_of(a.state_idx, a.n_states, p.s);
    float win[W][V], gw[W][V];
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) win[j][i] = gw[j][i] = 0.0f;
#pragma unroll
    for (int j = 0; j + 1 < W; ++j)
      if (j < halo) {
        float v[V];
        conv_input<T, V, ANY>(a, p.r, state, p.t0 - halo + j, c, v);
        shift_in<V, W>(win, v);
      }
    // g[t] of the segment's events and of the `halo` behind them completes dx[t - halo].  Behind the sequence's end g is zero.
    const bool silu = a.silu != 0;
    const int t_end = min(p.t1 + halo, p.r.len);   // events that g is formed of
    const int64_t step = a.q.newest_first ? -1 : 1;
    const T* x = static_cast<const T*>(a.x) + seq_row(a.q, p.r, p.t0) * a.ld_x + c;
    const T* dy = static_cast<const T*>(a.dy) + seq_row(a.q, p.r, p.t0) * a.ld_dy + c;
    T* dx = static_cast<T*>(a.y) + seq_row(a.q, p.r, p.t0) * a.ld_y + c;
    Pack<T, V> nx[AHEAD], ndy[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (p.t0 + u < t_end) {
        nx[u] = take<T, V, ANY>(x + u * step * a.ld_x, a.d - c);
        ndy[u] = take<T, V, ANY>(dy + u * step * a.ld_dy, a.d - c);
      }
    // one event; INSIDE: it is the segment's own, and dx[t - halo] as well
    auto event = [&](auto inside, int t, int u) {
      constexpr bool INSIDE = decltype(inside)::value;
      float g[V];
      if (INSIDE || t < t_end) {
        float v[V], pre[V];
#pragma unroll
        for (int i = 0; i < V; ++i) { v[i] = (float)nx[u].v[i]; g[i] = (float)ndy[u].v[i]; }
        shift_in<V, W>(win, v);
        conv_sum<V, W>(a, win, w, b, pre);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float sg = sigmoid(pre[i]);
          g[i] *= silu ? sg * fmaf(pre[i], 1.0f - sg, 1.0f) : 1.0f;
        }
        if (INSIDE || t < p.t1) {
#pragma unroll
          for (int j = 0; j < W; ++j)
            if (W != CONV_ANY || j >= W - a.width)
#pragma unroll
              for (int i = 0; i < V; ++i) dw[j][i] = fmaf(g[i], win[j][i], dw[j][i]);
#pragma unroll
          for (int i = 0; i < V; ++i) db[i] += g[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = 0.0f;
      }
      shift_in<V, W>(gw, g);
      if (INSIDE || (t >= p.t0 + halo && t < p.t1 + halo)) {
        // dx[t - halo] = sum over m of w[width - 1 - m] g[t - halo + m]: gw[j] is that with m = j - (W - width), its tap's place 2 W - 1 - width - j
        float o[V] = {};
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
          for (int k = W != CONV_ANY ? W - 1 - j : 0; k < (W != CONV_ANY ? W - j : W); ++k)
            if (W != CONV_ANY || (j >= W - a.width && k == 2 * W - 1 - a.width - j))
#pragma unroll
              for (int i = 0; i < V; ++i) o[i] = fmaf(w[k][i], gw[j][i], o[i]);
        put<T, V, ANY>(dx + (u - halo) * step * a.ld_y, o, a.d - c);
      }
    };
    auto ask = [&](int t4, int u) {
      const int ahead = min(u + AHEAD, t_end - 1 - t4);   // (past the end: a row that is there)
      nx[u] = take<T, V, ANY>(x + ahead * step * a.ld_x, a.d - c);
      ndy[u] = take<T, V, ANY>(dy + ahead * step * a.ld_dy, a.d - c);
    };
    auto on_to = [&]() {
      x += AHEAD * step * a.ld_x;
      dy += AHEAD * step * a.ld_dy;
      dx += AHEAD * step * a.ld_y;
    };
    int t4 = p.t0;
    auto border = [&]() {   // a group that is not all inside
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (t4 + u < p.t1 + halo) event(std::false_type(), t4 + u, u);
        if (t4 + AHEAD < t_end) ask(t4, u);
      }
      on_to();
      t4 += AHEAD;
    };
    while (t4 < p.t0 + halo && t4 < p.t1 + halo) border();
    for (; t4 + AHEAD <= p.t1; t4 += AHEAD) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        event(std::true_type(), t4 + u, u);
        ask(t4, u);
      }
      on_to();
    }
    while (t4 < p.t1 + halo) border();
    if (p.last) {
      float zero[V] = {};
      for (int t = p.r.len; t < p.r.slot; ++t) put<T, V, ANY>(static_cast<T*>(a.y) + (p.r.begin + t) * a.ld_y + c, zero, a.d - c);
    }
  }
  if (a.part == nullptr) return;
  // the threads of a column in the workgroup, added up in order; laid out like dw [d, width], then db [d]
  float* part = a.part + (int64_t)worker * (a.d * (int64_t)(a.width + 1));
#pragma unroll
  for (int j = 0; j <= W; ++j) {
    if (j < W - a.width) continue;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < V; ++i) acc[threadIdx.x * V + i] = j < W ? dw[j < W ? j : 0][i] : db[i];
    __syncthreads();
    if (ty == 0 && on)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if (ANY && c + i >= a.d) continue;
        float sum = 0.0f;
        for (int r = 0; r < per_y; ++r) sum += acc[(r * a.per_x + tx) * V + i];
        if (j < W) part[(int64_t)(c + i) * a.width + j - (W - a.width)] = sum;
        else part[(int64_t)a.d * a.width + c + i] = sum;
      }
  }
}

// f(T(), V, W, ANY): packs of 16 bytes, or of four values (FOUR: with eight the backward pass has two wavefronts to a vector
// unit instead of three, and takes 101 us for 63)
template <bool FOUR, class F> static void conv_shape(int dtype, int width, int d, int64_t rows, const void* const* p, const int64_t* ld, int n, F f) {
  with_type(dtype, [&](auto t) {
    constexpr int V = FOUR ? 4 : 16 / sizeof(t);
    const std::integral_constant<int, V> v;
    auto by_width = [&](auto any) {
      if (width == 2) f(t, v, std::integral_constant<int, 2>(), any);
      else if (width == 3) f(t, v, std::integral_constant<int, 3>(), any);
      else if (width == 4) f(t, v, std::integral_constant<int, 4>(), any);
      else f(t, v, std::integral_constant<int, CONV_ANY>(), any);
    };
    if (packs_fit(dtype, V, d, rows, p, ld, n)) by_width(std::false_type());
    else by_width(std::true_type());
  });
}

// Rows of a segment, 2^4 to 2^6: as many as leave `waves` wavefronts with four rows each on their way.  What is read
// twice is 5 per cent with 64 rows and four taps, 20 per cent (out of the L2) with 16.  (29,000 rows of 1,024 columns in bfloat16, backward, on
// one set of inputs: 57 us with 3,000, 53 with 1,500, 63 with 6,000; forward, and 7,000 to 120,000 rows of 1,024 to 100 columns,
// within one per cent of each other with half or twice as many.)
static int conv_bits(const tgnn_seqs& q, int d, int v, int waves) {
  const int64_t rows = q.indptr == nullptr ? (int64_t)q.n_seqs * q.max_len : q.n_rows, packs = (d + v - 1) / v;
  int bits = 6;
  while (bits > 4 && (rows >> bits) * packs < (int64_t)waves * 64) --bits;
  return bits;
}

static int conv_columns(int d, int v) {   // threads of a workgroup along the columns: a power of two, at most all
  int n = 1;
  while (n < 256 && n * v < d) n *= 2;
  return n;
}

int check_seqs(const tgnn_seqs* q) {
  if (q == nullptr) return set_error(TGNN_E_NULL_PTR, "seqs is NULL");
  if (q->n_seqs < 0 || q->max_len < 0 || q->n_rows < 0)
    return set_error(TGNN_E_INVALID_ARG, "a negative count in seqs (%d sequences, max_len %d, %lld rows)", q->n_seqs, q->max_len, (long long)q->n_rows);
  if (q->newest_first != 0 && q->newest_first != 1) return set_error(TGNN_E_INVALID_ARG, "newest_first = %d", q->newest_first);
  if (!aligned_to(q->indptr, 8) || !aligned_to(q->cnt, 4)) return set_error(TGNN_E_MISALIGNED, "indptr or cnt is not aligned to its type");
  if (q->indptr == nullptr && (int64_t)q->n_seqs * q->max_len > q->n_rows)
    return set_error(TGNN_E_OUT_OF_RANGE, "%d sequences of %d rows do not fit %lld rows", q->n_seqs, q->max_len, (long long)q->n_rows);
  if (q->n_rows >= (int64_t(1) << 33) || seg_total(*q, MIN_SEG_BITS) > INT_MAX)   // (segments are numbered by 31 bits)
    return set_error(TGNN_E_OUT_OF_RANGE, "%lld rows in %d sequences", (long long)q->n_rows, q->n_seqs);
  return TGNN_OK;
}

static int check_conv(int32_t dtype, int32_t d, int32_t width, const float* w, const float* bias, int32_t n_states, const int32_t* idx) {
  if (!type_known(dtype)) return set_error(TGNN_E_INVALID_ARG, "dtype = %d is none of TGNN_F32, TGNN_BF16, TGNN_F16", dtype);
  if (d < 1 || d > TGNN_MAX_SEQ_WIDTH) return set_error(TGNN_E_UNSUPPORTED_DIM, "d = %d outside [1, %d]", d, TGNN_MAX_SEQ_WIDTH);
  if (width < 1 || width > TGNN_MAX_CONV_WIDTH)
    return set_error(TGNN_E_UNSUPPORTED_DIM, "width = %d outside [1, %d]", width, TGNN_MAX_CONV_WIDTH);
  if (w == nullptr) return set_error(TGNN_E_NULL_PTR, "weight is NULL");
  if (!aligned_to(w, 4) || !aligned_to(bias, 4) || !aligned_to(idx, 4))
    return set_error(TGNN_E_MISALIGNED, "weight, bias or state_idx is not aligned to its type");
  if (n_states < 0) return set_error(TGNN_E_INVALID_ARG, "n_states = %d is negative", n_states);
  return TGNN_OK;
}

int check_row_array(const char* name, const void* p, int64_t ld, int64_t rows, int cols, int dtype) {
  if (rows > 0 && p == nullptr) return set_error(TGNN_E_NULL_PTR, "%s is NULL", name);
  if (!aligned_to(p, type_size(dtype))) return set_error(TGNN_E_MISALIGNED, "%s is not aligned to its type", name);
  if (ld < cols) return set_error(TGNN_E_INVALID_ARG, "the rows of %s are %lld apart and %d long", name, (long long)ld, cols);
  if (ld > (int64_t(1) << 27)) return set_error(TGNN_E_OUT_OF_RANGE, "the rows of %s are %lld apart", name, (long long)ld);
  return TGNN_OK;
}

}  // namespace tgnn

using namespace tgnn;

static int conv_grid(int64_t groups, int col_tiles, dim3* out) {
  const int64_t n = groups * col_tiles;
  if (n > INT_MAX) return set_error(TGNN_E_OUT_OF_RANGE, "%lld workgroups", (long long)n);
  *out = group_grid(n);
  return TGNN_OK;
}

extern "C" int32_t tgnn_causal_conv_fwd(const tgnn_seqs* seqs, int32_t dtype, int32_t d, int32_t width, const void* x, int64_t ld_x,
                                        const float* weight, const float* bias, int32_t silu, const void* state_in, void* state_out,
                                        const int32_t* state_idx, int32_t n_states, void* y, int64_t ld_y, void* stream) {
  if (int rc = check_seqs(seqs)) return rc;
  if (int rc = check_conv(dtype, d, width, weight, bias, n_states, state_idx)) return rc;
  if (int rc = check_row_array("x", x, ld_x, seqs->n_rows, d, dtype)) return rc;
  if (int rc = check_row_array("y", y, ld_y, seqs->n_rows, d, dtype)) return rc;
  const int size = type_size(dtype);
  if (!aligned_to(state_in, size) || !aligned_to(state_out, size)) return set_error(TGNN_E_MISALIGNED, "a state is not aligned to its type");
  const size_t state_bytes = (size_t)n_states * (width - 1) * d * size;
  if (spans_overlap(state_in, state_bytes, state_out, state_bytes)) return set_error(TGNN_E_INVALID_ARG, "state_out overlaps state_in");
  if (rows_overlap(seqs->n_rows, size, {x, d, ld_x}, {y, d, ld_y}))
    return set_error(TGNN_E_INVALID_ARG, "y overlaps x");
  if (seqs->n_seqs == 0) return TGNN_OK;
  ConvArgs a = {};
  a.q = *seqs; a.x = x; a.w = weight; a.bias = bias; a.y = y;
  a.state_in = width > 1 ? state_in : nullptr; a.state_out = width > 1 ? state_out : nullptr; a.state_idx = state_idx;
  a.ld_x = ld_x; a.ld_y = ld_y; a.d = d; a.width = width; a.n_states = n_states; a.silu = silu != 0;
  const void* p[] = {x, y, a.state_in, a.state_out};
  const int64_t ld[] = {ld_x, ld_y, d, d};
  int rc = TGNN_OK;
  conv_shape<false>(dtype, width, d, seqs->n_rows, p, ld, 4, [&](auto t, auto v, auto wd, auto any) {
    using T = decltype(t);
    constexpr int V = decltype(v)::value, W = decltype(wd)::value;
    constexpr bool ANY = decltype(any)::value;
    a.bits = conv_bits(*seqs, d, V, 4096);
    a.items = seg_total(*seqs, a.bits);
    a.per_x = conv_columns(d, V);
    const int per_y = 256 / a.per_x, tiles = (d + a.per_x * V - 1) / (a.per_x * V);
    dim3 grid;
    rc = conv_grid((a.items + per_y - 1) / per_y, tiles, &grid);
    if (rc != TGNN_OK) return;
    if (a.per_x >= 64) hipLaunchKernelGGL((conv_fwd_kernel<T, V, W, true, ANY>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
    else hipLaunchKernelGGL((conv_fwd_kernel<T, V, W, false, ANY>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
  });
  if (rc != TGNN_OK) return rc;
  TGNN_LAUNCH_CHECK();
  return TGNN_OK;
}

extern "C" int32_t tgnn_causal_conv_step(int32_t dtype, int64_t n_rows, int32_t d, int32_t width, const void* x, int64_t ld_x,
                                         const float* weight, const float* bias, int32_t silu, const void* state_in, void* state_out,
                                         const int32_t* state_idx, int32_t n_states, void* y, int64_t ld_y, void* stream) {
  if (n_rows < 0 || n_rows > INT_MAX) return set_error(TGNN_E_OUT_OF_RANGE, "n_rows = %lld outside [0, 2^31)", (long long)n_rows);
  if (int rc = check_conv(dtype, d, width, weight, bias, n_states, state_idx)) return rc;
  if (int rc = check_row_array("x", x, ld_x, n_rows, d, dtype)) return rc;
  if (int rc = check_row_array("y", y, ld_y, n_rows, d, dtype)) return rc;
  const int size = type_size(dtype);
  if (!aligned_to(state_in, size) || !aligned_to(state_out, size)) return set_error(TGNN_E_MISALIGNED, "a state is not aligned to its type");
  const size_t state_bytes = (size_t)n_states * (width - 1) * d * size;
  if (state_in != state_out && spans_overlap(state_in, state_bytes, state_out, state_bytes))
    return set_error(TGNN_E_INVALID_ARG, "state_out overlaps state_in without being it");
  if (!(x == y && ld_x == ld_y) && rows_overlap(n_rows, size, {x, d, ld_x}, {y, d, ld_y}))
    return set_error(TGNN_E_INVALID_ARG, "y overlaps x without being it");
  if (n_rows == 0) return TGNN_OK;
  ConvArgs a = {};
  a.x = x; a.w = weight; a.bias = bias; a.y = y;
  a.state_in = width > 1 ? state_in : nullptr; a.state_out = width > 1 ? state_out : nullptr; a.state_idx = state_idx;
  a.ld_x = ld_x; a.ld_y = ld_y; a.items = n_rows;
  a.d = d; a.width = width; a.n_states = n_states; a.silu = silu != 0;
  const void* p[] = {x, y, a.state_in, a.state_out};
  const int64_t ld[] = {ld_x, ld_y, d, d};
  int rc = TGNN_OK;
  conv_shape<false>(dtype, width, d, n_rows, p, ld, 4, [&](auto t, auto v, auto wd, auto any) {
    using T = decltype(t);
    constexpr int V = decltype(v)::value, W = decltype(wd)::value;
    dim3 grid;
    rc = conv_grid((n_rows * ((d + V - 1) / V) + 255) / 256, 1, &grid);
    if (rc == TGNN_OK) hipLaunchKernelGGL((conv_step_kernel<T, V, W, decltype(any)::value>), grid, dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a);
  });
  if (rc != TGNN_OK) return rc;
  TGNN_LAUNCH_CHECK();
  return TGNN_OK;
}

extern "C" int64_t tgnn_causal_conv_workspace_bytes(int32_t d, int32_t width) {
  return (int64_t)CONV_GRID * (d > 0 ? d : 1) * ((width > 0 ? width : 1) + 1) * (int64_t)sizeof(float);
}

extern "C" int32_t tgnn_causal_conv_bwd(const tgnn_seqs* seqs, int32_t dtype, int32_t d, int32_t width, const void* dy, int64_t ld_dy,
                                        const void* x, int64_t ld_x, const float* weight, const float* bias, int32_t silu,
                                        const void* state_in, const int32_t* state_idx, int32_t n_states, void* dx, int64_t ld_dx,
                                        float* d_weight, float* d_bias, int32_t accumulate, void* workspace, int64_t workspace_bytes,
                                        void* stream) {
  if (int rc = check_seqs(seqs)) return rc;
  if (int rc = check_conv(dtype, d, width, weight, bias, n_states, state_idx)) return rc;
  if (int rc = check_row_array("dy", dy, ld_dy, seqs->n_rows, d, dtype)) return rc;
  if (int rc = check_row_array("x", x, ld_x, seqs->n_rows, d, dtype)) return rc;
  if (int rc = check_row_array("dx", dx, ld_dx, seqs->n_rows, d, dtype)) return rc;
  if (!aligned_to(state_in, type_size(dtype)) || !aligned_to(d_weight, 4) || !aligned_to(d_bias, 4))
    return set_error(TGNN_E_MISALIGNED, "state_in, d_weight or d_bias is not aligned to its type");
  const int size = type_size(dtype);
  if (rows_overlap(seqs->n_rows, size, {dx, d, ld_dx}, {x, d, ld_x}) || rows_overlap(seqs->n_rows, size, {dx, d, ld_dx}, {dy, d, ld_dy}))
    return set_error(TGNN_E_INVALID_ARG, "dx overlaps x or dy");
  const bool weights = d_weight != nullptr || d_bias != nullptr;
  if (weights) {
    if (workspace == nullptr) return set_error(TGNN_E_NULL_PTR, "workspace is NULL");
    if (!aligned_to(workspace, 16)) return set_error(TGNN_E_MISALIGNED, "workspace is not 16-byte aligned");
    if (workspace_bytes < tgnn_causal_conv_workspace_bytes(d, width))
      return set_error(TGNN_E_WORKSPACE, "workspace of %lld bytes, %lld are needed", (long long)workspace_bytes,
                       (long long)tgnn_causal_conv_workspace_bytes(d, width));
  }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  ConvArgs a = {};
  a.q = *seqs; a.x = x; a.dy = dy; a.w = weight; a.bias = bias; a.y = dx; a.part = weights ? static_cast<float*>(workspace) : nullptr;
  a.state_in = width > 1 ? state_in : nullptr; a.state_idx = state_idx;
  a.ld_x = ld_x; a.ld_dy = ld_dy; a.ld_y = ld_dx;
  a.d = d; a.width = width; a.n_states = n_states; a.silu = silu != 0;
  const void* p[] = {x, dy, dx, a.state_in};
  const int64_t ld[] = {ld_x, ld_dy, ld_dx, d};
  int64_t workers = 0;
  if (seqs->n_seqs > 0) {
    conv_shape<true>(dtype, width, d, seqs->n_rows, p, ld, 4, [&](auto t, auto v, auto wd, auto any) {
      using T = decltype(t);
      constexpr int V = decltype(v)::value, W = decltype(wd)::value;
      constexpr bool ANY = decltype(any)::value;
      a.bits = conv_bits(*seqs, d, V, 3000);
      a.items = seg_total(*seqs, a.bits);
      a.per_x = conv_columns(d, V);
      const int per_y = 256 / a.per_x, tiles = (d + a.per_x * V - 1) / (a.per_x * V);
      workers = std::min<int64_t>((a.items + per_y - 1) / per_y, std::max(1, CONV_GRID / tiles));
      if (a.per_x >= 64) hipLaunchKernelGGL((conv_bwd_kernel<T, V, W, true, ANY>), dim3((unsigned)(workers * tiles)), dim3(256), 0, s, a);
      else hipLaunchKernelGGL((conv_bwd_kernel<T, V, W, false, ANY>), dim3((unsigned)(workers * tiles)), dim3(256), 0, s, a);
    });
    TGNN_LAUNCH_CHECK();
  }
  if (weights) {
    column_sum(ColumnSum{a.part, (int)workers, (int64_t)d * (width + 1), {d_weight, d_bias, nullptr}, {(int64_t)d * width, d, 0}, accumulate}, s);
    TGNN_LAUNCH_CHECK();
  }
  return TGNN_OK;
}
