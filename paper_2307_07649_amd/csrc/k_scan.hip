// Selective state space scan over the events of a sequence (tgnn_selective_scan_fwd, _bwd, _step).  Per column c with N states:
//
//   delta = softplus(dt + bias) (or dt + bias),  a[n] = exp(delta A[c, n]),  h[t, n] = a[n] h[t - 1, n] + delta x B[t, n]
//   y0 = sum over n of C[t, n] h[t, n] + D[c] x,  y = y0 silu(z) (or y0)
//
// and backwards, with gy = dy silu(z) and lam[t, n] = d loss / d h[t, n]:
//
//   lam[t] = C[t] gy[t] + a[t + 1] lam[t + 1]
//   dC[t, n] = sum over c of gy h,  dB[t, n] = sum over c of lam delta x,  s1 = sum over n of lam B,  s2 = sum over n of A lam a h[t - 1]
//   dx = D gy + delta s1,  ddelta = x s1 + s2,  ddt = ddelta sigmoid(dt + bias),  dz = dy y0 silu'(z)
//   dA[c, n] = sum over t of delta lam a h[t - 1],  dD = sum of gy x,  dbias = sum of ddt
//
// The state a sequence starts from is a constant, as stored memories are everywhere in this library.
//
// Bound by the vector units: an event costs every state of every column an exponential (quarter rate) and four multiplications
// or additions, some 32 cycles for 64 of them, against 8 to 16 bytes of memory per column.
//
// Forward, a lane has a column with all its states in registers: no sum crosses lanes, and B and C of an event are the same for
// the whole wavefront.  The recurrence along the events is what limits how many wavefronts there are; long sequences are
// cut into segments whose states are formed in three launches: each segment's own part (from a zero state) with the sum of
// its deltas, then from segment to segment h = exp(A sum of delta) h + part, then the outputs, every segment from its own
// first state.  Sequences that are short against the whole of the work are walked in one launch.
//
// Backward, four lanes have a column, N / 4 states each: a wavefront has 16 columns, so that sums over the states and over the
// columns each cross few lanes, and the four lanes form softplus and the gates of four events, one each.  The states come
// again from those saved every 32 events: a pass over the 32 leaves the state before every fourth event in LDS, then the
// groups of four are taken from the last to the first.
#include <math.h>

#include <algorithm>

#include "device_math.h"
#include "seq_device.h"

namespace tgnn {

constexpr int CHUNK = 32;               // events between two saved states
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct ScanArgs {
  tgnn_seqs q;
  const void *x, *dt, *B, *C, *z, *dy;
  const float *A, *D, *bias;
  const float* state_in;
  float* state_out;
  const int32_t* state_idx;
  void *y, *dx, *ddt, *dz, *dB, *dC;
  float* saved;                         // [chunks, d, n] state before every chunk
  float *seg_state, *seg_delta;         // [segments, d, n], [segments, d]
  float* part;                          // [workers, d n + 2 d] partial sums of dA, dD, dbias
  float* part_bc;                       // [column tiles of a group, rows, 2, groups n]; NULL: dB and dC are written directly
  int64_t ld_x, ld_dt, ld_b, ld_c, ld_z, ld_dy, ld_y, ld_dx, ld_ddt, ld_dz, ld_db, ld_dc, items;
  int d, n, groups, dg, n_states, softplus;
  int seg;                              // events of a segment, 0: sequences are not cut
  int tiles;                            // column tiles of a group
};

// log(1 + exp(v)) = max(v, 0) + log1p(e), e = exp(-|v|); log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3, by its series up to s^15
// (the next term is 2^-29 of the first).  Relative to the value, for large negative v too.
__device__ __forceinline__ float softplus(float v) {
  const float e = __builtin_amdgcn_exp2f(-fabsf(v) * LOG2E);
  const float s = e * __builtin_amdgcn_rcpf(2.0f + e), q = s * s;
  float p = fmaf(q, 1.0f / 15, 1.0f / 13);
  p = fmaf(q, p, 1.0f / 11);
  p = fmaf(q, p, 1.0f / 9);
  p = fmaf(q, p, 1.0f / 7);
  p = fmaf(q, p, 1.0f / 5);
  p = fmaf(q, p, 1.0f / 3);
  p = fmaf(q, p, 1.0f);
  return fmaf(2.0f * s, p, fmaxf(v, 0.0f));
}
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v * LOG2E)); }

__device__ __forceinline__ float lane_value(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }

__device__ __forceinline__ int64_t state_of(const ScanArgs& a, int s) {
  const int64_t i = a.state_idx != nullptr ? a.state_idx[s] : s;
  return i >= 0 && i < a.n_states ? i : -1;
}

// N states of a column from and to memory
template <int NP> __device__ __forceinline__ void load_states(const float* p, int n, float (&h)[NP]) {
  if (n == NP && NP % 4 == 0 && (n & 3) == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
    for (int i = 0; i + 3 < NP; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p + i);
      h[i] = v.x; h[i + 1] = v.y; h[i + 2] = v.z; h[i + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NP; ++i) h[i] = i < n ? p[i] : 0.0f;
  }
}
template <int NP> __device__ __forceinline__ void store_states(float* p, int n, const float (&h)[NP]) {
  if (n == NP && NP % 4 == 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
    for (int i = 0; i + 3 < NP; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(h[i], h[i + 1], h[i + 2], h[i + 3]);
  } else {
#pragma unroll
    for (int i = 0; i < NP; ++i)
      if (i < n) p[i] = h[i];
  }
}

enum { SCAN_Y, SCAN_STATES, SCAN_PART };   // outputs; saved states only; a segment's own part

// What a wavefront asks for of an event before it needs it
template <class T> struct Event { T x, dt, z; T b, c; };

// One wavefront: 64 columns of a group over a segment (or a whole sequence).
template <class T, int NP, int MODE>
__global__ __launch_bounds__(256) void scan_fwd_kernel(ScanArgs a) {
  const unsigned wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const unsigned all = (unsigned)(a.groups * a.tiles), item = wave / all, tile = wave - item * all;
  if (item >= a.items) return;
  const Piece p = piece_at(a.q, item, a.seg);
  if (p.none || (MODE == SCAN_PART && p.last)) return;
  const int g = tile / a.tiles, col = (tile - g * a.tiles) * 64 + lane;
  const bool on = col < a.dg;
  const unsigned c = g * a.dg + (on ? col : a.dg - 1);
  const int64_t state = state_of(a, p.s);
  float A[NP], h[NP];
  load_states<NP>(a.A + (int64_t)c * a.n, a.n, A);
  if (MODE != SCAN_PART && a.seg != 0) load_states<NP>(a.seg_state + (p.slot * a.d + c) * a.n, a.n, h);
  else if (MODE != SCAN_PART && state >= 0 && a.state_in != nullptr) load_states<NP>(a.state_in + (state * a.d + c) * a.n, a.n, h);
  else
#pragma unroll
    for (int i = 0; i < NP; ++i) h[i] = 0.0f;
  const float bias = a.bias ? a.bias[c] : 0.0f, D = a.D ? a.D[c] : 0.0f;
  const bool gated = MODE == SCAN_Y && a.z != nullptr;
  const unsigned bl = g * a.n + (lane < (unsigned)a.n ? lane : a.n - 1);   // lane n holds B and C of state n
  float total = 0.0f;   // of the deltas
  auto ask = [&](int t, Event<T>& e) {
    const int64_t row = seq_row(a.q, p.r, t);
    e.x = (static_cast<const T*>(a.x) + row * a.ld_x)[c];
    e.dt = (static_cast<const T*>(a.dt) + row * a.ld_dt)[c];
    if (gated) e.z = (static_cast<const T*>(a.z) + row * a.ld_z)[c];
    e.b = (static_cast<const T*>(a.B) + row * a.ld_b)[bl];
    if (MODE == SCAN_Y) e.c = (static_cast<const T*>(a.C) + row * a.ld_c)[bl];
  };
  constexpr int U = 4;
  Event<T> next[U];
  if (p.t0 < p.t1)
#pragma unroll
    for (int u = 0; u < U; ++u) ask(min(p.t0 + u, p.t1 - 1), next[u]);
  for (int t4 = p.t0; t4 < p.t1; t4 += U) {
    Event<T> e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) e[u] = next[u];
    if (t4 + U < p.t1)
#pragma unroll
      for (int u = 0; u < U; ++u) ask(min(t4 + U + u, p.t1 - 1), next[u]);
    if (MODE != SCAN_PART && a.saved != nullptr && t4 % CHUNK == 0 && on)
      store_states<NP>(a.saved + ((seg_base(a.q, p.s, CHUNK) + t4 / CHUNK) * a.d + c) * a.n, a.n, h);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t4 + u < p.t1) {
      const float x = (float)e[u].x, raw = (float)e[u].dt + bias, delta = a.softplus ? softplus(raw) : raw;
      const float d2 = delta * LOG2E, in = delta * x, bv = lane < (unsigned)a.n ? (float)e[u].b : 0.0f;
      if (MODE == SCAN_PART) total += delta;
      float y[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < NP; ++i) {   // (states beyond n stay zero)
        h[i] = fmaf(__builtin_amdgcn_exp2f(d2 * A[i]), h[i], in * lane_value(bv, i));
        if (MODE == SCAN_Y) y[i & 1] = fmaf(h[i], lane_value((float)e[u].c, i), y[i & 1]);
      }
      if (MODE == SCAN_Y) {
        float out = fmaf(D, x, y[0] + y[1]);
        if (gated) out *= (float)e[u].z * sigmoid((float)e[u].z);
        if (on) (static_cast<T*>(a.y) + seq_row(a.q, p.r, t4 + u) * a.ld_y)[c] = (T)out;
      }
      }
    }
  }
  if (!on) return;
  if (MODE == SCAN_PART) {
    store_states<NP>(a.seg_state + (p.slot * a.d + c) * a.n, a.n, h);
    a.seg_delta[p.slot * a.d + c] = total;
  }
  if (MODE == SCAN_Y && p.last) {
    for (int t = p.r.len; t < p.r.slot; ++t) (static_cast<T*>(a.y) + (p.r.begin + t) * a.ld_y)[c] = (T)0.0f;
    if (state >= 0 && a.state_out != nullptr) store_states<NP>(a.state_out + (state * a.d + c) * a.n, a.n, h);
  }
}

// The way back through a segment, for its own part of what reaches the segment before it: g = a[t] (C[t] gy[t] + g), from zero.
template <class T, int NP>
__global__ __launch_bounds__(256) void scan_back_part_kernel(ScanArgs a) {
  const unsigned wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const unsigned all = (unsigned)(a.groups * a.tiles), item = wave / all, tile = wave - item * all;
  if (item >= a.items) return;
  const Piece p = piece_at(a.q, item, a.seg);
  if (p.none || p.t0 == 0) return;
  const int grp = tile / a.tiles, col = (tile - grp * a.tiles) * 64 + lane;
  const bool on = col < a.dg;
  const unsigned c = grp * a.dg + (on ? col : a.dg - 1);
  float A[NP], g[NP];
  load_states<NP>(a.A + (int64_t)c * a.n, a.n, A);
#pragma unroll
  for (int i = 0; i < NP; ++i) g[i] = 0.0f;
  const float bias = a.bias ? a.bias[c] : 0.0f;
  const unsigned bl = grp * a.n + (lane < (unsigned)a.n ? lane : a.n - 1);
  float total = 0.0f;
  auto ask = [&](int t, Event<T>& e) {
    const int64_t row = seq_row(a.q, p.r, t);
    e.x = (static_cast<const T*>(a.dy) + row * a.ld_dy)[c];
    e.dt = (static_cast<const T*>(a.dt) + row * a.ld_dt)[c];
    if (a.z) e.z = (static_cast<const T*>(a.z) + row * a.ld_z)[c];
    e.c = (static_cast<const T*>(a.C) + row * a.ld_c)[bl];
  };
  constexpr int U = 4;
  Event<T> next[U];
#pragma unroll
  for (int u = 0; u < U; ++u) ask(max(p.t1 - 1 - u, p.t0), next[u]);
  for (int t4 = p.t1 - 1; t4 >= p.t0; t4 -= U) {
    Event<T> e[U];
#pragma unroll
    for (int u = 0; u < U; ++u) e[u] = next[u];
    if (t4 - U >= p.t0)
#pragma unroll
      for (int u = 0; u < U; ++u) ask(max(t4 - U - u, p.t0), next[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t4 - u >= p.t0) {
      const float raw = (float)e[u].dt + bias, delta = a.softplus ? softplus(raw) : raw, d2 = delta * LOG2E;
      const float cv = lane < (unsigned)a.n ? (float)e[u].c : 0.0f;
      float gy = (float)e[u].x;
      if (a.z) gy *= (float)e[u].z * sigmoid((float)e[u].z);
      total += delta;
#pragma unroll
      for (int i = 0; i < NP; ++i) g[i] = __builtin_amdgcn_exp2f(d2 * A[i]) * fmaf(gy, lane_value(cv, i), g[i]);
      }
    }
  }
  if (!on) return;
  store_states<NP>(a.seg_state + (p.slot * a.d + c) * a.n, a.n, g);
  a.seg_delta[p.slot * a.d + c] = total;
}

// From segment to segment.  Forward: seg_state[k] becomes the state before segment k, from the sequence's first state; backward: what
// reaches segment k from behind, from zero.  A thread per sequence, column and state.
template <bool BACK>
__global__ __launch_bounds__(256) void scan_chain_kernel(ScanArgs a) {
  const int64_t dn = (int64_t)a.d * a.n, i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= a.q.n_seqs * dn) return;
  const int s = (int)(i / dn);
  const int64_t e = i - s * dn;
  const int c = (int)(e / a.n);
  const Seq r = seq_at(a.q, s);
  const int64_t base = seg_base(a.q, s, a.seg);
  const int count = r.len > 0 ? (int)(((int64_t)r.len + a.seg - 1) / a.seg) : 1;
  const int64_t state = state_of(a, s);
  float cur = !BACK && state >= 0 && a.state_in != nullptr ? a.state_in[state * dn + e] : 0.0f;
  const float A = a.A[e];
  for (int k = 0; k < count; ++k) {
    const int64_t at = base + (BACK ? count - 1 - k : k);
    float* p = a.seg_state + at * dn + e;
    // (forward the last segment's part is not formed, backward the first one's)
    const float part = k + 1 < count ? *p : 0.0f, delta = k + 1 < count ? a.seg_delta[at * a.d + c] : 0.0f;
    *p = cur;
    cur = fmaf(__builtin_amdgcn_exp2f(delta * LOG2E * A), cur, part);
  }
}

// ---- backward ----
template <int CTRL> __device__ __forceinline__ float dpp_get(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xf, 0xf, true));
}
constexpr int QUAD_XOR1 = 0xB1, QUAD_XOR2 = 0x4E, ROW_ROR4 = 0x124, ROW_ROR8 = 0x128;
// the value that lane I of the four has
template <int I> __device__ __forceinline__ float quad_get(float v) { return dpp_get<I * 0x55>(v); }
// v[i] summed over the four lanes: lane i gets the sum of v[i]
__device__ __forceinline__ float quad_scatter_sum(const float (&v)[4], bool odd, bool high) {
  const float p = (odd ? v[1] : v[0]) + dpp_get<QUAD_XOR1>(odd ? v[0] : v[1]);
  const float q = (odd ? v[3] : v[2]) + dpp_get<QUAD_XOR1>(odd ? v[2] : v[3]);
  return (high ? q : p) + dpp_get<QUAD_XOR2>(high ? p : q);
}
// u of the lower and v of the upper half of the wavefront, each summed with the other half's
__device__ __forceinline__ float halves_sum(float u, float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(u), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// the same for the even and odd rows of 16 lanes
__device__ __forceinline__ float rows_sum(float u, float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(u), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Wavefronts of a workgroup: as many as 48 KB of LDS hold the states of (three workgroups to a compute unit)
constexpr int bwd_waves(int np) { return np <= 4 ? 4 : np == 8 ? 2 : 1; }

// A workgroup: 16 columns per wavefront of one group, over the pieces worker, worker + workers, ...
template <class T, int NP>
__global__ __launch_bounds__(64 * bwd_waves(NP)) void scan_bwd_kernel(ScanArgs a) {
  constexpr int WAVES = bwd_waves(NP), THREADS = 64 * WAVES, N4 = 4 * NP;
  __shared__ float bound[CHUNK / 4][THREADS * NP];   // a lane's states before every fourth event
  __shared__ float sB[CHUNK][N4], sC[CHUNK][N4];     // of the chunk's events
  __shared__ float red[WAVES][CHUNK][2][N4];         // dB, dC summed over a wavefront's columns
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, q = lane & 3;
  const int all = a.groups * a.tiles, tile = blockIdx.x % all, worker = blockIdx.x / all, workers = gridDim.x / all;
  const int grp = tile / a.tiles, sub = tile - grp * a.tiles;
  const int col = sub * 16 * WAVES + wave * 16 + (lane >> 2);
  const bool on = col < a.dg, full = __all(on), odd = (q & 1) != 0, high = (q & 2) != 0;
  const unsigned c = grp * a.dg + (on ? col : a.dg - 1);
  float A[NP], dA[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    A[i] = q * NP + i < a.n ? a.A[(int64_t)c * a.n + q * NP + i] : 0.0f;
    dA[i] = 0.0f;
  }
  const float bias = a.bias ? a.bias[c] : 0.0f, D = a.D ? a.D[c] : 0.0f;
  float dD = 0.0f, dbias = 0.0f;
  auto at = [&](const void* p, int64_t ld, int64_t row) -> float { return (float)(static_cast<const T*>(p) + row * ld)[c]; };

  for (int64_t item = worker; item < a.items; item += workers) {
    const Piece p = piece_at(a.q, item, a.seg);
    if (p.none) continue;
    float g[NP];   // what reaches the state behind the event in hand from the events after it
#pragma unroll
    for (int i = 0; i < NP; ++i)
      g[i] = a.seg != 0 && on && q * NP + i < a.n ? a.seg_state[(p.slot * a.d + c) * a.n + q * NP + i] : 0.0f;
    const int64_t chunk0 = seg_base(a.q, p.s, CHUNK);
    for (int tb = p.t1 > p.t0 ? p.t0 + (p.t1 - 1 - p.t0) / CHUNK * CHUNK : p.t0 - CHUNK; tb >= p.t0; tb -= CHUNK) {
      const int n_ev = min(CHUNK, p.t1 - tb), n_sub = (n_ev + 3) / 4;
      for (int i = tid; i < CHUNK * N4; i += THREADS) {
        const int t = i / N4, n = i - t * N4;
        float b = 0.0f, cc = 0.0f;
        if (t < n_ev && n < a.n) {
          const int64_t row = seq_row(a.q, p.r, tb + t);
          b = (float)(static_cast<const T*>(a.B) + row * a.ld_b)[grp * a.n + n];
          cc = (float)(static_cast<const T*>(a.C) + row * a.ld_c)[grp * a.n + n];
        }
        sB[t][n] = b;
        sC[t][n] = cc;
      }
      __syncthreads();
      float h[NP];
      const float* sv = a.saved + ((chunk0 + tb / CHUNK) * a.d + c) * a.n + q * NP;
#pragma unroll
      for (int i = 0; i < NP; ++i) h[i] = on && q * NP + i < a.n ? sv[i] : 0.0f;
      // forward over the chunk: the state before every fourth event
      for (int j = 0; j < n_sub; ++j) {
#pragma unroll
        for (int i = 0; i < NP; ++i) bound[j][tid * NP + i] = h[i];
        if (j + 1 == n_sub) break;
        const int t = 4 * j + q;
        const int64_t row = seq_row(a.q, p.r, tb + t);
        const float x = on ? at(a.x, a.ld_x, row) : 0.0f, raw = at(a.dt, a.ld_dt, row) + bias;
        const float delta = a.softplus ? softplus(raw) : raw, d2 = delta * LOG2E, in = delta * x;
        const float d2s[4] = {quad_get<0>(d2), quad_get<1>(d2), quad_get<2>(d2), quad_get<3>(d2)};
        const float ins[4] = {quad_get<0>(in), quad_get<1>(in), quad_get<2>(in), quad_get<3>(in)};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < NP; ++i)
            h[i] = fmaf(__builtin_amdgcn_exp2f(d2s[e] * A[i]), h[i], ins[e] * sB[4 * j + e][q * NP + i]);
      }
      // and back, four events at a time; a lane has the event's own quantities of event 4 j + q
      for (int j = n_sub - 1; j >= 0; --j) {
        const int t = 4 * j + q;
        const bool there = t < n_ev;
        const int64_t row = seq_row(a.q, p.r, tb + (there ? t : 0));
        float x = 0.0f, raw = 0.0f, z = 0.0f, dy = 0.0f, delta = 0.0f, sg = 0.0f, gy = 0.0f;
        if (there && on) {
          x = at(a.x, a.ld_x, row);
          raw = at(a.dt, a.ld_dt, row) + bias;
          dy = at(a.dy, a.ld_dy, row);
          delta = a.softplus ? softplus(raw) : raw;
          gy = dy;
          if (a.z) {
            z = at(a.z, a.ld_z, row);
            sg = sigmoid(z);
            gy = dy * z * sg;
          }
        }
        const float d2 = delta * LOG2E, in = delta * x;
        const float d2s[4] = {quad_get<0>(d2), quad_get<1>(d2), quad_get<2>(d2), quad_get<3>(d2)};
        const float ins[4] = {quad_get<0>(in), quad_get<1>(in), quad_get<2>(in), quad_get<3>(in)};
        const float gys[4] = {quad_get<0>(gy), quad_get<1>(gy), quad_get<2>(gy), quad_get<3>(gy)};
        float dec[4][NP], ah[4][NP], vB[4][NP], vC[4][NP], y[4], s1[4], s2[4];
#pragma unroll
        for (int i = 0; i < NP; ++i) h[i] = bound[j][tid * NP + i];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = 0.0f;
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            dec[e][i] = __builtin_amdgcn_exp2f(d2s[e] * A[i]);
            ah[e][i] = dec[e][i] * h[i];
            h[i] = fmaf(ins[e], sB[4 * j + e][q * NP + i], ah[e][i]);
            vC[e][i] = gys[e] * h[i];
            y[e] = fmaf(h[i], sC[4 * j + e][q * NP + i], y[e]);
          }
        }
#pragma unroll
        for (int e = 3; e >= 0; --e) {
          s1[e] = s2[e] = 0.0f;
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            const float lam = fmaf(sC[4 * j + e][q * NP + i], gys[e], g[i]), lah = lam * ah[e][i];
            s1[e] = fmaf(lam, sB[4 * j + e][q * NP + i], s1[e]);
            s2[e] = fmaf(A[i], lah, s2[e]);
            dA[i] = fmaf(d2s[e], lah, dA[i]);
            vB[e][i] = lam * ins[e];
            g[i] = dec[e][i] * lam;
          }
        }
        const float y0 = quad_scatter_sum(y, odd, high), t1 = quad_scatter_sum(s1, odd, high), t2 = quad_scatter_sum(s2, odd, high);
        if (there && on) {
          const float dd = fmaf(x, t1, t2), draw = a.softplus ? dd * sigmoid(raw) : dd;
          (static_cast<T*>(a.dx) + row * a.ld_dx)[c] = (T)fmaf(D, gy, delta * t1);
          (static_cast<T*>(a.ddt) + row * a.ld_ddt)[c] = (T)draw;
          if (a.z) (static_cast<T*>(a.dz) + row * a.ld_dz)[c] = (T)(dy * fmaf(D, x, y0) * (sg * fmaf(z, 1.0f - sg, 1.0f)));
          dD = fmaf(gy, x, dD);
          dbias += draw;
        }
        if (!full)   // a column that is none adds nothing (not even where C is infinite)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < NP; ++i) {
              vB[e][i] = on ? vB[e][i] : 0.0f;
              vC[e][i] = on ? vC[e][i] : 0.0f;
            }
        // sums over the wavefront's 16 columns: lower half dB, upper half dC; even rows events 0 and 1, odd rows 2 and 3
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            float v = rows_sum(halves_sum(vB[e][i], vC[e][i]), halves_sum(vB[e + 2][i], vC[e + 2][i]));
            v += dpp_get<ROW_ROR8>(v);
            v += dpp_get<ROW_ROR4>(v);
            if ((lane & 12) == 0) red[wave][4 * j + e + 2 * ((lane >> 4) & 1)][lane >> 5][q * NP + i] = v;
          }
      }
      __syncthreads();
      for (int i = tid; i < n_ev * 2 * N4; i += THREADS) {
        const int t = i / (2 * N4), kind = i / N4 & 1, n = i % N4;
        if (n >= a.n) continue;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += red[w][t][kind][n];
        const int64_t row = seq_row(a.q, p.r, tb + t);
        const int k = grp * a.n + n;
        if (a.part_bc != nullptr) a.part_bc[((sub * a.q.n_rows + row) * 2 + kind) * a.groups * a.n + k] = sum;
        else if (kind == 0) (static_cast<T*>(a.dB) + row * a.ld_db)[k] = (T)sum;
        else (static_cast<T*>(a.dC) + row * a.ld_dc)[k] = (T)sum;
      }
    }
    if (p.last) {   // padding rows
      for (int t = p.r.len + q; t < p.r.slot; t += 4) {
        if (!on) continue;
        const int64_t row = p.r.begin + t;
        (static_cast<T*>(a.dx) + row * a.ld_dx)[c] = (T)0.0f;
        (static_cast<T*>(a.ddt) + row * a.ld_ddt)[c] = (T)0.0f;
        if (a.z) (static_cast<T*>(a.dz) + row * a.ld_dz)[c] = (T)0.0f;
      }
      if (sub == 0)
        for (int64_t i = tid; i < (int64_t)(p.r.slot - p.r.len) * a.n; i += THREADS) {
          const int64_t row = p.r.begin + p.r.len + i / a.n;
          const int k = grp * a.n + (int)(i % a.n);
          (static_cast<T*>(a.dB) + row * a.ld_db)[k] = (T)0.0f;
          (static_cast<T*>(a.dC) + row * a.ld_dc)[k] = (T)0.0f;
        }
    }
  }
  if (a.part == nullptr) return;
  float* part = a.part + (int64_t)worker * ((int64_t)a.d * a.n + 2 * a.d);
  dD += dpp_get<QUAD_XOR1>(dD);
  dD += dpp_get<QUAD_XOR2>(dD);
  dbias += dpp_get<QUAD_XOR1>(dbias);
  dbias += dpp_get<QUAD_XOR2>(dbias);
  if (!on) return;
#pragma unroll
  for (int i = 0; i < NP; ++i)
    if (q * NP + i < a.n) part[(int64_t)c * a.n + q * NP + i] = dA[i] * LN2;   // (it was summed up with delta log2 e)
  if (q == 0) {
    part[(int64_t)a.d * a.n + c] = dD;
    part[(int64_t)a.d * a.n + a.d + c] = dbias;
  }
}

// dB and dC of the rows of sequences: the column tiles' parts in order
template <class T>
__global__ __launch_bounds__(256) void scan_bc_sum_kernel(ScanArgs a) {
  const Piece p = piece_at(a.q, blockIdx.x, CHUNK);
  if (p.none) return;
  const int per = a.groups * a.n;
  for (int i = threadIdx.x; i < (p.t1 - p.t0) * 2 * per; i += 256) {
    const int t = i / (2 * per), r = i - t * 2 * per, kind = r / per, k = r - kind * per;
    const int64_t row = seq_row(a.q, p.r, p.t0 + t);
    float sum = 0.0f;
    for (int w = 0; w < a.tiles; ++w) sum += a.part_bc[((w * a.q.n_rows + row) * 2 + kind) * per + k];
    if (kind == 0) (static_cast<T*>(a.dB) + row * a.ld_db)[k] = (T)sum;
    else (static_cast<T*>(a.dC) + row * a.ld_dc)[k] = (T)sum;
  }
}

// One event of each of `items` nodes: LC neighbouring lanes have a column, NP states each, next to each other in memory.
template <class T, int NP>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a, int lc_bits) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> lc_bits;
  const int part = threadIdx.x & ((1 << lc_bits) - 1);
  const bool on = i < a.items * a.d;
  const int64_t row = on ? i / a.d : 0;
  const int c = on ? (int)(i - row * a.d) : 0;
  const int g = c / a.dg;
  const int64_t state = state_of(a, (int)row);
  const float x = (float)(static_cast<const T*>(a.x) + row * a.ld_x)[c];
  const float raw = (float)(static_cast<const T*>(a.dt) + row * a.ld_dt)[c] + (a.bias ? a.bias[c] : 0.0f);
  const float delta = a.softplus ? softplus(raw) : raw, in = delta * x, d2 = delta * LOG2E;
  float y = 0.0f;
  float h[NP];
  const bool stored = state >= 0 && a.state_in != nullptr;
  const int64_t s0 = (state * a.d + c) * a.n + part * NP;
#pragma unroll
  for (int k = 0; k < NP; ++k) {
    const int n = part * NP + k;
    h[k] = 0.0f;
    if (n >= a.n) continue;
    const float h0 = stored ? a.state_in[s0 + k] : 0.0f;
    const float B = (float)(static_cast<const T*>(a.B) + row * a.ld_b)[g * a.n + n], C = (float)(static_cast<const T*>(a.C) + row * a.ld_c)[g * a.n + n];
    h[k] = fmaf(__builtin_amdgcn_exp2f(d2 * a.A[(int64_t)c * a.n + n]), h0, in * B);
    y = fmaf(h[k], C, y);
  }
  for (int o = 1; o < 1 << lc_bits; o <<= 1) y += __shfl_xor(y, o);
  if (!on) return;
  if (state >= 0 && a.state_out != nullptr)
#pragma unroll
    for (int k = 0; k < NP; ++k)
      if (part * NP + k < a.n) a.state_out[s0 + k] = h[k];
  if (part != 0) return;
  y = fmaf(a.D ? a.D[c] : 0.0f, x, y);
  if (a.z) {
    const float z = (float)(static_cast<const T*>(a.z) + row * a.ld_z)[c];
    y *= z * sigmoid(z);
  }
  (static_cast<T*>(a.y) + row * a.ld_y)[c] = (T)y;
}

// ---- host side ----
int check_row_array(const char* name, const void* p, int64_t ld, int64_t rows, int cols, int dtype);

static int check_scan(const tgnn_scan* p, int64_t rows) {
  if (p == nullptr) return set_error(TGNN_E_NULL_PTR, "scan is NULL");
  if (!type_known(p->dtype)) return set_error(TGNN_E_INVALID_ARG, "dtype = %d is none of TGNN_F32, TGNN_BF16, TGNN_F16", p->dtype);
  if (p->d < 1 || p->d > TGNN_MAX_SEQ_WIDTH) return set_error(TGNN_E_UNSUPPORTED_DIM, "d = %d outside [1, %d]", p->d, TGNN_MAX_SEQ_WIDTH);
  if (p->n_state < 1 || p->n_state > TGNN_MAX_SCAN_STATES)
    return set_error(TGNN_E_UNSUPPORTED_DIM, "n_state = %d outside [1, %d]", p->n_state, TGNN_MAX_SCAN_STATES);
  if (p->n_groups < 1 || p->d % p->n_groups != 0) return set_error(TGNN_E_UNSUPPORTED_DIM, "%d groups of %d columns", p->n_groups, p->d);
  if (int rc = check_row_array("x", p->x, p->ld_x, rows, p->d, p->dtype)) return rc;
  if (int rc = check_row_array("dt", p->dt, p->ld_dt, rows, p->d, p->dtype)) return rc;
  if (int rc = check_row_array("B", p->B, p->ld_b, rows, p->n_groups * p->n_state, p->dtype)) return rc;
  if (int rc = check_row_array("C", p->C, p->ld_c, rows, p->n_groups * p->n_state, p->dtype)) return rc;
  if (p->z != nullptr)
    if (int rc = check_row_array("z", p->z, p->ld_z, rows, p->d, p->dtype)) return rc;
  if (p->A == nullptr) return set_error(TGNN_E_NULL_PTR, "A is NULL");
  if (!aligned_to(p->A, 4) || !aligned_to(p->D, 4) || !aligned_to(p->dt_bias, 4) || !aligned_to(p->state_in, 4) || !aligned_to(p->state_idx, 4))
    return set_error(TGNN_E_MISALIGNED, "A, D, dt_bias, state_in or state_idx is not aligned to its type");
  if (p->n_states < 0) return set_error(TGNN_E_INVALID_ARG, "n_states = %d is negative", p->n_states);
  return TGNN_OK;
}

static ScanArgs scan_args(const tgnn_seqs* q, const tgnn_scan* p) {
  ScanArgs a = {};
  if (q) a.q = *q;
  a.x = p->x; a.dt = p->dt; a.B = p->B; a.C = p->C; a.z = p->z; a.A = p->A; a.D = p->D; a.bias = p->dt_bias;
  a.ld_x = p->ld_x; a.ld_dt = p->ld_dt; a.ld_b = p->ld_b; a.ld_c = p->ld_c; a.ld_z = p->ld_z;
  a.state_in = p->state_in; a.state_idx = p->state_idx; a.n_states = p->n_states;
  a.d = p->d; a.n = p->n_state; a.groups = p->n_groups; a.dg = p->d / p->n_groups; a.softplus = p->softplus != 0;
  return a;
}

// Rows that a call's sequences hold at most, and the longest of them as far as the caller says
static int64_t scan_rows(const tgnn_seqs& q) { return q.indptr == nullptr ? (int64_t)q.n_seqs * q.max_len : q.n_rows; }

// Events of a segment (a multiple of CHUNK), 0: sequences are walked whole.  `units` wavefronts (forward) or workgroups
// (backward) have a sequence between them, `spread` of them run side by side at full speed, `fill` times as many hide each other's
// latencies.  Whole, a call takes as many steps as the longest sequence has events, or as all of them share out; in segments it
// takes 1.8 times the shared work (every event once more for the segments' parts), some 40 steps' time for two more launches,
// and the walk over one segment.
static int scan_segment(const tgnn_seqs& q, int64_t units, int64_t spread, int64_t fill) {
  const int64_t rows = scan_rows(q), longest = std::min<int64_t>(q.max_len, rows), work = rows * units / spread;
  const int64_t seg = std::min<int64_t>(std::max<int64_t>((work / fill + CHUNK - 1) / CHUNK * CHUNK, CHUNK), 4096);
  return std::max(longest, work) > work + work * 4 / 5 + 40 + seg ? (int)seg : 0;
}

template <class F> static void scan_shape(int dtype, int n, F f) {   // f(T(), states of a lane that has them all)
  with_type(dtype, [&](auto t) {
    if (n <= 4) f(t, std::integral_constant<int, 4>());
    else if (n <= 8) f(t, std::integral_constant<int, 8>());
    else if (n <= 16) f(t, std::integral_constant<int, 16>());
    else if (n <= 32) f(t, std::integral_constant<int, 32>());
    else f(t, std::integral_constant<int, 64>());
  });
}

struct Take {   // pieces of a workspace
  char* base;
  int64_t off = 0;
  float* floats(int64_t n) {
    float* p = base ? reinterpret_cast<float*>(base + off) : nullptr;
    off += (n * (int64_t)sizeof(float) + 255) / 256 * 256;
    return p;
  }
};

constexpr int FWD_SPREAD = 1024, FWD_FILL = 4;   // wavefronts: one, and four, to a vector unit
static int fwd_tiles(int dg) { return (dg + 63) / 64; }
static int fwd_segment(const tgnn_seqs& q, int groups, int dg) { return scan_segment(q, (int64_t)groups * fwd_tiles(dg), FWD_SPREAD, FWD_FILL); }

static int64_t fwd_bytes(const tgnn_seqs& q, int d, int n, int groups, ScanArgs* a, void* ws) {
  Take t{static_cast<char*>(ws)};
  const int seg = fwd_segment(q, groups, d / groups);
  if (seg != 0) {
    float *st = t.floats(seg_total(q, seg) * d * n), *dl = t.floats(seg_total(q, seg) * d);
    if (a) { a->seg_state = st; a->seg_delta = dl; }
  }
  return t.off;
}

static int launch_grid(int64_t n, unsigned* out) {
  if (n > INT_MAX) return set_error(TGNN_E_OUT_OF_RANGE, "%lld workgroups", (long long)n);
  *out = (unsigned)n;
  return TGNN_OK;
}

// The launches of a forward pass; MODE: SCAN_Y or SCAN_STATES
template <int MODE> static int scan_forward(ScanArgs a, hipStream_t s, int dtype) {
  a.tiles = fwd_tiles(a.dg);
  a.seg = fwd_segment(a.q, a.groups, a.dg);
  a.items = a.seg ? seg_total(a.q, a.seg) : a.q.n_seqs;
  const int64_t waves = a.items * a.groups * a.tiles;
  if (waves > INT_MAX) return set_error(TGNN_E_OUT_OF_RANGE, "%lld wavefronts", (long long)waves);
  const dim3 grid((unsigned)((waves + 3) / 4));
  unsigned chain = 0;
  if (a.seg)
    if (int rc = launch_grid(((int64_t)a.q.n_seqs * a.d * a.n + 255) / 256, &chain)) return rc;
  scan_shape(dtype, a.n, [&](auto t, auto np) {
    using T = decltype(t);
    constexpr int NP = decltype(np)::value;
    if (a.seg) {
      hipLaunchKernelGGL((scan_fwd_kernel<T, NP, SCAN_PART>), grid, dim3(256), 0, s, a);
      hipLaunchKernelGGL((scan_chain_kernel<false>), dim3(chain), dim3(256), 0, s, a);
    }
    hipLaunchKernelGGL((scan_fwd_kernel<T, NP, MODE>), grid, dim3(256), 0, s, a);
  });
  TGNN_LAUNCH_CHECK();
  return TGNN_OK;
}

constexpr int BWD_SPREAD = 256, BWD_FILL = 3;   // workgroups: one, and three, to a compute unit
constexpr int BWD_WORKERS = 1024;   // at most as many partial sums of the weights' gradients

struct BwdPlan { int np, tiles, seg, workers; int64_t items; };
static BwdPlan bwd_plan(const tgnn_seqs& q, int d, int n, int groups) {
  BwdPlan p;
  p.np = n <= 4 ? 1 : n <= 8 ? 2 : n <= 16 ? 4 : n <= 32 ? 8 : 16;
  const int cols = 16 * bwd_waves(p.np), dg = d / groups;
  p.tiles = (dg + cols - 1) / cols;
  const int64_t all = (int64_t)groups * p.tiles;
  p.seg = scan_segment(q, all, BWD_SPREAD, BWD_FILL);
  p.items = p.seg ? seg_total(q, p.seg) : q.n_seqs;
  p.workers = (int)std::max<int64_t>(1, std::min<int64_t>(p.items, std::min<int64_t>(BWD_WORKERS, 2 * BWD_SPREAD * BWD_FILL / all)));
  return p;
}
static int64_t bwd_bytes(const tgnn_seqs& q, int d, int n, int groups, bool saved, ScanArgs* a, void* ws, ScanArgs* fwd) {
  const BwdPlan p = bwd_plan(q, d, n, groups);
  Take t{static_cast<char*>(ws)};
  if (!saved) {   // the states are formed here
    float* sv = t.floats(seg_total(q, CHUNK) * d * n);
    if (a) a->saved = fwd->saved = sv;
    const int64_t bytes = fwd_bytes(q, d, n, groups, fwd, ws ? static_cast<char*>(ws) + t.off : nullptr);
    t.off += bytes;
  }
  if (p.seg) {
    float *st = t.floats(seg_total(q, p.seg) * d * n), *dl = t.floats(seg_total(q, p.seg) * d);
    if (a) { a->seg_state = st; a->seg_delta = dl; }
  }
  float* part = t.floats((int64_t)p.workers * ((int64_t)d * n + 2 * d));
  if (a) a->part = part;
  if (p.tiles > 1) {
    float* bc = t.floats((int64_t)p.tiles * q.n_rows * 2 * groups * n);
    if (a) a->part_bc = bc;
  }
  return t.off;
}

static int check_sizes(const tgnn_seqs* q, int32_t d, int32_t n, int32_t groups) {
  if (int rc = check_seqs(q)) return rc;
  if (d < 1 || d > TGNN_MAX_SEQ_WIDTH || n < 1 || n > TGNN_MAX_SCAN_STATES || groups < 1 || d % groups != 0)
    return set_error(TGNN_E_UNSUPPORTED_DIM, "d = %d, n_state = %d, n_groups = %d", d, n, groups);
  return TGNN_OK;
}

static int check_workspace(const void* ws, int64_t have, int64_t need) {
  if (need <= 0) return TGNN_OK;
  if (ws == nullptr) return set_error(TGNN_E_NULL_PTR, "workspace is NULL");
  if (!aligned_to(ws, 16)) return set_error(TGNN_E_MISALIGNED, "workspace is not 16-byte aligned");
  if (have < need) return set_error(TGNN_E_WORKSPACE, "workspace of %lld bytes, %lld are needed", (long long)have, (long long)need);
  return TGNN_OK;
}

}  // namespace tgnn

using namespace tgnn;

extern "C" int64_t tgnn_selective_scan_saved_bytes(const tgnn_seqs* seqs, int32_t d, int32_t n_state) {
  if (int rc = check_sizes(seqs, d, n_state, 1)) return rc;
  return seg_total(*seqs, CHUNK) * d * n_state * (int64_t)sizeof(float);
}

extern "C" int64_t tgnn_selective_scan_workspace_bytes(const tgnn_seqs* seqs, int32_t d, int32_t n_state, int32_t n_groups, int32_t backward,
                                                       int32_t saved) {
  if (int rc = check_sizes(seqs, d, n_state, n_groups)) return rc;
  return backward ? bwd_bytes(*seqs, d, n_state, n_groups, saved != 0, nullptr, nullptr, nullptr)
                  : fwd_bytes(*seqs, d, n_state, n_groups, nullptr, nullptr);
}

extern "C" int32_t tgnn_selective_scan_fwd(const tgnn_seqs* seqs, const tgnn_scan* scan, void* y, int64_t ld_y, float* state_out,
                                           float* saved, int64_t saved_bytes, void* workspace, int64_t workspace_bytes, void* stream) {
  if (int rc = check_seqs(seqs)) return rc;
  if (int rc = check_scan(scan, seqs->n_rows)) return rc;
  if (int rc = check_row_array("y", y, ld_y, seqs->n_rows, scan->d, scan->dtype)) return rc;
  if (!aligned_to(state_out, 4)) return set_error(TGNN_E_MISALIGNED, "state_out is not aligned to its type");
  if (!aligned_to(saved, 16)) return set_error(TGNN_E_MISALIGNED, "saved is not 16-byte aligned");
  if (saved != nullptr && saved_bytes < tgnn_selective_scan_saved_bytes(seqs, scan->d, scan->n_state))
    return set_error(TGNN_E_WORKSPACE, "saved has %lld bytes, %lld are needed", (long long)saved_bytes,
                     (long long)tgnn_selective_scan_saved_bytes(seqs, scan->d, scan->n_state));
  const size_t states = (size_t)scan->n_states * scan->d * scan->n_state * sizeof(float);
  if (spans_overlap(scan->state_in, states, state_out, states)) return set_error(TGNN_E_INVALID_ARG, "state_out overlaps state_in");
  const int size = type_size(scan->dtype), bc = scan->n_groups * scan->n_state;
  const int64_t rows = seqs->n_rows;
  const size_t span = rows_span(rows, scan->d, ld_y, size);
  if (spans_overlap(y, span, scan->x, rows_span(rows, scan->d, scan->ld_x, size)) || spans_overlap(y, span, scan->dt, rows_span(rows, scan->d, scan->ld_dt, size)) ||
      spans_overlap(y, span, scan->z, rows_span(rows, scan->d, scan->ld_z, size)) || spans_overlap(y, span, scan->B, rows_span(rows, bc, scan->ld_b, size)) ||
      spans_overlap(y, span, scan->C, rows_span(rows, bc, scan->ld_c, size)))
    return set_error(TGNN_E_INVALID_ARG, "y overlaps an input");
  ScanArgs a = scan_args(seqs, scan);
  const int64_t need = fwd_bytes(*seqs, a.d, a.n, a.groups, &a, workspace);
  if (int rc = check_workspace(workspace, workspace_bytes, need)) return rc;
  if (seqs->n_seqs == 0) return TGNN_OK;
  a.y = y; a.ld_y = ld_y; a.state_out = state_out; a.saved = saved;
  return scan_forward<SCAN_Y>(a, reinterpret_cast<hipStream_t>(stream), scan->dtype);
}

extern "C" int32_t tgnn_selective_scan_step(const tgnn_scan* scan, int64_t n_rows, void* y, int64_t ld_y, float* state_out, void* stream) {
  if (n_rows < 0 || n_rows > INT_MAX) return set_error(TGNN_E_OUT_OF_RANGE, "n_rows = %lld outside [0, 2^31)", (long long)n_rows);
  if (int rc = check_scan(scan, n_rows)) return rc;
  if (int rc = check_row_array("y", y, ld_y, n_rows, scan->d, scan->dtype)) return rc;
  if (!aligned_to(state_out, 4)) return set_error(TGNN_E_MISALIGNED, "state_out is not aligned to its type");
  const size_t states = (size_t)scan->n_states * scan->d * scan->n_state * sizeof(float);
  if (scan->state_in != state_out && spans_overlap(scan->state_in, states, state_out, states))
    return set_error(TGNN_E_INVALID_ARG, "state_out overlaps state_in without being it");
  const int size = type_size(scan->dtype), bc = scan->n_groups * scan->n_state;
  const size_t span = rows_span(n_rows, scan->d, ld_y, size);
  if (spans_overlap(y, span, scan->x, rows_span(n_rows, scan->d, scan->ld_x, size)) || spans_overlap(y, span, scan->dt, rows_span(n_rows, scan->d, scan->ld_dt, size)) ||
      spans_overlap(y, span, scan->z, rows_span(n_rows, scan->d, scan->ld_z, size)) || spans_overlap(y, span, scan->B, rows_span(n_rows, bc, scan->ld_b, size)) ||
      spans_overlap(y, span, scan->C, rows_span(n_rows, bc, scan->ld_c, size)))
    return set_error(TGNN_E_INVALID_ARG, "y overlaps an input");
  if (n_rows == 0) return TGNN_OK;
  ScanArgs a = scan_args(nullptr, scan);
  a.y = y; a.ld_y = ld_y; a.state_out = state_out; a.items = n_rows;
  int bits = 0;
  const int np = a.n >= 4 ? 4 : 1;
  while ((np << bits) < a.n) ++bits;
  unsigned grid;
  if (int rc = launch_grid(((n_rows * a.d << bits) + 255) / 256, &grid)) return rc;
  with_type(scan->dtype, [&](auto t) {
    using T = decltype(t);
    if (np == 4) hipLaunchKernelGGL((scan_step_kernel<T, 4>), dim3(grid), dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a, bits);
    else hipLaunchKernelGGL((scan_step_kernel<T, 1>), dim3(grid), dim3(256), 0, reinterpret_cast<hipStream_t>(stream), a, bits);
  });
  TGNN_LAUNCH_CHECK();
  return TGNN_OK;
}

extern "C" int32_t tgnn_selective_scan_bwd(const tgnn_seqs* seqs, const tgnn_scan* scan, const void* dy, int64_t ld_dy, const float* saved,
                                           int64_t saved_bytes, const tgnn_scan_grads* grads, int32_t accumulate, void* workspace,
                                           int64_t workspace_bytes, void* stream) {
  if (int rc = check_seqs(seqs)) return rc;
  const int64_t rows = seqs->n_rows;
  if (int rc = check_scan(scan, rows)) return rc;
  if (grads == nullptr) return set_error(TGNN_E_NULL_PTR, "grads is NULL");
  const int d = scan->d, bc = scan->n_groups * scan->n_state, size = type_size(scan->dtype);
  struct Rows { const char* name; const void* p; int64_t ld; int cols; };
  const Rows out[] = {{"dx", grads->dx, grads->ld_dx, d}, {"ddt", grads->ddt, grads->ld_ddt, d}, {"dB", grads->dB, grads->ld_db, bc},
                      {"dC", grads->dC, grads->ld_dc, bc}, {"dz", grads->dz, grads->ld_dz, d}};
  const Rows in[] = {{"dy", dy, ld_dy, d}, {"x", scan->x, scan->ld_x, d}, {"dt", scan->dt, scan->ld_dt, d}, {"B", scan->B, scan->ld_b, bc},
                     {"C", scan->C, scan->ld_c, bc}, {"z", scan->z, scan->ld_z, d}};
  if (int rc = check_row_array("dy", dy, ld_dy, rows, d, scan->dtype)) return rc;
  const int n_out = scan->z != nullptr ? 5 : 4;
  for (int i = 0; i < n_out; ++i) {
    if (int rc = check_row_array(out[i].name, out[i].p, out[i].ld, rows, out[i].cols, scan->dtype)) return rc;
    for (const Rows& r : in)
      if (spans_overlap(out[i].p, rows_span(rows, out[i].cols, out[i].ld, size), r.p, rows_span(rows, r.cols, r.ld, size)))
        return set_error(TGNN_E_INVALID_ARG, "%s overlaps %s", out[i].name, r.name);
  }
  if (!aligned_to(grads->dA, 4) || !aligned_to(grads->dD, 4) || !aligned_to(grads->ddt_bias, 4))
    return set_error(TGNN_E_MISALIGNED, "dA, dD or ddt_bias is not aligned to its type");
  if (!aligned_to(saved, 16)) return set_error(TGNN_E_MISALIGNED, "saved is not 16-byte aligned");
  if (saved != nullptr && saved_bytes < tgnn_selective_scan_saved_bytes(seqs, d, scan->n_state))
    return set_error(TGNN_E_WORKSPACE, "saved has %lld bytes, %lld are needed", (long long)saved_bytes,
                     (long long)tgnn_selective_scan_saved_bytes(seqs, d, scan->n_state));
  ScanArgs a = scan_args(seqs, scan), fwd = a;
  const int64_t need = bwd_bytes(*seqs, d, a.n, a.groups, saved != nullptr, &a, workspace, &fwd);
  if (int rc = check_workspace(workspace, workspace_bytes, need)) return rc;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const BwdPlan plan = bwd_plan(*seqs, d, a.n, a.groups);
  if (saved != nullptr) a.saved = const_cast<float*>(saved);
  else if (seqs->n_seqs > 0)
    if (int rc = scan_forward<SCAN_STATES>(fwd, s, scan->dtype)) return rc;
  a.dy = dy; a.ld_dy = ld_dy;
  a.dx = grads->dx; a.ddt = grads->ddt; a.dz = grads->dz; a.dB = grads->dB; a.dC = grads->dC;
  a.ld_dx = grads->ld_dx; a.ld_ddt = grads->ld_ddt; a.ld_dz = grads->ld_dz; a.ld_db = grads->ld_db; a.ld_dc = grads->ld_dc;
  a.seg = plan.seg; a.items = plan.items;
  const bool weights = grads->dA != nullptr || grads->dD != nullptr || grads->ddt_bias != nullptr;
  if (!weights) a.part = nullptr;
  if (seqs->n_seqs > 0) {
    unsigned chain = 0, back = 0, sum = 0;
    const int64_t waves = plan.items * a.groups * fwd_tiles(a.dg);
    if (plan.seg) {
      if (int rc = launch_grid(((int64_t)seqs->n_seqs * d * a.n + 255) / 256, &chain)) return rc;
      if (int rc = launch_grid(waves, &back)) return rc;
    }
    if (int rc = launch_grid(seg_total(*seqs, CHUNK), &sum)) return rc;
    scan_shape(scan->dtype, a.n, [&](auto t, auto np) {
      using T = decltype(t);
      constexpr int NP = decltype(np)::value;
      if (plan.seg) {
        a.tiles = fwd_tiles(a.dg);
        hipLaunchKernelGGL((scan_back_part_kernel<T, NP>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, a);
        hipLaunchKernelGGL((scan_chain_kernel<true>), dim3(chain), dim3(256), 0, s, a);
      }
      a.tiles = plan.tiles;
      hipLaunchKernelGGL((scan_bwd_kernel<T, NP / 4>), dim3((unsigned)(plan.workers * a.groups * plan.tiles)), dim3(64 * bwd_waves(NP / 4)), 0, s, a);
      if (a.part_bc) hipLaunchKernelGGL((scan_bc_sum_kernel<T>), dim3(sum), dim3(256), 0, s, a);
    });
    TGNN_LAUNCH_CHECK();
  }
  if (weights) {
    const int64_t dn = (int64_t)d * a.n;
    column_sum(ColumnSum{a.part, seqs->n_seqs > 0 ? plan.workers : 0, dn + 2 * d, {grads->dA, grads->dD, grads->ddt_bias}, {dn, d, d}, accumulate}, s);
    TGNN_LAUNCH_CHECK();
  }
  return TGNN_OK;
}
