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
// Bound by the vector units: an event costs every state of every column an exponential, two multiplications and two fused ones, forward,
// and three times as much backward, against 8 to 16 bytes of memory per column.  32 sequences, 29,000 events of 1,024 columns in
// bfloat16 with 16 states: the segments' own parts 111 us, from segment to segment 22, the outputs 145, the vector units busy in all
// cycles of the first and last (their memory would take 52); of the 131 instructions that an event costs a wavefront in the outputs 80
// are the states', the others the step size, the gate, conversions, loads and the way through LDS.  A sequence of 8,191 events, 512 columns
// in two groups: forward 63 us with the states saved, backward 145, of which 99 in the last walk (busy in 79 per cent of its cycles at the
// two wavefronts that 212 registers leave a vector unit).  12,000 lists of ten events, 100 columns of float, states in and out: 89 us, 3.8
// TB/s, busy in 77 per cent.
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

constexpr int CHUNK_BITS = 5, CHUNK = 32;   // events between two saved states
constexpr int SUM_BITS = 3;                 // rows that a workgroup adds up the column tiles' parts of dB and dC of
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
  float* part;                          // [workers, d n + 2 d] partial sums of dA, dD, dbias (of slices: dA alone)
  float* part_y;                        // [3, slices, rows, d] the slices' parts of y0, s1, s2
  float* part_bc;                       // [column tiles of a group, rows, 2, groups n]; NULL: dB and dC are written directly
  int64_t ld_x, ld_dt, ld_b, ld_c, ld_z, ld_dy, ld_y, ld_dx, ld_ddt, ld_dz, ld_db, ld_dc, items;
  int d, n, groups, dg, n_states, softplus;
  int bits;                             // a segment has 2^bits events; WHOLE: sequences are not cut
  int tiles;                            // column tiles of a group
  int slices;                           // of the states
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

__device__ __forceinline__ int64_t state_of(const ScanArgs& a, int s) {
  const int64_t i = a.state_idx != nullptr ? a.state_idx[s] : s;
  return i >= 0 && i < a.n_states ? i : -1;
}

// N states of a column from and to memory, four at a time at any address: a column's neighbours in the wavefront are n floats away, so
// that every instruction touches 64 lines, and one float per instruction is four times as many of them (lists of one event,
// 623 columns of 63 states: 253 us a forward call with saved states, and 618).
typedef float Quad __attribute__((ext_vector_type(4), aligned(4)));
template <int NP> __device__ __forceinline__ void load_states(const float* p, int n, float (&h)[NP]) {
  static_assert(NP % 4 == 0, "in fours");
#pragma unroll
  for (int i = 0; i < NP; i += 4) {
    if (i + 4 <= n) {
      const Quad v = *reinterpret_cast<const Quad*>(p + i);
      h[i] = v.x; h[i + 1] = v.y; h[i + 2] = v.z; h[i + 3] = v.w;
    } else {
#pragma unroll
      for (int k = i; k < i + 4; ++k) h[k] = k < n ? p[k] : 0.0f;
    }
  }
}
template <int NP> __device__ __forceinline__ void store_states(float* p, int n, const float (&h)[NP]) {
#pragma unroll
  for (int i = 0; i < NP; i += 4) {
    if (i + 4 <= n) {
      *reinterpret_cast<Quad*>(p + i) = Quad{h[i], h[i + 1], h[i + 2], h[i + 3]};
    } else {
#pragma unroll
      for (int k = i; k < i + 4; ++k)
        if (k < n) p[k] = h[k];
    }
  }
}

enum { SCAN_Y, SCAN_STATES, SCAN_PART, SCAN_BACK_PART };   // outputs; saved states only; a segment's own part, forward and backward

// Four events of a wavefront on their way to the registers: the columns' values, one event per register, and the events' B and C,
// one value of the 4 x NP per lane (and register)
template <class T, int NP> struct Events {
  static constexpr int R = NP > 16 ? NP / 16 : 1;
  T x[4], dt[4], z[4], b[R], c[R];
};

// One wavefront: 64 columns of a group over a segment (or a whole sequence), four events at a time, the next four on their way.  The
// events' B and C go through a piece of LDS that only this wavefront uses: read back, every lane has all of them (a vector
// read of the same address for all lanes; taking them lane by lane from a register instead cost 16 per cent of a step).  Lanes
// without a column do what the last column's lane does, so that nothing in a step is conditional.
// USUAL: with softplus and gate, otherwise as the arguments say (which costs 2 to 4 per cent of these with up to 16 states, and
// spills 30 to 170 registers with 33 and more).
// SCAN_BACK_PART goes from the last event to the first, for the segment's own part of what reaches the segment before it:
// g = a[t] (C[t] gy[t] + g), from zero.
template <class T, int NP, int MODE, bool USUAL>
__global__ __launch_bounds__(256) void scan_fwd_kernel(ScanArgs a) {
  using E = Events<T, NP>;
  constexpr bool BACK = MODE == SCAN_BACK_PART, OUT = MODE == SCAN_Y, NEED_B = !BACK, NEED_C = OUT || BACK, PART = MODE == SCAN_PART || BACK;
  __shared__ float stage[4][2][4 * NP];
  const unsigned w4 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, wave = group_number() * 4 + w4;
  const unsigned all = (unsigned)(a.groups * a.tiles), item = wave / all, tile = wave - item * all;
  if (item >= a.items) return;
  const Piece p = piece_at(a.q, (int)item, a.bits);
  if (p.none || (MODE == SCAN_PART && p.last) || (BACK && p.t0 == 0)) return;
  const int g = tile / a.tiles, col = (tile - g * a.tiles) * 64 + lane;
  const unsigned c = g * a.dg + min(col, a.dg - 1);
  const int64_t state = state_of(a, p.s);
  float A[NP], h[NP];
  load_states<NP>(a.A + (int64_t)c * a.n, a.n, A);
  if (!PART && a.bits != WHOLE) load_states<NP>(a.seg_state + ((int64_t)p.slot * a.d + c) * a.n, a.n, h);
  else if (!PART && state >= 0 && a.state_in != nullptr) load_states<NP>(a.state_in + (state * a.d + c) * a.n, a.n, h);
  else
#pragma unroll
    for (int i = 0; i < NP; ++i) h[i] = 0.0f;
  const float bias = a.bias ? a.bias[c] : 0.0f, D = OUT && a.D ? a.D[c] : 0.0f;
  const bool soft = USUAL || a.softplus, gated = (OUT || BACK) && (USUAL || a.z != nullptr);
  float* sB = stage[w4][0];
  float* sC = stage[w4][1];
  // (the row, relative to the lowest of the four, and state of this lane's B and C)
  unsigned off_b[E::R], off_c[E::R];
#pragma unroll
  for (int r = 0; r < E::R; ++r) {
    const int idx = (lane + 64 * r) % (4 * NP), e = idx / NP, n = g * a.n + min(idx % NP, a.n - 1);
    off_b[r] = (a.q.newest_first ? 3 - e : e) * (unsigned)a.ld_b + n;
    off_c[r] = (a.q.newest_first ? 3 - e : e) * (unsigned)a.ld_c + n;
  }
  // the events t .. t + n - 1 of a group of four, first in front
  auto ask = [&](int t, int n, E& v) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t row = seq_row(a.q, p.r, t + (n == 4 ? u : min(u, n - 1)));
      v.x[u] = (static_cast<const T*>(BACK ? a.dy : a.x) + row * (BACK ? a.ld_dy : a.ld_x))[c];
      v.dt[u] = (static_cast<const T*>(a.dt) + row * a.ld_dt)[c];
      if (gated) v.z[u] = (static_cast<const T*>(a.z) + row * a.ld_z)[c];
    }
#pragma unroll
    for (int r = 0; r < E::R; ++r) {
      if (n == 4) {
        const int64_t low = seq_row(a.q, p.r, a.q.newest_first ? t + 3 : t);
        if (NEED_B) v.b[r] = (static_cast<const T*>(a.B) + low * a.ld_b)[off_b[r]];
        if (NEED_C) v.c[r] = (static_cast<const T*>(a.C) + low * a.ld_c)[off_c[r]];
      } else {
        const int idx = (lane + 64 * r) % (4 * NP), s = g * a.n + min(idx % NP, a.n - 1);
        const int64_t row = seq_row(a.q, p.r, t + min(idx / NP, n - 1));
        if (NEED_B) v.b[r] = (static_cast<const T*>(a.B) + row * a.ld_b)[s];
        if (NEED_C) v.c[r] = (static_cast<const T*>(a.C) + row * a.ld_c)[s];
      }
    }
  };
  float total = 0.0f;   // of the deltas
  auto work = [&](int t, int n, const E& v) {   // n < 4: the rest of the group changes nothing
#pragma unroll
    for (int r = 0; r < E::R; ++r) {
      const int idx = (lane + 64 * r) % (4 * NP);
      const bool in = idx % NP < a.n && (n == 4 || idx / NP < n);
      if (NEED_B) sB[idx] = in ? (float)v.b[r] : 0.0f;
      if (NEED_C) sC[idx] = in ? (float)v.c[r] : 0.0f;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int u = BACK ? 3 - k : k;
      const float raw = (float)v.dt[u] + bias;
      float x = (float)v.x[u], delta = soft ? softplus(raw) : raw, gate = 1.0f;
      if (gated) gate = (float)v.z[u] * sigmoid((float)v.z[u]);
      if (n < 4 && u >= n) x = delta = 0.0f;
      const float d2 = delta * LOG2E;
      if (PART) total += delta;
      if constexpr (BACK) {
        const float gy = n < 4 && u >= n ? 0.0f : x * gate;
#pragma unroll
        for (int i = 0; i < NP; ++i) h[i] = __builtin_amdgcn_exp2f(d2 * A[i]) * fmaf(gy, sC[u * NP + i], h[i]);
      } else {
        const float in = delta * x;
        float y[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NP; ++i) {   // (states beyond n stay zero)
          h[i] = fmaf(__builtin_amdgcn_exp2f(d2 * A[i]), h[i], in * sB[u * NP + i]);
          if (OUT) y[i & 1] = fmaf(h[i], sC[u * NP + i], y[i & 1]);
        }
        if (OUT && (n == 4 || u < n))
          (static_cast<T*>(a.y) + seq_row(a.q, p.r, t + u) * a.ld_y)[c] = (T)(fmaf(D, x, y[0] + y[1]) * gate);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  // whole groups, and what is left of them at the end (of the segment: the first thing on the way back)
  const int n_ev = p.t1 - p.t0, whole = n_ev / 4, left = n_ev & 3;
  float* saved = !PART && a.saved != nullptr ? a.saved + ((int64_t)(seg_base(a.q, p.s, CHUNK_BITS) + p.t0 / CHUNK) * a.d + c) * a.n : nullptr;
  const int64_t saved_step = (int64_t)a.d * a.n;
  E next;
  if (left != 0 && (BACK || whole == 0)) ask(p.t0 + 4 * whole, left, next);
  if (BACK && left != 0) work(p.t0 + 4 * whole, left, next);
  if (whole > 0) ask(BACK ? p.t0 + 4 * (whole - 1) : p.t0, 4, next);
  for (int j = 0; j < whole; ++j) {
    const E v = next;
    const int t = p.t0 + 4 * (BACK ? whole - 1 - j : j);
    if (j + 1 < whole) ask(BACK ? t - 4 : t + 4, 4, next);
    else if (!BACK && left != 0) ask(t + 4, left, next);
    if (!PART && saved != nullptr && (t & (CHUNK - 1)) == 0) {
      store_states<NP>(saved, a.n, h);
      saved += saved_step;
    }
    work(t, 4, v);
  }
  if (!BACK && left != 0) {
    if (!PART && saved != nullptr && ((p.t0 + 4 * whole) & (CHUNK - 1)) == 0) store_states<NP>(saved, a.n, h);
    work(p.t0 + 4 * whole, left, next);
  }
  if (PART) {
    store_states<NP>(a.seg_state + ((int64_t)p.slot * a.d + c) * a.n, a.n, h);
    a.seg_delta[(int64_t)p.slot * a.d + c] = total;
  }
  if (OUT && p.last) {
    for (int t = p.r.len; t < p.r.slot; ++t) (static_cast<T*>(a.y) + (p.r.begin + t) * a.ld_y)[c] = (T)0.0f;
    if (state >= 0 && a.state_out != nullptr) store_states<NP>(a.state_out + (state * a.d + c) * a.n, a.n, h);
  }
}

// v 2^s for the deltas of a whole segment or run: the factor may be more (or less) than a float holds where no event's is, and where the
// product is not (zero, a state that grows from 1e-30 to 1e11); outside [-400, 400] the product is zero or infinite whatever v is.
__device__ __forceinline__ float times_exp2(float v, float s) {
  s = fminf(fmaxf(s, -400.0f), 400.0f);
  const float whole = floorf(s);
  return ldexpf(v * __builtin_amdgcn_exp2f(s - whole), (int)whole);
}

// From segment to segment.  Forward: seg_state[k] becomes the state before segment k, from the sequence's first state; backward: what
// reaches segment k from behind, from zero.  A thread has a column and state of a sequence and asks for eight segments at a time;
// where there are many of them (RUNS = 8) eight threads cut them into runs: each run's own part and the sum of its
// deltas, the run's first state from those before it, then the states.  256 segments of 8,192 columns and states: 13 us,
// one thread for all, one segment after the other, 87; up to 32 segments of 32 sequences of 16,384: 37 us with runs, 22 without.
template <bool BACK, int RUNS>
__global__ __launch_bounds__(256) void scan_chain_kernel(ScanArgs a) {
  constexpr int COLS = 256 / RUNS;
  __shared__ float part[RUNS][COLS], sum[RUNS][COLS];
  const int64_t dn = (int64_t)a.d * a.n, per = (dn + COLS - 1) / COLS;
  const int64_t number = group_number();
  const int s = (int)(number / per), x = threadIdx.x % COLS, run = threadIdx.x / COLS;
  if (s >= a.q.n_seqs) return;
  const int64_t e = (number - s * per) * COLS + x;
  const bool on = e < dn;
  const int c = on ? (int)(e / a.n) : 0;
  const Seq r = seq_at(a.q, s);
  const int64_t base = seg_base(a.q, s, a.bits);
  const int count = seg_count(r.len, a.bits);
  const int64_t state = state_of(a, s);
  const float A = on ? a.A[e] * LOG2E : 0.0f;
  // segment k in the order of the recurrence; the last one's part was not formed (and is not needed)
  auto at = [&](int k) { return base + (BACK ? count - 1 - k : k); };
  const int each = (count + RUNS - 1) / RUNS, k0 = min(run * each, count), k1 = min(k0 + each, count);
  constexpr int U = 8;
  float cur = 0.0f, total = 0.0f;
  for (int k = k0; RUNS > 1 && on && k < min(k1, count - 1); k += U) {
    float v[U], d[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = at(min(k + u, count - 1));
      const bool in = k + u < min(k1, count - 1);
      v[u] = in ? a.seg_state[i * dn + e] : 0.0f;
      d[u] = in ? a.seg_delta[i * a.d + c] : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      cur = times_exp2(cur, d[u] * A) + v[u];
      total += d[u];
    }
  }
  if (RUNS > 1) {
    part[run][x] = cur;
    sum[run][x] = total;
    __syncthreads();
  }
  if (!on) return;
  cur = !BACK && state >= 0 && a.state_in != nullptr ? a.state_in[state * dn + e] : 0.0f;
  for (int i = 0; i < run; ++i) cur = times_exp2(cur, sum[i][x] * A) + part[i][x];
  for (int k = k0; k < k1; k += U) {
    float v[U], d[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = at(min(k + u, count - 1));
      const bool in = k + u < min(k1, count - 1);
      v[u] = in ? a.seg_state[i * dn + e] : 0.0f;
      d[u] = in ? a.seg_delta[i * a.d + c] : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k + u < k1) a.seg_state[at(k + u) * dn + e] = cur;
      cur = times_exp2(cur, d[u] * A) + v[u];
    }
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

// Wavefronts and columns of a workgroup.  Wavefronts share what is read of B and C, the sums over columns, and barriers: 1,800 lists of up to ten
// events, 100 columns, 73 us, one sequence of 8,191 events, 512 columns, 99; with eight 87 and 116, with two 79 and 114, with one 74 and 110.
constexpr int BWD_WAVES = 4, BWD_COLS = 16 * BWD_WAVES;
constexpr int FINISH_BITS = 3;
constexpr int SLICE = 16;                                 // states of a column that a workgroup has at most

// v[e][i] of four events and NP states, summed over the wavefront's 16 columns: every lane gets the sums of its four states for
// one event, event_of_sum(lane)
template <int NP> __device__ __forceinline__ void column_sums(const float (&v)[4][NP], float (&s)[NP]) {
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    float x = rows_sum(halves_sum(v[0][i], v[2][i]), halves_sum(v[1][i], v[3][i]));
    x += dpp_get<ROW_ROR8>(x);
    s[i] = x + dpp_get<ROW_ROR4>(x);
  }
}
__device__ __forceinline__ int event_of_sum(int lane) { return 2 * (lane >> 5) + (lane >> 4 & 1); }

// A workgroup: 16 columns per wavefront of one group, over the pieces worker, worker + workers, ...  With more than 16 states (SLICED)
// it has 16 of them, n0 .. n0 + 15, and leaves its part of the sums over the states (y0, s1, s2) for scan_finish_kernel.  (With all 64
// states of a column in four lanes, spilled, one wavefront to a vector unit, forward and backward over 10,000 events of 86 columns and 37
// states took 419 us, now 235; 1,126 lists of one event, 623 columns, 63 states: 1,311 and 594.  Narrow models lose by it, since they have
// wavefronts without a column in every slice: 163 sequences, 40,000 events of 13 columns and 56 states 278 and 366.)
template <class T, int NP, bool USUAL, bool SLICED>
__global__ __launch_bounds__(64 * BWD_WAVES, 2) void scan_bwd_kernel(ScanArgs a) {
  constexpr int WAVES = BWD_WAVES, THREADS = 64 * WAVES, N4 = 4 * NP, STAGE = CHUNK * N4 / THREADS > 0 ? CHUNK * N4 / THREADS : 1;
  __shared__ float bound[CHUNK / 4][THREADS * NP];   // a lane's states before every fourth event
  __shared__ float sB[CHUNK * N4], sC[CHUNK * N4];   // of the chunk's events
  __shared__ float red[WAVES][2][CHUNK * N4];        // dB, dC summed over a wavefront's columns
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane & 3;
  const int per = a.groups * a.tiles, all = SLICED ? per * a.slices : per;
  const int worker = blockIdx.x / all, workers = gridDim.x / all, at_all = blockIdx.x - worker * all, slice = SLICED ? at_all / per : 0;
  const int tile = at_all - slice * per, grp = tile / a.tiles, sub = tile - grp * a.tiles;
  const int n0 = slice * SLICE, n_here = SLICED ? min(a.n - n0, SLICE) : a.n;
  const int col = sub * BWD_COLS + wave * 16 + (lane >> 2);
  const bool on = col < a.dg, full = __all(on), odd = (q & 1) != 0, high = (q & 2) != 0;
  const bool soft = USUAL || a.softplus, gated = USUAL || a.z != nullptr, newest = a.q.newest_first != 0;
  const unsigned c = grp * a.dg + (on ? col : a.dg - 1);
  float A[NP], dA[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    A[i] = q * NP + i < n_here ? a.A[(int64_t)c * a.n + n0 + q * NP + i] : 0.0f;
    dA[i] = 0.0f;
  }
  const float bias = a.bias ? a.bias[c] : 0.0f, D = a.D ? a.D[c] : 0.0f;
  float dD = 0.0f, dbias = 0.0f;
  // A lane has the values of event q of a group of four: their distance from the lowest row of the group's four.
  const unsigned up = newest ? 3 - q : q;
  const unsigned ox = up * (unsigned)a.ld_x + c, odt = up * (unsigned)a.ld_dt + c, oz = up * (unsigned)a.ld_z + c, ody = up * (unsigned)a.ld_dy + c;

  // The next piece that has events; padding rows are cleared on the way.
  int64_t item = worker;
  auto advance = [&](Piece& p) -> bool {
    for (; item < a.items; item += workers) {
      p = piece_at(a.q, (int)item, a.bits);
      if (p.none) continue;
      if (p.last && p.r.slot > p.r.len) {
        for (int t = p.r.len + q; on && slice == 0 && t < p.r.slot; t += 4) {
          const int64_t row = p.r.begin + t;
          (static_cast<T*>(a.dx) + row * a.ld_dx)[c] = (T)0.0f;
          (static_cast<T*>(a.ddt) + row * a.ld_ddt)[c] = (T)0.0f;
          if (gated) (static_cast<T*>(a.dz) + row * a.ld_dz)[c] = (T)0.0f;
        }
        if (sub == 0)
          for (int t = p.r.len + wave; t < p.r.slot; t += WAVES)
            for (int n = lane; n < n_here; n += 64) {
              const int64_t row = p.r.begin + t;
              (static_cast<T*>(a.dB) + row * a.ld_db)[grp * a.n + n0 + n] = (T)0.0f;
              (static_cast<T*>(a.dC) + row * a.ld_dc)[grp * a.n + n0 + n] = (T)0.0f;
            }
      }
      if (p.t0 < p.t1) {
        item += workers;
        return true;
      }
    }
    return false;
  };
  // The chunk in hand and the next one (of the same piece, or the last chunk of the next piece): its B, C and first states, and its
  // first four events, are asked for while the one in hand is worked on.
  {
    Piece p, np;
    bool more = advance(p);
    int tb = more ? p.t0 + (p.t1 - 1 - p.t0) / CHUNK * CHUNK : 0;
    float g[NP];   // what reaches the state behind the event in hand from the events after it
    T rb[STAGE], rc[STAGE];
    float hn[NP];
    auto ask_chunk = [&](const Piece& p, int tb) {
      const int n_ev = min(CHUNK, p.t1 - tb);
#pragma unroll
      for (int r = 0; r < STAGE; ++r) {
        const int i = tid + r * THREADS, e = i / N4, n = i % N4;
        rb[r] = rc[r] = (T)0.0f;
        if (e < n_ev && n < n_here) {
          const int64_t row = seq_row(a.q, p.r, tb + e);
          rb[r] = (static_cast<const T*>(a.B) + row * a.ld_b)[grp * a.n + n0 + n];
          rc[r] = (static_cast<const T*>(a.C) + row * a.ld_c)[grp * a.n + n0 + n];
        }
      }
      const float* sv = a.saved + ((int64_t)(seg_base(a.q, p.s, CHUNK_BITS) + tb / CHUNK) * a.d + c) * a.n + n0 + q * NP;
#pragma unroll
      for (int i = 0; i < NP; ++i) hn[i] = on && q * NP + i < n_here ? sv[i] : 0.0f;
    };
    auto ask_back = [&](const Piece& p) {   // what reaches a piece from behind
#pragma unroll
      for (int i = 0; i < NP; ++i)
        g[i] = a.bits != WHOLE && on && q * NP + i < n_here ? a.seg_state[((int64_t)p.slot * a.d + c) * a.n + n0 + q * NP + i] : 0.0f;
    };
    struct Own { T x, dt, z, dy; };
    auto low_row = [&](const Piece& p, int t) { return p.r.begin + (newest ? p.r.len - 4 - t : t); };   // of the events t .. t + 3
    auto ask = [&](const Piece& p, int t, bool back, Own& v) {
      const int64_t row = low_row(p, t);
      v.x = v.dt = v.z = v.dy = (T)0.0f;
      if (on && t + q < p.t1) {
        v.x = (static_cast<const T*>(a.x) + row * a.ld_x)[ox];
        v.dt = (static_cast<const T*>(a.dt) + row * a.ld_dt)[odt];
        if (back) {
          v.dy = (static_cast<const T*>(a.dy) + row * a.ld_dy)[ody];
          if (gated) v.z = (static_cast<const T*>(a.z) + row * a.ld_z)[oz];
        }
      }
    };

    Own nx;
    if (more) {
      ask_chunk(p, tb);
      ask_back(p);
      ask(p, tb, p.t1 - tb <= 4, nx);
    }
    while (more) {
      const int n_ev = min(CHUNK, p.t1 - tb), n_sub = (n_ev + 3) / 4;
#pragma unroll
      for (int r = 0; r < STAGE; ++r)
        if (CHUNK * N4 >= THREADS || tid < CHUNK * N4) {
          sB[tid + r * THREADS] = (float)rb[r];
          sC[tid + r * THREADS] = (float)rc[r];
        }
      float h[NP];
#pragma unroll
      for (int i = 0; i < NP; ++i) h[i] = hn[i];
      __syncthreads();
      // forward over the chunk: the state before every fourth event
#pragma unroll
      for (int i = 0; i < NP; ++i) bound[0][tid * NP + i] = h[i];
      for (int j = 0; j + 1 < n_sub; ++j) {
        const Own v = nx;
        ask(p, tb + 4 * j + 4, j + 2 == n_sub, nx);
        const float raw = (float)v.dt + bias, delta = soft ? softplus(raw) : raw, d2 = delta * LOG2E, in = delta * (float)v.x;
        const float d2s[4] = {quad_get<0>(d2), quad_get<1>(d2), quad_get<2>(d2), quad_get<3>(d2)};
        const float ins[4] = {quad_get<0>(in), quad_get<1>(in), quad_get<2>(in), quad_get<3>(in)};
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < NP; ++i)
            h[i] = fmaf(__builtin_amdgcn_exp2f(d2s[e] * A[i]), h[i], ins[e] * sB[(4 * j + e) * N4 + q * NP + i]);
#pragma unroll
        for (int i = 0; i < NP; ++i) bound[j + 1][tid * NP + i] = h[i];
      }
      const bool next_piece = tb == p.t0;
      int next_tb = tb - CHUNK;
      np = p;
      if (next_piece) {
        more = advance(np);
        next_tb = more ? np.t0 + (np.t1 - 1 - np.t0) / CHUNK * CHUNK : 0;
      }
      if (more) ask_chunk(np, next_tb);
      // and back, four events at a time
      for (int j = n_sub - 1; j >= 0; --j) {
        const Own v = nx;
        if (j > 0) ask(p, tb + 4 * j - 4, true, nx);
        else if (more) ask(np, next_tb, np.t1 - next_tb <= 4, nx);
        const bool there = on && 4 * j + q < n_ev;
        const float x = (float)v.x, raw = (float)v.dt + bias, z = (float)v.z, dy = (float)v.dy;
        const float delta = there ? (soft ? softplus(raw) : raw) : 0.0f, sg = gated ? sigmoid(z) : 1.0f, gy = gated ? dy * z * sg : dy;
        const float d2 = delta * LOG2E, in = delta * x;
        const float d2s[4] = {quad_get<0>(d2), quad_get<1>(d2), quad_get<2>(d2), quad_get<3>(d2)};
        const float ins[4] = {quad_get<0>(in), quad_get<1>(in), quad_get<2>(in), quad_get<3>(in)};
        const float gys[4] = {quad_get<0>(gy), quad_get<1>(gy), quad_get<2>(gy), quad_get<3>(gy)};
        float dec[4][NP], ah[4][NP], v4[4][NP], y[4], s1[4], s2[4], sum[NP];
#pragma unroll
        for (int i = 0; i < NP; ++i) h[i] = bound[j][tid * NP + i];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = 0.0f;
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            dec[e][i] = __builtin_amdgcn_exp2f(d2s[e] * A[i]);
            ah[e][i] = dec[e][i] * h[i];
            h[i] = fmaf(ins[e], sB[(4 * j + e) * N4 + q * NP + i], ah[e][i]);
            v4[e][i] = gys[e] * h[i];
            y[e] = fmaf(h[i], sC[(4 * j + e) * N4 + q * NP + i], y[e]);
          }
        }
        auto columns_only = [&]() {   // a column that is none adds nothing, also where B (its state is not zero then) or C is infinite
          if (full) return;
          asm volatile("");   // (a branch, not 16 selects for every wavefront)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < NP; ++i) v4[e][i] = on ? v4[e][i] : 0.0f;
        };
        columns_only();
        column_sums<NP>(v4, sum);
        const int at = (4 * j + event_of_sum(lane)) * N4 + q * NP;
        if ((lane & 12) == 0)
#pragma unroll
          for (int i = 0; i < NP; ++i) red[wave][1][at + i] = sum[i];
#pragma unroll
        for (int e = 3; e >= 0; --e) {
          s1[e] = s2[e] = 0.0f;
#pragma unroll
          for (int i = 0; i < NP; ++i) {
            const float lam = fmaf(sC[(4 * j + e) * N4 + q * NP + i], gys[e], g[i]), lah = lam * ah[e][i];
            s1[e] = fmaf(lam, sB[(4 * j + e) * N4 + q * NP + i], s1[e]);
            s2[e] = fmaf(A[i], lah, s2[e]);
            dA[i] = fmaf(d2s[e], lah, dA[i]);
            v4[e][i] = lam * ins[e];
            g[i] = dec[e][i] * lam;
          }
        }
        columns_only();
        column_sums<NP>(v4, sum);
        if ((lane & 12) == 0)
#pragma unroll
          for (int i = 0; i < NP; ++i) red[wave][0][at + i] = sum[i];
        const float t1 = quad_scatter_sum(s1, odd, high), t2 = quad_scatter_sum(s2, odd, high);
        if constexpr (SLICED) {
          const float y0 = quad_scatter_sum(y, odd, high);
          if (there) {
            float* o = a.part_y + ((int64_t)slice * a.q.n_rows + low_row(p, tb + 4 * j) + up) * a.d + c;
            const int64_t all_rows = (int64_t)a.slices * a.q.n_rows * a.d;
            o[0] = y0;
            o[all_rows] = t1;
            o[2 * all_rows] = t2;
          }
          continue;
        }
        const float dd = fmaf(x, t1, t2), draw = soft ? dd * sigmoid(raw) : dd;
        float dz = 0.0f;
        if (gated) dz = dy * fmaf(D, x, quad_scatter_sum(y, odd, high)) * (sg * fmaf(z, 1.0f - sg, 1.0f));
        if (there) {
          const int64_t row = low_row(p, tb + 4 * j);
          (static_cast<T*>(a.dx) + row * a.ld_dx)[up * (unsigned)a.ld_dx + c] = (T)fmaf(D, gy, delta * t1);
          (static_cast<T*>(a.ddt) + row * a.ld_ddt)[up * (unsigned)a.ld_ddt + c] = (T)draw;
          if (gated) (static_cast<T*>(a.dz) + row * a.ld_dz)[up * (unsigned)a.ld_dz + c] = (T)dz;
          dD = fmaf(gy, x, dD);
          dbias += draw;
        }
      }
      if (next_piece && more) ask_back(np);
      __syncthreads();
      for (int i = tid; i < n_ev * 2 * N4; i += THREADS) {
        const int kind = i >= n_ev * N4, at = kind ? i - n_ev * N4 : i, e = at / N4, n = at % N4;
        if (n >= n_here) continue;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += red[w][kind][at];
        const int64_t row = seq_row(a.q, p.r, tb + e);
        const int k = grp * a.n + n0 + n;
        if (a.part_bc != nullptr) a.part_bc[((sub * a.q.n_rows + row) * 2 + kind) * a.groups * a.n + k] = sum;
        else if (kind == 0) (static_cast<T*>(a.dB) + row * a.ld_db)[k] = (T)sum;
        else (static_cast<T*>(a.dC) + row * a.ld_dc)[k] = (T)sum;
      }
      p = np;
      tb = next_tb;
    }
  }
  if (a.part == nullptr) return;
  float* part = a.part + (int64_t)worker * ((int64_t)a.d * a.n + (SLICED ? 0 : 2 * a.d));
  dD += dpp_get<QUAD_XOR1>(dD);
  dD += dpp_get<QUAD_XOR2>(dD);
  dbias += dpp_get<QUAD_XOR1>(dbias);
  dbias += dpp_get<QUAD_XOR2>(dbias);
  if (!on) return;
#pragma unroll
  for (int i = 0; i < NP; ++i)
    if (q * NP + i < n_here) part[(int64_t)c * a.n + n0 + q * NP + i] = dA[i] * LN2;   // (it was summed up with delta log2 e)
  if (!SLICED && q == 0) {
    part[(int64_t)a.d * a.n + c] = dD;
    part[(int64_t)a.d * a.n + a.d + c] = dbias;
  }
}

// What is left of a row once the slices' sums over their states are there: a thread has a column, a workgroup walks over pieces of 8
// events (of 32, 10,000 events of 86 columns took 31 us); dD and dbias per workgroup.
template <class T>
__global__ __launch_bounds__(256) void scan_finish_kernel(ScanArgs a, int per_x, int col_tiles) {
  __shared__ float acc[2][256];
  const int tx = threadIdx.x % per_x, ty = threadIdx.x / per_x, per_y = 256 / per_x;
  const int tile = blockIdx.x % col_tiles, worker = blockIdx.x / col_tiles, workers = gridDim.x / col_tiles;
  const int col = tile * per_x + tx, c = min(col, a.d - 1);
  const bool on = col < a.d;
  const float bias = a.bias ? a.bias[c] : 0.0f, D = a.D ? a.D[c] : 0.0f;
  const int64_t per_slice = a.q.n_rows * a.d, per_kind = a.slices * per_slice;
  float dD = 0.0f, dbias = 0.0f;
  for (int64_t item = worker; item < a.items; item += workers) {
    const Piece p = piece_at(a.q, (int)item, FINISH_BITS);
    if (p.none) continue;
    for (int t = p.t0 + ty; on && t < p.t1; t += per_y) {
      const int64_t row = seq_row(a.q, p.r, t);
      float y0 = 0.0f, s1 = 0.0f, s2 = 0.0f;
      for (int k = 0; k < a.slices; ++k) {
        const float* o = a.part_y + k * per_slice + row * a.d + c;
        y0 += o[0];
        s1 += o[per_kind];
        s2 += o[2 * per_kind];
      }
      const float x = (float)(static_cast<const T*>(a.x) + row * a.ld_x)[c], raw = (float)(static_cast<const T*>(a.dt) + row * a.ld_dt)[c] + bias;
      const float dy = (float)(static_cast<const T*>(a.dy) + row * a.ld_dy)[c], delta = a.softplus ? softplus(raw) : raw;
      float gy = dy;
      if (a.z) {
        const float z = (float)(static_cast<const T*>(a.z) + row * a.ld_z)[c], sg = sigmoid(z);
        gy = dy * z * sg;
        (static_cast<T*>(a.dz) + row * a.ld_dz)[c] = (T)(dy * fmaf(D, x, y0) * (sg * fmaf(z, 1.0f - sg, 1.0f)));
      }
      const float dd = fmaf(x, s1, s2), draw = a.softplus ? dd * sigmoid(raw) : dd;
      (static_cast<T*>(a.dx) + row * a.ld_dx)[c] = (T)fmaf(D, gy, delta * s1);
      (static_cast<T*>(a.ddt) + row * a.ld_ddt)[c] = (T)draw;
      dD = fmaf(gy, x, dD);
      dbias += draw;
    }
  }
  if (a.part == nullptr) return;
  acc[0][threadIdx.x] = dD;
  acc[1][threadIdx.x] = dbias;
  __syncthreads();
  if (ty != 0 || !on) return;
  for (int r = 1; r < per_y; ++r) {
    dD += acc[0][r * per_x + tx];
    dbias += acc[1][r * per_x + tx];
  }
  float* part = a.part + (int64_t)worker * 2 * a.d;
  part[c] = dD;
  part[a.d + c] = dbias;
}

// dB and dC of the rows of sequences: the column tiles' parts in order
template <class T>
__global__ __launch_bounds__(256) void scan_bc_sum_kernel(ScanArgs a) {
  const unsigned item = group_number();
  if (item >= a.items) return;
  const Piece p = piece_at(a.q, (int)item, SUM_BITS);
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

// One event of each of `items` rows, on the rows' states.  LC = 2^bits neighbouring lanes have a column, four states each, next to each
// other in memory; a workgroup has 256 / LC columns of four rows, whose states are asked for together.  With four lanes and
// more to a column (QUAD) every one of four neighbouring lanes forms the step size and the gate of one of the rows.  4,000
// rows of 256 columns and 16 states, 131 MB of states in and out: 35 us, 3.8 TB/s; with the states through the caches, which no other
// row of the call wants, 47; every lane forming all four rows' step sizes (no QUAD), 40; walking over the rows with the next four's states on their way, 65 (138 registers, half the
// wavefronts).
template <class T, bool QUAD>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a, int bits, int tiles) {
  const unsigned number = group_number();
  const int tile = number % tiles, part = threadIdx.x & ((1 << bits) - 1), q = threadIdx.x & 3;
  const int64_t row0 = (int64_t)(number / tiles) * 4, last = a.items - 1;
  if (row0 > last) return;
  const int col = tile * (256 >> bits) + (int)(threadIdx.x >> bits), c = min(col, a.d - 1), n0 = part * 4;
  const bool on = col < a.d, whole = n0 + 4 <= a.n;
  const int s0 = min(n0, a.n - 1), bc = c / a.dg * a.n + s0;   // (lanes without a state read another's)
  auto floats = [&](const float* p, float (&v)[4], auto once) {
    if (whole) {
      const FloatRun<4>* at = reinterpret_cast<const FloatRun<4>*>(p);
      const FloatRun<4> r = decltype(once)::value ? stream_load(at) : *at;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = r.v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = n0 + i < a.n ? p[i] : 0.0f;
    }
  };
  auto values = [&](const void* base, int64_t at, float (&v)[4]) {
    const T* p = static_cast<const T*>(base) + at;
    if (whole) {
      const Run<T, 4> r = *reinterpret_cast<const Run<T, 4>*>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = (float)r.v[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = n0 + i < a.n ? (float)p[i] : 0.0f;
    }
  };
  float A[4], h[4][4], B[4][4], C[4][4], y[4];
  int64_t state[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t row = min(row0 + e, last);
    state[e] = state_of(a, (int)row);
    if (state[e] >= 0 && a.state_in != nullptr) floats(a.state_in + (state[e] * a.d + c) * a.n + s0, h[e], std::true_type());
    else
#pragma unroll
      for (int i = 0; i < 4; ++i) h[e][i] = 0.0f;
    values(a.B, row * a.ld_b + bc, B[e]);
    values(a.C, row * a.ld_c + bc, C[e]);
  }
  floats(a.A + (int64_t)c * a.n + s0, A, std::false_type());
  const float bias = a.bias ? a.bias[c] : 0.0f, D = a.D ? a.D[c] : 0.0f;
  struct Own { float x, d2, in, gate; };   // of one row
  auto own = [&](int64_t r) {
    const int64_t row = min(r, last);
    Own o;
    o.x = (float)(static_cast<const T*>(a.x) + row * a.ld_x)[c];
    const float raw = (float)(static_cast<const T*>(a.dt) + row * a.ld_dt)[c] + bias, delta = a.softplus ? softplus(raw) : raw;
    o.d2 = delta * LOG2E;
    o.in = delta * o.x;
    o.gate = 1.0f;
    if (a.z) {
      const float z = (float)(static_cast<const T*>(a.z) + row * a.ld_z)[c];
      o.gate = z * sigmoid(z);
    }
    return o;
  };
  auto event = [&](int e, float d2, float in) {
    y[e] = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[e][i] = fmaf(__builtin_amdgcn_exp2f(d2 * A[i]), h[e][i], in * B[e][i]);
      y[e] = fmaf(h[e][i], C[e][i], y[e]);
    }
  };
  Own o[QUAD ? 1 : 4];
  if constexpr (QUAD) {
    o[0] = own(row0 + q);
    event(0, quad_get<0>(o[0].d2), quad_get<0>(o[0].in));
    event(1, quad_get<1>(o[0].d2), quad_get<1>(o[0].in));
    event(2, quad_get<2>(o[0].d2), quad_get<2>(o[0].in));
    event(3, quad_get<3>(o[0].d2), quad_get<3>(o[0].in));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] = own(row0 + e);
      event(e, o[e].d2, o[e].in);
    }
  }
  if (on && n0 < a.n && a.state_out != nullptr)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (row0 + e > last || state[e] < 0) continue;
      float* p = a.state_out + (state[e] * a.d + c) * a.n + n0;
      if (whole) {
        FloatRun<4> r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r.v[i] = h[e][i];
        stream_store(reinterpret_cast<FloatRun<4>*>(p), r);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n0 + i < a.n) p[i] = h[e][i];
      }
    }
  if constexpr (QUAD) {
    float sum = quad_scatter_sum(y, (q & 1) != 0, (q & 2) != 0);   // lane q: of row q
    for (int s = 4; s < 1 << bits; s <<= 1) sum += __shfl_xor(sum, s);
    if (on && part < 4 && row0 + q <= last) (static_cast<T*>(a.y) + (row0 + q) * a.ld_y)[c] = (T)(fmaf(D, o[0].x, sum) * o[0].gate);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float sum = y[e];
      for (int s = 1; s < 1 << bits; s <<= 1) sum += __shfl_xor(sum, s);
      if (on && part == 0 && row0 + e <= last) (static_cast<T*>(a.y) + (row0 + e) * a.ld_y)[c] = (T)(fmaf(D, o[e].x, sum) * o[e].gate);
    }
  }
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

// Bits of a segment's length, or WHOLE.  `units` wavefronts (forward) or workgroups (backward) have a sequence between them, `spread`
// of them run side by side at full speed, `fill` times as many hide each other's latencies and even out the segments' lengths.  Whole, a call
// takes as many steps as the longest sequence has events, or as all of them share out; in segments it takes 1.8 times the
// shared work (every event once more for the segments' parts), some 40 steps' time for two more launches, and the walk over
// one segment.
static int scan_segment(const tgnn_seqs& q, int64_t units, int64_t spread, int64_t fill) {
  const int64_t rows = scan_rows(q), longest = std::min<int64_t>(q.max_len, rows), work = rows * units / spread;
  int bits = CHUNK_BITS;
  while (bits < 12 && (int64_t(3) << bits) / 2 <= work / fill) ++bits;   // (the nearest power of two)
  return std::max(longest, work) > work + work * 4 / 5 + 40 + (1 << bits) ? bits : WHOLE;
}

// (1,792 lists of up to 21 events, 271 columns, 38 states: 183 us in 48 places and two wavefronts to a vector unit, 310 in 64 and one)
template <class F> static void scan_shape(int dtype, int n, F f) {   // f(T(), states of a lane that has them all)
  with_type(dtype, [&](auto t) {
    if (n <= 4) f(t, std::integral_constant<int, 4>());
    else if (n <= 8) f(t, std::integral_constant<int, 8>());
    else if (n <= 16) f(t, std::integral_constant<int, 16>());
    else if (n <= 32) f(t, std::integral_constant<int, 32>());
    else if (n <= 48) f(t, std::integral_constant<int, 48>());
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

constexpr int FWD_SPREAD = 1024, FWD_FILL = 6;   // wavefronts: one, and six, to a vector unit
static int fwd_tiles(int dg) { return (dg + 63) / 64; }
static int fwd_segment(const tgnn_seqs& q, int groups, int dg) { return scan_segment(q, (int64_t)groups * fwd_tiles(dg), FWD_SPREAD, FWD_FILL); }

static int64_t fwd_bytes(const tgnn_seqs& q, int d, int n, int groups, ScanArgs* a, void* ws) {
  Take t{static_cast<char*>(ws)};
  const int bits = fwd_segment(q, groups, d / groups);
  if (bits != WHOLE) {
    float *st = t.floats(seg_total(q, bits) * d * n), *dl = t.floats(seg_total(q, bits) * d);
    if (a) { a->seg_state = st; a->seg_delta = dl; }
  }
  return t.off;
}

static int launch_grid(int64_t n, dim3* out) {
  if (n > INT_MAX) return set_error(TGNN_E_OUT_OF_RANGE, "%lld workgroups", (long long)n);
  *out = group_grid(n);
  return TGNN_OK;
}

// Runs from 64 segments of the longest sequence on
static bool chain_runs(const ScanArgs& a) { return std::min<int64_t>(a.q.max_len, scan_rows(a.q)) > int64_t(64) << a.bits; }
static int chain_grid(const ScanArgs& a, dim3* out) {
  const int cols = chain_runs(a) ? 32 : 256;
  return launch_grid(a.q.n_seqs * (((int64_t)a.d * a.n + cols - 1) / cols), out);
}
template <bool BACK> static void launch_chain(const ScanArgs& a, dim3 grid, hipStream_t s) {
  if (chain_runs(a)) hipLaunchKernelGGL((scan_chain_kernel<BACK, 8>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((scan_chain_kernel<BACK, 1>), grid, dim3(256), 0, s, a);
}

template <class T, int NP, int MODE> static void launch_scan(const ScanArgs& a, dim3 grid, hipStream_t s) {
  constexpr bool GATED = MODE == SCAN_Y || MODE == SCAN_BACK_PART;
  if (a.softplus && (!GATED || a.z != nullptr)) hipLaunchKernelGGL((scan_fwd_kernel<T, NP, MODE, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((scan_fwd_kernel<T, NP, MODE, false>), grid, dim3(256), 0, s, a);
}

// The launches of a forward pass; MODE: SCAN_Y or SCAN_STATES
template <int MODE> static int scan_forward(ScanArgs a, hipStream_t s, int dtype) {
  a.tiles = fwd_tiles(a.dg);
  a.bits = fwd_segment(a.q, a.groups, a.dg);
  a.items = a.bits != WHOLE ? seg_total(a.q, a.bits) : a.q.n_seqs;
  const int64_t waves = a.items * a.groups * a.tiles;
  if (waves > INT_MAX) return set_error(TGNN_E_OUT_OF_RANGE, "%lld wavefronts", (long long)waves);
  const dim3 grid = group_grid((waves + 3) / 4);
  dim3 chain;
  if (a.bits != WHOLE)
    if (int rc = chain_grid(a, &chain)) return rc;
  scan_shape(dtype, a.n, [&](auto t, auto np) {
    using T = decltype(t);
    constexpr int NP = decltype(np)::value;
    if (a.bits != WHOLE) {
      launch_scan<T, NP, SCAN_PART>(a, grid, s);
      launch_chain<false>(a, chain, s);
    }
    launch_scan<T, NP, MODE>(a, grid, s);
  });
  TGNN_LAUNCH_CHECK();
  return TGNN_OK;
}

constexpr int BWD_SPREAD = 256, BWD_FILL = 5;   // workgroups: one, and five, to a compute unit
constexpr int BWD_WORKERS = 1024;   // at most as many partial sums of the weights' gradients

struct BwdPlan { int tiles, slices, bits, workers, finish_x, finish_tiles, finishers; int64_t items; };
static BwdPlan bwd_plan(const tgnn_seqs& q, int d, int n, int groups) {
  BwdPlan p = {};
  const int dg = d / groups;
  p.tiles = (dg + BWD_COLS - 1) / BWD_COLS;
  p.slices = (n + SLICE - 1) / SLICE;
  const int64_t all = (int64_t)groups * p.tiles * p.slices;
  p.bits = scan_segment(q, all, BWD_SPREAD, BWD_FILL);
  p.items = p.bits != WHOLE ? seg_total(q, p.bits) : q.n_seqs;
  p.workers = (int)std::max<int64_t>(1, std::min<int64_t>(p.items, std::min<int64_t>(BWD_WORKERS, 2 * BWD_SPREAD * BWD_FILL / all)));
  for (p.finish_x = 1; p.finish_x < 256 && p.finish_x < d;) p.finish_x *= 2;
  p.finish_tiles = (d + p.finish_x - 1) / p.finish_x;
  p.finishers = (int)std::max<int64_t>(1, std::min<int64_t>(seg_total(q, FINISH_BITS), 2048 / p.finish_tiles));
  return p;
}
struct BwdSpace { float *saved = nullptr, *part = nullptr, *part2 = nullptr, *part_y = nullptr, *part_bc = nullptr, *seg_state = nullptr, *seg_delta = nullptr; };
// Bytes of a backward call's workspace, and where its parts are; fwd: of the forward pass that forms the states (saved == false)
static int64_t bwd_bytes(const tgnn_seqs& q, int d, int n, int groups, bool saved, BwdSpace* s, void* ws, ScanArgs* fwd) {
  const BwdPlan p = bwd_plan(q, d, n, groups);
  BwdSpace none;
  if (s == nullptr) s = &none;
  Take t{static_cast<char*>(ws)};
  if (!saved) {
    s->saved = t.floats(seg_total(q, CHUNK_BITS) * d * n);
    t.off += fwd_bytes(q, d, n, groups, fwd, ws ? static_cast<char*>(ws) + t.off : nullptr);
  }
  if (p.bits != WHOLE) {
    s->seg_state = t.floats(seg_total(q, p.bits) * d * n);
    s->seg_delta = t.floats(seg_total(q, p.bits) * d);
  }
  s->part = t.floats((int64_t)p.workers * ((int64_t)d * n + 2 * d));
  if (p.tiles > 1) s->part_bc = t.floats((int64_t)p.tiles * q.n_rows * 2 * groups * n);
  if (p.slices > 1) {
    s->part2 = t.floats((int64_t)p.finishers * 2 * d);
    s->part_y = t.floats((int64_t)3 * p.slices * q.n_rows * d);
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
  return seg_total(*seqs, CHUNK_BITS) * d * n_state * (int64_t)sizeof(float);
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
  for (const RowArray& in : {RowArray{scan->x, scan->d, scan->ld_x}, RowArray{scan->dt, scan->d, scan->ld_dt}, RowArray{scan->z, scan->d, scan->ld_z},
                             RowArray{scan->B, bc, scan->ld_b}, RowArray{scan->C, bc, scan->ld_c}})
    if (rows_overlap(rows, size, {y, scan->d, ld_y}, in)) return set_error(TGNN_E_INVALID_ARG, "y overlaps an input");
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
  for (const RowArray& in : {RowArray{scan->x, scan->d, scan->ld_x}, RowArray{scan->dt, scan->d, scan->ld_dt}, RowArray{scan->z, scan->d, scan->ld_z},
                             RowArray{scan->B, bc, scan->ld_b}, RowArray{scan->C, bc, scan->ld_c}})
    if (rows_overlap(n_rows, size, {y, scan->d, ld_y}, in)) return set_error(TGNN_E_INVALID_ARG, "y overlaps an input");
  if (n_rows == 0) return TGNN_OK;
  ScanArgs a = scan_args(nullptr, scan);
  a.y = y; a.ld_y = ld_y; a.state_out = state_out; a.items = n_rows;
  int bits = 0;
  while ((4 << bits) < a.n) ++bits;
  const int tiles = (a.d + (256 >> bits) - 1) / (256 >> bits);
  dim3 grid;
  if (int rc = launch_grid((n_rows + 3) / 4 * tiles, &grid)) return rc;
  with_type(scan->dtype, [&](auto t) {
    using T = decltype(t);
    hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    if (bits >= 2) hipLaunchKernelGGL((scan_step_kernel<T, true>), grid, dim3(256), 0, s, a, bits, tiles);
    else hipLaunchKernelGGL((scan_step_kernel<T, false>), grid, dim3(256), 0, s, a, bits, tiles);
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
  struct Named { const char* name; RowArray a; };
  const Named out[] = {{"dx", {grads->dx, d, grads->ld_dx}}, {"ddt", {grads->ddt, d, grads->ld_ddt}}, {"dB", {grads->dB, bc, grads->ld_db}},
                       {"dC", {grads->dC, bc, grads->ld_dc}}, {"dz", {grads->dz, d, grads->ld_dz}}};
  const Named in[] = {{"dy", {dy, d, ld_dy}}, {"x", {scan->x, d, scan->ld_x}}, {"dt", {scan->dt, d, scan->ld_dt}},
                      {"B", {scan->B, bc, scan->ld_b}}, {"C", {scan->C, bc, scan->ld_c}}, {"z", {scan->z, d, scan->ld_z}}};
  if (int rc = check_row_array("dy", dy, ld_dy, rows, d, scan->dtype)) return rc;
  const int n_out = scan->z != nullptr ? 5 : 4;
  for (int i = 0; i < n_out; ++i) {
    if (int rc = check_row_array(out[i].name, out[i].a.p, out[i].a.ld, rows, (int)out[i].a.cols, scan->dtype)) return rc;
    for (const Named& r : in)
      if (rows_overlap(rows, size, out[i].a, r.a)) return set_error(TGNN_E_INVALID_ARG, "%s overlaps %s", out[i].name, r.name);
  }
  if (!aligned_to(grads->dA, 4) || !aligned_to(grads->dD, 4) || !aligned_to(grads->ddt_bias, 4))
    return set_error(TGNN_E_MISALIGNED, "dA, dD or ddt_bias is not aligned to its type");
  if (!aligned_to(saved, 16)) return set_error(TGNN_E_MISALIGNED, "saved is not 16-byte aligned");
  if (saved != nullptr && saved_bytes < tgnn_selective_scan_saved_bytes(seqs, d, scan->n_state))
    return set_error(TGNN_E_WORKSPACE, "saved has %lld bytes, %lld are needed", (long long)saved_bytes,
                     (long long)tgnn_selective_scan_saved_bytes(seqs, d, scan->n_state));
  ScanArgs a = scan_args(seqs, scan), fwd = a;
  BwdSpace space;
  const int64_t need = bwd_bytes(*seqs, d, a.n, a.groups, saved != nullptr, &space, workspace, &fwd);
  if (int rc = check_workspace(workspace, workspace_bytes, need)) return rc;
  for (int i = 1; i < n_out; ++i)
    for (int k = 0; k < i; ++k)
      if (rows_overlap(rows, size, out[i].a, out[k].a)) return set_error(TGNN_E_INVALID_ARG, "%s overlaps %s", out[i].name, out[k].name);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const BwdPlan plan = bwd_plan(*seqs, d, a.n, a.groups);
  a.saved = saved != nullptr ? const_cast<float*>(saved) : space.saved;
  fwd.saved = a.saved;
  if (saved == nullptr && seqs->n_seqs > 0)
    if (int rc = scan_forward<SCAN_STATES>(fwd, s, scan->dtype)) return rc;
  a.dy = dy; a.ld_dy = ld_dy;
  a.dx = grads->dx; a.ddt = grads->ddt; a.dz = grads->dz; a.dB = grads->dB; a.dC = grads->dC;
  a.ld_dx = grads->ld_dx; a.ld_ddt = grads->ld_ddt; a.ld_dz = grads->ld_dz; a.ld_db = grads->ld_db; a.ld_dc = grads->ld_dc;
  a.seg_state = space.seg_state; a.seg_delta = space.seg_delta; a.part_bc = space.part_bc; a.part_y = space.part_y;
  a.bits = plan.bits; a.items = plan.items; a.slices = plan.slices;
  const bool weights = grads->dA != nullptr || grads->dD != nullptr || grads->ddt_bias != nullptr, sliced = plan.slices > 1;
  if (seqs->n_seqs > 0) {
    dim3 chain, back, sum;
    const int64_t waves = plan.items * a.groups * fwd_tiles(a.dg);
    if (plan.bits != WHOLE) {
      if (int rc = chain_grid(a, &chain)) return rc;
      if (waves > INT_MAX) return set_error(TGNN_E_OUT_OF_RANGE, "%lld wavefronts", (long long)waves);
      back = group_grid((waves + 3) / 4);
    }
    const int64_t sums = seg_total(*seqs, SUM_BITS);
    if (int rc = launch_grid(sums, &sum)) return rc;
    scan_shape(scan->dtype, a.n, [&](auto t, auto np) {
      using T = decltype(t);
      constexpr int NP = decltype(np)::value, LANE = NP < SLICE ? NP / 4 : SLICE / 4;
      constexpr bool SLICED = NP > SLICE;
      if (plan.bits != WHOLE) {
        a.tiles = fwd_tiles(a.dg);
        launch_scan<T, NP, SCAN_BACK_PART>(a, back, s);
        launch_chain<true>(a, chain, s);
      }
      a.tiles = plan.tiles;
      a.part = weights ? space.part : nullptr;
      const dim3 grid((unsigned)(plan.workers * a.groups * plan.tiles * plan.slices)), block(64 * BWD_WAVES);
      if (a.softplus && a.z != nullptr) hipLaunchKernelGGL((scan_bwd_kernel<T, LANE, true, SLICED>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((scan_bwd_kernel<T, LANE, false, SLICED>), grid, block, 0, s, a);
      if (a.part_bc) {
        a.items = sums;
        hipLaunchKernelGGL((scan_bc_sum_kernel<T>), sum, dim3(256), 0, s, a);
      }
      if constexpr (SLICED) {
        a.items = seg_total(*seqs, FINISH_BITS);
        a.part = weights ? space.part2 : nullptr;
        hipLaunchKernelGGL((scan_finish_kernel<T>), dim3((unsigned)(plan.finishers * plan.finish_tiles)), dim3(256), 0, s, a, plan.finish_x,
                           plan.finish_tiles);
      }
    });
    TGNN_LAUNCH_CHECK();
  }
  if (weights) {
    const int64_t dn = (int64_t)d * a.n;
    const int n_part = seqs->n_seqs > 0 ? plan.workers : 0, n_part2 = seqs->n_seqs > 0 ? plan.finishers : 0;
    if (!sliced) {
      column_sum(ColumnSum{space.part, n_part, dn + 2 * d, {grads->dA, grads->dD, grads->ddt_bias}, {dn, d, d}, accumulate}, s);
    } else {
      column_sum(ColumnSum{space.part, n_part, dn, {grads->dA, nullptr, nullptr}, {dn, 0, 0}, accumulate}, s);
      column_sum(ColumnSum{space.part2, n_part2, 2 * (int64_t)d, {grads->dD, grads->ddt_bias, nullptr}, {d, d, 0}, accumulate}, s);
    }
    TGNN_LAUNCH_CHECK();
  }
  return TGNN_OK;
}
