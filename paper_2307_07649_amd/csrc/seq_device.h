// Where the rows of a call's sequences are (tgnn_seqs), and how long sequences are cut into segments.
#pragma once
#include "ops_device.h"

namespace tgnn {

struct Seq {
  int64_t begin;   // first row of the sequence's slot
  int len, slot;   // rows that belong to it, in front; rows of the slot
};

// Whatever the arrays on the device hold, begin .. begin + slot stays within the rows of the call: a range outside is an empty slot,
// a count outside [0, slot] an empty sequence.
__device__ __forceinline__ Seq seq_at(const tgnn_seqs& q, int s) {
  Seq r;
  if (q.indptr != nullptr) {
    const int64_t b = q.indptr[s], e = q.indptr[s + 1];
    const bool ok = b >= 0 && e >= b && e <= q.n_rows && e - b <= INT_MAX;
    r.begin = ok ? b : 0;
    r.slot = ok ? (int)(e - b) : 0;
  } else {
    r.begin = (int64_t)s * q.max_len;
    r.slot = q.max_len;
  }
  r.len = r.slot;
  if (q.cnt != nullptr) {
    const int c = q.cnt[s];
    r.len = c < 0 || c > r.slot ? 0 : c;
  }
  return r;
}

// row of the event at place t in time, t < len
__device__ __forceinline__ int64_t seq_row(const tgnn_seqs& q, const Seq& r, int t) {
  return r.begin + (q.newest_first ? r.len - 1 - t : t);
}

// Segments of 2^bits rows are numbered through all sequences: those of sequence s begin at seg_base(s) and are at most as many as
// lie between that and seg_base(s + 1).  With row ranges the numbers come from the ranges themselves, (begin >> bits) + s,
// which grows by at least one and at least by the segments of its rows from a sequence to the next: no counting pass, and at
// most (n_rows >> bits) + n_seqs of them (the host makes sure that they fit 31 bits).
__host__ __device__ __forceinline__ int seg_per(const tgnn_seqs& q, int bits) {
  return q.max_len > 0 ? (int)(((unsigned)q.max_len + (1u << bits) - 1) >> bits) : 1;
}
__device__ __forceinline__ int seg_base(const tgnn_seqs& q, int s, int bits) {
  if (q.indptr == nullptr) return s * seg_per(q, bits);
  const int64_t b = q.indptr[s];
  return (int)((b < 0 ? 0 : b > q.n_rows ? q.n_rows : b) >> bits) + s;
}
inline int64_t seg_total(const tgnn_seqs& q, int bits) {
  return q.indptr == nullptr ? (int64_t)q.n_seqs * seg_per(q, bits) : (q.n_rows >> bits) + q.n_seqs;
}
// The sequence of a segment, the same one for all 64 lanes of a wavefront: the lanes look at 64 places at a time, so that 64
// sequences take one load and 4,096 two.  (All lanes have to be there.)
__device__ __forceinline__ int seg_find(const tgnn_seqs& q, int slot, int bits) {
  if (q.indptr == nullptr) return (int)((unsigned)slot / (unsigned)seg_per(q, bits));
  const int lane = threadIdx.x & 63;
  int lo = 0, n = q.n_seqs;
  while (n > 1) {
    const int step = (n + 63) / 64, at = lo + min(lane * step, n - 1);
    const bool before = lane * step < n && seg_base(q, at, bits) <= slot;
    const int hits = __popcll(__ballot(before)), k = hits > 0 ? hits - 1 : 0;   // (the bases ascend: the hits come first)
    lo += k * step;
    n = min(step, n - k * step);
  }
  return __builtin_amdgcn_readfirstlane(lo);
}
// The same for a segment at or a little behind one whose sequence is known.
__device__ __forceinline__ int seg_find_from(const tgnn_seqs& q, int slot, int bits, int s) {
  if (q.indptr == nullptr) return (int)((unsigned)slot / (unsigned)seg_per(q, bits));
  while (s + 1 < q.n_seqs && seg_base(q, s + 1, bits) <= slot) ++s;
  return s;
}
// segments of a sequence of `len` events; an empty one has one
__device__ __forceinline__ int seg_count(int len, int bits) { return len > 0 ? (int)(((unsigned)len + (1u << bits) - 1) >> bits) : 1; }

// Work of one workgroup or wavefront: a segment of a sequence, or a whole one.
constexpr int MIN_SEG_BITS = 3;   // the shortest segments that anything is cut into
constexpr int WHOLE = -1;   // for `bits`: sequences are not cut
struct Piece {
  Seq r;
  int s;
  int slot;         // number of the segment
  int t0, t1;       // its events
  bool last;        // the sequence ends here: final state and padding rows are this piece's
  bool none;        // a number without a segment
};
// The piece of number `item`, a segment of sequence s or the whole of it
__device__ __forceinline__ Piece piece_of(const tgnn_seqs& q, int item, int bits, int s) {
  Piece p;
  p.slot = item;
  p.s = s;
  const int k = bits == WHOLE ? 0 : item - seg_base(q, s, bits);
  p.r = seq_at(q, s);
  const int need = bits == WHOLE ? 1 : seg_count(p.r.len, bits);
  p.last = k == need - 1;
  p.none = k < 0 || k >= need;
  p.t0 = p.none || bits == WHOLE ? 0 : k << bits;
  p.t1 = p.none ? 0 : p.last ? p.r.len : (k + 1) << bits;
  return p;
}
// (for a number that is the same for the whole wavefront)
__device__ __forceinline__ Piece piece_at(const tgnn_seqs& q, int item, int bits) {
  return piece_of(q, item, bits, bits == WHOLE ? item : seg_find(q, item, bits));
}

int check_seqs(const tgnn_seqs* q);

}  // namespace tgnn
