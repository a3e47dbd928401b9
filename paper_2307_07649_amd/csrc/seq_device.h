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

// Segments of `seg` rows are numbered through all sequences: those of sequence s begin at seg_base(s) and are at most as many as lie
// between that and seg_base(s + 1).  With row ranges the numbers come from the ranges themselves, begin / seg + s, which grows
// by at least one and at least ceil(rows / seg) from a sequence to the next: no counting pass, and at most n_rows / seg + n_seqs
// of them.
__host__ __device__ __forceinline__ int64_t seg_per(const tgnn_seqs& q, int seg) {
  return q.max_len > 0 ? ((int64_t)q.max_len + seg - 1) / seg : 1;
}
__device__ __forceinline__ int64_t seg_base(const tgnn_seqs& q, int s, int seg) {
  if (q.indptr == nullptr) return (int64_t)s * seg_per(q, seg);
  const int64_t b = q.indptr[s];
  return (b < 0 ? 0 : b > q.n_rows ? q.n_rows : b) / seg + s;
}
inline int64_t seg_total(const tgnn_seqs& q, int seg) {
  return q.indptr == nullptr ? q.n_seqs * seg_per(q, seg) : q.n_rows / seg + q.n_seqs;
}
// The sequence of a segment, and which one of its own it is.
__device__ __forceinline__ void seg_find(const tgnn_seqs& q, int64_t slot, int seg, int& s, int64_t& k) {
  if (q.indptr == nullptr) {
    const int64_t per = seg_per(q, seg);
    s = (int)(slot / per);
    k = slot - s * per;
    return;
  }
  int lo = 0, hi = q.n_seqs - 1;
  while (lo < hi) {
    const int mid = lo + (hi - lo + 1) / 2;
    if (seg_base(q, mid, seg) <= slot) lo = mid; else hi = mid - 1;
  }
  s = lo;
  k = slot - seg_base(q, lo, seg);
}

// Work of one workgroup or wavefront: a segment of a sequence, or (seg == 0) a whole one.
struct Piece {
  Seq r;
  int s;
  int64_t slot;     // number of the segment (seg != 0)
  int t0, t1;       // its events
  bool last;        // the sequence ends here: final state and padding rows are this piece's
  bool none;        // a number without a segment
};
__device__ __forceinline__ Piece piece_at(const tgnn_seqs& q, int64_t item, int seg) {
  Piece p;
  p.slot = item;
  int64_t k = 0;
  if (seg == 0) p.s = (int)item;
  else seg_find(q, item, seg, p.s, k);
  p.r = seq_at(q, p.s);
  if (seg == 0) {
    p.t0 = 0;
    p.t1 = p.r.len;
    p.last = true;
    p.none = false;
    return p;
  }
  const int64_t need = p.r.len > 0 ? ((int64_t)p.r.len + seg - 1) / seg : 1;
  p.none = k < 0 || k >= need;
  p.t0 = p.none ? 0 : (int)(k * seg);
  p.t1 = p.none ? 0 : (int)(k == need - 1 ? p.r.len : (k + 1) * seg);
  p.last = k == need - 1;
  return p;
}

int check_seqs(const tgnn_seqs* q);

}  // namespace tgnn
