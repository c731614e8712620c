// Index arithmetic of the paged window cache, for the kernels and for host tests
// (plain C++ without HIP types).  Every value that comes from device arrays of
// the caller (starts, lengths, page numbers) is bounded here.
#pragma once

#include <stddef.h>
#include <stdint.h>

#if defined(__HIPCC__)
#define DKV_HD __host__ __device__ __forceinline__
#else
#define DKV_HD inline
#endif

namespace dkv {

// A dkv_cache and its chunk as the kernels take them.
struct Pages {
  unsigned char *k, *v;   // [P, H, 2^lps, row bytes]
  uint8_t *ks, *vs;       // [P, H, 2^lps, d / 32]
  const int32_t *table;   // [S, cols]
  const int32_t *length;  // [S]
  const int32_t *start;   // [S + 1] or null
  int S, H, P, cols, lps, T, max_new;
  // Places of the chunk's tokens in a launch: max_new for each sequence where those are no more than T (token i of s at
  // s max_new + i), else the T packed rows, whose sequence is searched for.
  bool by_seq;
};
DKV_HD int64_t places(const Pages &c) { return c.by_seq ? (int64_t)c.S * c.max_new : c.T; }

DKV_HD int bound(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// Tokens of sequence s.
DKV_HD int seq_length(const Pages &c, int s) { return bound(c.length[s], 0, c.cols << c.lps); }

// First packed row of sequence s and its number of new tokens.
struct NewRows {
  int first, n;
};
DKV_HD NewRows new_rows(const Pages &c, int s) {
  if (!c.start) return NewRows{s * (c.T / c.S), c.T / c.S};
  const int a = bound(c.start[s], 0, c.T);
  return NewRows{a, bound(c.start[s + 1], a, c.T) - a};
}

// Largest s in [0, S) with at_most(s), -1 if there is none, where at_most holds up to some s and no further.  probe(lo,
// step, hi) gives the largest k < N with lo + k step < hi and at_most(lo + k step), or -1: N places side by side, the
// lanes of a group in the kernels.
template <int N, class F>
DKV_HD int last_at_most(int S, F probe) {
  int lo = 0, hi = S;
  do {
    const int step = (hi - lo + N - 1) / N, k = probe(lo, step, hi);
    if (k < 0) return -1;
    lo += k * step;
    hi = hi < lo + step ? hi : lo + step;
  } while (hi - lo > 1);
  return lo;
}

// First slot of sequence s where the row blocks (R rows, `rows` for each token) of packed sequences are numbered one after
// the other: [slot_base(s), slot_base(s + 1)) holds all of those of s, and one slot at most stays empty.  T rows / R + S
// slots in all.
DKV_HD int slot_base(const Pages &c, int rows, int R, int s) {
  return (int)((uint32_t)bound(c.start[s], 0, c.T) * (uint32_t)rows / (uint32_t)R) + s;
}
DKV_HD int64_t packed_slots(const Pages &c, int rows, int R) { return (int64_t)c.T * rows / R + c.S; }

// Page that holds position pos (0 <= pos < cols << lps) of sequence s, -1 if absent.
DKV_HD int page_of(const Pages &c, int s, int pos) {
  const int p = c.table[(size_t)s * c.cols + (pos >> c.lps)];
  return (unsigned)p < (unsigned)c.P ? p : -1;
}

// Row of the pool: head h of position pos in page p.
DKV_HD size_t pool_row(const Pages &c, int p, int h, int pos) {
  return ((((size_t)p * c.H + h) << c.lps) + (size_t)(pos & ((1 << c.lps) - 1)));
}

// Tokens that new token i of n sees in a sequence of len tokens: the positions j < hi
// with j >= lo or j < sink.
struct Mask {
  int window, sink, causal;
};
struct Seen {
  int lo, hi;
};
DKV_HD Seen seen_by(const Mask &m, int len, int n, int i) {
  const int at = m.causal ? len - n + i : len - 1;
  const int lo = m.window > 0 ? at - m.window + 1 : 0;
  return Seen{lo > 0 ? lo : 0, at + 1 > 0 ? at + 1 : 0};
}
DKV_HD bool sees(const Seen &r, int sink, int j) { return j < r.hi && (j >= r.lo || j < sink); }

}  // namespace dkv
