// What the kernels of attention with shaped scores share: where a packed sequence lies, and which keys a query sees.
#pragma once
#include "common.h"

namespace stg {

// Rows [lo, hi) of one packed sequence and the number of its leading keys that all of its queries see.
struct SeqSpan { int lo, hi, prefix; };

// Sequence i.  Offsets that do not ascend or leave [0, rows] are brought into it: what such a call computes is undefined, what it
// touches is not.
__device__ __forceinline__ SeqSpan seq_span(const ScoreArgs& a, int i) {
  SeqSpan s;
  if (a.seq_start) {
    s.lo = min(max(a.seq_start[i], 0), a.rows);
    s.hi = min(max(a.seq_start[i + 1], s.lo), a.rows);
  } else {
    const int n = a.rows / a.n_seq;
    s.lo = i * n;
    s.hi = s.lo + n;
  }
  s.prefix = a.prefix ? min(max(a.prefix[i], 0), s.hi - s.lo) : 0;
  return s;
}

// The sequence that a row lies in; false for a row before the first or behind the last.
__device__ __forceinline__ bool seq_of_row(const ScoreArgs& a, int row, SeqSpan& s) {
  int i = 0;
  if (a.seq_start) {                   // the last one that starts at or before the row: empty sequences share their start with the next
    int n = a.n_seq;
    while (n > 1) {
      const int half = n >> 1;
      if (a.seq_start[i + half] <= row) { i += half; n -= half; }
      else n = half;
    }
  } else i = row / (a.rows / a.n_seq);
  s = seq_span(a, i);
  return row >= s.lo && row < s.hi;
}

// The keys that query `row` sees are [s.lo, keys_end): a mask here is an interval from the sequence's first key on.
__device__ __forceinline__ int keys_end(const ScoreArgs& a, const SeqSpan& s, int row) { return a.causal ? max(row + 1, s.lo + s.prefix) : s.hi; }
// The queries that see key `row` are [queries_begin, s.hi).
__device__ __forceinline__ int queries_begin(const ScoreArgs& a, const SeqSpan& s, int row) { return a.causal && row >= s.lo + s.prefix ? row : s.lo; }

// Score of a product x, exact to a few roundings (the bf16 kernels have faster forms), and the cap's derivative there: 1 - t^2 in fp32, here as there, so
// 2^-23 off, and of a score of eight caps, whose derivative is that small itself, next to nothing is left.
__device__ __forceinline__ float shaped(float x, const ScoreArgs& a, float slope, int dist, float& dcap) {
  float s = x * a.scale;
  dcap = 1.f;
  if (a.cap > 0.f) {
    const float t = tanhf(s / a.cap);
    s = a.cap * t;
    dcap = fmaf(-t, t, 1.f);
  }
  return a.slope ? s - slope * (float)abs(dist) : s;
}

}  // namespace stg
