// Rows of new tokens, packed over ragged sequences: which sequence a workgroup works on.
//
// Rows first[b] .. first[b + 1] - 1 of the packed buffers belong to sequence b (first == NULL: s_q rows each).  Work is dealt out in
// runs of 2^shift rows without a scan of the run lengths: sequence b's runs are numbered from floor(first[b] * mul / 2^shift) + EXTRA * b, and
// floor(x + y) >= floor(x) + floor(y) leaves room for floor(n mul / 2^shift) + EXTRA of them; a run that its sequence does not need is
// left at once.  Finding the sequence is then one comparison per sequence, 64 at a time, instead of a prefix sum.
// Values of `first` are clamped into [0, total], and where one falls the count of sequences at or before x may name one behind x (k < 0) or
// one without rows: neither is worked on, so that whatever `first` holds stays in bounds.
#pragma once

#include "gqla_device.h"

namespace gqla {

struct RowSpan {
  int b, first, n, len;  // sequence, its first packed row, its rows, its cached tokens (the new ones included)
  int k;                 // which of the sequence's runs
};

template <int EXTRA>
__device__ __forceinline__ bool find_rows(const int32_t* first, const int32_t* seq_lens, int batch, int total, int s_q, int mul, int shift, int x, RowSpan& r) {
  const int lane = threadIdx.x & 63;
  auto begin = [&](int b) { return first ? min(max(first[b], 0), total) : b * s_q; };
  auto run = [&](int f, int b) { return (int)((int64_t)f * mul >> shift) + EXTRA * b; };
  if (batch < 64) {  // everything with one latency
    const int f = begin(min(lane, batch));
    const int l = seq_lens[min(lane, batch - 1)];
    const uint64_t mask = __builtin_amdgcn_ballot_w64(lane < batch && run(f, lane) <= x);
    if (mask == 0) return false;
    r.b = __builtin_popcountll(mask) - 1;
    r.first = __builtin_amdgcn_readlane(f, r.b);
    r.n = __builtin_amdgcn_readlane(f, r.b + 1) - r.first;
    r.len = __builtin_amdgcn_readlane(l, r.b);
  } else {
    int count = 0;
    for (int base = 0; base < batch; base += 64) {
      const int b = base + lane;
      const uint64_t mask = __builtin_amdgcn_ballot_w64(b < batch && run(begin(min(b, batch)), b) <= x);
      count += __builtin_popcountll(mask);
      if (mask != ~0ull) break;
    }
    if (count == 0) return false;
    r.b = __builtin_amdgcn_readfirstlane(count - 1);
    r.first = __builtin_amdgcn_readfirstlane(begin(r.b));
    r.n = __builtin_amdgcn_readfirstlane(begin(r.b + 1)) - r.first;
    r.len = __builtin_amdgcn_readfirstlane(seq_lens[r.b]);
  }
  r.k = x - run(r.first, r.b);
  return r.n > 0 && r.k >= 0;
}

// Runs of the whole batch, for the grid.
inline int64_t row_runs(int64_t total, int64_t mul, int shift, int64_t extra, int64_t batch) { return (total * mul >> shift) + extra * batch; }

}  // namespace gqla
