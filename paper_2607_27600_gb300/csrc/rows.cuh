// rows.cuh -- packed rows of new tokens (cc_rows), shared by the kernels of a
// serving step.
#pragma once
#include "cc_common.cuh"

namespace cc {

struct StepRows {
  int n_rows, max_rows, batch, cap;
  const int32_t *row_start;   // device [batch + 1], or nullptr: row b
  const int32_t *seq_len;     // device [batch]
};

// Sequence b's rows [r0, r0 + count), which take slots seq, seq + 1, ...  ok:
// in order and inside the buffers; `fit`: they have to fit in cap too.  A
// sequence that is not ok has no rows.
struct SeqRows {
  int r0, count, seq;
  bool ok;
};
CC_DEV SeqRows seq_rows(const StepRows &p, int b, bool fit) {
  SeqRows s;
  const int lo = p.row_start ? p.row_start[b] : b;
  const int hi = p.row_start ? p.row_start[b + 1] : b + 1;
  s.seq = p.seq_len[b];
  s.r0 = lo;
  s.ok = lo >= 0 && lo <= hi && hi <= p.n_rows && hi - lo <= p.max_rows && s.seq >= 0 &&
         s.seq <= p.cap && (!fit || hi - lo <= p.cap - s.seq);
  s.count = s.ok ? hi - lo : 0;
  return s;
}

}  // namespace cc
