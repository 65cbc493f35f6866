// Argument checks shared by the layer operators' entry points.
#pragma once

#include "bkmoo.h"
#include "internal.h"

namespace bkmoo {

inline bool valid_elem(int dt) { return dt == BKMOO_F32 || dt == BKMOO_BF16; }
inline bool natural(const void *p, int dt) { return (uintptr_t)p % (uintptr_t)elem_bytes(dt) == 0; }
inline bool at4(const void *p) { return (uintptr_t)p % 4 == 0; }

// Bytes [p, p + n) of a call's inputs and outputs.
struct Range {
  const void *p;
  size_t n;
};
inline bool ranges_overlap(const Range &a, const Range &b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && a.n && b.n && x < y + b.n && y < x + a.n;
}
// Some output overlaps an input or another output.
template <int NI, int NO>
bool any_overlap(const Range (&in)[NI], const Range (&out)[NO]) {
  for (int o = 0; o < NO; ++o) {
    for (int i = 0; i < NI; ++i)
      if (ranges_overlap(out[o], in[i])) return true;
    for (int q = o + 1; q < NO; ++q)
      if (ranges_overlap(out[o], out[q])) return true;
  }
  return false;
}

// The tasks' rows: K + 1 offsets (host) from 0 to M.
inline bool valid_task_rows(int32_t K, const int64_t *rows, int64_t M) {
  if (!rows || rows[0] != 0 || rows[K] != M) return false;
  for (int k = 0; k < K; ++k)
    if (rows[k] > rows[k + 1]) return false;
  return true;
}

inline bkmoo_status status_of(hipError_t e) { return e == hipSuccess ? BKMOO_OK : BKMOO_EHIP; }

}  // namespace bkmoo
