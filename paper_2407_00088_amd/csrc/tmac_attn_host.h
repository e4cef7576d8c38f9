// Checks of the views that the attention and cache entry points take (host code).
#ifndef TMAC_ATTN_HOST_H_
#define TMAC_ATTN_HOST_H_

#include <cstdint>

#include "tmac_attn.h"

namespace tmac {
namespace attn {

// Rows of 16-bit elements that the kernels can read 8 bytes at a time.
inline bool rows_ok(const tmac_view* v, bool seq, bool token, bool head) {
  if (!v || !v->data || (reinterpret_cast<uintptr_t>(v->data) & 7)) return false;
  auto fits = [](int64_t s) { return s >= 0 && s % 4 == 0 && s < ((int64_t)1 << 40); };
  return (!seq || fits(v->seq)) && (!token || fits(v->token)) && (!head || fits(v->head));
}

// Lengths up to which whole tiles past the end are still within 32-bit indexes.
inline bool long_axis(int64_t n) { return n > (int64_t)1 << 30; }

// Threads of a launch are counted in 32 bits.
inline bool launchable(int64_t workgroups, int threads) { return workgroups <= (int64_t)0xffffffff / threads; }

// 128 rows span more than a buffer's range.
inline bool far_rows(const tmac_view* v) { return v->token >= ((int64_t)1 << 22); }

// Rows that can be moved 16 bytes at a time.
inline bool wide_rows(const tmac_view* v, int D) {
  return (reinterpret_cast<uintptr_t>(v->data) & 15) == 0 && D % 8 == 0 && v->seq % 8 == 0 && v->token % 8 == 0 && v->head % 8 == 0;
}

}  // namespace attn
}  // namespace tmac
#endif
