// Whether two sets of rows in memory meet (internal, host; also compiled as plain C++).
#pragma once

#include <cstddef>
#include <cstdint>

namespace ptd {

// `count` rows of `bytes` bytes (0: none), `step` >= bytes apart (rows that touch, or a single one, count as one long
// row).  The last byte's offset fits in 63 bits.
struct MemoryRows {
  uintptr_t at;
  int64_t bytes, step, count;
};
inline MemoryRows memory_rows(const void* at, int64_t bytes, int64_t step = 0, int64_t count = 1) {
  if (count > 1 && step > bytes) return {reinterpret_cast<uintptr_t>(at), bytes, step, count};
  return {reinterpret_cast<uintptr_t>(at), bytes * count, bytes * count, 1};
}

// Exact where one set is a single row or both have the same step; sets of different steps are taken to meet where
// the memory from their first row to their last does.
inline bool rows_meet(const MemoryRows& a, const MemoryRows& b) {
  if (a.bytes <= 0 || b.bytes <= 0) return false;
  const int64_t span_a = (a.count - 1) * a.step + a.bytes, span_b = (b.count - 1) * b.step + b.bytes;
  if (a.at < b.at ? b.at - a.at >= (uintptr_t)span_a : a.at - b.at >= (uintptr_t)span_b) return false;
  if (a.count > 1 && b.count > 1 && a.step != b.step) return true;
  if (a.count == 1 && b.count == 1) return true;
  // Row i of a meets row k of b if -b.bytes < d - m step < a.bytes with d = b.at - a.at, m = i - k: the least m with
  // d - m step < a.bytes has to do, within what i and k allow.
  const int64_t step = a.count > 1 ? a.step : b.step, d = (int64_t)(b.at - a.at);
  const int64_t x = d - a.bytes;   // m step > x
  int64_t m = x / step + (x % step >= 0 ? 1 : 0);
  if (m < -(b.count - 1)) m = -(b.count - 1);
  return m <= a.count - 1 && d - m * step > -b.bytes;
}

}  // namespace ptd
