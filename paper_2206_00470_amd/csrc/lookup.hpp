// The ids of a lookup, from a store's table or a quantised one.
#pragma once

#include "common.hpp"

namespace adapm {

// Vectors in flight per thread: 65,536 rows of 2,048 floats to bf16 106 us with
// four, 89 with two or one; a table of 4.6M x 256 4-bit values restored to bf16
// 483 with four, 470 with two, 554 with one.
constexpr int LOOKUP_FLIGHT = 2;

// Outputs beyond this are written past the caches: from here on a lookup alone
// gains a quarter and more, and one with a kernel behind it that reads the output
// loses 3% at most. Measured, through them and past them, alone and with that kernel:
// 61 MB (rows of 512 floats to bf16) 24.7 and 21.6 us, 47.2 and 48.9; 85 MB (100
// floats) 30.9 and 22.5, 57.3 and 58.7; 127 MB (300 4-bit values to bf16) 49.2
// and 29.2, 93.7 and 85.7; 240 MB (301 floats) 90.7 and 57.1, 172 and 156.
constexpr int64_t LOOKUP_STREAMS = int64_t(80) << 20;

// The row of vector q, d vectors a row (a 64-bit division takes several times as
// long as one of 32 bits).
__device__ __forceinline__ int64_t row_of(int64_t q, uint32_t d) {
  return q <= UINT32_MAX ? (int64_t)((uint32_t)q / d) : q / d;
}

struct LookupIds {
  const int64_t* ids;   // NULL: row i of the table
  int64_t n;
  int64_t pad;
  int64_t num_rows;
  const int32_t* map;   // a staged store's key -> slot map, or NULL
  int64_t map_keys;
  int32_t* err;
};

// The table row of output row i, or -1 for a row of zeros.
__device__ __forceinline__ int64_t lookup_row(const LookupIds& l, int64_t i, int& bad, int& miss) {
  if (!l.ids) return i;
  const int64_t id = l.ids[i];
  if (id == l.pad && id != INT64_MIN) return -1;   // (INT64_MIN: there is none)
  if (id < 0 || id >= (l.map ? l.map_keys : l.num_rows)) {
    bad = 1;
    return -1;
  }
  if (!l.map) return id;
  const int32_t slot = l.map[id];
  miss |= slot < 0;
  return slot;
}

}  // namespace adapm
