// The ids of a lookup, from a store's table or a quantised one.
#pragma once

#include "common.hpp"

namespace adapm {

constexpr int EMBED_FLIGHT = 4;   // vectors in flight per thread

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
  if (id == l.pad) return -1;
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
