// What the sources of the library share on the host besides the C ABI: the
// error message, a store's table, and the sort of a list of ids.  Defined in
// library.hip.
#pragma once

#include "adapm.h"

#include <hip/hip_runtime.h>

#include "common.hpp"

#define ADAPM_HIDDEN __attribute__((visibility("hidden")))

namespace adapm {

// Sets the calling thread's error message and returns st.
ADAPM_HIDDEN ps_status raise(ps_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

#define RAISE_HIP(expr)                                                                                    \
  do {                                                                                                     \
    const hipError_t e_ = (expr);                                                                          \
    if (e_ != hipSuccess) return ::adapm::raise(PS_ERR_DEVICE, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

// The value table of a store.  A staged store's ids index its map_keys home
// keys and are translated by `map` to slots (num_keys of them).
struct TableView {
  const void* values;
  int64_t ld;
  int64_t num_keys;
  int32_t dim;
  bool bf16;
  int32_t* status;
  const int32_t* map;
  int64_t map_keys;
};

ADAPM_HIDDEN TableView table_view(const ps_store* s);

// A stable sort of n ids in [0, num_keys): sorted keys (num_keys marks the
// ids that take no part: `pad` silently, others outside the range with
// *err raised) and the occurrence of each sorted position.  With `runs` (n up to
// ORDER_RUNS_MAX) also the runs of equal keys: their distinct keys in uniq,
// their first positions in seg_off (seg_off[U] = ids that take part), U in
// hdr->num_unique; else seg_off is room for n + 1 positions.
// *counter, if given, is set to zero.
constexpr int64_t ORDER_RUNS_MAX = 8192;

struct Order {
  const uint32_t* keys;
  const uint32_t* perm;
  int32_t* seg_off;
  const SegHeader* hdr;
};

ADAPM_HIDDEN size_t order_bytes(int64_t n);
ADAPM_HIDDEN ps_status order_ids(const int64_t* ids, int64_t n, int64_t pad, int64_t num_keys, void* ws, bool runs,
                                 int64_t* uniq, uint32_t* counter, int32_t* err, hipStream_t st, Order* out);

// Largest number of occurrences of one call.
constexpr int64_t OCC_MAX = (int64_t(1) << 31) - (int64_t(1) << 20);

// Largest grid of workgroups of BLOCK threads (a launch counts its threads in 32
// bits).
constexpr int64_t GRID_MAX = (int64_t(1) << 32) / BLOCK - 1;

inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool on_bytes(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace adapm
