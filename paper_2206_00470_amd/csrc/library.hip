// The store (api.hip) and what it lends to the other sources of the library
// (internal.hpp).
#include "api.hip"

#include "internal.hpp"

namespace {

// Ids in which `pad` stands for no occurrence.  The intake calls it once for
// every id before anything later on the stream runs, so that it can also clear
// a counter of a later kernel.
struct KeysPadded {
  const int64_t* ids;
  int64_t pad;
  uint32_t* counter;
  __device__ int64_t operator()(int64_t i) const {
    if (counter && i == 0) *counter = 0u;
    const int64_t id = ids[i];
    if (id == ABSENT) return -1;   // as a pad it says that there is none, as an id it is outside
    return id == pad ? ABSENT : id;
  }
};

}  // namespace

namespace adapm {

ps_status raise(ps_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return fail(st, "%s", buf);
}

TableView table_view(const ps_store* s) {
  return TableView{s->W, s->ld, s->num_keys, s->dim, s->bf16, s->status, s->stg ? s->stg->map : nullptr,
                   s->stg ? s->stg->num_keys : int64_t(0)};
}

size_t order_bytes(int64_t n) {
  SortBufs b;
  Carver c(nullptr);
  carve_sort(c, n, 1, false, true, &b);
  return (c.off + 255) & ~size_t(255);
}

ps_status order_ids(const int64_t* ids, int64_t n, int64_t pad, int64_t num_keys, void* ws, bool runs, int64_t* uniq,
                    uint32_t* counter, int32_t* err, hipStream_t st, Order* out) {
  SortBufs b;
  Carver c(ws);
  carve_sort(c, n, 1, false, true, &b);
  uint32_t *ks, *perm;
  static_assert(ORDER_RUNS_MAX == SMALL_KEYS_MAX, "one workgroup gives the runs with the sort");
  if (n > SMALL_KEYS_MAX) {
    if (runs) return fail(PS_ERR_UNSUPPORTED, "runs of %lld ids", (long long)n);
    // the sort alone: run_keywork's without its last kernels
    const KeysPadded keys{ids, pad, counter};
    if (n > MID_KEYS_MAX) {
      if (ps_status r = run_sort(nullptr, keys, n, num_keys, b, err, nullptr, false, st, &ks, &perm)) return r;
      *out = Order{ks, perm, b.seg_off, nullptr};
      return PS_OK;
    }
    const RadixPlan plan = radix_plan(num_keys);
    const int tiles = (int)ceil_div(n, MID_TILE);
    hipLaunchKernelGGL((k_mid_intake<KeysPadded>), dim3(tiles), dim3(SMALL_BLOCK), 0, st, keys, (int)n,
                       (uint32_t)num_keys, plan.bits[0], b.k[0], b.counts, err);
    LAUNCHED(k_mid_intake);
    for (int p = 0; p < plan.passes; ++p) {
      if (p > 0) {
        hipLaunchKernelGGL(k_mid_count, dim3(tiles), dim3(SMALL_BLOCK), 0, st, b.k[p % 2], (int)n, plan.shift[p],
                           plan.bits[p], b.counts);
        LAUNCHED(k_mid_count);
      }
      hipLaunchKernelGGL(k_mid_scatter, dim3(tiles), dim3(SMALL_BLOCK), 0, st, b.k[p % 2],
                         p > 0 ? b.v[p % 2] : nullptr, (int)n, plan.shift[p], plan.bits[p], b.counts, tiles,
                         b.k[1 - p % 2], b.v[1 - p % 2], nullptr);
      LAUNCHED(k_mid_scatter);
    }
    *out = Order{b.k[plan.passes % 2], b.v[plan.passes % 2], b.seg_off, nullptr};
    return PS_OK;
  }
  if (ps_status r = run_keywork(nullptr, KeysPadded{ids, pad, counter}, n, num_keys, b, err, nullptr, false, st, &ks,
                                &perm, false, b.seg_off, uniq))
    return r;
  *out = Order{ks, perm, b.seg_off, b.hdr};
  return PS_OK;
}

}  // namespace adapm
