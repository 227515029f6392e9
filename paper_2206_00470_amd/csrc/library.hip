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
  (void)runs;
  if (ps_status r = run_keywork(nullptr, KeysPadded{ids, pad, counter}, n, num_keys, b, err, nullptr, false, st, &ks,
                                &perm, false, b.seg_off, uniq))
    return r;
  *out = Order{ks, perm, b.seg_off, b.hdr};
  return PS_OK;
}

ps_status fork_side(ps_store* s, hipStream_t st, hipStream_t* side) {
  *side = s->aux;
  return fork_aux(s, st);
}

ps_status join_side(ps_store* s, hipStream_t st) { return join_aux(s, st); }

}  // namespace adapm
