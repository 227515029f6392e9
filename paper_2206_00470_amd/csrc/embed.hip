// Entry points of the token table's lookup and of its gradient.
#include "embed.hpp"

#include <algorithm>
#include <chrono>
#include <thread>

#include "internal.hpp"
#include "rules.hpp"

using namespace adapm;

namespace {

ps_status check_type(int32_t type) {
  if (type != PS_F32 && type != PS_BF16 && type != PS_F16) return raise(PS_ERR_INVALID, "unknown element type %d", type);
  return PS_OK;
}

ps_status check_count(int64_t n) {
  if (n < 0) return raise(PS_ERR_INVALID, "negative size %lld", (long long)n);
  if (n > OCC_MAX) return raise(PS_ERR_UNSUPPORTED, "%lld ids exceed the 32-bit occurrence index", (long long)n);
  return PS_OK;
}

template <class F>
ps_status with_width(int vw, F&& f) {
  if (vw == 8) return f.template operator()<8>();
  if (vw == 4) return f.template operator()<4>();
  return f.template operator()<1>();
}

}  // namespace

extern "C" {

ps_status ps_embed(ps_store* s, const int64_t* ids, int64_t n, int64_t pad, float scale, int32_t out_type, void* out,
                   int64_t out_stride, void* stream) {
  if (!s) return raise(PS_ERR_INVALID, "store is NULL");
  if (ps_status r = check_count(n)) return r;
  if (ps_status r = check_type(out_type)) return r;
  const TableView t = table_view(s);
  if (out_stride < t.dim) return raise(PS_ERR_INVALID, "out_stride %lld < dim %d", (long long)out_stride, t.dim);
  if (n == 0) return PS_OK;
  if (!ids || !out) return raise(PS_ERR_INVALID, "ids or out is NULL");
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int ob = type_bytes(out_type);
  if (!on_bytes(out, ob)) return raise(PS_ERR_INVALID, "out is not aligned to its elements");
  // stores of 16 bytes (to bf16 from fp32 in vectors of four: 105 us instead of 89 as in lookup.hpp)
  const int vw = t.dim >= 8 && ob == 2 ? 8 : t.dim >= 4 ? 4 : 1;
  const SmallDiv nv = small_div((uint32_t)div_up(t.dim, vw));
  const int64_t grid = div_up(n * nv.d, int64_t(BLOCK) * LOOKUP_FLIGHT);
  if (grid > GRID_MAX) return raise(PS_ERR_UNSUPPORTED, "%lld rows of %d exceed the lookup's grid", (long long)n, t.dim);
  const LookupIds l{ids, n, pad, t.num_keys, t.map, t.map_keys, t.status};
  return with_type(out_type, [&]<class OT>(OT) -> ps_status {
    return with_width(vw, [&]<int VW>() -> ps_status {
      auto launch = [&](auto kernel, auto values) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(BLOCK), 0, st, values, t.ld, l, nv, t.dim, scale, static_cast<OT*>(out),
                           out_stride);
      };
      auto launch_values = [&]<class VT>(const VT* values) {
        if (n * int64_t(t.dim) * ob > LOOKUP_STREAMS) launch(k_embed<VT, OT, VW, true>, values);
        else launch(k_embed<VT, OT, VW, false>, values);
      };
      if (t.bf16) launch_values(static_cast<const bf16_t*>(t.values));
      else launch_values(static_cast<const float*>(t.values));
      RAISE_HIP(hipGetLastError());
      return PS_OK;
    });
  });
}

}  // extern "C"

// ======================================================================== gradient
namespace {

// Blocks folded together: a run over x blocks is finished from about x / f + 2 f
// partial rows, sixteen of them at a time, and the commonest token has a tenth
// or so of a batch.  Up to 256 blocks none are, which saves a launch.
int log_fold(int64_t blocks) { return blocks <= 256 ? 10 : blocks < 16384 ? 4 : blocks < (1 << 20) ? 6 : 8; }

// Positions of a block: fewer rows are added one after another where there are
// not enough blocks of 16 to fill the units, which costs more partial rows.
// Measured, with 8 and with 16: 1,021 ids of 300 floats 20.9 and 24.2 us, 8,192
// of 768 bf16 values 44.9 and 47.3 (but 400,000 of 16 floats over 1,000 rows 69
// and 64); 20,000 of 2,048 63.6 and 55.0, 300,000 of 64 95 and 85, 1M of 100
// floats 270 and 255.
int log_block(int64_t n, int dim) { return n * int64_t(dim) < (int64_t(1) << 24) ? 3 : 4; }

struct GradPlan {
  size_t order = 0;        // the sort's share, at the start
  int log_block = 0;       // positions of a block, as a power of two
  double* partial = nullptr;
  double* fold = nullptr;
  int4* split_list = nullptr;
  uint32_t* split_count = nullptr;
  uint32_t* tile_heads = nullptr;   // rows form
  int32_t* block_run = nullptr;
  size_t bytes = 0;
};

GradPlan plan_grad(void* ws, int64_t n, int dim) {
  GradPlan p;
  p.order = order_bytes(n);
  size_t off = p.order;
  auto take = [&](size_t bytes) {
    off = (off + 255) & ~size_t(255);
    char* q = ws ? static_cast<char*>(ws) + off : nullptr;
    off += bytes;
    return q;
  };
  p.log_block = log_block(n, dim);
  const int64_t blocks = div_up(n, int64_t(1) << p.log_block);
  p.partial = reinterpret_cast<double*>(take(size_t(2) * blocks * dim * sizeof(double)));
  p.fold = reinterpret_cast<double*>(take(size_t(blocks >> log_fold(blocks)) * dim * sizeof(double)));
  p.split_list = reinterpret_cast<int4*>(take(size_t(blocks) * sizeof(int4)));
  p.split_count = reinterpret_cast<uint32_t*>(take(sizeof(uint32_t)));
  p.tile_heads = reinterpret_cast<uint32_t*>(take(size_t(div_up(n, RUNS_TILE)) * sizeof(uint32_t)));
  p.block_run = reinterpret_cast<int32_t*>(take(size_t(blocks) * sizeof(int32_t)));
  p.bytes = off + 256;
  return p;
}

struct GradCall {
  const int64_t* ids;
  int64_t n;
  int64_t pad;
  double scale;
  int32_t in_type;
  const void* dout;
  int64_t in_ld;
  GradOut out;
  int64_t* uniq;         // rows form
  int32_t* num_unique;   // rows form
};

ps_status clear_rows(const GradOut& o, int64_t rows, int dim, hipStream_t st) {
  const int h = o.type == PS_F32 ? 2 : 1;   // 16-bit words per element
  int64_t halves = int64_t(dim) * h, ld = o.ld * h;
  if (ld == halves || rows == 1) {   // one stretch
    halves *= rows;
    rows = 1;
    ld = halves;
  }
  const int vec = halves % 8 == 0 && ld % 8 == 0 && on_bytes(o.p, 16) ? 8
                  : halves % 2 == 0 && ld % 2 == 0 && on_bytes(o.p, 4) ? 2 : 1;
  const int64_t grid = std::min<int64_t>(div_up(rows * (halves / vec), BLOCK), 8192);
  hipLaunchKernelGGL(k_grad_clear, dim3(grid), dim3(BLOCK), 0, st, static_cast<uint16_t*>(o.p), rows, halves, ld, vec);
  RAISE_HIP(hipGetLastError());
  return PS_OK;
}

ps_status embed_grad(ps_store* s, const GradCall& c, void* ws, size_t ws_bytes, hipStream_t st) {
  if (!s) return raise(PS_ERR_INVALID, "store is NULL");
  const TableView t = table_view(s);
  if (t.map) return raise(PS_ERR_UNSUPPORTED, "the lookup's gradient is not available on a staged store");
  if (ps_status r = check_count(c.n)) return r;
  if (ps_status r = check_type(c.in_type)) return r;
  if (ps_status r = check_type(c.out.type)) return r;
  if ((c.in_ld < t.dim && c.in_ld != 0) || c.out.ld < t.dim)   // (0: one row for all ids)
    return raise(PS_ERR_INVALID, "a row stride is smaller than dim %d", t.dim);
  if (!c.out.p) return raise(PS_ERR_INVALID, "grad is NULL");
  const bool rows = c.num_unique != nullptr;
  const int ib = type_bytes(c.in_type), ob = type_bytes(c.out.type);
  if (!on_bytes(c.out.p, ob)) return raise(PS_ERR_INVALID, "grad is not aligned to its elements");
  if (c.n == 0) {
    if (rows) {
      hipLaunchKernelGGL(k_grad_clear, dim3(1), dim3(BLOCK), 0, st, reinterpret_cast<uint16_t*>(c.num_unique),
                         int64_t(1), int64_t(2), int64_t(2), 2);
      RAISE_HIP(hipGetLastError());
      return PS_OK;
    }
    return c.out.accumulate ? PS_OK : clear_rows(c.out, t.num_keys, t.dim, st);
  }
  if (!c.ids || !c.dout || (rows && !c.uniq)) return raise(PS_ERR_INVALID, "ids, dout or uniq is NULL");
  if (!on_bytes(c.dout, ib)) return raise(PS_ERR_INVALID, "dout is not aligned to its elements");
  const GradPlan p = plan_grad(ws, c.n, t.dim);
  if (!ws) return raise(PS_ERR_INVALID, "workspace pointer is NULL");
  if (ws_bytes < p.bytes) return raise(PS_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, p.bytes);
  if (!on_bytes(ws, 16)) return raise(PS_ERR_INVALID, "the workspace must be 16-byte aligned");

  // 16 bytes of the wider side; where sums are added to a row, vectors that lie
  // over each other would add twice
  const bool apart = c.out.accumulate != 0;
  auto fits = [&](int w) { return apart ? t.dim % w == 0 : t.dim >= w; };
  const int vw = ib + ob == 4 && fits(8) ? 8 : fits(4) ? 4 : 1;
  const int vectors = (int)div_up(t.dim, vw);
  int log_lanes = 2;
  while ((1 << log_lanes) < WAVE && (1 << log_lanes) < vectors) ++log_lanes;
  const int slices = (int)div_up(vectors, 1 << log_lanes);
  const int64_t blocks = div_up(c.n, int64_t(1) << p.log_block);
  const int64_t grid = div_up(blocks, BLOCK >> log_lanes);
  if (grid > GRID_MAX || div_up(c.n, BLOCK) > GRID_MAX) return raise(PS_ERR_UNSUPPORTED, "%lld ids of %d exceed the merge's grid", (long long)c.n, t.dim);

  if (!rows && !c.out.accumulate)
    if (ps_status r = clear_rows(c.out, t.num_keys, t.dim, st)) return r;
  // where one workgroup sorts the ids it also gives the runs; else the rows form
  // finds them itself, and the index of each block's first one with them
  const bool own_runs = rows && c.n > ORDER_RUNS_MAX;
  Order o;
  if (ps_status r = order_ids(c.ids, c.n, c.pad, t.num_keys, ws, rows && !own_runs, c.uniq, p.split_count, t.status, st,
                              &o))
    return r;
  if (own_runs) {
    const int64_t tiles = div_up(c.n, RUNS_TILE);
    const bool scan = tiles > 4096;
    hipLaunchKernelGGL(k_runs_count, dim3(tiles), dim3(BLOCK), 0, st, o.keys, c.n, (uint32_t)t.num_keys, p.tile_heads);
    RAISE_HIP(hipGetLastError());
    if (scan) {
      hipLaunchKernelGGL(k_runs_scan, dim3(1), dim3(BLOCK), 0, st, p.tile_heads, tiles);
      RAISE_HIP(hipGetLastError());
    }
    hipLaunchKernelGGL(k_runs_write, dim3(tiles), dim3(BLOCK), 0, st, o.keys, c.n, (uint32_t)t.num_keys, p.tile_heads,
                       (int)scan, p.log_block, c.uniq, o.seg_off, p.block_run, c.num_unique);
    RAISE_HIP(hipGetLastError());
  }
  const GradRuns g{o.keys, o.perm, c.n, (uint32_t)t.num_keys, rows ? o.seg_off : nullptr, o.hdr,
                   own_runs ? p.block_run : nullptr, c.num_unique, p.partial, p.log_block, log_fold(blocks),
                   p.split_list, p.split_count};
  const ps_status r = with_type(c.in_type, [&]<class IT>(IT) -> ps_status {
    return with_width(vw, [&]<int VW>() -> ps_status {
      if constexpr (sizeof(IT) * VW <= 16) {
        auto kernel = p.log_block == 3 ? k_grad_merge<IT, VW, 8> : k_grad_merge<IT, VW, 16>;
        hipLaunchKernelGGL(kernel, dim3(grid, slices), dim3(BLOCK), (BLOCK >> log_lanes) * sizeof(GradMeta), st, g,
                           static_cast<const IT*>(c.dout), c.in_ld, t.dim, log_lanes, c.scale, c.out);
        RAISE_HIP(hipGetLastError());
      }
      return PS_OK;
    });
  });
  if (r) return r;
  if (blocks < 3) return PS_OK;   // no run is longer than its block and the next
  const int col_slices = (int)div_up(t.dim, WAVE);
  const int64_t supers = blocks >> log_fold(blocks);
  if (supers > 1) {   // (the first is never folded)
    hipLaunchKernelGGL(k_grad_fold, dim3(std::min<int64_t>(supers * col_slices, 2048)), dim3(BLOCK), 0, st, g, (int)supers,
                       t.dim, col_slices, p.fold);
    RAISE_HIP(hipGetLastError());
  }
  hipLaunchKernelGGL(k_grad_finish, dim3(std::min<int64_t>(blocks * col_slices, 2048)), dim3(BLOCK), 0, st, g, t.dim, col_slices,
                     p.fold, c.scale, c.out);
  RAISE_HIP(hipGetLastError());
  return PS_OK;
}

}  // namespace

extern "C" {

size_t ps_embed_grad_workspace_bytes(int32_t dim, int64_t n) {
  if (dim < 1 || n < 1 || n > OCC_MAX) return 0;
  return plan_grad(nullptr, n, dim).bytes;
}

ps_status ps_embed_grad(ps_store* s, const int64_t* ids, int64_t n, int64_t pad, double scale, int32_t in_type,
                        const void* dout, int64_t dout_stride, int32_t out_type, void* grad, int64_t grad_stride,
                        int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  return embed_grad(s, GradCall{ids, n, pad, scale, in_type, dout, dout_stride,
                                GradOut{grad, grad_stride, out_type, accumulate != 0}, nullptr, nullptr},
                    ws, ws_bytes, static_cast<hipStream_t>(stream));
}

ps_status ps_embed_grad_rows(ps_store* s, const int64_t* ids, int64_t n, int64_t pad, double scale, int32_t in_type,
                             const void* dout, int64_t dout_stride, int32_t out_type, int64_t* uniq, void* rows,
                             int64_t rows_stride, int32_t* num_unique, void* ws, size_t ws_bytes, void* stream) {
  if (!num_unique) return raise(PS_ERR_INVALID, "num_unique is NULL");
  return embed_grad(s, GradCall{ids, n, pad, scale, in_type, dout, dout_stride,
                                GradOut{rows, rows_stride, out_type, 0}, uniq, num_unique},
                    ws, ws_bytes, static_cast<hipStream_t>(stream));
}

ps_status ps_wait_count(const int32_t* count, void* stream) {
  if (!count) return raise(PS_ERR_INVALID, "count is NULL");
  // The number is mostly there within some 100 us, and a nap ends up to 70 us late.  Behind a stream
  // that has much to do before the call, the processor is left to others.
  using clock = std::chrono::steady_clock;
  constexpr std::chrono::microseconds SPIN(2000), NAP(20);
  const auto there = [&] { return __atomic_load_n(count, __ATOMIC_ACQUIRE) >= 0; };
  const auto start = clock::now();
  while (!there()) {
    if (clock::now() - start < SPIN)
      for (int i = 0; i < 1024 && !there(); ++i) __builtin_ia32_pause();   // some 30 us between two looks at the stream
    else
      std::this_thread::sleep_for(NAP);
    if (there()) break;   // (to ask a stream takes some 20 us)
    const hipError_t e = hipStreamQuery(static_cast<hipStream_t>(stream));
    if (e == hipErrorNotReady) {
      (void)hipGetLastError();   // no error, and none that a later call should report
      continue;
    }
    RAISE_HIP(e);
    if (!there()) return raise(PS_ERR_INVALID, "the stream is through and count is still negative");
  }
  return PS_OK;
}

}  // extern "C"
