// Entry points of the microscaled 4-bit tables.
#include "mx4.hpp"

#include <algorithm>

#include "internal.hpp"
#include "lookup.hpp"
#include "rules.hpp"

using namespace adapm;

namespace {

constexpr int MX_DIM_MAX = 16384;

ps_status check_dim(int32_t dim) {
  if (dim < 1 || dim > MX_DIM_MAX) return raise(PS_ERR_UNSUPPORTED, "dim %d outside [1, %d]", dim, MX_DIM_MAX);
  return PS_OK;
}

ps_status check_type(int32_t type) {
  if (type != PS_F32 && type != PS_BF16 && type != PS_F16) return raise(PS_ERR_INVALID, "unknown element type %d", type);
  return PS_OK;
}

int blocks_of(int dim) { return (dim + MX_BLOCK - 1) / MX_BLOCK; }

}  // namespace

extern "C" {

ps_status ps_mx4_quantize(int64_t rows, int32_t dim, int32_t type, const void* x, int64_t row_stride, uint8_t* codes,
                          uint8_t* scales, void* stream) {
  if (rows < 0) return raise(PS_ERR_INVALID, "negative size %lld", (long long)rows);
  if (ps_status r = check_dim(dim)) return r;
  if (ps_status r = check_type(type)) return r;
  if (row_stride < dim) return raise(PS_ERR_INVALID, "row_stride %lld < dim %d", (long long)row_stride, dim);
  if (rows == 0) return PS_OK;
  if (!x || !codes || !scales) return raise(PS_ERR_INVALID, "x, codes or scales is NULL");
  const int b = type_bytes(type);
  if (!on_bytes(x, b)) return raise(PS_ERR_INVALID, "x is not aligned to its elements");
  if (!on_bytes(codes, 16)) return raise(PS_ERR_INVALID, "codes must be 16-byte aligned");
  const SmallDiv per_row = small_div((uint32_t)blocks_of(dim) * 4);
  if (rows > INT64_MAX / (4 * per_row.d)) return raise(PS_ERR_UNSUPPORTED, "%lld rows", (long long)rows);
  const int64_t grid = div_up(rows * per_row.d, BLOCK);
  if (grid > GRID_MAX) return raise(PS_ERR_UNSUPPORTED, "%lld rows of %d exceed the grid", (long long)rows, dim);
  return with_type(type, [&]<class T>(T) -> ps_status {
    auto kernel = rows * per_row.d * 4 > LOOKUP_STREAMS ? k_mx4_quantize<T, true> : k_mx4_quantize<T, false>;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(BLOCK), 0, static_cast<hipStream_t>(stream),
                       static_cast<const T*>(x), rows, dim, row_stride, per_row, reinterpret_cast<uint32_t*>(codes),
                       scales);
    RAISE_HIP(hipGetLastError());
    return PS_OK;
  });
}

ps_status ps_mx4_embed(const uint8_t* codes, const uint8_t* scales, int64_t num_rows, int32_t dim, const int64_t* ids,
                       int64_t n, int64_t pad, float scale, int32_t out_type, void* out, int64_t out_stride,
                       int32_t* err, void* stream) {
  if (num_rows < 0) return raise(PS_ERR_INVALID, "negative size %lld", (long long)num_rows);
  if (n < 0) return raise(PS_ERR_INVALID, "negative size %lld", (long long)n);
  if (ps_status r = check_dim(dim)) return r;
  if (ps_status r = check_type(out_type)) return r;
  if (out_stride < dim) return raise(PS_ERR_INVALID, "out_stride %lld < dim %d", (long long)out_stride, dim);
  if (!ids && n > num_rows) return raise(PS_ERR_INVALID, "%lld rows of a table of %lld", (long long)n, (long long)num_rows);
  if (n == 0) return PS_OK;
  if (!out || (num_rows > 0 && (!codes || !scales))) return raise(PS_ERR_INVALID, "codes, scales or out is NULL");
  if (ids && !err) return raise(PS_ERR_INVALID, "err is NULL");
  if (!on_bytes(codes, 16)) return raise(PS_ERR_INVALID, "codes must be 16-byte aligned");
  const int b = type_bytes(out_type);
  if (!on_bytes(out, b)) return raise(PS_ERR_INVALID, "out is not aligned to its elements");
  const SmallDiv nv = small_div((uint32_t)div_up(dim, 16 / b));
  if (n > INT64_MAX / (4 * nv.d)) return raise(PS_ERR_UNSUPPORTED, "%lld rows", (long long)n);
  const int64_t grid = div_up(n * nv.d, int64_t(BLOCK) * LOOKUP_FLIGHT);
  if (grid > GRID_MAX) return raise(PS_ERR_UNSUPPORTED, "%lld rows of %d exceed the grid", (long long)n, dim);
  const LookupIds l{ids, n, pad, num_rows, nullptr, 0, err};
  return with_type(out_type, [&]<class OT>(OT) -> ps_status {
    auto launch = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3(grid), dim3(BLOCK), 0, static_cast<hipStream_t>(stream),
                         codes, scales, blocks_of(dim), dim, l, nv, scale,
                         static_cast<OT*>(out), out_stride);
    };
    if (n * int64_t(dim) * b > LOOKUP_STREAMS) launch(k_mx4_embed<OT, true>);
    else launch(k_mx4_embed<OT, false>);
    RAISE_HIP(hipGetLastError());
    return PS_OK;
  });
}

ps_status ps_mx4_product(int64_t m, int64_t n, int32_t dim, const uint8_t* a_codes, const uint8_t* a_scales,
                         const uint8_t* b_codes, const uint8_t* b_scales, float scale, int32_t out_type, void* out,
                         int64_t out_stride, void* stream) {
  if (m < 0 || n < 0) return raise(PS_ERR_INVALID, "negative size %lld x %lld", (long long)m, (long long)n);
  if (ps_status r = check_dim(dim)) return r;
  if (ps_status r = check_type(out_type)) return r;
  if (out_stride < n) return raise(PS_ERR_INVALID, "out_stride %lld < %lld", (long long)out_stride, (long long)n);
  if (m == 0 || n == 0) return PS_OK;
  if (!a_codes || !a_scales || !b_codes || !b_scales || !out)
    return raise(PS_ERR_INVALID, "codes, scales or out is NULL");
  if (!on_bytes(a_codes, 16) || !on_bytes(b_codes, 16)) return raise(PS_ERR_INVALID, "codes must be 16-byte aligned");
  if (!on_bytes(out, type_bytes(out_type))) return raise(PS_ERR_INVALID, "out is not aligned to its elements");
  constexpr int64_t kRows = int64_t(1) << 40;
  if (m > kRows || n > kRows) return raise(PS_ERR_UNSUPPORTED, "%lld x %lld rows", (long long)m, (long long)n);
  const MxRows A{a_codes, a_scales, m}, B{b_codes, b_scales, n};
  return with_type(out_type, [&]<class OT>(OT) -> ps_status {
    auto launch = [&](auto kernel, int tile_q, int tile_t) -> ps_status {
      const int64_t tq = div_up(m, tile_q), tt = div_up(n, tile_t);
      if (tq > (GRID_MAX - NUM_XCD) / tt) return raise(PS_ERR_UNSUPPORTED, "%lld x %lld exceed the grid", (long long)m, (long long)n);
      hipLaunchKernelGGL(kernel, dim3(div_up(tq * tt, NUM_XCD) * NUM_XCD), dim3(BLOCK), 0,
                         static_cast<hipStream_t>(stream), A, B, blocks_of(dim),
                         scale, static_cast<OT*>(out), out_stride, (uint32_t)tq, (uint32_t)tt);
      RAISE_HIP(hipGetLastError());
      return PS_OK;
    };
    // past the caches where C fills the last-level one and its rows are whole lines
    // (1,024 x 65,536 in fp32 of dim 1,024 108 us through the caches, 77 past them;
    // rows that share lines, 2,048 x 50,021 in fp32 131 and 173)
    const int64_t bytes = m * n * (int64_t)sizeof(OT);
    const bool lines = on_bytes(out, 64) && out_stride * sizeof(OT) % 64 == 0, nt = bytes >= LLC_BYTES && lines;
    // few queries: 32 of them by 256 rows a workgroup. Both sides of the line, in
    // tiles of 32 and of 128 queries, us in fp32: 24 queries x 200,000 rows of 256 9.5
    // and 10.3, x 1M of 512 74 and 70; 48 queries 12.9 and 13.8, 94 and 89; 30,000 rows
    // of 1,024 8.2 and 7.9, 9.0 and 8.5
    if (m <= 32) {
      if (nt) return launch(k_mx4_product<OT, 1, 2, 1, 4, true>, 32, 256);
      return launch(k_mx4_product<OT, 1, 2, 1, 4, false>, 32, 256);
    }
    if (nt) return launch(k_mx4_product<OT, 2, 2, 2, 2, true>, 128, 128);
    // rows that share lines, many and long: wider tiles share fewer, and cost more
    // loads, which count where rows are wide (tiles of 128 x 128 and 64 x 256, us:
    // 2,048 x 100,043 in bf16 of dim 64, 300 and 512 130 and 106, 143 and 133, 149
    // and 148, 2,048 x 20,011 of 256 35 and 23, 256 x 300,003 in fp32 of 256 101 and
    // 91; but 2,048 x 50,021 in bf16 of 2,048 157 and 185, 200 x 100,003 in fp32 of
    // 128 17.4 and 18.2, 2,048 x 10,007 in bf16 of 64 12.7 and 13.7)
    if (!lines && bytes >= LLC_BYTES / 4 && m >= 256 && dim <= 512)
      return launch(k_mx4_product<OT, 2, 2, 1, 4, false>, 64, 256);
    return launch(k_mx4_product<OT, 2, 2, 2, 2, false>, 128, 128);
  });
}

}  // extern "C"
