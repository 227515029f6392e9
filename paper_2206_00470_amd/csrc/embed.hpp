// The token table's lookup with scaling and its gradient by sorted tokens.
#pragma once

#include "elem.hpp"
#include "lookup.hpp"

namespace adapm {

// ------------------------------------------------------------------ lookup
//   out[i] = T( scale * W[ids[i]] ),   zero where ids[i] == pad
// (the product is rounded to fp32, then to T).  Bound by the rows read and
// written.  The rows are cut into vectors of VW elements and the vectors of
// the whole output dealt out in order, EMBED_FLIGHT in flight per thread: every
// lane has a vector whatever the row's width, a row of any width is spread
// over as many workgroups as it fills, and a workgroup writes one stretch.
template <class VT, class OT, int VW, bool NT>
__global__ __launch_bounds__(BLOCK) void k_embed(const VT* __restrict__ W, int64_t ld, LookupIds l, SmallDiv nv,
                                                 float scale, OT* __restrict__ out, int64_t out_ld) {
  constexpr int U = EMBED_FLIGHT;
  const int64_t q0 = (int64_t)blockIdx.x * (BLOCK * U);
  const int64_t row0 = q0 / nv.d;
  const uint32_t first = (uint32_t)(q0 - row0 * nv.d) + threadIdx.x;
  int bad = 0, miss = 0;
  int64_t src[U], dst[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t x = first + u * BLOCK;
    const uint32_t dr = quotient(x, nv);
    const uint32_t c = (x - dr * nv.d) * VW;
    const int64_t i = row0 + dr;
    src[u] = -2;   // nothing to write
    if (i < l.n) {
      const int64_t r = lookup_row(l, i, bad, miss);
      src[u] = r < 0 ? -1 : r * ld + c;
      dst[u] = i * out_ld + c;
    }
  }
  raw_t<VT, VW> w[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    w[u] = raw_t<VT, VW>{};
    if (src[u] >= 0) w[u] = load_raw<VT, VW>(W + src[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (src[u] == -2) continue;
    float x[VW];
#pragma unroll
    for (int e = 0; e < VW; ++e) x[e] = src[u] < 0 ? 0.0f : scale * raw_get<VT, VW>(w[u], e);
    store_raw<OT, VW, NT>(out + dst[u], raw_make<OT, VW>(x));
  }
  if (bad) atomicOr(l.err, 1);
  if (miss) atomicOr(l.err + 1, 1);
}

// ------------------------------------------------------------------ gradient
//   dW[v] = scale * sum of dout[i] over the i with ids[i] == v
// over the ids' stable sort: the occurrences of a token are a run of sorted
// positions, added in their order in fp64, scaled and rounded to fp32 and then
// to the gradient's type (rounding twice costs at most 2^-24 of the value more
// than rounding once).  No atomics: the sums have one order.
//
// The sorted positions are cut into blocks of GRAD_BLOCK, one row group of
// lanes per block and column slice, so that the rows in flight do not depend
// on how long the runs are (most tokens of a batch come once or twice, the
// commonest thousands of times).  A run inside a block is written at once.  A
// run over several blocks leaves one fp64 partial row per block: in the even
// slot of the block where it comes in from the block before or starts with the
// block, in the odd slot where it starts inside.  k_grad_fold adds the even
// slots of GRAD_FOLD blocks that one run fills, k_grad_finish adds the rest.
constexpr int GRAD_BLOCK = 32;
constexpr int GRAD_FOLD = 64;
constexpr int GRAD_FLIGHT = 8;   // rows in flight per group

// Where a token's gradient row goes: row `key` of the dense form, or the
// run's index in the rows form (seg_off != NULL).
struct GradOut {
  void* p;
  int64_t ld;
  int32_t type;
  int32_t accumulate;
};

template <class OT, int VW>
__device__ __forceinline__ void write_grad(const GradOut& o, int64_t row, int col, const double* acc, double scale) {
  OT* p = static_cast<OT*>(o.p) + row * o.ld + col;
  float x[VW];
  if (o.accumulate) {
    const raw_t<OT, VW> old = load_raw<OT, VW>(p);
#pragma unroll
    for (int e = 0; e < VW; ++e) x[e] = (float)((double)raw_get<OT, VW>(old, e) + scale * acc[e]);
  } else {
#pragma unroll
    for (int e = 0; e < VW; ++e) x[e] = (float)(scale * acc[e]);
  }
  store_raw<OT, VW>(p, raw_make<OT, VW>(x));
}

template <int VW>
__device__ __forceinline__ void write_grad_any(const GradOut& o, int64_t row, int col, const double* acc,
                                               double scale) {
  if (o.type == 0) write_grad<float, VW>(o, row, col, acc, scale);
  else if (o.type == 1) write_grad<bf16_t, VW>(o, row, col, acc, scale);
  else write_grad<f16_t, VW>(o, row, col, acc, scale);
}

// Index of the run that holds sorted position p: the last u with
// seg_off[u] <= p.
__device__ __forceinline__ int32_t run_at(const int32_t* seg_off, int32_t num_runs, int32_t p) {
  int32_t lo = 0, hi = num_runs;   // seg_off[lo] <= p < seg_off[hi]
  while (hi - lo > 1) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (seg_off[mid] <= p) lo = mid;
    else hi = mid;
  }
  return lo;
}

struct GradRuns {
  const uint32_t* keys;    // sorted, `sentinel` and above last
  const uint32_t* perm;
  int64_t n;
  uint32_t sentinel;
  const int32_t* seg_off;  // rows form only
  const SegHeader* hdr;
  int32_t* num_unique;     // rows form: receives the number of rows
  double* partial;         // [2 * blocks][dim]
  int32_t* split_list;     // first positions of the runs over several blocks
  uint32_t* split_count;
};

template <class IT, int VW>
__global__ __launch_bounds__(BLOCK) void k_grad_merge(GradRuns g, const IT* __restrict__ dout, int64_t in_ld, int dim,
                                                      int lanes, int slices, double scale, GradOut out) {
  constexpr int U = GRAD_FLIGHT;
  const int64_t group = (int64_t)blockIdx.x * (BLOCK / lanes) + threadIdx.x / lanes;
  const int gl = threadIdx.x & (lanes - 1);
  const int64_t b = group / slices;
  const int slice = (int)(group - b * slices);
  const int col = (slice * lanes + gl) * VW;
  if (g.seg_off && group == 0 && gl == 0) *g.num_unique = (int32_t)g.hdr->num_unique;
  const int64_t p0 = b * GRAD_BLOCK;
  if (p0 >= g.n) return;
  const int64_t p1 = p0 + GRAD_BLOCK < g.n ? p0 + GRAD_BLOCK : g.n;
  uint32_t key = g.keys[p0];
  if (key >= g.sentinel) return;
  bool came_in = p0 > 0 && g.keys[p0 - 1] == key;   // the run began in an earlier block
  int64_t start = p0;                               // the run's first position here
  int64_t u = g.seg_off ? run_at(g.seg_off, (int32_t)g.hdr->num_unique, (int32_t)p0) : 0;
  const bool active = col < dim;
  double acc[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) acc[e] = 0.0;
  for (int64_t p = p0; p < p1; p += U) {
    uint32_t k[U + 1], r[U];
#pragma unroll
    for (int i = 0; i <= U; ++i) k[i] = p + i < g.n ? g.keys[p + i] : 0xffffffffu;
#pragma unroll
    for (int i = 0; i < U; ++i) r[i] = p + i < g.n ? g.perm[p + i] : 0u;
    raw_t<IT, VW> x[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      x[i] = raw_t<IT, VW>{};
      if (active && k[i] < g.sentinel) x[i] = load_raw<IT, VW>(dout + (int64_t)r[i] * in_ld + col);
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (k[i] >= g.sentinel) return;   // the rest are too, and the last run has been written
#pragma unroll
      for (int e = 0; e < VW; ++e) acc[e] += (double)raw_get<IT, VW>(x[i], e);
      const bool ends = k[i + 1] != k[i];
      const bool leaves = !ends && p + i + 1 == p1;
      if (!ends && !leaves) continue;
      if (ends && !came_in) {
        if (active) write_grad_any<VW>(out, g.seg_off ? u : (int64_t)k[i], col, acc, scale);
      } else {
        if (active) {
          double* q = g.partial + (2 * b + (start != p0 ? 1 : 0)) * dim + col;
#pragma unroll
          for (int e = 0; e < VW; ++e) q[e] = acc[e];
        }
        if (leaves && !came_in && gl == 0 && slice == 0)
          g.split_list[atomicAdd(g.split_count, 1u)] = (int32_t)start;
      }
#pragma unroll
      for (int e = 0; e < VW; ++e) acc[e] = 0.0;
      came_in = false;
      start = p + i + 1;
      ++u;
    }
  }
}

// Adds rows row(k), k = 0 .. count-1, of fp64 columns col, by the block's
// four waves (wave w the rows w, w + 4, ..., FU in flight, then the waves'
// sums in wave order); the total is valid in wave 0.
template <class RowAt>
__device__ __forceinline__ double sum_rows_by_waves(RowAt row, int64_t count, bool active, int col, double* smem) {
  constexpr int FU = 8;
  const int w = threadIdx.x / WAVE;
  double acc = 0.0;
  int64_t k = w;
  for (; k + (FU - 1) * WAVES_PER_BLOCK < count; k += FU * WAVES_PER_BLOCK) {
    double x[FU];
#pragma unroll
    for (int f = 0; f < FU; ++f) x[f] = active ? row(k + f * WAVES_PER_BLOCK)[col] : 0.0;
#pragma unroll
    for (int f = 0; f < FU; ++f) acc += x[f];
  }
  for (; k < count; k += WAVES_PER_BLOCK) acc += active ? row(k)[col] : 0.0;
  smem[threadIdx.x] = acc;
  __syncthreads();
  double t = 0.0;
  if (w == 0)
#pragma unroll
    for (int i = 0; i < WAVES_PER_BLOCK; ++i) t += smem[i * WAVE + lane_id()];
  __syncthreads();
  return t;
}

// fold[s] = the even slots of blocks [s * GRAD_FOLD, (s + 1) * GRAD_FOLD)
// where one run comes into the first of them and into the last (so into all).
__global__ __launch_bounds__(BLOCK) void k_grad_fold(GradRuns g, int64_t supers, int dim, int slices,
                                                     double* __restrict__ fold) {
  __shared__ double smem[BLOCK];
  for (int64_t e = blockIdx.x; e < supers * slices; e += gridDim.x) {
    const int64_t s = e / slices;
    const int col = (int)(e - s * slices) * WAVE + lane_id();
    const int64_t b0 = s * GRAD_FOLD;
    if (b0 == 0) continue;
    const uint32_t key = g.keys[b0 * GRAD_BLOCK];   // uniform over the block, as what follows
    if (key >= g.sentinel || g.keys[b0 * GRAD_BLOCK - 1] != key ||
        g.keys[(b0 + GRAD_FOLD - 1) * GRAD_BLOCK] != key)
      continue;
    const double t = sum_rows_by_waves([&](int64_t k) { return g.partial + 2 * (b0 + k) * dim; }, GRAD_FOLD,
                                       col < dim, col, smem);
    if (threadIdx.x < WAVE && col < dim) fold[s * dim + col] = t;
  }
}

// The runs over several blocks: partial of the first block, of the blocks up
// to the first folded ones, the folds, and the blocks after them, added in
// this order by sum_rows_by_waves.
__global__ __launch_bounds__(BLOCK) void k_grad_finish(GradRuns g, int dim, int slices,
                                                       const double* __restrict__ fold, double scale, GradOut out) {
  __shared__ double smem[BLOCK];
  const int64_t items = (int64_t)*g.split_count * slices;
  for (int64_t e = blockIdx.x; e < items; e += gridDim.x) {
    const int64_t r = e / slices;
    const int col = (int)(e - r * slices) * WAVE + lane_id();
    const int64_t s0 = g.split_list[r];
    const uint32_t key = g.keys[s0];
    int64_t u = key, s1;
    if (g.seg_off) {
      u = run_at(g.seg_off, (int32_t)g.hdr->num_unique, (int32_t)s0);
      s1 = g.seg_off[u + 1];
    } else {   // the first position with a larger key
      int64_t lo = s0, hi = g.n;
      while (hi - lo > 1) {
        const int64_t mid = lo + (hi - lo) / 2;
        if (g.keys[mid] <= key) lo = mid;
        else hi = mid;
      }
      s1 = hi;
    }
    const int64_t f = s0 / GRAD_BLOCK + 1, l = (s1 - 1) / GRAD_BLOCK;   // blocks it comes into
    const int64_t sa = (f + GRAD_FOLD - 1) / GRAD_FOLD, sb = (l + 1) / GRAD_FOLD;
    const int64_t nf = sb > sa ? sb - sa : 0;
    const int64_t n1 = nf ? sa * GRAD_FOLD - f : l - f + 1;
    const int64_t n3 = nf ? l - sb * GRAD_FOLD + 1 : 0;
    auto row = [&](int64_t k) -> const double* {
      if (k == 0) return g.partial + (2 * (s0 / GRAD_BLOCK) + (s0 % GRAD_BLOCK != 0 ? 1 : 0)) * dim;
      if (k <= n1) return g.partial + 2 * (f + k - 1) * dim;
      if (k <= n1 + nf) return fold + (sa + k - 1 - n1) * dim;
      return g.partial + 2 * (sb * GRAD_FOLD + k - 1 - n1 - nf) * dim;
    };
    const double t = sum_rows_by_waves(row, 1 + n1 + nf + n3, col < dim, col, smem);
    if (threadIdx.x < WAVE && col < dim) write_grad_any<1>(out, u, col, &t, scale);
  }
}

// Zero rows: the dense form before its tokens' rows are written.  A row is
// `halves` 16-bit words, stored `vec` at a time (8, 2 or 1).
__global__ __launch_bounds__(BLOCK) void k_grad_clear(uint16_t* __restrict__ p, int64_t rows, int64_t halves,
                                                      int64_t ld_halves, int vec) {
  const int64_t per = halves / vec;
  const int64_t total = rows * per;
  for (int64_t i = (int64_t)blockIdx.x * BLOCK + threadIdx.x; i < total; i += (int64_t)gridDim.x * BLOCK) {
    const int64_t r = per == total ? 0 : i / per;
    uint16_t* q = p + r * ld_halves + (i - r * per) * vec;
    if (vec == 8) *reinterpret_cast<words4*>(q) = words4{0u, 0u, 0u, 0u};
    else if (vec == 2) *reinterpret_cast<uint32_t*>(q) = 0u;
    else *q = 0;
  }
}

}  // namespace adapm
