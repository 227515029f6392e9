// The token table's lookup with scaling and its gradient by sorted tokens.
#pragma once

#include "elem.hpp"
#include "lookup.hpp"

namespace adapm {

// ------------------------------------------------------------------ lookup
//   out[i] = T( scale * W[ids[i]] ),   zero where ids[i] == pad
// (the product is rounded to fp32, then to T).  Bound by the rows read and
// written.  The rows are cut into vectors of VW elements and the vectors of
// the whole output dealt out in order, LOOKUP_FLIGHT in flight per thread: every
// lane has a vector whatever the row's width, a row of any width is spread
// over as many workgroups as it fills, and a workgroup writes one stretch.  A
// row that is no multiple of VW has its last vector end with the row, over some
// elements of the one before: both write the same.
template <class VT, class OT, int VW, bool NT>
__global__ __launch_bounds__(BLOCK) void k_embed(const VT* __restrict__ W, int64_t ld, LookupIds l, SmallDiv nv,
                                                 int dim, float scale, OT* __restrict__ out, int64_t out_ld) {
  constexpr int U = LOOKUP_FLIGHT;
  const int64_t q0 = (int64_t)blockIdx.x * (BLOCK * U);
  const int64_t row0 = row_of(q0, nv.d);
  const uint32_t first = (uint32_t)(q0 - row0 * nv.d) + threadIdx.x;
  int bad = 0, miss = 0;
  int64_t src[U], dst[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t x = first + u * BLOCK;
    const uint32_t dr = quotient(x, nv);
    const int at = (int)(x - dr * nv.d) * VW;
    const int c = at + VW <= dim ? at : dim - VW;
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
    if (src[u] >= 0) w[u] = load_any<VT, VW>(W + src[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (src[u] == -2) continue;
    float x[VW];
#pragma unroll
    for (int e = 0; e < VW; ++e) x[e] = src[u] < 0 ? 0.0f : scale * raw_get<VT, VW>(w[u], e);
    store_any<OT, VW, NT>(out + dst[u], raw_make<OT, VW>(x));
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
// The sorted positions are cut into blocks, one row group of
// lanes per block and column slice, so that the rows in flight do not depend
// on how long the runs are (most tokens of a batch come once or twice, the
// commonest thousands of times).  A run inside a block is written at once, and
// so is one that ends in the block after: the block where it starts takes it
// whole.  A longer run leaves one fp64 partial row per block: in the even slot
// of the block where it comes in from the block before or starts with the
// block, in the odd slot where it starts inside.  k_grad_fold adds the even
// slots of as many blocks (a power of two) as one run fills, k_grad_finish adds the rest.
constexpr int GRAD_BLOCK_MAX = 16;   // positions of a block: 16, or 8 in small calls

// Where a token's gradient row goes: row `key` of the dense form, or the
// run's index in the rows form (seg_off != NULL).
struct GradOut {
  void* p;
  int64_t ld;
  int32_t type;
  int32_t accumulate;
};

template <int VW>
__device__ __forceinline__ void write_row_any(const GradOut& o, int64_t row, int col, const float* x) {
  const int64_t at = row * o.ld + col;
  if (o.type == 0) store_any<float, VW>(static_cast<float*>(o.p) + at, raw_make<float, VW>(x));
  else if (o.type == 1) store_any<bf16_t, VW>(static_cast<bf16_t*>(o.p) + at, raw_make<bf16_t, VW>(x));
  else store_any<f16_t, VW>(static_cast<f16_t*>(o.p) + at, raw_make<f16_t, VW>(x));
}

template <class OT, int VW>
__device__ __forceinline__ void add_old(const GradOut& o, int64_t at, double* x) {
  const raw_t<OT, VW> old = load_any<OT, VW>(static_cast<const OT*>(o.p) + at);
#pragma unroll
  for (int e = 0; e < VW; ++e) x[e] += (double)raw_get<OT, VW>(old, e);
}

template <int VW>
__device__ __forceinline__ void write_grad_any(const GradOut& o, int64_t row, int col, const double* acc,
                                               double scale) {
  double x[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) x[e] = scale * acc[e];
  if (o.accumulate) {
    const int64_t at = row * o.ld + col;
    if (o.type == 0) add_old<float, VW>(o, at, x);
    else if (o.type == 1) add_old<bf16_t, VW>(o, at, x);
    else add_old<f16_t, VW>(o, at, x);
  }
  float y[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) y[e] = (float)x[e];
  write_row_any<VW>(o, row, col, y);
}

// The number of runs, for a host that reads it while the rows are being written.
__device__ __forceinline__ void write_count(int32_t* num_unique, int32_t u) {
  __hip_atomic_store(num_unique, u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
}

// The runs of the sorted keys, for the rows form of calls whose sort does not
// give them: tiles of RUNS_TILE positions count the runs that start in them;
// then every tile adds up the counts before its own and writes its runs' keys
// and first positions, and the run that each of its blocks starts in.
constexpr int RUNS_ITEMS = 16;
constexpr int RUNS_TILE = BLOCK * RUNS_ITEMS;

// The keys of a thread's positions and the bits of those that start a run.
__device__ __forceinline__ uint32_t run_heads(const uint32_t* __restrict__ keys, int64_t n, uint32_t sentinel,
                                              int64_t p, uint32_t (&k)[RUNS_ITEMS + 1]) {
  const uint32_t before = p > 0 && p <= n ? keys[p - 1] : 0xffffffffu;
#pragma unroll
  for (int i = 0; i <= RUNS_ITEMS; ++i) k[i] = p + i < n ? keys[p + i] : 0xffffffffu;
  uint32_t heads = 0;
#pragma unroll
  for (int i = 0; i < RUNS_ITEMS; ++i)
    heads |= (uint32_t)(k[i] < sentinel && (i ? k[i - 1] : before) != k[i]) << i;
  return heads;
}

__global__ __launch_bounds__(BLOCK) void k_runs_count(const uint32_t* __restrict__ keys, int64_t n, uint32_t sentinel,
                                                      uint32_t* __restrict__ tile_heads) {
  __shared__ uint32_t smem[WAVES_PER_BLOCK + 1];
  uint32_t k[RUNS_ITEMS + 1], total;
  const int64_t p = (int64_t)blockIdx.x * RUNS_TILE + threadIdx.x * RUNS_ITEMS;
  block_exclusive_scan(__popc(run_heads(keys, n, sentinel, p, k)), smem, &total);
  if (threadIdx.x == 0) tile_heads[blockIdx.x] = total;
}

// One workgroup: tile_heads becomes the runs before each tile (where there are
// so many tiles that adding them up in each would take longer).
__global__ __launch_bounds__(BLOCK) void k_runs_scan(uint32_t* __restrict__ tile_heads, int64_t tiles) {
  __shared__ uint32_t smem[WAVES_PER_BLOCK + 1];
  uint32_t carry = 0;
  for (int64_t t0 = 0; t0 < tiles; t0 += BLOCK) {
    const int64_t t = t0 + threadIdx.x;
    uint32_t total;
    const uint32_t before = block_exclusive_scan(t < tiles ? tile_heads[t] : 0u, smem, &total);
    if (t < tiles) tile_heads[t] = carry + before;
    carry += total;
  }
}

__global__ __launch_bounds__(BLOCK) void k_runs_write(const uint32_t* __restrict__ keys, int64_t n, uint32_t sentinel,
                                                      const uint32_t* __restrict__ tile_heads, int scanned, int log_block,
                                                      int64_t* __restrict__ uniq, int32_t* __restrict__ seg_off,
                                                      int32_t* __restrict__ block_run,
                                                      int32_t* __restrict__ num_unique) {
  __shared__ uint32_t smem[WAVES_PER_BLOCK + 1];
  uint32_t before = 0, total;
  if (scanned) {
    before = tile_heads[blockIdx.x];
  } else {
    for (int t = threadIdx.x; t < (int)blockIdx.x; t += BLOCK) before += tile_heads[t];
    block_exclusive_scan(before, smem, &total);
    before = total;
  }
  uint32_t k[RUNS_ITEMS + 1];
  const int64_t p = (int64_t)blockIdx.x * RUNS_TILE + threadIdx.x * RUNS_ITEMS;
  const uint32_t heads = run_heads(keys, n, sentinel, p, k);
  uint32_t u = before + block_exclusive_scan(__popc(heads), smem, &total);   // runs that start before position p + i
#pragma unroll
  for (int i = 0; i < RUNS_ITEMS; ++i) {
    const bool head = (heads >> i) & 1u;
    if (((p + i) & ((1 << log_block) - 1)) == 0 && p + i < n) block_run[(p + i) >> log_block] = (int32_t)(u + head) - 1;
    if (head) {
      uniq[u] = (int64_t)k[i];
      seg_off[u] = (int32_t)(p + i);
      ++u;
    }
    if (k[i] < sentinel && k[i + 1] >= sentinel) {   // the last position of the last run
      seg_off[u] = (int32_t)(p + i) + 1;
      write_count(num_unique, (int32_t)u);
    }
  }
  if (p == 0 && k[0] >= sentinel) write_count(num_unique, 0);
}

// Index of the run that holds sorted position p, the last u with
// seg_off[u] <= p, by the `lanes` lanes of a group together: each round they
// probe as many places, so that a million runs take four rounds of 32 lanes
// instead of twenty of one.
__device__ __forceinline__ int32_t run_at(const int32_t* seg_off, int32_t num_runs, int32_t p, int lanes, int gl) {
  int32_t lo = 0, len = num_runs;   // seg_off[lo] <= p < seg_off[lo + len]
  const int shift = lane_id() - gl;
  while (len > 1) {
    const int32_t step = (len + lanes - 1) / lanes;
    const int32_t at = (gl + 1) * step;
    const bool below = at < len && seg_off[lo + at] <= p;
    const uint64_t m = __ballot(below) >> shift;
    const int k = __popcll(lanes == WAVE ? m : m & ((1ull << lanes) - 1));
    lo += k * step;
    len = len - k * step < step ? len - k * step : step;
  }
  return lo;
}

struct GradRuns {
  const uint32_t* keys;    // sorted, `sentinel` and above last
  const uint32_t* perm;
  int64_t n;
  uint32_t sentinel;
  const int32_t* seg_off;  // rows form only
  const SegHeader* hdr;    // rows form, from the sort: the number of runs;
  const int32_t* block_run;  // or, from k_runs_write, the run of each block's first position
  int32_t* num_unique;     // rows form: receives the number of rows
  double* partial;         // [2 * blocks][dim]
  int log_block;           // positions of a block, and blocks folded together, as powers of two
  int log_fold;
  int4* split_list;        // the longer runs: first position, key, index of the run
  uint32_t* split_count;
};

// Keys and occurrences of a group's positions: its block, the one after and
// the key behind them.
struct alignas(16) GradMeta {
  uint32_t key[2 * GRAD_BLOCK_MAX + 4];
  uint32_t occ[2 * GRAD_BLOCK_MAX];
};

// All rows of a block are in flight at once and have arrived before the first
// sum is written: the vector memory counter retires loads and stores in their
// order, so a group that waited for a row behind a store would wait for the
// store.  The positions of a run taken whole beyond the block are a second such
// round.
template <class IT, int VW, int BLK>
__global__ __launch_bounds__(BLOCK) void k_grad_merge(GradRuns g, const IT* __restrict__ dout, int64_t in_ld, int dim,
                                                      int log_lanes, double scale, GradOut out) {
  constexpr int U = BLK;
  extern __shared__ GradMeta grad_meta[];   // one per group
  const int lanes = 1 << log_lanes;
  const int gl = threadIdx.x & (lanes - 1);
  const int64_t b = (int64_t)blockIdx.x * (BLOCK >> log_lanes) + (threadIdx.x >> log_lanes);
  const int slice = blockIdx.y;
  const int at = (slice * lanes + gl) * VW;
  const bool active = at < dim;
  const int col = at + VW <= dim ? at : dim - VW;   // the last vector ends with the row, as in k_embed
  const int64_t p0 = b * BLK;
  if (p0 >= g.n) return;
  const uint32_t before = p0 > 0 ? g.keys[p0 - 1] : 0xffffffffu;
  const uint32_t before2 = p0 > BLK ? g.keys[p0 - BLK - 1] : 0xffffffffu;
  int32_t u = g.block_run ? g.block_run[b] : 0;   // the run's index (rows form)
  GradMeta& m = grad_meta[threadIdx.x >> log_lanes];
  for (int i = gl; i <= 2 * BLK; i += lanes) m.key[i] = p0 + i < g.n ? g.keys[p0 + i] : 0xffffffffu;
  for (int i = gl; i < 2 * BLK; i += lanes) m.occ[i] = p0 + i < g.n ? g.perm[p0 + i] : 0u;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // a group's lanes are of one wave
  __builtin_amdgcn_wave_barrier();
  const int count = g.n - p0 < BLK ? (int)(g.n - p0) : BLK;
  const uint32_t first = m.key[0], last = m.key[count - 1], next = m.key[count];
  if (g.seg_off && !g.block_run) {
    if (b == 0 && slice == 0 && gl == 0) write_count(g.num_unique, (int32_t)g.hdr->num_unique);
    // (before the rows are asked for: behind them its loads would wait for them)
    u = run_at(g.seg_off, (int32_t)g.hdr->num_unique, (int32_t)p0, lanes, gl);
  }
  if (first >= g.sentinel) return;
  bool came_in = before == first;                                     // the run began in an earlier block
  const bool taken = came_in && before2 != first && next != first;    // which takes it whole
  const bool extend = count == BLK && next == last && !(came_in && last == first) &&
                      m.key[2 * BLK] != last;                         // as this block does its own last run
  const int stop = extend ? 2 * BLK : count;
  int start = 0;   // the run's first position here
  const IT* src = dout + col;
  double acc[VW];
#pragma unroll
  for (int e = 0; e < VW; ++e) acc[e] = 0.0;
  for (int p = 0; p < stop; p += U) {
    uint32_t k[U + 1], r[U];
#pragma unroll
    for (int i = 0; i < U; i += 4) {
      const words4 a = *reinterpret_cast<const words4*>(m.key + p + i);
      const words4 c = *reinterpret_cast<const words4*>(m.occ + p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) k[i + e] = a[e], r[i + e] = c[e];
    }
    k[U] = m.key[p + U];
    // every position's row, its own or not: an occurrence is a row of dout
    // (the first one stands for those beyond the last)
    raw_t<IT, VW> x[U];
#pragma unroll
    for (int i = 0; i < U; ++i) x[i] = load_any<IT, VW>(src + (int64_t)r[i] * in_ld);
    int mine = 0;   // positions that are this group's: the first of them
#pragma unroll
    for (int i = 0; i < U; ++i) mine += k[i] < g.sentinel && (p == 0 || k[i] == last) ? 1 : 0;
#pragma unroll
    for (int i = 0; i < U; ++i) asm volatile("" : "+v"(x[i]));
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (i >= mine) return;   // nothing of this group's follows
      const bool ends = k[i + 1] != k[i];
      if (ends && start == p + i && !came_in && !out.accumulate) {
        // a token that comes once: no sum
        float y[VW];
#pragma unroll
        for (int e = 0; e < VW; ++e) y[e] = (float)(scale * (double)raw_get<IT, VW>(x[i], e));
        if (active) write_row_any<VW>(out, g.seg_off ? (int64_t)u : (int64_t)k[i], col, y);
        start = p + i + 1;
        ++u;
        continue;
      }
#pragma unroll
      for (int e = 0; e < VW; ++e) acc[e] += (double)raw_get<IT, VW>(x[i], e);
      const bool leaves = !ends && p + i + 1 == count && !extend;
      if (!ends && !leaves) continue;
      if (taken && k[i] == first) {
      } else if (ends && !came_in) {
        if (active) write_grad_any<VW>(out, g.seg_off ? (int64_t)u : (int64_t)k[i], col, acc, scale);
      } else {
        if (active) {
          double* q = g.partial + (2 * b + (start != 0 ? 1 : 0)) * dim + col;
#pragma unroll
          for (int e = 0; e < VW; ++e) q[e] = acc[e];
        }
        if (leaves && !came_in && gl == 0 && slice == 0)
          g.split_list[atomicAdd(g.split_count, 1u)] = int4{(int)p0 + start, (int)k[i], u, 0};
      }
#pragma unroll
      for (int e = 0; e < VW; ++e) acc[e] = 0.0;
      came_in = false;
      start = p + i + 1;
      ++u;
    }
  }
}

// Adds rows row(k), k = 0 .. count-1, of fp64 column col: wave w of the
// workgroup the rows w, w + 4, ... in their order, SUM_FLIGHT of them in flight,
// then the waves' sums in wave order.  The time of a long run is that of a chain
// of loads, hence a workgroup for each (a wave each, and all waves on one run of
// few rows only where it is long: 400,000 ids of 16 floats over 1,000 rows 83
// and 71 us against 69, 300,000 of 64 over 50,000 96 and 88 against 84,
// 20,000 of 2,048 over 500, many runs of few rows, 55 and 59 against 55).
constexpr int SUM_FLIGHT = 8;

template <class RowAt>
__device__ __forceinline__ double sum_rows(RowAt row, int count, bool active, int col, double* smem) {
  const int w = threadIdx.x / WAVE;
  double acc = 0.0;
  for (int k = w; k < count; k += SUM_FLIGHT * WAVES_PER_BLOCK) {
    double x[SUM_FLIGHT];
#pragma unroll
    for (int f = 0; f < SUM_FLIGHT; ++f)
      x[f] = active && k + f * WAVES_PER_BLOCK < count ? row(k + f * WAVES_PER_BLOCK)[col] : 0.0;
#pragma unroll
    for (int f = 0; f < SUM_FLIGHT; ++f) acc += k + f * WAVES_PER_BLOCK < count ? x[f] : 0.0;
  }
  smem[threadIdx.x] = acc;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int i = 0; i < WAVES_PER_BLOCK; ++i) t += smem[i * WAVE + lane_id()];
  __syncthreads();
  return t;
}

// fold[s] = the even slots of blocks [s << g.log_fold, (s + 1) << g.log_fold)
// where one run comes into the first of them and into the last (so into all).
// One workgroup per 64 columns, here and below.
__global__ __launch_bounds__(BLOCK) void k_grad_fold(GradRuns g, int supers, int dim, int slices,
                                                     double* __restrict__ fold) {
  __shared__ double smem[BLOCK];
  for (uint32_t e = blockIdx.x; e < (uint32_t)supers * (uint32_t)slices; e += gridDim.x) {
    const uint32_t s = e / (uint32_t)slices;
    const int col = (int)(e - s * (uint32_t)slices) * WAVE + lane_id();
    const int64_t b0 = (int64_t)s << g.log_fold;
    if (b0 == 0) continue;
    const uint32_t key = g.keys[b0 << g.log_block];
    if (key >= g.sentinel || g.keys[(b0 << g.log_block) - 1] != key ||
        g.keys[(b0 + (1 << g.log_fold) - 1) << g.log_block] != key)
      continue;
    const double t =
        sum_rows([&](int k) { return g.partial + 2 * (b0 + k) * dim; }, 1 << g.log_fold, col < dim, col, smem);
    if (threadIdx.x < WAVE && col < dim) fold[(int64_t)s * dim + col] = t;
  }
}

// The last block that the run of `key`, which comes into block f, comes into,
// by the wave's lanes together as in run_at.
__device__ __forceinline__ int32_t last_block(const GradRuns& g, uint32_t key, int32_t f) {
  const int32_t blocks = (int32_t)((g.n + (1 << g.log_block) - 1) >> g.log_block);
  int32_t lo = f, len = blocks - f;   // it comes into lo, not into lo + len
  while (len > 1) {
    const int32_t step = (len + WAVE - 1) / WAVE;
    const int32_t at = (lane_id() + 1) * step;
    const int k = __popcll(__ballot(at < len && g.keys[(int64_t)(lo + at) << g.log_block] == key));
    lo += k * step;
    len = len - k * step < step ? len - k * step : step;
  }
  return lo;
}

// The runs over three blocks and more: partial of the first block, of the
// blocks up to the first folded ones, the folds, and the blocks after them.
__global__ __launch_bounds__(BLOCK) void k_grad_finish(GradRuns g, int dim, int slices,
                                                       const double* __restrict__ fold, double scale, GradOut out) {
  __shared__ double smem[BLOCK];
  const int64_t items = (int64_t)*g.split_count * slices;
  for (int64_t e = blockIdx.x; e < items; e += gridDim.x) {
    const int64_t r = items <= UINT32_MAX ? (int64_t)((uint32_t)e / (uint32_t)slices) : e / slices;
    const int col = (int)(e - r * slices) * WAVE + lane_id();
    const int4 run = g.split_list[r];
    const int32_t s0 = run.x;
    const uint32_t key = (uint32_t)run.y;
    const int32_t b0 = s0 >> g.log_block, f = b0 + 1;   // the blocks it comes into: f to l
    const int32_t l = g.seg_off ? (g.seg_off[run.z + 1] - 1) >> g.log_block : last_block(g, key, f);
    const int32_t sa = (f + (1 << g.log_fold) - 1) >> g.log_fold, sb = (l + 1) >> g.log_fold;   // folds [sa, sb)
    const int32_t nf = sb > sa ? sb - sa : 0;
    const int32_t n1 = nf ? (sa << g.log_fold) - f : l - f + 1;
    const int32_t n3 = nf ? l - (sb << g.log_fold) + 1 : 0;
    auto row = [&](int32_t k) -> const double* {
      int64_t slot;
      if (k == 0) slot = 2 * (int64_t)b0 + ((s0 & ((1 << g.log_block) - 1)) != 0 ? 1 : 0);
      else if (k <= n1) slot = 2 * (int64_t)(f + k - 1);
      else if (k <= n1 + nf) return fold + (int64_t)(sa + k - 1 - n1) * dim;
      else slot = 2 * (int64_t)((sb << g.log_fold) + k - 1 - n1 - nf);
      return g.partial + slot * dim;
    };
    const double t = sum_rows(row, 1 + n1 + nf + n3, col < dim, col, smem);
    if (threadIdx.x < WAVE && col < dim)
      write_grad_any<1>(out, g.seg_off ? (int64_t)run.z : (int64_t)key, col, &t, scale);
  }
}

// Zero rows: the dense form before its tokens' rows are written.  On the same
// stream as the rest: beside the sort (a second stream) or among the merge's
// workgroups (which then leave the rows with ids to it) the whole takes as long,
// 117 and 114 us against 114 for 32,768 ids x 1,024 over 65,536 rows, as the
// zeros (6.1 TB/s) and the merge both fill the memory.  A row is
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
