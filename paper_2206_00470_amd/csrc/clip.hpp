// The global norm of the gradients of many tensors, and clipping by it.
//   norm = sqrt( sum over tensors and elements of g^2 )
//   out  = T( coef * g ),   coef = max_norm / norm where norm > max_norm, else 1
// A norm that is NaN gives NaN everywhere, an infinite one coef = 0.
// Squares and their sum are fp64, so that no finite fp32 gradient overflows or
// vanishes in them; coef and the product are rounded to fp32, then to T.
// A coef that fp32 holds as a subnormal only is applied in two factors, the
// first a power of two, so that it keeps its 24 bits.
//
// The tensors are cut into chunks of CLIP_CHUNK elements and the chunks of all
// of them dealt out over one grid.  A plan has a list of its chunks in device
// memory: one launch for the norm and one for the scaling, however many tensors
// there are.  A call without a plan carries its tensors' addresses in the
// launches' arguments, CLIP_TENSORS at a time: nothing is copied to the device
// (a plan's call and one of ps_clip_grads, us: 397 tensors of 26,610 floats in all
// 45 and 45, of 10.6M floats 44 and 66, 291 of 500M bf16 values 511 and 523; from
// Python the latter also checks each tensor anew, 427, 409 and 527).
// Each workgroup of the norm leaves one
// partial sum; each workgroup of the scaling adds all of them up again by
// itself, in one order, instead of waiting for another launch to do so.
#pragma once

#include "elem.hpp"

namespace adapm {

constexpr int CLIP_TENSORS = 128;
constexpr int64_t CLIP_CHUNK = 16384;
constexpr int64_t CLIP_GRID = 768;   // workgroups of a launch, at most: three a compute unit

// A part of a tensor.
struct ClipChunk {
  const void* in;
  void* out;
  uint32_t count;   // elements
  uint32_t type;
};

struct ChunkList {
  const ClipChunk* list;
  uint32_t n;
  __device__ __forceinline__ uint32_t chunks() const { return n; }
  __device__ __forceinline__ ClipChunk at(uint32_t c) const { return list[c]; }
};

struct TensorList {
  const void* in[CLIP_TENSORS];
  void* out[CLIP_TENSORS];
  int64_t numel[CLIP_TENSORS];
  uint32_t first[CLIP_TENSORS + 1];   // first chunk of each tensor; the last entry: chunks in all
  uint8_t type[CLIP_TENSORS];
  int32_t count;
  __device__ __forceinline__ uint32_t chunks() const { return first[count]; }
  __device__ __forceinline__ ClipChunk at(uint32_t c) const {   // (uniform over the workgroup)
    int k = 0, hi = count;   // first[k] <= c < first[hi]
    while (hi - k > 1) {
      const int mid = (k + hi) / 2;
      if (first[mid] <= c) k = mid;
      else hi = mid;
    }
    const int64_t i0 = (int64_t)(c - first[k]) * CLIP_CHUNK, left = numel[k] - i0;
    const int64_t byte = i0 * (type[k] == 0 ? 4 : 2);
    return ClipChunk{static_cast<const char*>(in[k]) + byte, static_cast<char*>(out[k]) + byte,
                     (uint32_t)(left < CLIP_CHUNK ? left : CLIP_CHUNK), type[k]};
  }
};

// f(p, n) over the elements [i0, i1) of a tensor: VW at a time from the first
// address that is aligned for them, the rest one by one.
template <class T, class Vec, class One>
__device__ __forceinline__ void over_elements(const T* p, int64_t count, Vec&& vec, One&& one) {
  constexpr int VW = 16 / sizeof(T);
  const int64_t head = ((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / sizeof(T);
  const int64_t h = head < count ? head : count;
  if ((int64_t)threadIdx.x < h) one(threadIdx.x);
  const int64_t nv = (count - h) / VW;
  constexpr int U = 4;
  int64_t v = threadIdx.x;
  for (; v + (U - 1) * BLOCK < nv; v += U * BLOCK) vec.template operator()<U>(h + v * VW, BLOCK * VW);
  for (; v < nv; v += BLOCK) vec.template operator()<1>(h + v * VW, 0);
  const int64_t tail = h + nv * VW + threadIdx.x;
  if (tail < count) one(tail);
}

template <class T>
__device__ __forceinline__ double chunk_squares(const T* p, int64_t count) {
  constexpr int VW = 16 / sizeof(T);
  double s0 = 0.0, s1 = 0.0;
  over_elements(
      p, count,
      [&]<int U>(int64_t i, int64_t step) {
        raw_t<T, VW> w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = load_raw<T, VW>(p + i + u * step);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int e = 0; e < VW; e += 2) {
            const double a = raw_get<T, VW>(w[u], e), b = raw_get<T, VW>(w[u], e + 1);
            s0 = __builtin_fma(a, a, s0);
            s1 = __builtin_fma(b, b, s1);
          }
      },
      [&](int64_t i) {
        const double a = raw_get<T, 1>(load_raw<T, 1>(p + i), 0);
        s0 = __builtin_fma(a, a, s0);
      });
  return s0 + s1;
}

template <class List>
__global__ __launch_bounds__(BLOCK) void k_norm_part(const List t, double* __restrict__ part) {
  __shared__ double smem[WAVES_PER_BLOCK];
  double s = 0.0;
  const uint32_t chunks = t.chunks();
  for (uint32_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const ClipChunk x = t.at(c);
    if (x.type == 0) s += chunk_squares(static_cast<const float*>(x.in), x.count);
    else if (x.type == 1) s += chunk_squares(static_cast<const bf16_t*>(x.in), x.count);
    else s += chunk_squares(static_cast<const f16_t*>(x.in), x.count);
  }
  s = block_sum_double(s, smem);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The norm from the partial sums, the same in every workgroup (in thread 0).
__device__ __forceinline__ double total_norm(const double* __restrict__ part, int64_t parts, double* smem) {
  double s = 0.0;
  int64_t i = threadIdx.x;
  for (; i + 3 * BLOCK < parts; i += 4 * BLOCK) {
    double x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = part[i + k * BLOCK];
#pragma unroll
    for (int k = 0; k < 4; ++k) s += x[k];
  }
  for (; i < parts; i += BLOCK) s += part[i];
  return __builtin_sqrt(block_sum_double(s, smem));
}

__global__ __launch_bounds__(BLOCK) void k_norm_total(const double* __restrict__ part, int64_t parts,
                                                      double* __restrict__ norm) {
  __shared__ double smem[WAVES_PER_BLOCK];
  const double t = total_norm(part, parts, smem);
  if (threadIdx.x == 0) *norm = t;
}

struct Coef {
  float unit;   // 1, or 2^-100 where the factor is below it
  float c;      // (1 too where a factor just below 2^-100 is rounded to it)
  __device__ __forceinline__ bool is_one() const { return unit == 1.0f && c == 1.0f; }
  __device__ __forceinline__ float operator()(float x) const { return x * unit * c; }
};

__device__ __forceinline__ Coef coef_of(double norm, double max_norm) {
  if (norm <= max_norm) return Coef{1.0f, 1.0f};
  const double c = max_norm / norm;   // NaN where the norm is
  if (c < 0x1p-100) return Coef{0x1p-100f, (float)(c * 0x1p100)};
  return Coef{1.0f, (float)c};
}

template <class T, bool NT>
__device__ __forceinline__ void chunk_scale(const T* p, T* o, int64_t count, Coef coef) {
  constexpr int VW = 16 / sizeof(T);
  // out may be aligned otherwise than in: then one element at a time
  const bool vec = ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(o)) & 15) == 0;
  auto one = [&](int64_t i) {
    const float x = coef(raw_get<T, 1>(load_raw<T, 1>(p + i), 0));
    store_raw<T, 1>(o + i, raw_make<T, 1>(&x));
  };
  if (!vec) {
    for (int64_t i = threadIdx.x; i < count; i += BLOCK) one(i);
    return;
  }
  over_elements(
      p, count,
      [&]<int U>(int64_t i, int64_t step) {
        raw_t<T, VW> w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = load_raw<T, VW>(p + i + u * step);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float x[VW];
#pragma unroll
          for (int e = 0; e < VW; ++e) x[e] = coef(raw_get<T, VW>(w[u], e));
          store_raw<T, VW, NT>(o + i + u * step, raw_make<T, VW>(x));
        }
      },
      one);
}

// The chunks go from the last to the first: the ones read last for the norm are
// still in the last-level cache.  NT (large outputs that are not their inputs)
// writes past the caches.  Measured without a plan, 500M bf16 values in 291 tensors: 567 us
// through the caches, 528 past them (174 of it the norm, 5.7 TB/s read; 5.6 TB/s
// read and written by the rest), 536 in the norm's order; 200M fp32 in 400 481,
// 444 and 450; in place 571 (556 by a plan; 581 and, in the norm's order, 590 when
// both were timed).
template <bool NT, class List>
__global__ __launch_bounds__(BLOCK) void k_clip_scale(const List t, const double* __restrict__ part, int64_t parts,
                                                      double max_norm, double* __restrict__ norm) {
  __shared__ double smem[WAVES_PER_BLOCK];
  __shared__ double norm_sh;
  const double nm = total_norm(part, parts, smem);
  if (threadIdx.x == 0) {
    norm_sh = nm;
    if (blockIdx.x == 0 && norm) *norm = nm;
  }
  __syncthreads();
  const Coef coef = coef_of(norm_sh, max_norm);
  const uint32_t chunks = t.chunks();
  for (uint32_t q = blockIdx.x; q < chunks; q += gridDim.x) {
    const ClipChunk x = t.at(chunks - 1 - q);
    if (coef.is_one() && x.in == x.out) continue;   // in place, and within the bound
    if (x.type == 0) chunk_scale<float, NT>(static_cast<const float*>(x.in), static_cast<float*>(x.out), x.count, coef);
    else if (x.type == 1)
      chunk_scale<bf16_t, NT>(static_cast<const bf16_t*>(x.in), static_cast<bf16_t*>(x.out), x.count, coef);
    else chunk_scale<f16_t, NT>(static_cast<const f16_t*>(x.in), static_cast<f16_t*>(x.out), x.count, coef);
  }
}

}  // namespace adapm
