// Tables in microscaled 4-bit floating point: quantisation, lookup, and the
// product of two of them.
//
// A row of `dim` values is cut into blocks of 32 (the last filled up with
// zeros).  A block holds 32 codes of sign, two exponent bits and one mantissa
// bit (0, 0.5, 1, 1.5, 2, 3, 4, 6), two to a byte, the first in the low half,
// and one scale byte s for 2^(s - 127), s = 255 for a block that is NaN:
//   s    = max(0, floor(log2 max|x|) - 2 + 127)
//   code = x / 2^(s - 127) to the nearest, ties to the even code, at most 6
// Codes are row-major, 16 bytes a block, scales one byte a block.
#pragma once

#include "elem.hpp"
#include "lookup.hpp"

namespace adapm {

constexpr int MX_BLOCK = 32;
constexpr int MX_BYTES = 16;      // of codes per block

// 2^(s - 127) as a float; s = 0 is subnormal, s = 255 NaN.
__device__ __forceinline__ float scale_value(uint32_t s) {
  return __builtin_bit_cast(float, s == 0 ? 0x00400000u : s == 255 ? 0x7fc00000u : s << 23);
}

// ------------------------------------------------------------------ quantisation
// Bound by the values read.  Four lanes share a block, eight values each: the
// block's largest magnitude takes two exchanges inside the four, the eight
// codes are one word.  Magnitudes are compared as integers (the bits of a
// float without its sign order like its value, infinities and NaN last).
constexpr int QUANT_FLIGHT = 2;

template <class T, bool VEC>
__global__ __launch_bounds__(BLOCK) void k_mx4_quantize(const T* __restrict__ x, int64_t rows, int dim, int64_t ld,
                                                        SmallDiv per_row, uint32_t* __restrict__ codes,
                                                        uint8_t* __restrict__ scales) {
  constexpr int U = QUANT_FLIGHT;
  const int64_t q0 = (int64_t)blockIdx.x * (BLOCK * U);
  const int64_t row0 = q0 / per_row.d;
  const uint32_t first = (uint32_t)(q0 - row0 * per_row.d) + threadIdx.x;
  float v[U][8];
  int64_t row[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t a = first + u * BLOCK;
    const uint32_t dr = quotient(a, per_row);
    const int c = (int)(a - dr * per_row.d) * 8;
    row[u] = row0 + dr;
    const T* p = x + row[u] * ld + c;
    const bool in = row[u] < rows;
    if constexpr (VEC) {   // rows are whole vectors of eight
      raw_t<T, 8> w{};
      if (in && c < dim) w = load_raw<T, 8>(p);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] = raw_get<T, 8>(w, e);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[u][e] = in && c + e < dim ? raw_get<T, 1>(load_raw<T, 1>(p + e), 0) : 0.0f;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t b = __builtin_bit_cast(uint32_t, v[u][e]) & 0x7fffffffu;
      m = m > b ? m : b;
    }
    const uint32_t m1 = lane_xor_word<1>(m);
    m = m > m1 ? m : m1;
    const uint32_t m2 = lane_xor_word<2>(m);
    m = m > m2 ? m : m2;
    const uint32_t top = m >> 23;   // floor(log2 max|x|) + 127, or 0 where that is below -126
    const uint32_t s = top == 255 ? 255u : top > 2 ? top - 2 : 0u;
    // x 2^(127 - s) is exact: a value that leaves the normal range is below
    // half the smallest code
    const float inv = __builtin_bit_cast(float, (254u - (s == 255 ? 127u : s)) << 23);
    uint32_t word = 0;
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][0] * inv, v[u][1] * inv, 1.0f, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][2] * inv, v[u][3] * inv, 1.0f, 1);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][4] * inv, v[u][5] * inv, 1.0f, 2);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][6] * inv, v[u][7] * inv, 1.0f, 3);
    if (s == 255) word = 0;
    if (row[u] >= rows) continue;
    const int64_t q = q0 + threadIdx.x + u * BLOCK;
    codes[q] = word;
    if ((q & 3) == 0) scales[q >> 2] = (uint8_t)s;
  }
}

// ------------------------------------------------------------------ lookup
// As k_embed over quantised rows, eight codes (one word) of a row per vector
// and stores of VW elements; ids NULL restores the whole table.
template <class OT, int VW>
__global__ __launch_bounds__(BLOCK) void k_mx4_embed(const uint32_t* __restrict__ codes,
                                                     const uint8_t* __restrict__ scales, int blocks_row, int dim,
                                                     LookupIds l, SmallDiv nv, float scale, OT* __restrict__ out,
                                                     int64_t out_ld) {
  constexpr int U = EMBED_FLIGHT;
  const int64_t q0 = (int64_t)blockIdx.x * (BLOCK * U);
  const int64_t row0 = q0 / nv.d;
  const uint32_t first = (uint32_t)(q0 - row0 * nv.d) + threadIdx.x;
  int bad = 0, miss = 0;
  uint32_t w[U], s[U];
  int64_t at[U];
  int col[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t x = first + u * BLOCK;
    const uint32_t dr = quotient(x, nv);
    const uint32_t c = x - dr * nv.d;   // word of the row
    const int64_t i = row0 + dr;
    col[u] = dim;   // nothing to write
    w[u] = 0;
    s[u] = 0;
    if (i < l.n) {
      col[u] = (int)c * 8;
      at[u] = i * out_ld + col[u];
      const int64_t r = lookup_row(l, i, bad, miss);
      if (r >= 0) {
        w[u] = codes[r * blocks_row * 4 + c];
        s[u] = scales[r * blocks_row + (c >> 2)];
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (col[u] >= dim) continue;
    const float f = scale_value(s[u]);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // the magnitude's bits below an exponent of zero are its value / 2^126
      const uint32_t m = (w[u] >> (4 * e)) & 7u, sign = (w[u] >> (4 * e + 3)) << 31;
      x[e] = __builtin_bit_cast(float, m << 22 | sign) * 0x1p126f * f * scale;
    }
    const int left = dim - col[u];
#pragma unroll
    for (int e = 0; e < 8; e += VW) {
      if (e < left) store_raw<OT, VW>(out + at[u] + e, raw_make<OT, VW>(x + e));
    }
  }
  if (bad) atomicOr(l.err, 1);
}

// ------------------------------------------------------------------ product
//   C[i][j] = T( scale * sum_k A[i][k] B[j][k] ),  A [m][dim], B [n][dim]
// on the block-scaled matrix instruction of 32 x 32 x 64: lane l of a wave
// gives block l / 32 of row l % 32 of each operand, 32 codes and their scale;
// the products are exact and summed in fp32.  The sum over k has no order, so
// a lane takes neighbouring blocks of its row.  B's rows run along the lanes of the result (column l % 32), so that stores of
// one register are 32 neighbouring elements of a row of C.
//
// Bound by C's bytes where there are many queries (a table's width is a few
// hundred), by B's where there are few.
typedef int mx_operand __attribute__((ext_vector_type(8)));
typedef float mx_acc __attribute__((ext_vector_type(16)));

struct MxRows {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t rows;
};

// The codes and scale of block kb of a row, zeros outside.
__device__ __forceinline__ void mx_load(const MxRows& t, int64_t row, int kb, int blocks_row, words4& c, int& s) {
  c = words4{0u, 0u, 0u, 0u};
  s = 127;
  if (row < t.rows && kb < blocks_row) {
    c = *reinterpret_cast<const words4*>(t.codes + (row * blocks_row + kb) * MX_BYTES);
    s = t.scales[row * blocks_row + kb];
  }
}

__device__ __forceinline__ mx_operand mx_words(const words4& c) {
  return mx_operand{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};
}

// A wave's tile: MT x 32 rows of A by NTL x 32 rows of B; a workgroup's waves
// are WM x WN such tiles.
template <class OT, int MT, int NTL, int WM, int WN>
__global__ __launch_bounds__(BLOCK) void k_mx4_product(MxRows A, MxRows B, int blocks_row, float scale,
                                                       OT* __restrict__ C, int64_t ldc, int64_t tiles_n) {
  static_assert(WM * WN == WAVES_PER_BLOCK, "four waves");
  const int w = threadIdx.x / WAVE, l = lane_id();
  const int64_t tm = blockIdx.x / tiles_n, tn = blockIdx.x - tm * tiles_n;
  const int64_t i0 = (tm * WM + w / WN) * (MT * 32), j0 = (tn * WN + w % WN) * (NTL * 32);
  const int half = l / 32, r = l % 32;
  mx_acc acc[MT][NTL];
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int b = 0; b < NTL; ++b)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[a][b][e] = 0.0f;
  for (int k0 = 0; k0 < blocks_row; k0 += 2) {
    const int kb = k0 + half;
    words4 ca[MT], cb[NTL];
    int sa[MT], sb[NTL];
#pragma unroll
    for (int a = 0; a < MT; ++a) mx_load(A, i0 + a * 32 + r, kb, blocks_row, ca[a], sa[a]);
#pragma unroll
    for (int b = 0; b < NTL; ++b) mx_load(B, j0 + b * 32 + r, kb, blocks_row, cb[b], sb[b]);
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
      for (int b = 0; b < NTL; ++b)
        acc[a][b] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_words(ca[a]), mx_words(cb[b]), acc[a][b], 4, 4,
                                                                   0, sa[a], 0, sb[b]);
  }
#pragma unroll
  for (int a = 0; a < MT; ++a)
#pragma unroll
    for (int b = 0; b < NTL; ++b) {
      const int64_t j = j0 + b * 32 + r;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int64_t i = i0 + a * 32 + 8 * (e / 4) + 4 * half + e % 4;
        const float x = scale * acc[a][b][e];
        if (i < A.rows && j < B.rows) store_raw<OT, 1>(C + i * ldc + j, raw_make<OT, 1>(&x));
      }
    }
}

}  // namespace adapm
