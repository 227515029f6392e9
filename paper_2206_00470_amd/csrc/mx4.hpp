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
// One vector a thread, as one of fp32 is two loads; NT writes the codes past the
// caches (LOOKUP_STREAMS).  Measured, 4.6M x 256 fp32 values: two vectors a
// thread 992 us, one 933, with NT 889 (6.0 TB/s); 1M x 301 bf16 values 198 and 196,
// 400,000 x 1,024 174 and 181.
template <class T, bool NT>
__global__ __launch_bounds__(BLOCK) void k_mx4_quantize(const T* __restrict__ x, int64_t rows, int dim, int64_t ld,
                                                        SmallDiv per_row, uint32_t* __restrict__ codes,
                                                        uint8_t* __restrict__ scales) {
  const int64_t q0 = (int64_t)blockIdx.x * BLOCK;
  const int64_t row0 = row_of(q0, per_row.d);
  const uint32_t a = (uint32_t)(q0 - row0 * per_row.d) + threadIdx.x;
  const uint32_t dr = quotient(a, per_row);
  const int c = (int)(a - dr * per_row.d) * 8;
  const int64_t row = row0 + dr;
  const T* p = x + row * ld + c;
  const bool in = row < rows;
  float v[8];
  {
    raw_t<T, 8> w{};
    if (in && c + 8 <= dim) w = load_any<T, 8>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = raw_get<T, 8>(w, e);
    if (in && c < dim && c + 8 > dim) {   // the row's last few
#pragma unroll
      for (int e = 0; e < 7; ++e)
        if (c + e < dim) v[e] = raw_get<T, 1>(load_raw<T, 1>(p + e), 0);
    }
  }
  uint32_t m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu;
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
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[0] * inv, v[1] * inv, 1.0f, 0);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[2] * inv, v[3] * inv, 1.0f, 1);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[4] * inv, v[5] * inv, 1.0f, 2);
  word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[6] * inv, v[7] * inv, 1.0f, 3);
  if (s == 255) word = 0;
  if (!in) return;
  const int64_t q = q0 + threadIdx.x;
  store_words<uint32_t, NT>(codes + q, word);
  if ((q & 3) == 0) scales[q >> 2] = (uint8_t)s;
}

// ------------------------------------------------------------------ lookup
// As k_embed over quantised rows, vectors of 16 bytes of the output (eight
// codes, or four); ids NULL restores the whole table.  Two codes become floats in
// one instruction, without their scale: the product with a subnormal one is
// rounded as fp32 products are.  Measured, to bf16: 212,992 rows of 300 29.2 us,
// 4.8 TB/s (32.5 with the codes put together from their bits), 4.6M x 256 restored
// 468 us, 6.4 TB/s.
template <class OT, bool NT>
__global__ __launch_bounds__(BLOCK) void k_mx4_embed(const uint8_t* __restrict__ codes,
                                                     const uint8_t* __restrict__ scales, int blocks_row, int dim,
                                                     LookupIds l, SmallDiv nv, float scale, OT* __restrict__ out,
                                                     int64_t out_ld) {
  constexpr int U = LOOKUP_FLIGHT;
  const int64_t q0 = (int64_t)blockIdx.x * (BLOCK * U);
  const int64_t row0 = row_of(q0, nv.d);
  const uint32_t first = (uint32_t)(q0 - row0 * nv.d) + threadIdx.x;
  int bad = 0, miss = 0;
  constexpr int VW = 16 / sizeof(OT);
  uint32_t w[U], s[U];
  float mul[U];   // scale, or 0 for a row of zeros: their codes and scale bytes are 0
  int64_t at[U];
  int col[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const uint32_t x = first + u * BLOCK;
    const uint32_t dr = quotient(x, nv);
    const uint32_t c = (x - dr * nv.d) * VW;
    const int64_t i = row0 + dr;
    col[u] = dim;   // nothing to write
    w[u] = 0;
    s[u] = 0;
    mul[u] = 0.0f;
    if (i < l.n) {
      col[u] = (int)c;
      at[u] = i * out_ld + c;
      const int64_t r = lookup_row(l, i, bad, miss);
      if (r >= 0) {
        const uint8_t* p = codes + (r * blocks_row * MX_BYTES + c / 2);
        if constexpr (VW == 8) w[u] = *reinterpret_cast<const uint32_t*>(p);
        else w[u] = *reinterpret_cast<const uint16_t*>(p);
        s[u] = scales[r * blocks_row + c / MX_BLOCK];
        mul[u] = scale;
      }
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (col[u] >= dim) continue;
    const float f = scale_value(s[u]);
    float x[VW];
    float_pair c[4];
    c[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.0f, 0);
    c[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.0f, 1);
    if constexpr (VW == 8) {
      c[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.0f, 2);
      c[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[u], 1.0f, 3);
    }
#pragma unroll
    for (int e = 0; e < VW; ++e) x[e] = c[e / 2][e % 2] * f * mul[u];
    const int left = dim - col[u];
    if (left >= VW) {
      store_any<OT, VW, NT>(out + at[u], raw_make<OT, VW>(x));
    } else {
#pragma unroll
      for (int e = 0; e < VW - 1; ++e)
        if (e < left) store_raw<OT, 1>(out + at[u] + e, raw_make<OT, 1>(x + e));
    }
  }
  if (bad) atomicOr(l.err, 1);
}

// ------------------------------------------------------------------ product
//   C[i][j] = T( scale * sum_k A[i][k] B[j][k] ),  A [m][dim], B [n][dim]
// on the block-scaled matrix instruction of 32 x 32 x 64: lane l of a wave
// gives one block (32 codes and their scale) of row l % 32 of each operand, the
// lanes from 32 on another block than those below.  Products are exact, sums
// fp32.  The sum over k has no order of its own, so a lane takes four
// neighbouring blocks of its row at a time: 64 bytes of codes, one word of
// scales, whose bytes the instruction selects.
//
// B's rows go in as the first operand, so that a lane's result registers are
// four neighbouring columns of a row of C; they pass through LDS to leave as
// whole stretches of a row, 16 bytes a lane.
//
// The codes are staged in LDS eight blocks of a row at a time, copied there
// without a detour through registers: read straight from memory, the fragments
// of one instruction lie in 32 lines (2,048 x 131,072 of dim 512 326 us, staged
// 153).  One buffer: other workgroups of the compute unit fill the wait better
// than a second buffer does, which leaves room for two of them instead of four
// (200 us against 153; four instead of three 136 against 146).  The scales pass
// through LDS too, each row's brought by one thread: a lane that reads those it
// needs asks for twice as many lines as the codes have (dim 2,048, 2,048 x 31,000:
// 127 us against 98; dim 512 143 against 133).
//
// Bound by C's bytes where there are many queries (a table's width is a few
// hundred: 2 dim operations per element written), by B's where there are few.
// Measured: one query x 4.6M rows of 256 110 us, 5.8 TB/s of rows read and
// scores written; 2,048 x 131,072 in bf16 of dim 64 105 us, 5.1 TB/s, of dim 512
// 130 to 144 us, 4.2 TB/s and 2,000 TFLOP/s; 2,048 x 31,000 of dim 2,048 91 us,
// 2,860 TFLOP/s.  The instruction alone, its operands in registers, reaches 9,800: the
// matrix units are busy 24% of the time at dim 512, 42% at 2,048.
typedef int mx_operand __attribute__((ext_vector_type(8)));
typedef float mx_acc __attribute__((ext_vector_type(16)));

struct MxRows {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t rows;
};

// A workgroup's rows of one operand: the first row's codes and scales, and the
// last row there is (rows beyond it are read as it, and not stored).  Offsets
// inside a tile are 32 bits.
struct MxTile {
  const uint8_t* codes;
  const uint8_t* scales;
  int last;
};

__device__ __forceinline__ MxTile mx_rows(const MxRows& t, int64_t row0, int rows, int blocks_row) {
  const int64_t left = t.rows - 1 - row0;
  return MxTile{t.codes + row0 * blocks_row * MX_BYTES, t.scales + row0 * blocks_row,
                left < rows - 1 ? (int)left : rows - 1};
}

// Staged codes: rows of eight blocks (128 bytes), block b of a row in slot
// b ^ (row / 2 % 8), so that the blocks of one number of sixteen rows lie in
// sixteen different slots of 256 bytes: reading them has no bank conflict.
__device__ __forceinline__ int mx_slot(int row, int b) { return row * 8 + (b ^ ((row >> 1) & 7)); }

// Copies blocks k0 .. k0+7 of the tile's ROWS rows into LDS, the eight rows of
// an instruction side by side.  Blocks beyond a row's end are taken from its
// last block.
template <int ROWS>
__device__ __forceinline__ void mx_stage(const MxTile& t, int k0, int blocks_row, words4* to) {
  const int w = threadIdx.x / WAVE, l = lane_id();
  // (the rows of one thread are 32 apart: their blocks have the same slots)
  const int kb = k0 + ((l % 8) ^ (((w * 8 + l / 8) >> 1) & 7));
  const uint32_t at = (kb < blocks_row ? kb : blocks_row - 1) * MX_BYTES;
#pragma unroll
  for (int i = 0; i < ROWS / 8; i += WAVES_PER_BLOCK) {
    const int row = (i + w) * 8 + l / 8;   // (ROWS / 8 is a multiple of the number of waves)
    const uint32_t off = (uint32_t)(row < t.last ? row : t.last) * (uint32_t)(blocks_row * MX_BYTES) + at;
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(t.codes + off),
                                     (__attribute__((address_space(3))) void*)(to + (i + w) * WAVE), 16, 0, 0);
  }
}

// A row's scale bytes from block k0 on, two words, 1 where they are beyond its end.
__device__ __forceinline__ void mx_scales(const MxTile& t, int row, int k0, int blocks_row, uint32_t (&s)[2]) {
  const uint8_t* p = t.scales + (uint32_t)((row < t.last ? row : t.last) * blocks_row + k0);
  const int left = blocks_row - k0;
  if (left >= 8) {
    __builtin_memcpy(s, p, 8);
    return;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int have = left - 4 * i;   // of the word's bytes, where below 4
    s[i] = 0x7f7f7f7fu;
    if (have >= 4) {
      __builtin_memcpy(&s[i], p + 4 * i, 4);
    } else if (have > 0 && blocks_row >= 4) {   // the row's last four, those before the word's shifted out
      uint32_t x;
      __builtin_memcpy(&x, p + left - 4, 4);
      s[i] = (uint32_t)((0x7f7f7f7full << 32 | x) >> (32 - 8 * have));
    } else if (have > 0) {
#pragma unroll
      for (int q = 0; q < 3; ++q)
        if (q < have) s[i] ^= (uint32_t)(p[4 * i + q] ^ 0x7fu) << (8 * q);
    }
  }
}

__device__ __forceinline__ mx_operand mx_words(const words4& c) {
  return mx_operand{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};
}

// The workgroup's tile.  With several tiles of queries each die takes one
// stretch of C's columns, in groups of MX_GROUP tiles, a group's tiles row after
// row: B's rows come into one die's cache once, the lines in which two
// neighbouring tiles' rows meet are put together there, and the tiles at work
// lie side by side (tiles under each other, 2^k bytes apart, meet in few
// channels of the memory).  Measured, 2,048 x 131,072 of dim 64 and 512, bf16:
// tiles under each other 128 and 152 us, groups 105 and 144.
constexpr uint32_t MX_GROUP = 16;

// (tiles are counted in 32 bits, as workgroups are)
__device__ __forceinline__ void mx_tile(uint32_t tiles_q, uint32_t tiles_b, uint32_t& tb, uint32_t& tq) {
  if (tiles_q == 1) {
    tb = blockIdx.x;
    tq = 0;
    return;
  }
  const uint32_t tile = (blockIdx.x % NUM_XCD) * (gridDim.x / NUM_XCD) + blockIdx.x / NUM_XCD;
  const uint32_t group = tile / (MX_GROUP * tiles_q), rest = tile - group * (MX_GROUP * tiles_q);
  const uint32_t before = group * MX_GROUP;
  const uint32_t wide = before >= tiles_b ? 1 : tiles_b - before < MX_GROUP ? tiles_b - before : MX_GROUP;
  tq = rest / wide;
  tb = before + (rest - tq * wide);
  if (tq >= tiles_q) tb = tiles_b;   // beyond the last tile
}

// A wave's tile is QT x 32 rows of A by TT x 32 rows of B; a workgroup's waves
// stand WQ x WT.  Rows of C are stored 16 bytes at a time wherever they start.
// Four workgroups stand in a compute unit, three of the widest tile (by their LDS).
template <class OT, int QT, int TT, int WQ, int WT, bool NT>
__global__ __launch_bounds__(BLOCK, WQ * QT + WT * TT <= 9 ? 4 : 3) void k_mx4_product(MxRows A, MxRows B, int blocks_row, float scale,
                                                       OT* __restrict__ C, int64_t ldc, uint32_t tiles_q,
                                                       uint32_t tiles_b) {
  constexpr int VW = 16 / sizeof(OT);
  constexpr int ET = sizeof(OT) == 2 && TT % 4 == 0 ? 4 : 2;   // tiles that leave together: rows of 256 or 128 bytes
  static_assert(WQ * WT == WAVES_PER_BLOCK && TT % ET == 0, "four waves, whole rows");
  constexpr int COLS = ET * 32, PITCH = COLS + VW;   // elements; rows start four banks apart
  constexpr int RA = WQ * QT * 32, RB = WT * TT * 32;   // rows of the workgroup's tile
  constexpr size_t kStage = (RA + RB) * 8 * sizeof(words4), kOut = WAVES_PER_BLOCK * 32 * PITCH * sizeof(OT);
  __shared__ words4 lds[(kStage > kOut ? kStage : kOut) / sizeof(words4)];
  __shared__ uint32_t scales[2][RA + RB];   // of the eight staged blocks
  const int w = threadIdx.x / WAVE, l = lane_id();
  uint32_t tb, tq;
  mx_tile(tiles_q, tiles_b, tb, tq);
  if (tb >= tiles_b) return;   // (the grid is a multiple of the dies)
  const int wa = w / WT * QT * 32, wb = w % WT * TT * 32;   // the wave's rows in the tile
  const int64_t i0 = (int64_t)tq * RA + wa, j0 = (int64_t)tb * RB + wb;
  const int half = l / 32, r = l % 32;
  words4 *sa = lds, *sb = lds + RA * 8;
  const MxTile ta = mx_rows(A, (int64_t)tq * RA, RA, blocks_row),
               tbl = mx_rows(B, (int64_t)tb * RB, RB, blocks_row);
  mx_acc acc[QT][TT];
#pragma unroll
  for (int q = 0; q < QT; ++q)
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[q][t][e] = 0.0f;
  uint32_t xa[QT], xb[TT];   // scales
  // block number K of the lane's blocks first .. first+3 of the staged ones
  auto multiply = [&]<int K, bool FULL>(int first, int rem) {
    mx_operand fa[QT], fb[TT];
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      words4 c = sa[mx_slot(wa + q * 32 + r, first + K)];
      if (!FULL && first + K >= rem) c = words4{0u, 0u, 0u, 0u};
      fa[q] = mx_words(c);
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) fb[t] = mx_words(sb[mx_slot(wb + t * 32 + r, first + K)]);
#pragma unroll
    for (int q = 0; q < QT; ++q)
#pragma unroll
      for (int t = 0; t < TT; ++t)
        acc[q][t] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[t], fa[q], acc[q][t], 4, 4, K, (int)xb[t], K,
                                                                    (int)xa[q]);
  };
  constexpr int SR = (RA + RB + BLOCK - 1) / BLOCK;   // rows whose scales a thread brings
  uint32_t sc[SR][2];
  auto stage = [&](int k0) {
    if (k0 > 0) __syncthreads();
    mx_stage<RB>(tbl, k0, blocks_row, sb);
    mx_stage<RA>(ta, k0, blocks_row, sa);
#pragma unroll
    for (int i = 0; i < SR; ++i) {
      const int row = i * BLOCK + threadIdx.x;
      if (row < RA) mx_scales(ta, row, k0, blocks_row, sc[i]);
      else if (row < RA + RB) mx_scales(tbl, row - RA, k0, blocks_row, sc[i]);
    }
#pragma unroll
    for (int i = 0; i < SR; ++i)
#pragma unroll
      for (int q = 0; q < 2; ++q)
        if (i * BLOCK + (int)threadIdx.x < RA + RB) scales[q][i * BLOCK + threadIdx.x] = sc[i][q];
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  int k0 = 0;
  for (; k0 + 8 <= blocks_row; k0 += 8) {
    stage(k0);
    const uint32_t* s = scales[half];
#pragma unroll
    for (int t = 0; t < TT; ++t) xb[t] = s[RA + wb + t * 32 + r];
#pragma unroll
    for (int q = 0; q < QT; ++q) xa[q] = s[wa + q * 32 + r];
    multiply.template operator()<0, true>(4 * half, 8);
    multiply.template operator()<1, true>(4 * half, 8);
    multiply.template operator()<2, true>(4 * half, 8);
    multiply.template operator()<3, true>(4 * half, 8);
  }
  if (k0 < blocks_row) {   // up to seven blocks, halved between the lanes below 32 and above
    const int rem = blocks_row - k0, per = (rem + 1) / 2;
    stage(k0);
    // four bytes from byte 0 or `per` (at most 4) of the eight
    auto scale_word = [&](int row) {
      return (uint32_t)(((uint64_t)scales[1][row] << 32 | scales[0][row]) >> (8 * per * half));
    };
#pragma unroll
    for (int t = 0; t < TT; ++t) xb[t] = scale_word(RA + wb + t * 32 + r);
#pragma unroll
    for (int q = 0; q < QT; ++q) xa[q] = scale_word(wa + q * 32 + r);
    multiply.template operator()<0, false>(per * half, rem);
    if (per > 1) multiply.template operator()<1, false>(per * half, rem);
    if (per > 2) multiply.template operator()<2, false>(per * half, rem);
    if (per > 3) multiply.template operator()<3, false>(per * half, rem);
  }
  __syncthreads();   // the staged codes make room for the results
  // register e of a tile: row r of A's 32, column 8 (e / 4) + 4 half + e % 4 of B's
  OT* my = reinterpret_cast<OT*>(lds) + w * 32 * PITCH;
#pragma unroll
  for (int q = 0; q < QT; ++q)
#pragma unroll
    for (int t = 0; t < TT; t += ET) {
      if (i0 + q * 32 >= A.rows || j0 + t * 32 >= B.rows) continue;   // (the same for the whole wave)
#pragma unroll
      for (int tt = 0; tt < ET; ++tt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = scale * acc[q][t + tt][4 * g + e];
          store_raw<OT, 4>(my + r * PITCH + tt * 32 + 8 * g + 4 * half, raw_make<OT, 4>(x));
        }
      // the wave reads what its own lanes wrote
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      constexpr int LR = COLS / VW;   // lanes per row
      const int c = l % LR * VW;
      const int64_t j = j0 + t * 32 + c;
#pragma unroll
      for (int g = 0; g < 32; g += WAVE / LR) {
        const int i = g + l / LR;
        const words4 v = *reinterpret_cast<const words4*>(my + i * PITCH + c);
        if (i0 + q * 32 + i >= A.rows) continue;
        OT* p = C + (i0 + q * 32 + i) * ldc + j;
        if (j + VW <= B.rows) store_words<words4_any, NT>(p, v);
        else
          for (int e = 0; e < VW && j + e < B.rows; ++e) p[e] = my[i * PITCH + c + e];
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
}

}  // namespace adapm
