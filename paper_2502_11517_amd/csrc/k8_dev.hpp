// Shared by the kernels of the 8-bit cache: its geometry, the plan's records, conversions of codes, sums over a work-group.
#pragma once
#include <hip/hip_runtime.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>

#include <utility>

#include "k8_split.hpp"

namespace k8 {

constexpr int kBlock = 16;           // tokens under one scale
constexpr int kEMin = -100, kEMax = 119;
constexpr int kRows = 32;            // stacked rows (query row x head of the kv head's group) of one wave
constexpr int kWideRows = 64;        // ... of one work-group, in requests that have more than kManyRows
constexpr int kManyRows = 128;
constexpr int kWholeTokens = 768, kWholeWide = 512;  // where the table has room for no more, no tile is split (with tiles of 32 rows; of 64 rows, too)
constexpr int kTaggedRows = 64;      // with a prefix and at most so many rows in a step, a request's rows are taken to be streams with tags
constexpr int kMostTokens = 1 << 27; // of a request: a plan's sums over 1024 tiles stay within 32 bits
constexpr int kUnitBlocks = 64;      // blocks of a unit that are listed with it
enum { kE4m3 = 0, kInt8 = 1 };
enum { kF32 = 0, kBf16 = 1, kF16 = 2 };

using half2v = __attribute__((ext_vector_type(2))) _Float16;
using int2v = __attribute__((ext_vector_type(2))) int;
using half8 = __attribute__((ext_vector_type(8))) _Float16;
using float2v = __attribute__((ext_vector_type(2))) float;
using float4v = __attribute__((ext_vector_type(4))) float;
using float16v = __attribute__((ext_vector_type(16))) float;
using uint4v = __attribute__((ext_vector_type(4))) uint32_t;
using uint2v = __attribute__((ext_vector_type(2))) uint32_t;

struct Geometry {
  int Hkv, G, D, page_tokens, page_shift;
  int blocks_per_page;  // page_tokens / 16
  int n_pages;          // of a layer
  int table_width;      // pages_per_request
};

// One piece of the attention's work, times Hkv.
struct Unit {
  int request;
  int s0;        // first stacked row: (row of the step) * G + head within the kv head's group
  int n_rows;    // stacked rows
  int pos0;      // token of the first row; stacked row i is token pos0 + i / G
  int lo, hi;    // tokens to read
  int prefix;    // tokens below see no tags and no order
  int part;      // first partial row, -1: the result goes to out
};
// The stacked rows whose tokens are split over several units: parts k = 0 .. n_parts-1 at partial rows part + k * n_rows.
struct Tile {
  int s0, n_rows, part, n_parts;
};

__device__ inline float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // e in [-126, 127]

// Least e with amax <= Q * 2^e, from the bits of a finite amax: Q = 448 = 1.75 * 2^8 or 127 = 1.984375 * 2^6.
template <int CODES>
__device__ inline int scale_exponent(uint32_t amax_bits) {
  constexpr int kTopExp = CODES == kE4m3 ? 8 : 6;
  constexpr uint32_t kTopMant = CODES == kE4m3 ? 0x600000u : 0x7e0000u;
  int x = (int)(amax_bits >> 23) - 127;  // a subnormal amax comes out below kEMin anyway
  int e = x - kTopExp + ((amax_bits & 0x7fffffu) > kTopMant ? 1 : 0);
  return min(max(e, kEMin), kEMax);
}

// Four values in units of the scale, at most Q in magnitude -> four codes; nearest, ties to even.
template <int CODES>
__device__ inline uint32_t encode4(float a, float b, float c, float d) {
  if constexpr (CODES == kE4m3) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  } else {
    // at 3 * 2^22 a step of fp32 is 1: the sum rounds to a whole number, whose low byte is the code
    auto whole = [](float x) { return __float_as_uint(x + 12582912.f); };
    const uint32_t lo = __builtin_amdgcn_perm(whole(b), whole(a), 0x0c0c0400u), hi = __builtin_amdgcn_perm(whole(d), whole(c), 0x04000c0cu);
    return lo | hi;
  }
}

// Four codes -> their values.
template <int CODES>
__device__ inline void decode4(uint32_t w, float (&x)[4]) {
  if constexpr (CODES == kE4m3) {
    float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0], x[1] = lo[1], x[2] = hi[0], x[3] = hi[1];
  } else {
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  }
}

// Eight codes -> the operand of a matrix instruction.  Every code is a whole number of fp16's bits in either type, so this is exact.
//   e4m3  one conversion for two codes
//   int8  with the sign bit turned, c + 128 is the low byte of the fp16 number 1024 + c + 128; one byte permutation and one
//         packed addition for two codes
template <int CODES>
__device__ inline half8 codes_to_half8(uint32_t a, uint32_t b) {
  union { half2v h[4]; half8 v; uint32_t u[4]; } r;
  if constexpr (CODES == kE4m3) {
    r.h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
    r.h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
    r.h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
    r.h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
  } else {
    const half2v off = {(_Float16)1152.f, (_Float16)1152.f};
    a ^= 0x80808080u, b ^= 0x80808080u;
    r.u[0] = __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u);
    r.u[1] = __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u);
    r.u[2] = __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u);
    r.u[3] = __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u);
    for (int i = 0; i < 4; ++i) r.h[i] -= off;
  }
  return r.v;
}

// Largest of the wave's 64 values, in every lane: rotations within rows of 16 lanes, then the rows.
__device__ inline uint32_t wave_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));  // row_ror:8
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, false));
  x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, false));
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max(b[0], b[1]);
}

// Sum over the lanes below and including this one: within rows of 16 lanes, then each row's end into the next row, then half into half.
__device__ inline int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15, rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31, rows 2 and 3
  return x;
}

// Inclusive sums over the work-group and their totals; `tmp` holds a pair per wave.  Every thread calls it; it ends with a barrier.
template <int NT>
__device__ inline int2v group_scan(int2v x, int2v* tmp, int2v& total) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  x[0] = wave_scan(x[0]), x[1] = wave_scan(x[1]);
  if constexpr (NT == 64) {
    total = int2v{__builtin_amdgcn_readlane(x[0], 63), __builtin_amdgcn_readlane(x[1], 63)};
    __syncthreads();
    return x;
  }
  if (lane == 63) tmp[wave] = x;
  __syncthreads();
  int2v before{0, 0}, all{0, 0};
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const int2v t = tmp[w];
    if (w < wave) before += t;
    all += t;
  }
  __syncthreads();
  total = all;
  return x + before;
}

template <int NT>
__device__ inline int group_scan(int x, int2v* tmp, int& total) {
  int2v all;
  const int2v y = group_scan<NT>(int2v{x, 0}, tmp, all);
  total = all[0];
  return y[0];
}

// How many of v[0 .. n) are <= x; v ascending.
template <class T>
__device__ inline int count_le(const T* v, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    int m = (lo + hi) >> 1;
    if (v[m] <= x) lo = m + 1; else hi = m;
  }
  return lo;
}

// The block that holds a token of a request, by its page table.
__device__ inline int block_of(const Geometry& g, const int* table, int request, int token, int hi) {
  const int t = max(min(token, hi - 1), 0);
  const int page = table[(int64_t)request * g.table_width + (t >> g.page_shift)];
  return token < hi && page >= 0 && page < g.n_pages ? page * g.blocks_per_page + ((token & (g.page_tokens - 1)) >> 4) : -1;
}

}  // namespace k8
