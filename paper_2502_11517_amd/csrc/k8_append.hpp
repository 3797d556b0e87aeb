// New rows of one layer into the cache, as 8-bit codes.
//
// A wave takes the rows that a call brings into one block (a run of at most 16 neighbouring slots) of one kv head, K or V: their
// largest magnitude gives the scale, codes ahead of the run are rounded again if the scale grew, and a block begun by the run is
// written whole.  Scales are powers of two, so x / scale is exact and a code is one rounding of its value.  Magnitudes are compared
// as bits: what is not finite is then larger than everything finite.
//
// Bound by memory for prompts: 8192 rows of 8 heads of 128, bf16, 50 MB in 13.0 us, 3.9 TB/s (K's half alone 4.0; a large copy 4.9).  A step of eight
// rows takes 3.0 us, its launch and two dependent reads (slots, then rows with scales and codes).  Loads that bypass the caches took 69 us instead of 77
// where the rows came from HBM, and 14 instead of 11 where they were near, as behind the projection that wrote them: not taken.
#pragma once
#include "k8_dev.hpp"

namespace k8 {

struct AppendArgs {
  Geometry g;
  int n_rows, group;  // rows that a work-group looks at
  const int* slot;
  const void *k_new, *v_new;
  uint8_t *k, *v;
  float *ks, *vs;
};

template <int IN, int N>
__device__ inline void load_row(const void* base, int64_t at, float (&x)[N]) {  // N neighbouring values
  if constexpr (IN == kF32) {
    const float* p = (const float*)base + at;
    if constexpr (N >= 4) {
      for (int i = 0; i < N; i += 4) {
        const float4v w = *(const float4v*)(p + i);
        for (int k = 0; k < 4; ++k) x[i + k] = w[k];
      }
    } else if constexpr (N == 2) {
      const float2v w = *(const float2v*)p;
      x[0] = w[0], x[1] = w[1];
    } else {
      x[0] = *p;
    }
  } else {
    const uint16_t* p = (const uint16_t*)base + at;
    uint32_t w[(N + 1) / 2];
    if constexpr (N >= 8) {
      for (int i = 0; i < N / 8; ++i) {
        const uint4v t = *((const uint4v*)p + i);
        for (int k = 0; k < 4; ++k) w[4 * i + k] = t[k];
      }
    } else if constexpr (N == 2) {
      w[0] = *(const uint32_t*)p;
    } else {
      w[0] = *p;
    }
    for (int i = 0; i < N; ++i) {
      const uint32_t b = (i & 1) ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
      if constexpr (IN == kBf16) {
        x[i] = __uint_as_float(b << 16);
      } else {
        union { uint16_t u; _Float16 h; } c{(uint16_t)b};
        x[i] = (float)c.h;
      }
    }
  }
}

// Bits of the largest magnitude of N values that load_row gave.
template <int N>
__device__ inline uint32_t magnitude(const float (&x)[N], uint32_t amax) {
#pragma unroll
  for (int i = 0; i < N; ++i) amax = max(amax, __float_as_uint(x[i]) & 0x7fffffffu);
  return amax;
}

// Past kEMax a value can be beyond Q times the scale, and is Q then.
template <int CODES, int N>
__device__ inline void hold(float (&x)[N], float inverse) {
  constexpr float kTop = CODES == kE4m3 ? 448.f : 127.f;
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = fminf(fmaxf(x[i], -kTop / inverse), kTop / inverse);
}

struct RunScale {
  bool held;      // the exponent is kEMax
  float inverse;  // 2^-e of the new codes
  float again;    // 2^(f-e) for the codes ahead of the run
  float scale;    // what the block gets
  bool regrown, lost;
};

template <int CODES>
__device__ inline RunScale run_scale(uint32_t amax, int offset, float was) {
  RunScale s{};
  const bool bad = amax >= 0x7f800000u;
  int e = bad ? kEMin : scale_exponent<CODES>(amax);
  s.lost = bad;
  if (offset > 0) {
    if (was != was) {
      s.lost = true;
    } else {
      const int f = min(max((int)(__float_as_uint(was) >> 23 & 255) - 127, kEMin), kEMax);
      s.regrown = !bad && e > f;
      s.again = s.regrown ? (e - f > 126 ? 0.f : pow2f(f - e)) : 1.f;
      e = max(e, f);
    }
  }
  s.held = e == kEMax;
  s.inverse = pow2f(-e);
  s.scale = s.lost ? __builtin_nanf("") : pow2f(e);
  return s;
}

// K: a lane holds 16 dims of a token, one piece of the block's layout (two pieces if D = 128).
template <int CODES, int D, int IN>
__device__ inline void append_k(const AppendArgs& a, int row, int n, int offset, int head, int64_t block) {
  constexpr int kPieces = D / 64;
  const int lane = threadIdx.x & 63, token = lane >> 2, part = lane & 3;
  uint8_t* codes = a.k + block * (kBlock * D);
  const float was = a.ks[block];
  float x[kPieces][16];
  uint32_t amax = 0;
  const bool mine = token >= offset && token < offset + n;
  for (int j = 0; j < kPieces; ++j) {
    for (int i = 0; i < 16; ++i) x[j][i] = 0.f;
    if (mine) load_row<IN, 16>(a.k_new, ((int64_t)(row + token - offset) * a.g.Hkv + head) * D + (part + 4 * j) * 16, x[j]);
    amax = magnitude(x[j], amax);
  }
  const RunScale s = run_scale<CODES>(wave_max(amax), offset, was);
  if (s.held)
    for (int j = 0; j < kPieces; ++j) hold<CODES>(x[j], s.inverse);
  const bool before = token < offset;
  for (int j = 0; j < kPieces; ++j) {
    uint4v* to = (uint4v*)(codes + ((part + 4 * j) * kBlock + token) * 16);
    if (before && !s.regrown) continue;
    if (!before && !mine && offset) continue;  // behind the run of a block that had begun
    uint4v w;
    if (before) {
      w = *to;
      for (int i = 0; i < 4; ++i) {
        float y[4];
        decode4<CODES>(w[i], y);
        w[i] = encode4<CODES>(y[0] * s.again, y[1] * s.again, y[2] * s.again, y[3] * s.again);
      }
    } else {
      for (int i = 0; i < 4; ++i)
        w[i] = s.lost ? 0u : encode4<CODES>(x[j][4 * i] * s.inverse, x[j][4 * i + 1] * s.inverse, x[j][4 * i + 2] * s.inverse, x[j][4 * i + 3] * s.inverse);
    }
    *to = w;
  }
  if (lane == 0) a.ks[block] = s.scale;
}

// V: a lane holds all 16 tokens of one dim (two if D = 128), rows of the block's layout.
template <int CODES, int D, int IN>
__device__ inline void append_v(const AppendArgs& a, int row, int n, int offset, int head, int64_t block) {
  constexpr int N = D / 64;
  const int lane = threadIdx.x & 63;
  uint4v* codes = (uint4v*)(a.v + block * (kBlock * D)) + lane * N;
  float x[kBlock][N];
  uint32_t amax = 0;
  // Places without a row get the nearest one's, which changes no maximum and is dropped below: loads under branches wait for one another (8192 rows of 8
  // heads, a layer: 19 us with them, 13 without; a step of eight rows 4.0 and 3.3).
#pragma unroll
  for (int t = 0; t < kBlock; ++t)
    load_row<IN, N>(a.v_new, ((int64_t)(row + min(max(t - offset, 0), n - 1)) * a.g.Hkv + head) * D + lane * N, x[t]);
  const float was = a.vs[block];
  uint4v old[N];
  for (int j = 0; j < N; ++j) old[j] = uint4v{0, 0, 0, 0};
  if (offset)
    for (int j = 0; j < N; ++j) old[j] = codes[j];
#pragma unroll
  for (int t = 0; t < kBlock; ++t) amax = magnitude(x[t], amax);
  const RunScale s = run_scale<CODES>(wave_max(amax), offset, was);
  if (s.held)
#pragma unroll
    for (int t = 0; t < kBlock; ++t) hold<CODES>(x[t], s.inverse);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    uint4v w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t fresh = s.lost ? 0u : encode4<CODES>(x[4 * i][j] * s.inverse, x[4 * i + 1][j] * s.inverse, x[4 * i + 2][j] * s.inverse, x[4 * i + 3][j] * s.inverse);
      uint32_t again = old[j][i];
      if (s.regrown) {
        float y[4];
        decode4<CODES>(again, y);
        again = encode4<CODES>(y[0] * s.again, y[1] * s.again, y[2] * s.again, y[3] * s.again);
      }
      uint32_t before = 0, run = 0;  // bytes ahead of the run, bytes of the run
      for (int k = 0; k < 4; ++k) {
        const int t = 4 * i + k;
        if (t < offset) before |= 255u << (8 * k);
        else if (t < offset + n) run |= 255u << (8 * k);
      }
      w[i] = (again & before) | (fresh & run) | (old[j][i] & ~(before | run));
    }
    codes[j] = w;
  }
  if (lane == 0) a.vs[block] = s.scale;
}

template <int CODES, int D, int IN>
__global__ __launch_bounds__(256) void k8_append(AppendArgs a) {
  const int lane = threadIdx.x & 63, task = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = task >> 1;
  if (head >= a.g.Hkv) return;
  const int n_slots = a.g.n_pages << a.g.page_shift;
  const int first = blockIdx.x * a.group, last = min(first + a.group, a.n_rows);
  // lane k: the slot of row first + k - 1; a run that begins within the group ends within 16 more rows
  const int row = first + lane - 1;
  const int mine = lane <= a.group + kBlock && row >= 0 && row < a.n_rows ? a.slot[row] : -1;
  int i = first;
  while (i < last) {
    const int at = i - first + 1, prev = __builtin_amdgcn_readlane(mine, at - 1), slot = __builtin_amdgcn_readlane(mine, at);
    if (slot < 0 || slot >= n_slots) {
      ++i;
      continue;
    }
    const bool goes_on = lane >= at && mine == slot + lane - at && (mine >> 4) == (slot >> 4);
    const int n = __builtin_ctzll(~(__ballot(goes_on) >> at));
    if (!(prev >= 0 && slot == prev + 1 && (slot & 15))) {  // the run begins here
      const int page = slot >> a.g.page_shift, b = (slot & (a.g.page_tokens - 1)) >> 4;
      const int64_t block = ((int64_t)page * a.g.Hkv + head) * a.g.blocks_per_page + b;
      if (task & 1)
        append_v<CODES, D, IN>(a, i, n, slot & 15, head, block);
      else
        append_k<CODES, D, IN>(a, i, n, slot & 15, head, block);
    }
    i += n;
  }
}

}  // namespace k8
