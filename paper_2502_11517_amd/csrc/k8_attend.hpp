// Attention over the 8-bit cache.
//
// With z = q . K8_j (codes), row factor c = |scale| * log2(e) * 2^-k (q is scaled by 2^k into fp16's range, and by the scale's sign),
// block scales ks, vs and running maximum m, all scores in log2 units:
//
//   t_j = z * c * ks            (capped, lowered by distance)        w_j = 2^(t_j - m)      l = sum w_j
//   O   = sum (w_j * vs * 2^-E) V8_j                                 out = O * 2^E / l      lse = ln 2 * (m + log2 l)
//
// Codes are whole fp16 numbers, so K and V enter the products exactly and the scales, powers of two, outside of them; E is the largest
// exponent of vs so far, so that what enters as fp16 (the softmax weight) stays within [0, 1].  Its rounding, 2^-12 of each weight, is
// the only one that fp32 does not see; it is half a bit of an fp16 output.
//
// Both products run transposed, S^T = K Q^T and O^T = V^T P^T, in 32x32x16 steps of a wave over 32 tokens x 32 stacked rows.  What row of
// the first product a token has is free, and so is the order of dims within it; both are chosen such that
//   * a lane's piece of K (16 dims of a token) and of V (16 tokens of a dim) are 16 neighbouring bytes of the cache: codes go from memory to
//     the products' operands through registers alone, in whole cache lines, with no transposition;
//   * the scores that a lane gets (16 tokens of one block, one row) are, as fp16, its operand of the second product.
//
// k8_attend, few rows (<= 32 stacked): every wave takes blocks of 32 tokens of its own, and the four meet once at the end.
// Many rows: four waves of 32 rows each take the same tokens; the codes are turned into fp16 once per work-group, by way of LDS.
#pragma once
#include "k8_dev.hpp"

namespace k8 {

struct AttendArgs {
  Geometry g;
  int Hq, g_shift, dtype, n_rows;
  float scale_log2;       // |softmax_scale| * log2(e)
  int negate;             // softmax_scale < 0
  float cap_log2, cap_in; // logit_cap * log2(e), 2 / logit_cap; 0: none
  const uint8_t *k, *v;
  const float *ks, *vs;
  const int* table;
  const uint8_t* slot_tag;
  const int *slot_position, *row_position;
  const uint64_t* row_see;
  const float* slopes;
  const int* n_units;
  const Unit* units;
  const Tile* tiles;
  const void* q;
  void* out;
  float* lse;
  float2v* part_ml;  // [partial row][Hkv]: m, l
  float* part_acc;   // ... [D]: O * 2^E
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ inline float other_half(float x) {  // of lane ^ 32
  return __shfl_xor(x, 32);
}

// A wave's 32 stacked rows: lane n and n + 32 hold row n, each half of the dims.
template <int D>
struct Rows {
  half8 q[D / 16];
  float c;      // score factor but for ks
  float slope;  // in log2 units
  int token;    // own place
  int position;
  uint64_t see;
  bool real;
};

__device__ inline int64_t row_address(const AttendArgs& a, int s, int head) {  // of stacked row s, in rows of D
  return (int64_t)(s >> a.g_shift) * a.Hq + head * a.g.G + (s & (a.g.G - 1));
}

template <int D>
__device__ inline void load_rows(const AttendArgs& a, const Unit& u, int head, int first, Rows<D>& r) {
  const int lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
  r.real = first + n < u.n_rows;
  const int s = u.s0 + (r.real ? first + n : 0);
  const uint4v* p = (const uint4v*)((const uint16_t*)a.q + row_address(a, s, head) * D);
  uint4v w[D / 16];
#pragma unroll
  for (int k = 0; k < D / 16; ++k) w[k] = p[(2 * (k >> 1) + half) * 2 + (k & 1)];
  r.token = u.pos0 + ((first + n) >> a.g_shift);
  r.see = a.row_see ? a.row_see[s >> a.g_shift] : 0;
  r.position = a.row_position ? a.row_position[s >> a.g_shift] : r.token;
  r.slope = a.slopes ? a.slopes[head * a.g.G + (s & (a.g.G - 1))] * kLog2e : 0.f;
  float x[D / 16][8];
  uint32_t amax = 0;
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t b = (i & 1) ? w[k][i / 2] >> 16 : w[k][i / 2] & 0xffffu;
      union { uint16_t u; _Float16 h; } c{(uint16_t)b};
      x[k][i] = a.dtype == kBf16 ? __uint_as_float(b << 16) : (float)c.h;
      amax = max(amax, __float_as_uint(x[k][i]) & 0x7fffffffu);
    }
  amax = max(amax, (uint32_t)__shfl_xor((int)amax, 32));
  // the largest value comes to [2^14, 2^15): bf16's 8 bits stay whole down to 2^-31 of it, fp16's 11 to 2^-28
  const int up = amax ? min(max(14 + 127 - (int)(amax >> 23), -126), 126) : 0;
  const float f = r.real ? (a.negate ? -pow2f(up) : pow2f(up)) : 0.f;
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) r.q[k][i] = r.real ? (_Float16)(x[k][i] * f) : (_Float16)0.f;
  r.c = a.scale_log2 * pow2f(-up);
}

// The blocks of a stretch of tokens, lane k the k-th of them: index into the scales (-1: none there), the scales, the first slot / 16.
struct Blocks {
  int at, slot16;
  float ks, vs;
};

__device__ inline Blocks load_blocks(const AttendArgs& a, int request, int head, int token, int hi) {
  Blocks b{-1, 0, 0.f, 0.f};
  if (token < hi) {
    const int page = a.table[(int64_t)request * a.g.table_width + (token >> a.g.page_shift)];
    if (page >= 0 && page < a.g.n_pages) {
      const int in = (token & (a.g.page_tokens - 1)) >> 4;
      b.at = (page * a.g.Hkv + head) * a.g.blocks_per_page + in;
      b.slot16 = page * a.g.blocks_per_page + in;
      b.ks = a.ks[b.at];
      b.vs = a.vs[b.at];
    }
  }
  return b;
}

// 32 tokens: two blocks.
struct Pair {
  int at[2], slot16[2];
  float ks[2], vs[2];
};

__device__ inline Pair pair_of(const Blocks& b, int k) {  // blocks 2k and 2k + 1 of the wave's lanes; k the same for all lanes
  Pair p;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    p.at[i] = __builtin_amdgcn_readlane(b.at, 2 * k + i);
    p.slot16[i] = __builtin_amdgcn_readlane(b.slot16, 2 * k + i);
    p.ks[i] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(b.ks), 2 * k + i));
    p.vs[i] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(b.vs), 2 * k + i));
  }
  return p;
}

// The codes of a pair, as this lane's pieces.  Row m = 8a + 4h + b of the first product is token 4a + b of block h.
template <int D>
__device__ inline void load_k(const AttendArgs& a, const Pair& p, uint4v (&k)[D / 32]) {
  const int lane = threadIdx.x & 63, m = lane & 31, half = lane >> 5;
  const int at = max((m & 4) ? p.at[1] : p.at[0], 0);
  const uint8_t* from = a.k + (int64_t)at * (kBlock * D) + half * 256 + ((m >> 3) * 4 + (m & 3)) * 16;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) k[i] = *(const uint4v*)(from + i * 512);
}

template <int D>
__device__ inline void load_v(const AttendArgs& a, const Pair& p, uint4v (&v)[D / 32]) {
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int at = max(half ? p.at[1] : p.at[0], 0);
  const uint8_t* from = a.v + (int64_t)at * (kBlock * D) + (lane & 31) * 16;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) v[i] = *(const uint4v*)(from + i * 512);
  if (p.at[0] < 0 || p.at[1] < 0) {  // what is not there must not be NaN: its weight is 0
    const bool none = (half ? p.at[1] : p.at[0]) < 0;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) v[i] = none ? uint4v{0, 0, 0, 0} : v[i];
  }
}

// Which of the lane's 16 tokens (base, base + 1, ...) its row sees, as bits.
__device__ inline uint32_t visible(const AttendArgs& a, const Unit& u, int hi, int base, int at, int slot16, int token, uint64_t see) {
  auto below = [](int n) { return n <= 0 ? 0u : n >= kBlock ? 0xffffu : (1u << n) - 1u; };
  uint32_t bits = below(token + 1 - base);
  if (a.row_see) {
    const uint4v t = at >= 0 ? *(const uint4v*)(a.slot_tag + (int64_t)slot16 * kBlock) : uint4v{0, 0, 0, 0};
    uint32_t tagged = 0;
    const uint32_t one = (t[0] & 255u) * 0x01010101u;
    if (__all(t[0] == one && t[1] == one && t[2] == one && t[3] == one)) {
      tagged = (see >> (one & 63u)) & 1 ? 0xffffu : 0u;
    } else {
#pragma unroll
      for (int i = 0; i < kBlock; ++i) tagged |= (uint32_t)((see >> ((t[i / 4] >> (8 * (i & 3))) & 63u)) & 1) << i;
    }
    bits &= tagged;
  }
  bits |= below(u.prefix - base);
  return at >= 0 ? bits & below(hi - base) : 0u;
}

// Scores of a pair (in the first product's units) -> log2 units, capped, lowered, hidden.
__device__ inline void finish_scores(const AttendArgs& a, const Unit& u, int hi, int t0, const Pair& p, float c, float slope, int token, int position,
                                     uint64_t see, bool masked, float16v& s) {
  const int half = (threadIdx.x >> 5) & 1, base = t0 + 16 * half;
  const float f = c * (half ? p.ks[1] : p.ks[0]);
  if (a.cap_log2 > 0.f) {
    // cap * tanh(x / cap) = cap - 2 cap / (1 + e^(2 x / cap))
    const float g = f * a.cap_in;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = fmaf(-2.f * a.cap_log2, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s[i] * g)), a.cap_log2);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] *= f;
  }
  const int at = half ? p.at[1] : p.at[0], slot16 = half ? p.slot16[1] : p.slot16[0];
  if (a.slopes) {
    if (a.row_position) {
      const int4* pos = (const int4*)(a.slot_position + (int64_t)slot16 * kBlock);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int4 w = pos[i];
        s[4 * i] -= slope * fabsf((float)(position - w.x));
        s[4 * i + 1] -= slope * fabsf((float)(position - w.y));
        s[4 * i + 2] -= slope * fabsf((float)(position - w.z));
        s[4 * i + 3] -= slope * fabsf((float)(position - w.w));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] -= slope * fabsf((float)(token - base - i));
    }
  }
  if (masked) {
    const uint32_t bits = visible(a, u, hi, base, at, slot16, token, see);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = (bits >> i) & 1 ? s[i] : -INFINITY;
  }
}

// Whether some row of the wave may not see some of the tokens [t0, t1).
__device__ inline bool needs_mask(const AttendArgs& a, const Unit& u, int hi, int t0, int t1, int first_token) {
  return t1 > hi || (t1 > u.prefix && (a.row_see || t1 - 1 > first_token));
}

// Running state of a wave's rows.
template <int D>
struct State {
  float16v o[D / 32];
  float m, l;  // l: of this lane's tokens
  int e;       // exponent of the values in o
};

template <int D>
__device__ inline void start(State<D>& z) {
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int k = 0; k < 16; ++k) z.o[i][k] = 0.f;
  z.m = -INFINITY, z.l = 0.f, z.e = -126;
}

// N pairs of blocks under one maximum: their scores become the second product's operands.
template <int D, int N>
__device__ inline void soften(State<D>& z, float16v (&s)[N], const Pair (&p)[N], half8 (&w)[N][2]) {
  const int half = (threadIdx.x >> 5) & 1;
  float m = s[0][0];
  int e = z.e;
  bool odd = false;
#pragma unroll
  for (int n = 0; n < N; ++n) {
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, s[n][i]);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int x = (int)((__float_as_uint(p[n].vs[b]) >> 23) & 255) - 127;
      if (x == 128) odd = true;  // the block reads as NaN
      else if (p[n].at[b] >= 0) e = max(e, x);
    }
  }
  m = fmaxf(m, other_half(m));
  m = fmaxf(m, z.m);
  const float base = m == -INFINITY ? 0.f : m;
  float alpha = __builtin_amdgcn_exp2f(z.m - base);
  z.l *= alpha;
  if (e != z.e) alpha *= z.e - e < -126 ? 0.f : pow2f(z.e - e);
  if (__any(alpha != 1.f)) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int k = 0; k < 16; ++k) z.o[i][k] *= alpha;
  }
  z.m = m, z.e = e;
  float sum = 0.f;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const float vs = half ? p[n].vs[1] : p[n].vs[0];
    const float f = vs * pow2f(-e);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = __builtin_amdgcn_exp2f(s[n][i] - base);
      sum += x;
      float y = x * f;
      if (odd) y = s[n][i] == -INFINITY ? 0.f : y;
      s[n][i] = y;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) w[n][i / 8][i % 8] = (_Float16)s[n][i];
  }
  z.l += sum;
}

template <int D>
__device__ inline float16v score(const Rows<D>& r, const half8 (&k)[D / 16]) {
  float16v s;
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
  for (int i = 0; i < D / 16; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[i], r.q[i], s, 0, 0, 0);
  return s;
}

__device__ inline void store_out(const AttendArgs& a, int64_t at, float4v x) {  // four neighbouring values of the result
  uint2v w;
  if (a.dtype == kBf16) {
    for (int i = 0; i < 2; ++i) {
      uint32_t b[2];
      for (int k = 0; k < 2; ++k) {
        const uint32_t y = __float_as_uint(x[2 * i + k]);
        b[k] = x[2 * i + k] != x[2 * i + k] ? 0x7fc0u : (y + 0x7fffu + ((y >> 16) & 1)) >> 16;
      }
      w[i] = b[0] | b[1] << 16;
    }
  } else {
    for (int i = 0; i < 2; ++i) {
      union { half2v h; uint32_t u; } c;
      c.h[0] = (_Float16)x[2 * i], c.h[1] = (_Float16)x[2 * i + 1];
      w[i] = c.u;
    }
  }
  *(uint2v*)((uint16_t*)a.out + at) = w;
}

template <int CODES, int D>
__device__ inline void attend_few(const AttendArgs& a, const Unit& u, int head, float* lds) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, half = lane >> 5;
  const int n_pairs = (u.hi - u.lo + 31) >> 5;  // of the unit; this wave takes wave, wave + 4, ...
  Rows<D> r;
  State<D> z;
  start(z);
  Blocks b = load_blocks(a, u.request, head, u.lo + (wave + 4 * (lane >> 1)) * 32 + (lane & 1) * 16, u.hi);
  load_rows<D>(a, u, head, 0, r);
  const int first_token = u.pos0;
  uint4v k[D / 32], v[D / 32];
  Pair p = pair_of(b, 0);
  if (wave < n_pairs) {
    load_k<D>(a, p, k);
    load_v<D>(a, p, v);
  }
  for (int j = wave, i = 0; j < n_pairs; j += 4) {
    half8 kk[D / 16];
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      kk[2 * x] = codes_to_half8<CODES>(k[x][0], k[x][1]);
      kk[2 * x + 1] = codes_to_half8<CODES>(k[x][2], k[x][3]);
    }
    half8 vv[D / 32][2];
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      vv[x][0] = codes_to_half8<CODES>(v[x][0], v[x][1]);
      vv[x][1] = codes_to_half8<CODES>(v[x][2], v[x][3]);
    }
    const Pair now[1] = {p};
    const int t0 = u.lo + j * 32;
    if (j + 4 < n_pairs) {
      if (++i == 32) {
        i = 0;
        b = load_blocks(a, u.request, head, u.lo + (j + 4 + 4 * (lane >> 1)) * 32 + (lane & 1) * 16, u.hi);
      }
      p = pair_of(b, i);
      load_k<D>(a, p, k);
      load_v<D>(a, p, v);
    }
    float16v s[1] = {score<D>(r, kk)};
    const bool masked = needs_mask(a, u, u.hi, t0, t0 + 32, first_token) || now[0].at[0] < 0 || now[0].at[1] < 0;
    finish_scores(a, u, u.hi, t0, now[0], r.c, r.slope, r.token, r.position, r.see, masked, s[0]);
    half8 w[1][2];
    soften<D, 1>(z, s, now, w);
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      z.o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vv[x][0], w[0][0], z.o[x], 0, 0, 0);
      z.o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vv[x][1], w[0][1], z.o[x], 0, 0, 0);
    }
  }
  // the four waves meet
  constexpr int kPitch = D + 4;
  float* s_o = lds;                                       // [4][32][kPitch]
  float2v* s_ml = (float2v*)(lds + 4 * kRows * kPitch);   // [4][32]
  float l = z.l + other_half(z.l);
  if (half == 0) s_ml[wave * kRows + n] = float2v{z.m, l};
  __syncthreads();
  float m = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) m = fmaxf(m, s_ml[w * kRows + n][0]);
  const float base = m == -INFINITY ? 0.f : m;
  if (r.real) {
    const float f = __builtin_amdgcn_exp2f(z.m - base) * pow2f(z.e);
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(float4v*)(s_o + (wave * kRows + n) * kPitch + 32 * x + 8 * q + 4 * half) =
            float4v{z.o[x][4 * q] * f, z.o[x][4 * q + 1] * f, z.o[x][4 * q + 2] * f, z.o[x][4 * q + 3] * f};
  }
  __syncthreads();
  for (int i = threadIdx.x; i < u.n_rows * (D / 4); i += 256) {
    const int row = i / (D / 4), d = i % (D / 4) * 4;
    float mm = -INFINITY, ll = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, s_ml[w * kRows + row][0]);
    const float bb = mm == -INFINITY ? 0.f : mm;
    float4v o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      ll += s_ml[w * kRows + row][1] * __builtin_amdgcn_exp2f(s_ml[w * kRows + row][0] - bb);
      o += *(const float4v*)(s_o + (w * kRows + row) * kPitch + d);
    }
    if (u.part < 0) {
      const int64_t to = row_address(a, u.s0 + row, head);
      const float inv = ll == 0.f ? 0.f : 1.f / ll;
      store_out(a, to * D + d, o * inv);
      if (a.lse && d == 0) a.lse[to] = ll == 0.f ? -INFINITY : kLn2 * (mm + __builtin_amdgcn_logf(ll));
    } else {
      const int64_t to = (int64_t)(u.part + row) * a.g.Hkv + head;
      *(float4v*)(a.part_acc + to * D + d) = o;
      if (d == 0) a.part_ml[to] = float2v{mm, ll};
    }
  }
}

// LDS of the shared tiles: two buffers of 64 tokens, K and V as the products' operands, a lane's 16 bytes next to its neighbour's.
template <int D>
constexpr int kTileHalfs = 2 * 64 * D;  // K and V

template <int CODES, int D>
__device__ inline void attend_many(const AttendArgs& a, const Unit& u, int head, half8* lds) {
  constexpr int kPieces = D / 64;               // pieces of K, and of V, that a wave brings of a tile
  constexpr int kK = 64 * 2 * (D / 16);         // half8's of K in a tile; as many of V behind
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, half = lane >> 5;
  const int n_tiles = (u.hi - u.lo + 63) >> 6;
  const int sub = wave >> 1, piece0 = (wave & 1) * kPieces;  // this wave's share: pieces piece0 .. of 32-token half `sub`
  Rows<D> r;
  State<D> z;
  start(z);
  const bool works = wave * kRows < u.n_rows;
  Blocks b = load_blocks(a, u.request, head, u.lo + lane * 16, u.hi), ahead = b;
  load_rows<D>(a, u, head, wave * kRows, r);
  const int first_token = u.pos0 + (wave * kRows >> a.g_shift);
  const int last_token = u.pos0 + ((min(wave * kRows + kRows, u.n_rows) - 1) >> a.g_shift);
  uint4v k[kPieces], v[kPieces];
  auto request = [&](int tile) {
    if (tile && (tile & 15) == 0) ahead = load_blocks(a, u.request, head, u.lo + tile * 64 + lane * 16, u.hi);
    const Pair p = pair_of(ahead, 2 * (tile & 15) + sub);
    const int m = lane & 31;
    const int at = max((m & 4) ? p.at[1] : p.at[0], 0), atv = half ? p.at[1] : p.at[0];
    const uint8_t* from = a.k + (int64_t)at * (kBlock * D) + half * 256 + ((m >> 3) * 4 + (m & 3)) * 16;
    const uint8_t* fromv = a.v + (int64_t)max(atv, 0) * (kBlock * D) + (lane & 31) * 16;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      k[i] = *(const uint4v*)(from + (piece0 + i) * 512);
      v[i] = *(const uint4v*)(fromv + (piece0 + i) * 512);
    }
    if (p.at[0] < 0 || p.at[1] < 0)
#pragma unroll
      for (int i = 0; i < kPieces; ++i) v[i] = atv < 0 ? uint4v{0, 0, 0, 0} : v[i];
  };
  auto publish = [&](int tile) {
    half8* to = lds + (tile & 1) * 2 * kK;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int step = (sub * (D / 32) + piece0 + i) * 2;
      to[step * 64 + lane] = codes_to_half8<CODES>(k[i][0], k[i][1]);
      to[(step + 1) * 64 + lane] = codes_to_half8<CODES>(k[i][2], k[i][3]);
      to[kK + step * 64 + lane] = codes_to_half8<CODES>(v[i][0], v[i][1]);
      to[kK + (step + 1) * 64 + lane] = codes_to_half8<CODES>(v[i][2], v[i][3]);
    }
  };
  if (n_tiles > 0) {
    request(0);
    publish(0);
    if (n_tiles > 1) request(1);
  }
  __syncthreads();
  for (int j = 0; j < n_tiles; ++j) {
    if (j && (j & 15) == 0) b = load_blocks(a, u.request, head, u.lo + j * 64 + lane * 16, u.hi);
    const int t0 = u.lo + j * 64;
    if (works && (t0 <= last_token || t0 < u.prefix)) {
      const half8* from = lds + (j & 1) * 2 * kK;
      const Pair p[2] = {pair_of(b, 2 * (j & 15)), pair_of(b, 2 * (j & 15) + 1)};
      float16v s[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        half8 kk[D / 16];
#pragma unroll
        for (int i = 0; i < D / 16; ++i) kk[i] = from[(x * (D / 16) + i) * 64 + lane];
        s[x] = score<D>(r, kk);
      }
      const bool gone = p[0].at[0] < 0 || p[0].at[1] < 0 || p[1].at[0] < 0 || p[1].at[1] < 0;
      const bool masked = gone || needs_mask(a, u, u.hi, t0, t0 + 64, first_token);
#pragma unroll
      for (int x = 0; x < 2; ++x) finish_scores(a, u, u.hi, t0 + 32 * x, p[x], r.c, r.slope, r.token, r.position, r.see, masked, s[x]);
      half8 w[2][2];
      soften<D, 2>(z, s, p, w);
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
          for (int y = 0; y < 2; ++y)
            z.o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(from[kK + ((x * (D / 32) + i) * 2 + y) * 64 + lane], w[x][y], z.o[i], 0, 0, 0);
    }
    if (j + 1 < n_tiles) {
      publish(j + 1);
      if (j + 2 < n_tiles) request(j + 2);
    }
    __syncthreads();
  }
  if (!works) return;
  const float l = z.l + other_half(z.l);
  if (!r.real) return;
  const int row = wave * kRows + n;
  const float up = pow2f(z.e);
  if (u.part < 0) {
    const int64_t to = row_address(a, u.s0 + row, head);
    const float f = l == 0.f ? 0.f : up / l;
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        store_out(a, to * D + 32 * x + 8 * q + 4 * half, float4v{z.o[x][4 * q] * f, z.o[x][4 * q + 1] * f, z.o[x][4 * q + 2] * f, z.o[x][4 * q + 3] * f});
    if (a.lse && half == 0) a.lse[to] = l == 0.f ? -INFINITY : kLn2 * (z.m + __builtin_amdgcn_logf(l));
  } else {
    const int64_t to = (int64_t)(u.part + row) * a.g.Hkv + head;
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(float4v*)(a.part_acc + to * D + 32 * x + 8 * q + 4 * half) =
            float4v{z.o[x][4 * q] * up, z.o[x][4 * q + 1] * up, z.o[x][4 * q + 2] * up, z.o[x][4 * q + 3] * up};
    if (half == 0) a.part_ml[to] = float2v{z.m, l};
  }
}

template <int CODES, int D, bool MANY>
__global__ __launch_bounds__(256, 2) void k8_attend(AttendArgs a) {
  constexpr int kFewBytes = 4 * kRows * (D + 4) * 4 + 4 * kRows * 8;
  constexpr int kManyBytes = 2 * kTileHalfs<D> * 2;
  __shared__ __attribute__((aligned(16))) uint8_t lds[MANY && kManyBytes > kFewBytes ? kManyBytes : kFewBytes];
  const int i = blockIdx.x / a.g.Hkv, head = blockIdx.x % a.g.Hkv;
  if (i >= a.n_units[0]) return;
  const Unit u = a.units[i];
  if (MANY && u.n_rows > kRows)
    attend_many<CODES, D>(a, u, head, (half8*)lds);
  else
    attend_few<CODES, D>(a, u, head, (float*)lds);
}

// Joins the partial rows of the tiles whose tokens are split.  Work-group (tile, head, z) takes every gridDim.z-th row; 32 lanes hold a row's
// parts four dims apiece (D = 128), and the 256 / (D / 4) groups of lanes take a share of the parts each.
template <int D>
__global__ __launch_bounds__(256) void k8_merge(AttendArgs a) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
  __shared__ float4v s_o[kGroups][kLanes];
  __shared__ float s_l[kGroups];
  const int t = blockIdx.x / a.g.Hkv, head = blockIdx.x % a.g.Hkv;
  if (t >= a.n_units[1]) return;
  const Tile tile = a.tiles[t];
  if (tile.n_parts < 2) return;
  const int group = threadIdx.x / kLanes, d = threadIdx.x % kLanes;
  for (int row = blockIdx.y; row < tile.n_rows; row += gridDim.y) {
    const float2v* ml = a.part_ml + ((int64_t)(tile.part + row) * a.g.Hkv + head);
    const float* acc = a.part_acc + ((int64_t)(tile.part + row) * a.g.Hkv + head) * D;
    const int64_t step = (int64_t)tile.n_rows * a.g.Hkv;
    float m = -INFINITY;
    for (int k = threadIdx.x & 63; k < tile.n_parts; k += 64) m = fmaxf(m, ml[k * step][0]);
    for (int x = 32; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
    const float base = m == -INFINITY ? 0.f : m;
    float4v o{0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll 4
    for (int k = group; k < tile.n_parts; k += kGroups) {
      const float2v x = ml[k * step];
      const float f = __builtin_amdgcn_exp2f(x[0] - base);
      l += x[1] * f;
      o += *(const float4v*)(acc + k * step * D + 4 * d) * f;
    }
    s_o[group][d] = o;
    if (d == 0) s_l[group] = l;
    __syncthreads();
    if (group == 0) {
      for (int x = 1; x < kGroups; ++x) o += s_o[x][d], l += s_l[x];
      const int64_t to = row_address(a, tile.s0 + row, head);
      const float inv = l == 0.f ? 0.f : 1.f / l;
      store_out(a, to * D + 4 * d, o * inv);
      if (a.lse && d == 0) a.lse[to] = l == 0.f ? -INFINITY : kLn2 * (m + __builtin_amdgcn_logf(l));
    }
    __syncthreads();
  }
}

}  // namespace k8
