// Attention over the 4-bit cache.
//
// Rows, units, marks and the hiding of scores are those of the 8-bit cache (k8_attend.hpp); codes and scales enter differently.  With f = |scale| * log2(e)
// and 2^ev_j the scale of token j's V, all scores in log2 units:
//
//   t_j = f * (q . K_j)   (capped, lowered by distance)       m ~ max (t_j + ev_j)         y_j = 2^(t_j + ev - m)
//   l   = 2^-ev sum y_j       O = sum y_j 2^(ev_j - ev) V4_j       out = O / l             lse = ln 2 * (m + log2 l)
//
// ev is the largest ev_j of 16 tokens.
//   q . K   operands of q's type, which enters as it is.  A code times its scale is a bf16 number, which one conversion gives of two codes: K's scales, one to a
//           token and 32 dims, cost nothing (and 255 among them gives numbers that are none).  In fp16 it is one, too, in units of a power of two from which the
//           scales are at most 2^13 away; a wave goes by that of its first token, and where scales are further away a pair's products are taken window by window.
//   P . V   fp16 operands.  A token's V scale must stay outside of the product over tokens: a power of two up to 2^-8 below the block's largest, times which
//           the weight, rounded to fp16 before that, stays as exact.  Where a block's scales are further apart, or one of them is further below the largest so
//           far, or not a number, the step takes scores t_j + ev_j instead, token by token, and sums l from t_j apart (rare: V's rows of a model differ by
//           a few powers of two).
// Weights rounded to fp16, each by at most 2^-11 of itself or 2^-25 (which is 2^-24 of the row's largest product of weight and scale, or less), are the only rounding
// that fp32 does not see.
//
// Products are transposed, S^T = K Q^T and O^T = V^T P^T, in 32x32x16 steps over 32 tokens x 32 stacked rows.  A lane's piece of K is 16 bytes, the 32 dims of
// one token under one scale; its piece of V 16 bytes, two neighbouring dims of a block's 16 tokens, which go to two products' rows: the dims of a product are
// every second of 64.  The scores that a lane gets (16 tokens of one block, one row) are its operand of the second product, as in the 8-bit cache.  Units with at
// most 16 rows go in steps of another shape (k4_few.hpp).
//
// What bounds it (8 kv heads of 128; a layer):
//   8 streams over 8k tokens, 11 MB        9.6 us: the ramp, as in the 8-bit cache (11.1): a work-group has 1.3 steps' worth to each wave; 2.5 of launch
//   16 ragged requests, capped, 50 MB      20.0 us: units with more than 16 rows, 15 of these us and more in a wave's chain from step to step, ramp and end 4; vector
//                                          instructions, 23 a score, are busy half of the time, and ten percent fewer (the cap by a series) changed nothing
//   2048 x 4 rows over 8k tokens, 309 GF   329 us once the card's clocks have settled (325 to 350 by the card; 360 to 416 in the first thirty launches), 880 to 950
//                                          TFLOP/s (740 to 860) against 1190 of a large library product: vector instructions busy 68% of the time, matrix
//                                          instructions 42%.  2048 rows that end 8k tokens: plain 264 us, with tags 340, capped 370; of 64 dims 178, with tags 235
// Tried and not taken: the scaled matrix instruction on the codes themselves with q split into e4m3 parts (its sums are off by 1.5e-4 of their terms' magnitudes,
// a hundred times as much as a sum in fp32), eight waves to a work-group (8 streams over 8k 109 -> 110 us a pass, the prompt 389 -> 415), the first blocks in scalar
// registers (no change), Q's rows loaded whole and turned in LDS (the prompt 333 -> 338).
#pragma once
#include "k4_dev.hpp"
#include "k8_attend.hpp"

namespace k4 {

struct AttendArgs : k8::AttendArgs {
  const uint8_t *k_scale, *v_scale;  // of the layer
};

constexpr int kNear = 8;      // powers of two between a block's V scales that its weights bear
constexpr float kLift = 7.f;  // The base of the scores is set 2^7 below their maximum and follows when that is 2^15 ahead, which fp16 still holds: so its
                              // smallest normal number is 2^-21 of the largest weight or less, times 2^kNear where that is one of a small V scale

// The sums l are held 2^-kRoom times: a token's term is between 2^-112 (V's scale 2^119, the weight 2^7) and 2^115 (2^-100, as of a V of zeros, and 2^15), of which
// 2^13 are no fp32 number, but 2^25 times 2^-12 are.  (A multiplication a step: prompts within 1.5% of what they took, the rest within what two runs differ by.)
constexpr float kRoom = 12.f, kLess = 0x1p-12f;

__device__ inline float lse_of(float m, float l) { return l == 0.f ? -INFINITY : kLn2 * (m + (__builtin_amdgcn_logf(l) + kRoom)); }

// A wave's rows of Q, as pieces of 8 dims: lane n and n + 32 hold row n, group 2x + half of the dims at 4x .. 4x + 3.  With 16 rows, lanes n, n + 16, ..
// each a quarter of the dims.
template <int D, bool MARKS, int ROWS = kRows>
__device__ inline void request_rows(const AttendArgs& a, const Unit& u, int head, int first, Rows<D>& r, uint4v (&raw)[D * ROWS / 512]) {
  const int lane = threadIdx.x & 63, n = lane & (ROWS - 1), part = lane / ROWS;
  r.real = first + n < u.n_rows;
  const int s = u.s0 + (r.real ? first + n : 0);  // (a lane without a row computes the first one's, and nobody looks)
  const uint4v* p = (const uint4v*)((const uint16_t*)a.q + row_address(a, s, head) * D);
#pragma unroll
  for (int k = 0; k < D * ROWS / 512; ++k) raw[k] = p[ROWS == kRows ? (2 * (k >> 2) + part) * 4 + (k & 3) : part * (D / 32) + k];
  r.token = u.pos0 + ((first + n) >> a.g_shift);
  r.first_token = u.pos0 + (first >> a.g_shift);
  r.slope = a.slopes[head * a.g.G + (s & (a.g.G - 1))] * kLog2e;
  if constexpr (MARKS) {
    r.see = a.row_see[s >> a.g_shift];
    r.position = (uint32_t)a.row_position[s >> a.g_shift] ^ 0x80000000u;
  } else {
    r.see = 0, r.position = 0;
  }
}

// 32 tokens whose codes and scales a lane holds its pieces of.
template <int D>
struct Codes {
  uint4v k[D / 64], v[D / 64];
  uint32_t ks;  // scales of the token of the lane's row of the first product, a byte to a group of dims
  uint32_t vs;  // V's scales of tokens 2i, 2i + 1 of block lane >> 5, i = lane & 7
};

// Row m = 8a + 4h + b of the first product is token 4a + b of block h.
template <int D>
__device__ inline void load_k(const AttendArgs& a, int at0, int at1, Codes<D>& c) {
  const int lane = threadIdx.x & 63, m = lane & 31, half = lane >> 5, token = (m >> 3) * 4 + (m & 3);
  const int64_t at = max((m & 4) ? at1 : at0, 0), block = max(half ? at1 : at0, 0);
  const uint8_t* from = a.k + at * kCodeBytes(D) + (half * kBlock + token) * 16;
#pragma unroll
  for (int x = 0; x < D / 64; ++x) c.k[x] = *(const uint4v*)(from + x * 2 * kBlock * 16);
  if constexpr (D == 128)
    c.ks = *(const uint32_t*)(a.k_scale + (at * kBlock + token) * 4);
  else
    c.ks = *(const uint16_t*)(a.k_scale + (at * kBlock + token) * 2);
  c.vs = *(const uint16_t*)(a.v_scale + block * kBlock + 2 * (lane & 7));
}

template <int D>
__device__ inline void load_v(const AttendArgs& a, int at0, int at1, Codes<D>& c) {
  const int lane = threadIdx.x & 63;
  const int64_t at = max((lane & 32) ? at1 : at0, 0);
  const uint8_t* from = a.v + at * kCodeBytes(D) + (lane & 31) * 16;
#pragma unroll
  for (int x = 0; x < D / 64; ++x) c.v[x] = *(const uint4v*)(from + x * 512);
}

// Eight codes of K under their scale (or that in other units), as an operand.
template <bool F16>
__device__ inline uint4v k_operand(uint32_t w, float scale) {
  if constexpr (F16) {
    union { half2v p[4]; uint4v v; } r;
    r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0);
    r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1);
    r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2);
    r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3);
    return r.v;
  } else {
    union { bf16x2 p[4]; uint4v v; } r;
    r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
    return r.v;
  }
}

__device__ inline float uniform(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }

template <bool F16>
__device__ inline float16v product(const uint4v& k, const uint4v& q, const float16v& s) {
  union { uint4v w; half8 h; bf16x8 b; } x{k}, y{q};
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(x.h, y.h, s, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.b, y.b, s, 0, 0, 0);
}

// fp16's window of K's scales: a code times 2^-13 .. 2^13 is a normal fp16 number.  (Down to 2^-23 it is one, too, but of those sums of products keep fewer bits:
// scores of 2^-23 were ten times as far off.)  `unit` is the byte of the scale that is 1.
constexpr int kAside = 13;
__device__ inline float unit_scale(int unit) { return pow2f(unit - 127); }

// Whether all scales of the lane's token lie in the window.
template <int D>
__device__ inline bool in_window(uint32_t ks, int unit) {
  using short2v = __attribute__((ext_vector_type(2))) unsigned short;
  union { uint32_t w; short2v v; } even, odd, low, high;
  even.w = ks & 0x00ff00ffu, odd.w = D == 128 ? ks >> 8 & 0x00ff00ffu : ks >> 8;
  if constexpr (D == 64) even.w |= even.w << 16, odd.w |= odd.w << 16;  // (two scales)
  low.w = (uint32_t)(unit - kAside) * 0x10001u, high.w = (uint32_t)(unit + kAside) * 0x10001u;
  const short2v most = __builtin_elementwise_max(even.v, odd.v), least = __builtin_elementwise_min(even.v, odd.v);
  union { short2v v; uint32_t w; } off{__builtin_elementwise_sub_sat(most, high.v) | __builtin_elementwise_sub_sat(low.v, least)};
  return off.w == 0;
}

__device__ inline half8 v_operand(uint32_t w) {
  union { half2v p[4]; half8 v; } r;
  r.p[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 0);
  r.p[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 1);
  r.p[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 2);
  r.p[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.f, 3);
  return r.v;
}

// What is known of a pair's tokens once their scales are there: lane i of each row of 16 lanes holds that of tokens 2i and 2i + 1 of its half's block.
struct Scales {
  float ev;      // largest exponent of the block's V scales (of none, the largest so far)
  uint32_t low;  // 2^(ev_j - ev) of the two tokens, as fp16
  uint32_t vs;   // their bytes; those that do not count are the block's largest
  bool rare;     // for the wave: more than the above is needed
};

__device__ inline int row_largest(int x) {  // of a row of 16 lanes, of which i and i + 8 hold the same
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x124, 0xf, 0xf, false));  // row_ror
  x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x122, 0xf, 0xf, false));
  return max(x, __builtin_amdgcn_update_dpp(0, x, 0x121, 0xf, 0xf, false));
}

template <int BLOCKS>
__device__ inline int largest_block(int x) {  // of what is the same in a block's lanes
  const auto halves = __builtin_amdgcn_permlane32_swap((uint32_t)x, (uint32_t)x, false, false);
  x = max((int)halves[0], (int)halves[1]);
  if constexpr (BLOCKS == 2) return x;
  const auto rows = __builtin_amdgcn_permlane16_swap((uint32_t)x, (uint32_t)x, false, false);
  return max((int)rows[0], (int)rows[1]);
}

template <int BLOCKS>
__device__ inline Scales scales_of(uint32_t vs, int absent, int t0, int hi, int& most) {
  Scales s;
  int b0 = vs & 255, b1 = vs >> 8;
  bool some = true, nan = false;
  int up = row_largest(max(b0, b1));
  const bool cut = t0 + BLOCKS * kBlock > hi || absent, all = !__any(up == kNone) && !cut;  // (the same for the whole wave)
  if (__builtin_expect(!all, 0)) {  // tokens that there are not, or whose V is not a number, are left out: they get the largest of the others
    const int block = lanes_block<BLOCKS>(), left = (absent >> block) & 1 ? 0 : min(max(hi - (t0 + 16 * block + 2 * (int)(threadIdx.x & 7)), 0), 2);
    const bool n0 = left > 0 && b0 == kNone, n1 = left > 1 && b1 == kNone;
    up = row_largest(max(left > 0 && !n0 ? b0 : 0, left > 1 && !n1 ? b1 : 0));
    some = up > 0, nan = n0 || n1;
    most = max(most, largest_block<BLOCKS>(up));
    up = some ? up : most;
    s.vs = (uint32_t)(n0 || left < 1 ? (n0 ? kNone : up) : b0) | (uint32_t)(n1 || left < 2 ? (n1 ? kNone : up) : b1) << 8;
    b0 = left < 1 || n0 ? up : b0, b1 = left < 2 || n1 ? up : b1;
  } else {
    most = max(most, largest_block<BLOCKS>(up));
    s.vs = vs;
  }
  s.ev = (float)(up - 127);
  s.low = 0x3c003c00u - ((uint32_t)(up - b0) << 10) - ((uint32_t)(up - b1) << 26);
  s.rare = __any(nan || max(up - b0, up - b1) > kNear || (some && up < most - kScaleSpan));
  return s;
}

template <int D>
__device__ inline void times(State<D>& z, float x) {
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int k = 0; k < 16; ++k) z.o[i][k] *= x;
}

// How far a maximum may be ahead of the scores' base before that follows.  Where a base is beyond kFar, nothing: there fp32's steps are half a unit and more, so
// that t_j + ev - m, rounded, and what it is compared with, rounded on its own way, may be any number of units apart; t_j + ev is rounded first there, and then
// no weight is above 2^8.  (Kept out of the way of all other steps: a prompt's pass 337 -> 338 us, the smallest call 14.7 -> 15.2, batches within 1%.)
constexpr float kAhead = kSlack + kLift, kFar = 0x1p22f;

// N pairs (of BLOCKS blocks) and G groups of rows: their scores (times f) become the second product's operands.
template <int BLOCKS, class Z, int G, int N>
__device__ inline void soften(Z (&z)[G], float& slack, float16v (&s)[G][N], float (&f)[G][N], Scales (&p)[N], half8 (&w)[G][N][2]) {
  bool rare = false;
#pragma unroll
  for (int n = 0; n < N; ++n) rare |= p[n].rare;
  float back[N], own_m[G][N], own_l[G][N];
#pragma unroll
  for (int n = 0; n < N; ++n) back[n] = __builtin_amdgcn_exp2f(-p[n].ev);
  if (__builtin_expect(rare, 0)) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        own_m[g][n] = -FLT_MAX, own_l[g][n] = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[g][n][i] *= f[g][n], own_m[g][n] = fmaxf(own_m[g][n], s[g][n][i]);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          own_l[g][n] += __builtin_amdgcn_exp2f(s[g][n][i] - own_m[g][n]);
          __builtin_amdgcn_sched_barrier(0);  // (one after the other, or registers run out)
        }
        f[g][n] = 1.f;
      }
      each<16>([&](auto i) {
        const int byte = of_row<i.value / 2>((int)p[n].vs) >> (8 * (i.value & 1)) & 255;
        const float e = byte == kNone ? p[n].ev : (float)(byte - 127);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const int seen = byte == kNone && s[g][n][i.value] != -INFINITY ? 0x7fc00000 : 0;  // (without a branch)
          z[g].bad = __uint_as_float(__float_as_uint(z[g].bad) | seen);
          s[g][n][i.value] += e;
        }
        __builtin_amdgcn_sched_barrier(0);
      });
      p[n].ev = 0.f, p[n].low = 0x3c003c00u, back[n] = 0.f;
    }
  }
  float m[G];
  bool ahead = false;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    m[g] = -FLT_MAX;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float most = s[g][n][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) most = fmaxf(most, s[g][n][i]);
      m[g] = fmaxf(m[g], fmaf(most, f[g][n], p[n].ev));
    }
    m[g] = fmaxf(m[g], other_half(m[g]));
    if constexpr (BLOCKS == 4) {
      const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(m[g]), __float_as_uint(m[g]), false, false);
      m[g] = fmaxf(__uint_as_float(rows[0]), __uint_as_float(rows[1]));
    }
    ahead |= m[g] > z[g].m + slack;
  }
  if (__builtin_expect(__any(ahead), 0)) {
    bool far = false;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const float to = fmaxf(m[g] - kLift, z[g].m), h = root_exp2(z[g].m - to), alpha = h * h;
      const bool fresh = z[g].m == -FLT_MAX;  // (nothing so far)
      z[g].m = to;
      z[g].l = z[g].l * h * h;
      if (!__all(fresh)) times(z[g], alpha);
      far |= fabsf(to) >= kFar && to != -FLT_MAX;
    }
    slack = __any(far) ? 0.f : kAhead;
  }
  if (__builtin_expect(slack == 0.f, 0)) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float to = f[g][n];
        asm volatile("" : "+v"(to));  // (or else this is done ahead of the branch)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[g][n][i] = fmaf(s[g][n][i], to, p[n].ev);
          __builtin_amdgcn_sched_barrier(0);
        }
        f[g][n] = 1.f;
      }
      p[n].ev = 0.f;
    }
  }
  if (__builtin_expect(rare, 0)) {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const float h = root_exp2(own_m[g][n] - z[g].m - kRoom);
        z[g].l = fmaf(own_l[g][n] * h, h, z[g].l);
      }
  }
#pragma unroll
  for (int n = 0; n < N; ++n) {
    float off[G], sum[G];
#pragma unroll
    for (int g = 0; g < G; ++g) off[g] = p[n].ev - z[g].m, sum[g] = 0.f;
    each<8>([&](auto i) {
      union { int w; half2v h; } low{of_row<i.value>((int)p[n].low)};
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const float y0 = __builtin_amdgcn_exp2f(fmaf(s[g][n][2 * i.value], f[g][n], off[g]));
        const float y1 = __builtin_amdgcn_exp2f(fmaf(s[g][n][2 * i.value + 1], f[g][n], off[g]));
        sum[g] += y0, sum[g] += y1;
        const half2v h = __builtin_convertvector((float2v{y0, y1}), half2v) * low.h;
        w[g][n][i.value / 4][2 * i.value % 8] = h[0], w[g][n][i.value / 4][2 * i.value % 8 + 1] = h[1];
      }
    });
#pragma unroll
    for (int g = 0; g < G; ++g) z[g].l = fmaf(sum[g] * kLess, back[n], z[g].l);
  }
}

// Scores of a pair whose K scales do not share a window, fp16: window by window, the smallest first, in units that go up with them (what gets lost so is 2^-126 of
// the next one's).  Returns the last one's unit.
template <int D, int G, int N>
__device__ inline int windows(const Codes<D>& c, bool there, const uint4v* q, float16v (&s)[G][N], int n) {
  constexpr int kWide = 2 * kAside, kWindows = 256 / kWide + 1;
  const int half = (threadIdx.x >> 5) & 1;
  int byte[D / 64], unit = -1;
#pragma unroll
  for (int x = 0; x < D / 64; ++x) byte[x] = there ? (int)(c.ks >> (8 * (2 * x + half)) & 255u) : kNone;  // (those have no window)
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int i = 0; i < 16; ++i) s[g][n][i] = 0.f;
#pragma unroll 1
  for (int w = 0; w < kWindows; ++w) {
    bool some = w == kWindows - 1 && unit < 0;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) some |= byte[x] != kNone && byte[x] / kWide == w;
    if (!__any(some)) continue;
    const int next = kWide * w + kAside;
    const float down = unit < 0 ? 1.f : pow2f(max(unit - next, -126));
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[g][n][i] *= down;
    unit = next;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) {
      const bool mine = byte[x] == kNone || byte[x] / kWide == w;  // (not a number: in every window)
      const float scale = __uint_as_float(byte[x] == kNone ? 0x7f800000u : (uint32_t)((mine ? byte[x] - next : 0) + 127) << 23);
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const uint4v codes = k_operand<true>(mine ? c.k[x][y] : 0u, scale);
#pragma unroll
        for (int g = 0; g < G; ++g) s[g][n] = product<true>(codes, q[(g * (D / 16) + 4 * x + y) * 64 + (threadIdx.x & 63)], s[g][n]);
      }
    }
  }
  return unit;
}

// One step of a wave: N pairs whose codes are in c, against G groups of 32 rows.  `ahead` is called when K may be overwritten, `behind` when V may.
template <int D, bool F16, int KIND, int G, int N, class Ahead, class Behind>
__device__ inline void step(const AttendArgs& a, const Unit& u, const Rows<D> (&r)[G], const uint4v* q, int unit, State<D> (&z)[G], Codes<D> (&c)[N],
                            const int (&absent)[N], const Marks (&marks)[N], const int (&t0)[N], int& most, float& slack, Ahead ahead, Behind behind) {
  float16v s[G][N];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[g][n][i] = 0.f;
  const int half = (threadIdx.x >> 5) & 1;
  // A wave at the matrix pipe goes first: else the older of a SIMD's two runs ahead, and the younger ends alone.
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int x = 0; x < D / 64; ++x) {
    float scale[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const uint32_t bits = (c[n].ks >> (8 * (2 * x + half)) & 255u) << 23;
      scale[n] = __uint_as_float(F16 ? bits + ((uint32_t)(127 - unit) << 23) : bits);
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      uint4v codes[N];
#pragma unroll
      for (int n = 0; n < N; ++n) codes[n] = k_operand<F16>(c[n].k[x][y], scale[n]);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const uint4v row = q[(g * (D / 16) + 4 * x + y) * 64 + (threadIdx.x & 63)];
#pragma unroll
        for (int n = 0; n < N; ++n) s[g][n] = product<F16>(codes[n], row, s[g][n]);
      }
    }
  }
  __builtin_amdgcn_s_setprio(0);
  float f[G][N];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int n = 0; n < N; ++n) f[g][n] = F16 ? uniform(a.scale_log2 * unit_scale(unit)) : a.scale_log2;
  if constexpr (F16) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int m = threadIdx.x & 31, at = t0[n] + (m & 4 ? 16 : 0) + (m >> 3) * 4 + (m & 3);  // the lane's token of the first product
      const bool there = at < u.hi && !(absent[n] >> (m >> 2 & 1) & 1);
      if (__builtin_expect(__any(there && !in_window<D>(c[n].ks, unit)), 0)) {
        const int last = windows(c[n], there, q, s, n);
#pragma unroll
        for (int g = 0; g < G; ++g) f[g][n] = uniform(a.scale_log2 * unit_scale(last));
      }
    }
  }
  Marks m[N];
  Scales p[N];
#pragma unroll
  for (int n = 0; n < N; ++n) m[n] = marks[n], p[n] = scales_of<2>(c[n].vs, absent[n], t0[n], u.hi, most);
  ahead();
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const Pair pair{1.f, 0.f, absent[n], 0, 0};
      if constexpr (KIND == kMarked)
        finish_scores<KIND>(a, u.prefix, u.hi, t0[n], pair, Marked{m[n], r[g].position, r[g].by_tag}, r[g].slope, r[g].token, r[g].first_token, f[g][n], s[g][n]);
      else
        finish_scores<KIND>(a, u.prefix, u.hi, t0[n], pair, Unmarked{}, r[g].slope, r[g].token, r[g].first_token, f[g][n], s[g][n]);
    }
  half8 w[G][N][2];
  k4::soften<2>(z, slack, s, f, p, w);
  __builtin_amdgcn_s_setprio(1);
  __builtin_amdgcn_sched_barrier(0);  // (V's codes are turned as they are needed: all at once they take 64 registers more)
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const half8 codes = v_operand(c[n].v[x / 2][2 * (x & 1) + y]);
#pragma unroll
        for (int g = 0; g < G; ++g) z[g].o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes, w[g][n][y], z[g].o[x], 0, 0, 0);
      }
  __builtin_amdgcn_s_setprio(0);
  behind();
}

// A unit of G groups of 32 rows.  Every wave takes a quarter of the tokens, pairs wave, wave + 4, ...; the four meet at the end.  Two pairs at a time, so that a
// softmax's way through its lanes is taken once for 64 tokens; with two groups and 128 dims there are registers for one.  Q's operands lie in LDS, a copy for
// each wave (where its output goes later).
template <int D, bool F16, int KIND, int G>
__device__ inline void attend_unit(const AttendArgs& a, const Unit& u, int listed, int head, float* lds) {
  constexpr bool MARKS = KIND == kMarked;
  constexpr int N = G == 1 || D == 64 ? 2 : 1;
  static_assert(G * (D / 16) * 64 * 16 <= kRows * kPitch<D> * 4, "Q's operands lie where the output goes");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 31, half = lane >> 5;
  const int n_pairs = max((((u.hi - u.lo + 31) >> 5) - wave + 3) >> 2, 0);  // this wave's
  uint4v* q = (uint4v*)(lds + wave * kRows * kPitch<D>);
  Rows<D> r[G];
  State<D> z[G];
  Blocks b;
  uint64_t gone;
  int most = kEMin + 127;  // largest byte of V's scales so far
  float slack = kAhead;
  Codes<D> c[N];
  Marks marks[N] = {};
  auto token = [&](int i) { return u.lo + (wave + 4 * i) * 32; };  // first of the wave's i-th pair
  auto find = [&](int i) { find_blocks(a, u.request, head, token(i + (lane >> 1)) + (lane & 1) * 16, u.hi, b), gone = __ballot(b.at < 0); };
  auto k_ahead = [&](int i, int to) {
    const int x = 2 * (i & 31);
    load_k<D>(a, __builtin_amdgcn_readlane(b.at, x), __builtin_amdgcn_readlane(b.at, x + 1), c[to]);
  };
  auto v_ahead = [&](int i, int to) {
    const int x = 2 * (i & 31);
    load_v<D>(a, __builtin_amdgcn_readlane(b.at, x), __builtin_amdgcn_readlane(b.at, x + 1), c[to]);
  };
  auto absent_of = [&](int i) { return (int)(gone >> (2 * (i & 31))) & 3; };
  {
    // Everything is asked for before anything is waited for: loads come back in their order.  (Where the wave has fewer than N pairs, block 0 is read in
    // their place.)
    uint4v raw[D / 16];
    k4::request_rows<D, MARKS>(a, u, head, 0, r[0], raw);
    __builtin_amdgcn_sched_barrier(0);
    if (u.hi - u.lo <= kUnitBlocks * kBlock)
      on_block(a, 2 * (wave + 4 * (lane >> 1)) + (lane & 1) < kUnitBlocks ? listed : -1, head, b), gone = __ballot(b.at < 0);
    else
      find(0);
#pragma unroll
    for (int n = 0; n < N; ++n)
      if constexpr (MARKS) marks[n] = load_marks(a, b, n);
#pragma unroll
    for (int n = 0; n < N; ++n) k_ahead(n, n);
#pragma unroll
    for (int n = 0; n < N; ++n) v_ahead(n, n);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      if (g) k4::request_rows<D, MARKS>(a, u, head, g * kRows, r[g], raw);
      if constexpr (MARKS) r[g].by_tag = rows_by_tag(r[g].see, a.g_shift);
      const uint32_t sign = a.negate ? 0x80008000u : 0u;
      if (a.negate)  // (the same for all lanes)
#pragma unroll
        for (int y = 0; y < D / 16; ++y) raw[y] ^= uint4v{sign, sign, sign, sign};
#pragma unroll
      for (int y = 0; y < D / 16; ++y) q[(g * (D / 16) + y) * 64 + lane] = raw[y];
    }
  }
  int unit = 127;
  if constexpr (F16) {
    const int byte = __builtin_amdgcn_readfirstlane(c[0].ks) & 255;  // of the wave's first token
    unit = (gone & 1) || byte == kNone ? 127 : min(max(byte, kEMin + 127), kNone - 1 - kAside);  // (kNone lies in no window)
  }
#pragma unroll
  for (int g = 0; g < G; ++g) start(z[g]);
  int i = 0;
  for (; i + N - 1 < n_pairs; i += N) {
    int t0[N], absent[N];
#pragma unroll
    for (int n = 0; n < N; ++n) t0[n] = token(i + n), absent[n] = absent_of(i + n);
    k4::step<D, F16, KIND, G, N>(a, u, r, q, unit, z, c, absent, marks, t0, most, slack,
      [&] {
        if (i + N >= n_pairs) return;
        if (((i + N) & 31) == 0) find(i + N);
#pragma unroll
        for (int n = 0; n < N; ++n)
          if constexpr (MARKS) marks[n] = load_marks(a, b, (i + N + n) & 31);
#pragma unroll
        for (int n = 0; n < N; ++n) k_ahead(i + N + n, n);
      },
      [&] {
        if (i + N >= n_pairs) return;
#pragma unroll
        for (int n = 0; n < N; ++n) v_ahead(i + N + n, n);
      });
  }
  if constexpr (N == 2) {
    if (i < n_pairs) {
      const int t0[1] = {token(i)}, absent[1] = {absent_of(i)};
      const Marks last[1] = {marks[0]};
      k4::step<D, F16, KIND, G, 1>(a, u, r, q, unit, z, *(Codes<D>(*)[1]) & c, absent, last, t0, most, slack, [] {}, [] {});
    }
  }
  // The four waves meet, group after group.  Each gives three quarters of its output to the others and joins the fourth with theirs: quarter y of a lane's
  // is o[..][4y .. 4y + 3], of each 64 dims the eight from 16 y + 8 half on, which go through LDS as they lie in the registers.
  constexpr int kPieces = D / 32;  // float4s of a quarter
  float4v* s_o = (float4v*)lds;    // [4] waves, kPitch * kRows floats apart: [4] quarters [kPieces][64]
  float2v* s_ml = (float2v*)(lds + 4 * kRows * kPitch<D>);  // [4][32]
  auto at = [&](int w, int y, int k) { return w * (kRows * kPitch<D> / 4) + (y * kPieces + k) * 64 + lane; };
#pragma unroll
  for (int g = 0; g < G; ++g) {
    if (g && u.n_rows <= g * kRows) break;
    const float l = z[g].l + other_half(z[g].l);
    poison(z[g]);
    if (g) __syncthreads();
    if (half == 0) s_ml[wave * kRows + row] = float2v{z[g].m, l};
    // o[2X + j][4y + b] is dim 64 X + 2 (8y + 4 half + b) + j
    auto piece = [&](int y, int k) {
      const int x = k / 2, b = 2 * (k % 2);
      return float4v{z[g].o[2 * x][4 * y + b], z[g].o[2 * x + 1][4 * y + b], z[g].o[2 * x][4 * y + b + 1], z[g].o[2 * x + 1][4 * y + b + 1]};
    };
    float4v own[kPieces];
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int k = 0; k < kPieces; ++k) {
        if (y == wave) own[k] = piece(y, k);  // (the same for the whole wave)
        else s_o[at(wave, y, k)] = piece(y, k);
      }
    __syncthreads();
    float2v ml[4];
    float4v part[3][kPieces];
#pragma unroll
    for (int w = 0; w < 4; ++w) ml[w] = s_ml[w * kRows + row];
#pragma unroll
    for (int i = 0; i < 3; ++i)
#pragma unroll
      for (int k = 0; k < kPieces; ++k) part[i][k] = s_o[at(i + (i >= wave), wave, k)];
    const float m = fmaxf(fmaxf(ml[0][0], ml[1][0]), fmaxf(ml[2][0], ml[3][0]));
    float all = 0.f, factor[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float h = root_exp2(ml[w][0] - m);
      all = fmaf(ml[w][1] * h, h, all);
      factor[w] = h * h;
    }
    const float mine = wave < 2 ? (wave == 0 ? factor[0] : factor[1]) : (wave == 2 ? factor[2] : factor[3]);
    if (!r[g].real) continue;
    const int s = u.s0 + g * kRows + row, first = 16 * wave + 8 * half;
    const int64_t to = u.part < 0 ? row_address(a, s, head) : (int64_t)(u.part + g * kRows + row) * a.g.Hkv + head;
    const float inverse = inverse_of(all) * kLess;
#pragma unroll
    for (int x = 0; x < D / 64; ++x) {
      float4v o[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        o[k] = own[2 * x + k] * mine;
#pragma unroll
        for (int i = 0; i < 3; ++i) o[k] += part[i][2 * x + k] * (i >= wave ? factor[i + 1] : factor[i]);
      }
      if (u.part < 0) {
        store_out(a, to * D + 64 * x + first, o[0] * inverse);
        store_out(a, to * D + 64 * x + first + 4, o[1] * inverse);
      } else {
        float4v* p = (float4v*)(a.part_acc + to * D + 64 * x + first);
        p[0] = o[0] * kLess, p[1] = o[1] * kLess;
      }
    }
    if (wave == 0 && half == 0) {
      if (u.part >= 0) a.part_ml[to] = float2v{m + kRoom, all};
      else if (a.lse) a.lse[to] = k4::lse_of(m, all);
    }
  }
}

// Two groups at a time do not fit the registers with 128 dims and scores that are capped, lowered or hidden by tags: then a work-group (blockIdx.y) takes each.
// (2048 rows over 8k tokens, plain: 336 us in bf16, 348 in fp16, which spills a few registers in `rare`; a work-group each 390.)
template <int D, int KIND>
constexpr bool kApart = D == 128 && KIND != kPlain;

}  // namespace k4

#include "k4_few.hpp"

namespace k4 {

template <int D, bool F16, bool MANY, int KIND>
__global__ __launch_bounds__(256, 2) void k4_attend(AttendArgs a) {
  __shared__ __attribute__((aligned(16))) float lds[4 * kRows * kPitch<D> + 4 * kRows * 2];
  const int head = blockIdx.x % a.g.Hkv, unit = blockIdx.x / a.g.Hkv, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Unit u = a.units[unit];
  // the lane's block, asked for together with the unit: pairs are dealt out to the four waves
  const int listed = a.unit_blocks[unit * kUnitBlocks + min(2 * (wave + 4 * (lane >> 1)) + (lane & 1), kUnitBlocks - 1)];
  const int few = MANY ? 0 : a.unit_blocks[unit * kUnitBlocks + min(4 * (wave + 4 * (lane >> 2)) + (lane & 3), kUnitBlocks - 1)];  // (fours, in attend_few)
  asm volatile("" ::"s"(u.request), "s"(u.s0), "s"(u.pos0), "s"(u.lo), "s"(u.hi), "s"(u.prefix), "s"(u.part));  // (one load, ahead of the branch)
  if constexpr (MANY && kApart<D, KIND>) {
    const int first = blockIdx.y * kRows;
    u.s0 += first, u.n_rows = min(u.n_rows - first, kRows), u.pos0 += first >> a.g_shift;
    if (u.part >= 0) u.part += first;
  }
  if (u.n_rows <= 0) return;
  if constexpr (MANY && !kApart<D, KIND>) {
    if (u.n_rows > kRows)
      k4::attend_unit<D, F16, KIND, 2>(a, u, listed, head, lds);
    else
      k4::attend_unit<D, F16, KIND, 1>(a, u, listed, head, lds);
  } else if (!MANY && u.n_rows <= kFewRows) {
    k4::attend_few<D, F16, KIND>(a, u, few, head, lds);
  } else {
    k4::attend_unit<D, F16, KIND, 1>(a, u, listed, head, lds);
  }
}

}  // namespace k4
