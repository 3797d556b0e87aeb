// Attention over the 8-bit cache.
//
// With z = q . K8_j (codes), row factor c = |scale| * log2(e) * 2^-k (q is scaled by 2^k into fp16's range, and by the scale's sign) and
// block scales ks, vs = 2^ev, all scores in log2 units:
//
//   t_j = z * c * ks            (capped, lowered by distance)        m = max (t_j + ev_j)        y_j = 2^(t_j + ev_j - m)
//   l   = sum y_j / vs          O = sum y_j V8_j                     out = O / l                 lse = ln 2 * (m + log2 l)
//
// Codes are whole fp16 numbers, so K and V enter the products exactly, and the scales, powers of two, stay outside of them: K's is a
// factor of the score, V's a term of the exponent, the same for 16 tokens.  The maximum that keeps y_j within [0, 1] is that of what
// enters the second product, row by row, so that its rounding to fp16, at most 2^-11 of each y_j, is small against the row's own result
// whatever the blocks' scales; it is the only rounding that fp32 does not see, half a step of an fp16 output.
//
// Both products run transposed, S^T = K Q^T and O^T = V^T P^T, in 32x32x16 steps of a wave over 32 tokens x 32 stacked rows.  What row of
// the first product a token has is free, and so is the order of dims within it; both are chosen such that
//   * a lane's piece of K (16 dims of a token) and of V (16 tokens of a dim) are 16 neighbouring bytes of the cache: codes go from memory to
//     the products' operands through registers alone, in whole cache lines, with no transposition;
//   * the scores that a lane gets (16 tokens of one block, one row) are, as fp16, its operand of the second product.
//
// A work-group takes 32 or 64 stacked rows; its four waves split the tokens, each with codes of its own in registers, and meet once at the end.
//
// What bounds it (8 kv heads of 128; a layer):
//   8 streams over 8k tokens, 21 MB        11.1 us: the ramp.  1.2 us to the first codes alone, 3.1 with the whole chip asking, 3.3 for the three pairs of a
//                                          wave, 1.5 for the waves' meeting, 2.5 of launch; the bytes are 4.3 us at a large copy's 4.9 TB/s
//   16 ragged requests, 95 MB              26.0 us, 3.7 TB/s: memory
//   16 x 8 rows over 51k tokens, 100 MB    59 us: vector instructions, 21 a score (codes to fp16, exponentials, distances, tags); the four tiles of rows
//                                          share codes through the L2 only, since two groups of rows with marks do not fit the registers
//   2048 x 4 rows over 8k tokens, 309 GF   322 to 354 us by the card, 870 to 960 TFLOP/s against 1190 to 1230 of a large library product: vector
//                                          instructions busy 64% of the time, matrix instructions 43%
// Tried and not taken: eight waves to a work-group (8 streams over 8k 123 -> 133 us a pass; 128 registers would be needed for four waves to a SIMD, and spill),
// one copy of Q's operands for all waves (a barrier; 1 to 3% more), touching the codes of the step after next ahead of their turn (4 to 7% more), three
// waves to a SIMD with 64 dims (spills), no priority for waves at the matrix pipe (nested forks over 35k 4% more).
#pragma once
#include <float.h>

#include "k8_dev.hpp"

namespace k8 {

struct AttendArgs {
  Geometry g;
  int Hq, g_shift, dtype, n_rows;
  float scale_log2;       // |softmax_scale| * log2(e)
  int negate;             // softmax_scale < 0
  float cap_log2, cap_in; // logit_cap * log2(e), 2 / logit_cap, both held within fp32; 0: none
  const uint8_t *k, *v;
  const float *ks, *vs;
  const int* table;
  // Arrays that the call does without are replaced by others that are as long, so that their loads need no branches (each of which would
  // wait for everything under way); the flags say whether what comes of them counts.
  bool tagged, placed, lowered;  // row_see, row_position, slopes are given
  const uint8_t* slot_tag;
  const int *slot_position, *row_position;
  const uint64_t* row_see;
  const float* slopes;
  int block_shift;  // page_tokens / 16 = 1 << block_shift
  const Unit* units;
  const int* unit_blocks;  // [unit][kUnitBlocks]
  const Tile* tiles;
  const void* q;
  void* out;
  float* lse;
  float2v* part_ml;  // [partial row][Hkv]: m, l
  float* part_acc;   // ... [D]: O
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;   // the base of the scores follows their maximum when that is 2^8 ahead: O is rescaled rarely, and weights up to 256
                                // lose nothing in fp16
constexpr float kLowCap = 128.f;  // caps up to this (log2 units) need no second form for small scores
constexpr int kScaleSpan = 60;  // blocks whose V scale is more powers of two than this below the largest so far have their part of l summed apart

__device__ inline float other_half(float x) {  // of lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32) ? r[0] : r[1]);
}

// 2^d as h * h.  O goes by the product; l, which carries the inverse of V's scales and may be 2^100 where 2^d is less than any number of fp32, by one
// factor after the other.
__device__ inline float root_exp2(float d) { return __builtin_amdgcn_exp2f(0.5f * d); }

// Lane i of each row of 16 lanes, for all lanes of the row.  The move stays one of its own: joined by the compiler with the subtraction that
// uses it (v_subrev_u32 with row_newbcast), every lane got its own value on this chip.
template <int I>
__device__ inline int of_row(int x) {
  int y = __builtin_amdgcn_update_dpp(0, x, 0x150 + I, 0xf, 0xf, true);
  asm("" : "+v"(y));
  return y;
}

template <class F, int... I>
__device__ inline void each(F f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ inline void each(F f) {  // f(0) ... f(N - 1), the numbers as constants
  each(f, std::make_integer_sequence<int, N>{});
}

// A wave's 32 stacked rows: lane n and n + 32 hold row n, each half of the dims.
template <int D>
struct Rows {
  float c;      // score factor but for ks
  float slope;  // in log2 units
  int token;    // own place
  int first_token;  // the wave's first row's
  uint32_t position;  // from -2^31 on
  uint64_t see;
  int by_tag;  // lane t: which of the wave's rows see tag t
  bool real;
};

__device__ inline int64_t row_address(const AttendArgs& a, int s, int head) {  // of stacked row s, in rows of D
  return (int64_t)(s >> a.g_shift) * a.Hq + head * a.g.G + (s & (a.g.G - 1));
}

template <int D, bool MARKS>
__device__ inline void request_rows(const AttendArgs& a, const Unit& u, int head, int first, Rows<D>& r, uint4v (&raw)[D / 16]) {
  const int lane = threadIdx.x & 63, n = lane & 31, half = lane >> 5;
  r.real = first + n < u.n_rows;
  const int s = u.s0 + (r.real ? first + n : 0);  // (a lane without a row computes the first one's, times 0)
  const uint4v* p = (const uint4v*)((const uint16_t*)a.q + row_address(a, s, head) * D);
#pragma unroll
  for (int k = 0; k < D / 16; ++k) raw[k] = p[(2 * (k >> 1) + half) * 2 + (k & 1)];
  r.token = u.pos0 + ((first + n) >> a.g_shift);
  r.first_token = u.pos0 + (first >> a.g_shift);
  r.slope = a.slopes[head * a.g.G + (s & (a.g.G - 1))];
  if constexpr (MARKS) {
    r.see = a.row_see[s >> a.g_shift];
    r.position = (uint32_t)a.row_position[s >> a.g_shift] ^ 0x80000000u;
  } else {
    r.see = 0, r.position = 0;
  }
}

// Lane t: which of the wave's rows see tag t; lane n's `see` is that of row n.
__device__ inline int rows_by_tag(uint64_t see, int g_shift) {
  const int heads = (1 << (1 << g_shift)) - 1;
  int rows = 0;
  for (int n = 0; n < kRows; n += 1 << g_shift) {
    const uint64_t tags = (uint32_t)__builtin_amdgcn_readlane((int)see, n) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(see >> 32), n) << 32;
    rows |= __builtin_amdgcn_inverse_ballot_w64(tags) ? heads << n : 0;
  }
  return rows;
}

template <int D>
__device__ inline void finish_rows(const AttendArgs& a, Rows<D>& r, const uint4v (&raw)[D / 16], half8 (&q)[D / 16]) {
  uint32_t amax = 0;  // largest magnitude: bits without the sign, of either type
#pragma unroll
  for (int k = 0; k < D / 16; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) amax = max(max(amax, raw[k][i] & 0x7fffu), raw[k][i] >> 16 & 0x7fffu);
  amax = max(amax, __float_as_uint(other_half(__uint_as_float(amax))));
  union { uint16_t u; _Float16 h; } c{(uint16_t)amax};
  amax = a.dtype == kBf16 ? amax << 16 : __float_as_uint((float)c.h);
  // the largest value comes to [2^14, 2^15): bf16's 8 bits stay whole down to 2^-31 of it, fp16's 11 to 2^-28
  const int up = amax ? min(max(14 + 127 - (int)(amax >> 23), -126), 126) : 0;
  const float f = !r.real ? 0.f : a.negate ? -pow2f(up) : pow2f(up);
  if (a.dtype == kBf16) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) q[k][i] = (_Float16)(__uint_as_float((i & 1) ? raw[k][i / 2] & 0xffff0000u : raw[k][i / 2] << 16) * f);
  } else {
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      union { uint4v w; half8 h; } x{raw[k]};
#pragma unroll
      for (int i = 0; i < 8; ++i) q[k][i] = (_Float16)((float)x.h[i] * f);
    }
  }
  r.c = a.scale_log2 * pow2f(-up);
  r.slope *= kLog2e;
}

// The blocks of a stretch of tokens, lane k the k-th of them: index into the scales (-1: none there), first slot / 16, K's scale, the exponent of
// V's as it enters the scores; and, for the wave, which blocks are absent, whose V reads as NaN, and whose V is too small to count.
struct Blocks {
  int at, slot16;
  float ks, vs, ev;
  uint64_t absent, nan, far;
};

// Block `number` of the layer's slots (slot / 16; negative: absent) for a kv head.
__device__ inline void on_block(const AttendArgs& a, int number, int head, Blocks& b) {
  const int page = number >> a.block_shift, in = number & (a.g.blocks_per_page - 1);
  b.at = number >= 0 ? (page * a.g.Hkv + head) * a.g.blocks_per_page + in : -1;
  b.slot16 = max(number, 0);
}

__device__ inline void find_blocks(const AttendArgs& a, int request, int head, int token, int hi, Blocks& b) {
  on_block(a, block_of(a.g, a.table, request, token, hi), head, b);
}

__device__ inline void load_scales(const AttendArgs& a, Blocks& b) {
  b.ks = a.ks[max(b.at, 0)];
  b.vs = a.vs[max(b.at, 0)];
}

// `most`: the largest exponent of V's scales so far; these blocks' are added to it.  (A block that is absent has no weight, one that reads as NaN any.)
__device__ inline void finish_scales(Blocks& b, int& most) {
  const int x = (int)((__float_as_uint(b.vs) >> 23) & 255) - 127;
  const bool there = b.at >= 0, nan = x == 128;
  most = max(most, (int)__builtin_amdgcn_readfirstlane(wave_max(there && !nan ? x + 127 : 0)) - 127);
  b.ev = (float)(there && !nan ? max(x, kEMin) : most);
  b.absent = __ballot(!there);
  b.nan = __ballot(there && nan);
  b.far = __ballot(there && x < most - kScaleSpan);
}

// 32 tokens: two blocks, of which the lane has to do with the one that its half of the wave holds scores of.  Of what is rare, bit h says it of
// block h.
struct Pair {
  float ks, ev;
  int absent, nan, far;
};

__device__ inline float of_lanes(float x, int low, int high) {  // of one lane for the lower half of the wave, of another for the upper half
  const float l = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), low)), h = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), high));
  return (threadIdx.x & 32) ? h : l;
}

__device__ inline Pair pair_of(const Blocks& b, int k) {  // blocks 2k and 2k + 1 of the wave's lanes; k the same for all lanes
  Pair p;
  p.ks = of_lanes(b.ks, 2 * k, 2 * k + 1), p.ev = of_lanes(b.ev, 2 * k, 2 * k + 1);
  p.absent = (int)(b.absent >> (2 * k)) & 3, p.nan = (int)(b.nan >> (2 * k)) & 3, p.far = (int)(b.far >> (2 * k)) & 3;
  return p;
}

__device__ inline bool of_half(int bits) { return (bits >> ((threadIdx.x >> 5) & 1)) & 1; }

// The codes of a pair, as this lane's pieces.  Row m = 8a + 4h + b of the first product is token 4a + b of block h.
__device__ inline const uint8_t* k_piece(const AttendArgs& a, int at0, int at1, int D) {
  const int lane = threadIdx.x & 63, m = lane & 31, half = lane >> 5;
  const int at = max((m & 4) ? at1 : at0, 0);
  return a.k + (int64_t)at * (kBlock * D) + half * 256 + ((m >> 3) * 4 + (m & 3)) * 16;
}

__device__ inline const uint8_t* v_piece(const AttendArgs& a, int at0, int at1, int D) {
  const int lane = threadIdx.x & 63;
  const int at = max((lane & 32) ? at1 : at0, 0);
  return a.v + (int64_t)at * (kBlock * D) + (lane & 31) * 16;
}

template <int N>
__device__ inline void load_pieces(const uint8_t* from, uint4v (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = *(const uint4v*)(from + i * 512);
}

template <int N>
__device__ inline void drop_absent(int absent, uint4v (&v)[N]) {  // what is not there must not be NaN: its weight is 0
  if (absent) {
    const bool none = of_half(absent);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = none ? uint4v{0, 0, 0, 0} : v[i];
  }
}

// Tag and position of a pair's tokens: lane l holds those of token l & 15 of block l >> 5.
struct Marks {
  int tag, position;
};

__device__ inline Marks load_marks(const AttendArgs& a, const Blocks& b, int k) {
  const int lane = threadIdx.x & 63;
  const int s0 = __builtin_amdgcn_readlane(b.slot16, 2 * k), s1 = __builtin_amdgcn_readlane(b.slot16, 2 * k + 1);
  const int64_t at = (int64_t)((lane & 32) ? s1 : s0) * kBlock + (lane & 15);
  return Marks{(int)a.slot_tag[at], a.slot_position[at]};
}

// What a call does to scores, which is known ahead of the launch: nothing but hide by order and prefix, cap or lower them by places too, or anything.
enum { kPlain = 0, kShaped = 1, kMarked = 2 };

// What the tokens of a pair are to the wave's rows: how far, and who sees them.
struct Unmarked {
  template <class F>
  __device__ void distances(F) const {}
  __device__ bool in_order(float&) const { return false; }
  __device__ int rows() const { return 0; }
};

struct Marked {
  int tag, by_tag;
  uint32_t mark, position;  // of the token and of the row, from -2^31 on: two of them can be up to 2^32 - 1 apart
  __device__ Marked(const Marks& m, uint32_t position, int by_tag)
      : tag(m.tag), by_tag(by_tag), mark((uint32_t)m.position ^ 0x80000000u), position(position) {}
  template <class F>
  __device__ void distances(F f) const {
    each<16>([&](auto i) {
      uint32_t far;
      asm("v_sad_u32 %0, %1, %2, 0" : "=v"(far) : "v"(position), "v"(of_row<i.value>((int)mark)));
      f(i.value, (float)far);
    });
  }
  // Whether the tokens' positions go up by one from each to the next, as in a prompt; then how far the lane's first token is from its row.
  __device__ bool in_order(float& far) const {
    const uint32_t first = (uint32_t)of_row<0>((int)mark);
    far = position >= first ? (float)(position - first) : -(float)(first - position);
    return __all(mark - first == (threadIdx.x & 15) && first <= UINT32_MAX - 15);
  }
  __device__ int rows() const { return __builtin_amdgcn_ds_bpermute((tag & 63) * 4, by_tag); }  // that see the lane's token
};

// f(i, whether the lane's row sees token i of its block: -1 or 0), from the rows that see the lane's token.
template <class F>
__device__ inline void sights(int rows, F f) {
  const int row = threadIdx.x & 31;
  each<16>([&](auto i) { f(i.value, __builtin_amdgcn_sbfe(of_row<i.value>(rows), row, 1)); });
}

__device__ inline float shown(float s, int seen) {  // where seen is -1, else -inf
  return __uint_as_float((__float_as_uint(s) & seen) | (0xff800000u & ~seen));
}

// Scores of a pair, tokens t0 .. t0 + 31: capped, lowered, hidden.  They come as the first product gives them (times f: log2 units) and are
// left so where nothing has to be done; else they come out in log2 units and f is 1.
template <int KIND, class Source>
__device__ inline void finish_scores(const AttendArgs& a, int prefix, int hi, int t0, const Pair& p, const Source& source, float slope, int token,
                                     int first_token, float& f, float16v& s) {
  const int half = (threadIdx.x >> 5) & 1, base = t0 + 16 * half;
  const bool ordered = t0 + 31 > first_token, cut = t0 + 32 > hi || p.absent;
  const bool masked = cut || (t0 + 32 > prefix && ((KIND == kMarked && a.tagged) || ordered));
  const bool shaped = KIND != kPlain && (a.cap_log2 > 0.f || a.lowered);
  if (KIND == kPlain ? __builtin_expect(!masked, 1) : !masked && !shaped) return;
  if (KIND != kPlain && a.cap_log2 > 0.f) {
    // cap * tanh(x / cap) = cap - 2 cap / (1 + e^(2 x / cap)), which is off by 2^-22 or so of the cap, whatever x
    const float g = f * a.cap_in;
    auto closed = [&](float y) { return fmaf(-2.f * a.cap_log2, __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(y)), a.cap_log2); };
    if (a.cap_log2 <= kLowCap) {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = closed(s[i] * g);
    } else {
      // where x is small beside a high cap: x * tanh(u) / u by its series in u = x / cap, off by 2^-28 at u = 1/8
      constexpr float kUnit = 0.25f * kLn2 * kLn2, c1 = -kUnit / 3.f, c2 = 2.f * kUnit * kUnit / 15.f, c3 = -17.f * kUnit * kUnit * kUnit / 315.f;
      float to = g;
      asm volatile("" : "+v"(to));  // (or else all sixteen s * g are made ahead of the branch, and s has to be kept beside them)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = s[i] * to, w = y * y;  // y = 2 u log2(e)
        s[i] = fabsf(y) < 0.25f * kLog2e ? s[i] * f * fmaf(fmaf(fmaf(c3, w, c2), w, c1), w, 1.f) : closed(y);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    f = 1.f;
  }
  if (KIND != kPlain && a.lowered) {
    float far = (float)(token - base);
    if (KIND != kMarked || !a.placed || source.in_order(far)) {
      if (KIND == kMarked && __all(far >= 15.f)) {  // the row is behind them all
        const float least = -slope * far;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], f, fmaf(slope, (float)i, least));
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], f, -slope * fabsf(far - (float)i));
      }
    } else {
      source.distances([&](int i, float far) { s[i] = fmaf(s[i], f, -slope * far); });
    }
    f = 1.f;
  }
  if (!masked) return;
  if (!shaped) {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] *= f;
    f = 1.f;
  }
  int rows = 0;
  if (KIND == kMarked && a.tagged) {
    rows = source.rows();
    if (t0 >= prefix && !ordered && !cut) {  // tags alone
      if (!__all(rows == -1)) sights(rows, [&](int i, int seen) { s[i] = shown(s[i], seen); });
      return;
    }
  }
  auto below = [](int n) { return n <= 0 ? 0u : n >= kBlock ? 0xffffu : (1u << n) - 1u; };
  uint32_t bits = below(token + 1 - base);
  if (KIND == kMarked && a.tagged) {
    uint32_t tagged = 0;
    sights(rows, [&](int i, int seen) { tagged |= (uint32_t)seen & (1u << i); });
    bits &= tagged;
  }
  bits |= below(prefix - base);
  bits = of_half(p.absent) ? 0u : bits & below(hi - base);
#pragma unroll
  for (int i = 0; i < 16; ++i) s[i] = shown(s[i], __builtin_amdgcn_sbfe((int)bits, i, 1));
}

// Running state of a wave's rows.
template <int D>
struct State {
  float16v o[D / 32];
  float m, l;  // the scores' base, at most kSlack below their maximum; l: of this lane's tokens
  float bad;   // NaN: the row sees a block whose V reads as NaN
};

template <int D>
__device__ inline void start(State<D>& z) {
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int k = 0; k < 16; ++k) z.o[i][k] = 0.f;
  z.m = -FLT_MAX, z.l = 0.f, z.bad = 0.f;
}

__device__ inline void to_half(const float16v& y, half8 (&w)[2]) {
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    const half2v h = __builtin_convertvector((float2v{y[i], y[i + 1]}), half2v);
    w[i / 8][i % 8] = h[0], w[i / 8][i % 8 + 1] = h[1];
  }
}

// N pairs of blocks and G groups of 32 rows: their scores (times f) become the second product's operands.
template <int D, int G, int N>
__device__ inline void soften(State<D> (&z)[G], const float16v (&s)[G][N], const float (&f)[G][N], const Pair (&p)[N], half8 (&w)[G][N][2]) {
  float m[G];
  bool ahead = false;
  int rare = 0;
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
    ahead |= m[g] > z[g].m + kSlack;
  }
#pragma unroll
  for (int n = 0; n < N; ++n) rare |= p[n].nan | p[n].far;
  if (__builtin_expect(__any(ahead), 0)) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const float to = fmaxf(m[g], z[g].m), h = root_exp2(z[g].m - to), alpha = h * h;
      z[g].m = to;
      z[g].l = z[g].l * h * h;
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int k = 0; k < 16; ++k) z[g].o[i][k] *= alpha;
    }
  }
  float off[G][N], back[N];
#pragma unroll
  for (int n = 0; n < N; ++n) back[n] = __builtin_amdgcn_exp2f(-p[n].ev);
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int n = 0; n < N; ++n) off[g][n] = p[n].ev - z[g].m;
  // Of a block whose scale is far below the largest, y may be less than any number of fp32 where y / vs still counts: its part of l goes by the
  // largest score of its own.
  if (__builtin_expect(rare, 0)) {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        bool sees = false;
        float most = -FLT_MAX, sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) sees |= s[g][n][i] != -INFINITY, most = fmaxf(most, s[g][n][i] * f[g][n]);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f(fmaf(s[g][n][i], f[g][n], -most));
        if (of_half(p[n].nan) && sees) z[g].bad = __builtin_nanf("");
        const float h = root_exp2(most - z[g].m);
        if (of_half(p[n].far)) z[g].l = fmaf(sum * h, h, z[g].l);
      }
#pragma unroll
    for (int n = 0; n < N; ++n) back[n] = of_half(p[n].far) ? 0.f : back[n];
  }
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float sum = 0.f;
      float16v y;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        y[i] = __builtin_amdgcn_exp2f(fmaf(s[g][n][i], f[g][n], off[g][n]));
        sum += y[i];
      }
      z[g].l = fmaf(sum, back[n], z[g].l);
      to_half(y, w[g][n]);
    }
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

template <int D>
__device__ inline void poison(State<D>& z) {
  const float bad = z.bad + other_half(z.bad);
  if (__any(bad != 0.f)) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int k = 0; k < 16; ++k) z.o[i][k] += bad;
  }
}

__device__ inline float lse_of(float m, float l) { return l == 0.f ? -INFINITY : kLn2 * (m + __builtin_amdgcn_logf(l)); }
__device__ inline float inverse_of(float l) { return l == 0.f ? 0.f : 1.f / l; }

// One step of a wave: N pairs whose codes are in k and v, against G groups of 32 rows.  `ahead` is called when k may be overwritten, `behind` when v may.
template <int CODES, int D, int KIND, int G, int N, class Ahead, class Behind>
__device__ inline void step(const AttendArgs& a, const Unit& u, const Rows<D> (&r)[G], const half8* q, State<D> (&z)[G], uint4v (&k)[N][D / 32],
                            uint4v (&v)[N][D / 32], const Pair (&p)[N], const Marks (&marks)[N], const int (&t0)[N], Ahead ahead, Behind behind) {
  float16v s[G][N];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[g][n][i] = 0.f;
  // A wave at the matrix pipe goes first: else the older of a SIMD's two runs ahead, and the younger ends alone.
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int x = 0; x < D / 32; ++x)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      half8 codes[N];
#pragma unroll
      for (int n = 0; n < N; ++n) codes[n] = codes_to_half8<CODES>(k[n][x][2 * y], k[n][x][2 * y + 1]);
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const half8 row = q[(g * (D / 16) + 2 * x + y) * 64 + (threadIdx.x & 63)];
#pragma unroll
        for (int n = 0; n < N; ++n) s[g][n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes[n], row, s[g][n], 0, 0, 0);
      }
    }
  __builtin_amdgcn_s_setprio(0);
  Marks m[N];
#pragma unroll
  for (int n = 0; n < N; ++n) m[n] = marks[n];
  ahead();
  float f[G][N];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int n = 0; n < N; ++n) {
      f[g][n] = r[g].c * p[n].ks;
      if constexpr (KIND == kMarked)
        finish_scores<KIND>(a, u.prefix, u.hi, t0[n], p[n], Marked{m[n], r[g].position, r[g].by_tag}, r[g].slope, r[g].token, r[g].first_token, f[g][n], s[g][n]);
      else
        finish_scores<KIND>(a, u.prefix, u.hi, t0[n], p[n], Unmarked{}, r[g].slope, r[g].token, r[g].first_token, f[g][n], s[g][n]);
    }
  half8 w[G][N][2];
  soften<D, G, N>(z, s, f, p, w);
  __builtin_amdgcn_s_setprio(1);
  __builtin_amdgcn_sched_barrier(0);  // (V's codes are turned as they are needed: all at once they take 64 registers more)
#pragma unroll
  for (int n = 0; n < N; ++n) {
    drop_absent(p[n].absent, v[n]);
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const half8 codes = codes_to_half8<CODES>(v[n][x][2 * y], v[n][x][2 * y + 1]);
#pragma unroll
        for (int g = 0; g < G; ++g) z[g].o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes, w[g][n][y], z[g].o[x], 0, 0, 0);
      }
  }
  __builtin_amdgcn_s_setprio(0);
  behind();
}

template <int D>
constexpr int kPitch = D + 4;  // of the rows that the waves put into LDS at the end

// A unit of G groups of 32 rows.  Every wave takes a quarter of the tokens, pairs wave, wave + 4, ...; the four meet at the end.
//   G = 1   two pairs at a time, so that a softmax's way through its lanes is taken once for 64 tokens
//   G = 2   what turning a pair's codes costs, and reading them, serves twice as many rows; with 128 dims there are registers for one pair at a time (with 64,
//           two instead of one are worth 5%: four requests' pieces of prompts 107 -> 102 us a pass)
// Q's operands lie in LDS, a copy for each wave (where its output goes later): in registers they would leave no room for that.
template <int CODES, int D, int KIND, int G>
__device__ inline void attend_unit(const AttendArgs& a, const Unit& u, int listed, int head, float* lds) {
  constexpr bool MARKS = KIND == kMarked;
  constexpr int N = G == 1 || D == 64 ? 2 : 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 31, half = lane >> 5;
  const int n_pairs = max((((u.hi - u.lo + 31) >> 5) - wave + 3) >> 2, 0);  // this wave's
  half8* q = (half8*)(lds + wave * kRows * kPitch<D>);
  Rows<D> r[G];
  State<D> z[G];
  Blocks b;
  int most = kEMin;  // largest exponent of V's scales so far
  uint4v k[N][D / 32], v[N][D / 32];
  Marks marks[N] = {};
  auto token = [&](int i) { return u.lo + (wave + 4 * i) * 32; };  // first of the wave's i-th pair
  auto find = [&](int i) { find_blocks(a, u.request, head, token(i + (lane >> 1)) + (lane & 1) * 16, u.hi, b); };
  auto load_k = [&](int i, int to) {
    const int x = 2 * (i & 31);
    load_pieces(k_piece(a, __builtin_amdgcn_readlane(b.at, x), __builtin_amdgcn_readlane(b.at, x + 1), D), k[to]);
  };
  auto load_v = [&](int i, int to) {
    const int x = 2 * (i & 31);
    load_pieces(v_piece(a, __builtin_amdgcn_readlane(b.at, x), __builtin_amdgcn_readlane(b.at, x + 1), D), v[to]);
  };
  {
    // Everything is asked for before anything is waited for: loads come back in their order.  (Where the wave has fewer than N pairs, block 0 is read in
    // their place.)
    uint4v raw[D / 16];
    request_rows<D, MARKS>(a, u, head, 0, r[0], raw);
    __builtin_amdgcn_sched_barrier(0);
    if (u.hi - u.lo <= kUnitBlocks * kBlock)
      on_block(a, 2 * (wave + 4 * (lane >> 1)) + (lane & 1) < kUnitBlocks ? listed : -1, head, b);
    else
      find(0);
    load_scales(a, b);
#pragma unroll
    for (int n = 0; n < N; ++n)
      if constexpr (MARKS) marks[n] = load_marks(a, b, n);
#pragma unroll
    for (int n = 0; n < N; ++n) load_k(n, n);
#pragma unroll
    for (int n = 0; n < N; ++n) load_v(n, n);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g < G; ++g) {
      half8 x[D / 16];
      if (g) request_rows<D, MARKS>(a, u, head, g * kRows, r[g], raw);
      finish_rows<D>(a, r[g], raw, x);
      if constexpr (MARKS) r[g].by_tag = rows_by_tag(r[g].see, a.g_shift);
#pragma unroll
      for (int y = 0; y < D / 16; ++y) q[(g * (D / 16) + y) * 64 + lane] = x[y];
    }
  }
  finish_scales(b, most);
#pragma unroll
  for (int g = 0; g < G; ++g) start(z[g]);
  int i = 0;
  for (; i + N - 1 < n_pairs; i += N) {
    Pair p[N];
    int t0[N];
#pragma unroll
    for (int n = 0; n < N; ++n) p[n] = pair_of(b, (i + n) & 31), t0[n] = token(i + n);
    step<CODES, D, KIND, G, N>(a, u, r, q, z, k, v, p, marks, t0,
      [&] {
        if (i + N >= n_pairs) return;
        if (((i + N) & 31) == 0) find(i + N), load_scales(a, b), finish_scales(b, most);
#pragma unroll
        for (int n = 0; n < N; ++n)
          if constexpr (MARKS) marks[n] = load_marks(a, b, (i + N + n) & 31);
#pragma unroll
        for (int n = 0; n < N; ++n) load_k(i + N + n, n);
      },
      [&] {
        if (i + N >= n_pairs) return;
#pragma unroll
        for (int n = 0; n < N; ++n) load_v(i + N + n, n);
      });
  }
  if constexpr (N == 2) {
    if (i < n_pairs) {
      const Pair p[1] = {pair_of(b, i & 31)};
      const int t0[1] = {token(i)};
      const Marks last[1] = {marks[0]};
      step<CODES, D, KIND, G, 1>(a, u, r, q, z, *(uint4v(*)[1][D / 32]) & k, *(uint4v(*)[1][D / 32]) & v, p, last, t0, [] {}, [] {});
    }
  }
  // the four waves meet, group after group
  float* s_o = lds;                                         // [4][32][kPitch]
  float2v* s_ml = (float2v*)(lds + 4 * kRows * kPitch<D>);  // [4][32]
#pragma unroll
  for (int g = 0; g < G; ++g) {
    if (g && u.n_rows <= g * kRows) break;
    const float l = z[g].l + other_half(z[g].l);
    poison(z[g]);
    if (g) __syncthreads();
    if (half == 0) s_ml[wave * kRows + row] = float2v{z[g].m, l};
    if (r[g].real) {
#pragma unroll
      for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y)
          *(float4v*)(s_o + (wave * kRows + row) * kPitch<D> + 32 * x + 8 * y + 4 * half) =
              float4v{z[g].o[x][4 * y], z[g].o[x][4 * y + 1], z[g].o[x][4 * y + 2], z[g].o[x][4 * y + 3]};
    }
    __syncthreads();
    // a thread takes the same four dims of several rows; what lies in LDS is read for rows that there are not, too
    constexpr int kLanes = D / 4, kAtOnce = 256 / kLanes;
    const int i0 = threadIdx.x / kLanes, d = threadIdx.x % kLanes * 4, rows = min(u.n_rows - g * kRows, kRows);
#pragma unroll
    for (int j = 0; j < kRows / kAtOnce; ++j) {
      const int i = i0 + j * kAtOnce;
      float2v ml[4];
      float4v part[4];
#pragma unroll
      for (int w = 0; w < 4; ++w) ml[w] = s_ml[w * kRows + i], part[w] = *(const float4v*)(s_o + (w * kRows + i) * kPitch<D> + d);
      const float m = fmaxf(fmaxf(ml[0][0], ml[1][0]), fmaxf(ml[2][0], ml[3][0]));
      float all = 0.f;
      float4v o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float h = root_exp2(ml[w][0] - m);
        all = fmaf(ml[w][1] * h, h, all);
        o += part[w] * (h * h);
      }
      if (i >= rows) continue;
      if (u.part < 0) {
        const int64_t to = row_address(a, u.s0 + g * kRows + i, head);
        store_out(a, to * D + d, o * inverse_of(all));
        if (a.lse && d == 0) a.lse[to] = lse_of(m, all);
      } else {
        const int64_t to = (int64_t)(u.part + g * kRows + i) * a.g.Hkv + head;
        *(float4v*)(a.part_acc + to * D + d) = o;
        if (d == 0) a.part_ml[to] = float2v{m, all};
      }
    }
  }
}

// Two groups at a time do not fit the registers with 128 dims and tags or positions, or int8 codes and a cap: then a work-group (blockIdx.y) takes each.
template <int CODES, int D, int KIND>
constexpr bool kApart = D == 128 && (KIND == kMarked || (KIND == kShaped && CODES == kInt8));

template <int CODES, int D, bool MANY, int KIND>
__global__ __launch_bounds__(256, 2) void k8_attend(AttendArgs a) {
  __shared__ __attribute__((aligned(16))) float lds[4 * kRows * kPitch<D> + 4 * kRows * 2];
  const int head = blockIdx.x % a.g.Hkv, unit = blockIdx.x / a.g.Hkv, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Unit u = a.units[unit];
  // the lane's block, asked for together with the unit: pairs are dealt out to the four waves
  const int listed = a.unit_blocks[unit * kUnitBlocks + min(2 * (wave + 4 * (lane >> 1)) + (lane & 1), kUnitBlocks - 1)];
  asm volatile("" ::"s"(u.request), "s"(u.s0), "s"(u.pos0), "s"(u.lo), "s"(u.hi), "s"(u.prefix), "s"(u.part));  // (one load, ahead of the branch)
  if constexpr (MANY && kApart<CODES, D, KIND>) {
    const int first = blockIdx.y * kRows;
    u.s0 += first, u.n_rows = min(u.n_rows - first, kRows), u.pos0 += first >> a.g_shift;
    if (u.part >= 0) u.part += first;
  }
  if (u.n_rows <= 0) return;
  if constexpr (MANY && !kApart<CODES, D, KIND>) {
    if (u.n_rows > kRows)
      attend_unit<CODES, D, KIND, 2>(a, u, listed, head, lds);
    else
      attend_unit<CODES, D, KIND, 1>(a, u, listed, head, lds);
  } else {
    attend_unit<CODES, D, KIND, 1>(a, u, listed, head, lds);
  }
}

// Joins the partial rows of the tiles whose tokens are split.  D / 4 lanes hold a row, four dims apiece; of the 1024 / D such groups of a
// work-group as many share a row's parts as leave each four of them, or all.  A group asks for its parts at once and goes by their own maximum, so
// that nothing waits for a maximum over all; the groups' results are joined in LDS.  Bound by its launch and one way to memory: 3.8 us for 32 rows x 28
// parts of 8 heads (3.8 MB), of which 2.5 are the launch.  Joining in k8_attend, by the last work-group to come, would need partial rows written past the
// L2s of eight dies and one CU to read all parts of a tile.
template <int D>
__global__ __launch_bounds__(256) void k8_merge(AttendArgs a) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes, kAtOnce = 4;
  __shared__ float4v s_o[kGroups][kLanes];
  __shared__ float2v s_ml[kGroups];
  const int t = blockIdx.x / a.g.Hkv, head = blockIdx.x % a.g.Hkv;
  const Tile tile = a.tiles[t];
  if (tile.n_parts < 2) return;
  const int group = threadIdx.x / kLanes, d = threadIdx.x % kLanes;
  const int share = tile.n_parts <= kAtOnce ? 1 : tile.n_parts <= 2 * kAtOnce ? 2 : tile.n_parts <= 4 * kAtOnce ? 4 : kGroups;  // groups to a row
  const int rows = kGroups / share;                                                                                         // rows at a time
  const int64_t step = (int64_t)tile.n_rows * a.g.Hkv;
  for (int row0 = blockIdx.y * rows; row0 < tile.n_rows; row0 += gridDim.y * rows) {
    const int row = row0 + group / share;
    const bool real = row < tile.n_rows;
    const int64_t at = (int64_t)(tile.part + (real ? row : 0)) * a.g.Hkv + head;
    const float2v* ml = a.part_ml + at;
    const float* acc = a.part_acc + at * D + 4 * d;
    float m = -FLT_MAX, l = 0.f;
    float4v o{0.f, 0.f, 0.f, 0.f};
    for (int k0 = group % share; k0 < tile.n_parts; k0 += kAtOnce * share) {
      float2v x[kAtOnce];
      float4v y[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int64_t k = min(k0 + i * share, tile.n_parts - 1);
        x[i] = ml[k * step], y[i] = *(const float4v*)(acc + k * step * D);
      }
      const float before = m;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) m = fmaxf(m, x[i][0]);
      const float h = root_exp2(before - m);
      l = l * h * h, o *= h * h;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (k0 + i * share >= tile.n_parts) continue;
        const float h = root_exp2(x[i][0] - m);
        l = fmaf(x[i][1] * h, h, l);
        o += y[i] * (h * h);
      }
    }
    if (share > 1) {
      __syncthreads();
      s_o[group][d] = o;
      if (d == 0) s_ml[group] = float2v{m, l};
      __syncthreads();
      if (group % share) continue;
      for (int x = 1; x < share; ++x) m = fmaxf(m, s_ml[group + x][0]);
      l = 0.f, o = float4v{0.f, 0.f, 0.f, 0.f};
      for (int x = 0; x < share; ++x) {
        const float2v y = s_ml[group + x];
        const float h = root_exp2(y[0] - m);
        l = fmaf(y[1] * h, h, l);
        o += s_o[group + x][d] * (h * h);
      }
    }
    if (!real) continue;
    const int64_t to = row_address(a, tile.s0 + row, head);
    store_out(a, to * D + 4 * d, o * inverse_of(l));
    if (a.lse && d == 0) a.lse[to] = lse_of(m, l);
  }
}

}  // namespace k8
