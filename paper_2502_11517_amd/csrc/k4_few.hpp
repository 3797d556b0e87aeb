// Attention over the 4-bit cache of units with at most 16 stacked rows: one or a few threads, where half of a tile of 32 rows and more would be empty.
//
// As k4_attend.hpp, in 16x16x32 steps over 64 tokens (four blocks) x 16 rows: half the scores, and so half the softmax, per lane and token.  Only in launches without
// tiles of 64 rows: beside those the registers do not hold both forms, and such units go in steps of 32 rows there.
//   S^T = K Q^T    four tiles of 16 tokens: row m of tile t is token 4t + m % 4 of block m / 4, so that lane row + 16 g gets the 16 scores of block g, its operand of
//                  the second product; a lane's piece of K is a quarter of a token's dims
//   O^T = V^T P^T  a lane's piece of V is two neighbouring dims of a block's 16 tokens, which go to two products: the dims of a product are every second of 32
//
// In steps of 32 rows and here (32 / 8 heads of 128 unless said; a pass with its plan and merges): one thread over 32k tokens, 4 layers, 70.7 / 61.1 us; four over
// 8k, 4 layers, 52.9 / 47.5; 16 requests of one over 32k, 2 layers, 239 / 221, 104 us a layer of 560 MB, 5.4 TB/s; 16 of four over 4k, 4 layers, 121 / 109, of 64 dims with caps and
// distances 129 / 92.
#pragma once
#include "k4_attend.hpp"

namespace k4 {

constexpr int kFewRows = 16;
constexpr int kFour = 4 * kBlock;  // tokens of a step


// Running state of a wave's 16 rows; members as in State.
template <int D>
struct FewState {
  float4v o[D / 16];  // [2c + e]: dims 32 c + 2 (4 (lane / 16) + i) + e of row lane % 16
  float m, l, bad;
};

template <int D>
__device__ inline void times(FewState<D>& z, float x) {
#pragma unroll
  for (int i = 0; i < D / 16; ++i) z.o[i] *= x;
}

template <int D>
struct FewCodes {
  uint32_t k[4][D / 32];  // by tile: a quarter of the dims of a token
  uint32_t ks[4];         // their scale
  uint4v v[D / 32];
  uint32_t vs;  // V's scales of tokens 2i, 2i + 1 of block lane / 16, i = lane % 8
};

// Blocks that the wave's lanes hold for it: `of` the index of the step's first.
__device__ inline int block_at(int x, int of, int block) { return __builtin_amdgcn_ds_bpermute(4 * (of + block), x); }

template <int D>
__device__ inline void few_k(const AttendArgs& a, const Blocks& b, int of, FewCodes<D>& c) {
  const int lane = threadIdx.x & 63, m = lane & 15, part = lane >> 4, group = part * (D / 32) / 4;
  const int64_t at = max(block_at(b.at, of, m >> 2), 0), own = max(block_at(b.at, of, part), 0);
  const uint8_t* codes = a.k + at * kCodeBytes(D) + group * 256 + (m & 3) * 16 + (D == 128 ? 0 : (part & 1) * 8);
  const uint8_t* scale = a.k_scale + (at * kBlock + (m & 3)) * (D / 32) + group;
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    if constexpr (D == 128) {
      const uint4v w = *(const uint4v*)(codes + t * 64);
      for (int y = 0; y < 4; ++y) c.k[t][y] = w[y];
    } else {
      const uint2v w = *(const uint2v*)(codes + t * 64);
      for (int y = 0; y < 2; ++y) c.k[t][y] = w[y];
    }
    c.ks[t] = scale[t * 4 * (D / 32)];
  }
  c.vs = *(const uint16_t*)(a.v_scale + own * kBlock + 2 * (lane & 7));
}

template <int D>
__device__ inline void few_v(const AttendArgs& a, const Blocks& b, int of, FewCodes<D>& c) {
  const int lane = threadIdx.x & 63;
  const uint8_t* from = a.v + (int64_t)max(block_at(b.at, of, lane >> 4), 0) * kCodeBytes(D) + (lane & 15) * 16;
#pragma unroll
  for (int x = 0; x < D / 32; ++x) c.v[x] = *(const uint4v*)(from + x * 256);
}

__device__ inline Marks few_marks(const AttendArgs& a, const Blocks& b, int of) {  // lane l: of token l % 16 of block l / 16
  const int lane = threadIdx.x & 63;
  const int64_t at = (int64_t)block_at(b.slot16, of, lane >> 4) * kBlock + (lane & 15);
  return Marks{(int)a.slot_tag[at], a.slot_position[at]};
}

template <bool F16>
__device__ inline float4v few_product(const uint4v& k, const uint4v& q, const float4v& s) {
  union { uint4v w; half8 h; bf16x8 b; } x{k}, y{q};
  if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(x.h, y.h, s, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x.b, y.b, s, 0, 0, 0);
}

// As windows() of k4_attend.hpp; kNone among the bytes of tokens that there are not.
template <int D>
__device__ inline int few_windows(const FewCodes<D>& c, const int (&byte)[4], const uint4v (&q)[D / 32], float4v (&s)[4]) {
  constexpr int kWide = 2 * kAside, kWindows = 256 / kWide + 1;
  int unit = -1;
#pragma unroll
  for (int t = 0; t < 4; ++t) s[t] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int w = 0; w < kWindows; ++w) {
    bool some = w == kWindows - 1 && unit < 0;
#pragma unroll
    for (int t = 0; t < 4; ++t) some |= byte[t] != kNone && byte[t] / kWide == w;
    if (!__any(some)) continue;
    const int next = kWide * w + kAside;
    const float down = unit < 0 ? 1.f : pow2f(max(unit - next, -126));
    unit = next;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bool mine = byte[t] == kNone || byte[t] / kWide == w;  // (not a number: in every window)
      const float scale = __uint_as_float(byte[t] == kNone ? 0x7f800000u : (uint32_t)((mine ? byte[t] - next : 0) + 127) << 23);
      s[t] *= down;
#pragma unroll
      for (int y = 0; y < D / 32; ++y) s[t] = few_product<true>(k_operand<true>(mine ? c.k[t][y] : 0u, scale), q[y], s[t]);
    }
  }
  return unit;
}

// One step of a wave.  `ahead` is called when K may be overwritten, `behind` when V may.
template <int D, bool F16, int KIND, class Ahead, class Behind>
__device__ inline void few_step(const AttendArgs& a, const Unit& u, const Rows<D>& r, const uint4v (&q)[D / 32], int unit, FewState<D> (&z)[1], FewCodes<D>& c,
                                int absent, const Marks& marks, int t0, int& most, float& slack, Ahead ahead, Behind behind) {
  float4v p[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) p[t] = float4v{0.f, 0.f, 0.f, 0.f};
  float scale[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) scale[t] = __uint_as_float((c.ks[t] << 23) + (F16 ? (uint32_t)(127 - unit) << 23 : 0u));
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int y = 0; y < D / 32; ++y)
#pragma unroll
    for (int t = 0; t < 4; ++t) p[t] = few_product<F16>(k_operand<F16>(c.k[t][y], scale[t]), q[y], p[t]);
  __builtin_amdgcn_s_setprio(0);
  float f[1][1] = {{F16 ? uniform(a.scale_log2 * unit_scale(unit)) : a.scale_log2}};
  if constexpr (F16) {
    const int m = threadIdx.x & 15, left = (absent >> (m >> 2)) & 1 ? 0 : u.hi - (t0 + 16 * (m >> 2) + (m & 3));  // tokens 4t < left are there
    bool in = true;
#pragma unroll
    for (int t = 0; t < 4; ++t) in &= 4 * t >= left || (uint32_t)((int)c.ks[t] - unit + kAside) <= 2 * kAside;
    if (__builtin_expect(!__all(in), 0)) {
      int byte[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) byte[t] = 4 * t >= left ? kNone : (int)c.ks[t];
      f[0][0] = uniform(a.scale_log2 * unit_scale(few_windows<D>(c, byte, q, p)));
    }
  }
  Scales scales[1] = {scales_of<4>(c.vs, absent, t0, u.hi, most)};
  const Marks m = marks;
  ahead();
  float16v s[1][1];
#pragma unroll
  for (int i = 0; i < 16; ++i) s[0][0][i] = p[i / 4][i % 4];
  const Pair pair{1.f, 0.f, absent, 0, 0};
  if constexpr (KIND == kMarked)
    finish_scores<KIND, 4>(a, u.prefix, u.hi, t0, pair, Marked{m, r.position, r.by_tag}, r.slope, r.token, r.first_token, f[0][0], s[0][0]);
  else
    finish_scores<KIND, 4>(a, u.prefix, u.hi, t0, pair, Unmarked{}, r.slope, r.token, r.first_token, f[0][0], s[0][0]);
  half8 w[1][1][2];
  k4::soften<4>(z, slack, s, f, scales, w);
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int y = 0; y < 2; ++y)
#pragma unroll
    for (int x = 0; x < D / 16; ++x)
      z[0].o[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v_operand(c.v[x / 2][2 * (x & 1) + y]), w[0][0][y], z[0].o[x], 0, 0, 0);
  __builtin_amdgcn_s_setprio(0);
  behind();
}

__device__ inline float sum_of_row(float x) {  // of a row's four lanes, the same in each
  const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
  const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(rows[0]) + __uint_as_float(rows[1]);
}

// A unit.  Every wave takes a quarter of the tokens, fours of blocks wave, wave + 4, ...; the four waves meet at the end.  `listed`: the lane's block of those that
// stand with the unit.
template <int D, bool F16, int KIND>
__device__ inline void attend_few(const AttendArgs& a, const Unit& u, int listed, int head, float* lds) {
  constexpr bool MARKS = KIND == kMarked;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, part = lane >> 4;
  const int n_steps = max((((u.hi - u.lo + kFour - 1) / kFour) - wave + 3) >> 2, 0);  // this wave's
  Rows<D> r;
  FewState<D> z[1];
  Blocks b;
  uint64_t gone;
  int most = kEMin + 127;  // largest byte of V's scales so far
  float slack = kAhead;
  FewCodes<D> c;
  Marks marks{};
  auto token = [&](int i) { return u.lo + (wave + 4 * i) * kFour; };  // first of the wave's i-th step
  auto find = [&](int i) { find_blocks(a, u.request, head, token(i + (lane >> 2)) + (lane & 3) * kBlock, u.hi, b), gone = __ballot(b.at < 0); };
  auto first_of = [](int i) { return 4 * (i & 15); };
  uint4v q[D / 32];
  // Everything is asked for before anything is waited for.  (Where the wave has no step, block 0 is read in its place.)
  k4::request_rows<D, MARKS, kFewRows>(a, u, head, 0, r, q);
  __builtin_amdgcn_sched_barrier(0);
  if (u.hi - u.lo <= kUnitBlocks * kBlock)
    on_block(a, 4 * (wave + 4 * (lane >> 2)) + (lane & 3) < kUnitBlocks ? listed : -1, head, b), gone = __ballot(b.at < 0);
  else
    find(0);
  if constexpr (MARKS) marks = few_marks(a, b, 0);
  few_k<D>(a, b, 0, c);
  few_v<D>(a, b, 0, c);
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (MARKS) r.by_tag = rows_by_tag(r.see, a.g_shift);  // (lanes 16 .. 31 hold rows 0 .. 15 again, and look at bits 16 .. 31)
  if (a.negate)  // (the same for all lanes)
#pragma unroll
    for (int y = 0; y < D / 32; ++y) q[y] ^= uint4v{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
  int unit = 127;
  if constexpr (F16) {
    const int byte = __builtin_amdgcn_readfirstlane(c.ks[0]);  // of the wave's first token
    unit = (gone & 1) || byte == kNone ? 127 : min(max(byte, kEMin + 127), kNone - 1 - kAside);  // (kNone lies in no window)
  }
#pragma unroll
  for (int i = 0; i < D / 16; ++i) z[0].o[i] = float4v{0.f, 0.f, 0.f, 0.f};
  z[0].m = -FLT_MAX, z[0].l = 0.f, z[0].bad = 0.f;
  for (int i = 0; i < n_steps; ++i)
    few_step<D, F16, KIND>(a, u, r, q, unit, z, c, (int)(gone >> first_of(i)) & 15, marks, token(i), most, slack,
      [&] {
        if (i + 1 >= n_steps) return;
        if (((i + 1) & 15) == 0) find(i + 1);
        if constexpr (MARKS) marks = few_marks(a, b, first_of(i + 1));
        few_k<D>(a, b, first_of(i + 1), c);
      },
      [&] {
        if (i + 1 < n_steps) few_v<D>(a, b, first_of(i + 1), c);
      });
  // The four waves meet: pieces of four dims of a lane's, two to 32 dims, of which each wave joins a quarter.
  constexpr int kPieces = D / 16, kOwn = kPieces / 4;
  float4v* s_o = (float4v*)lds;                             // [4] waves [kPieces][64]
  float2v* s_ml = (float2v*)(lds + 4 * kRows * kPitch<D>);  // [4][kRows]
  const float l = sum_of_row(z[0].l), bad = sum_of_row(z[0].bad);
  if (__any(bad != 0.f))
#pragma unroll
    for (int i = 0; i < D / 16; ++i) z[0].o[i] += bad;
  if (part == 0) s_ml[wave * kRows + row] = float2v{z[0].m, l};
  auto piece = [&](int k) {
    const int x = k / 2, i = 2 * (k % 2);
    return float4v{z[0].o[2 * x][i], z[0].o[2 * x + 1][i], z[0].o[2 * x][i + 1], z[0].o[2 * x + 1][i + 1]};
  };
  float4v own[kOwn];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    if (k / kOwn == wave) own[k % kOwn] = piece(k);  // (the same for the whole wave)
    else s_o[(wave * kPieces + k) * 64 + lane] = piece(k);
  }
  __syncthreads();
  float2v ml[4];
  float4v others[3][kOwn];
#pragma unroll
  for (int w = 0; w < 4; ++w) ml[w] = s_ml[w * kRows + row];
#pragma unroll
  for (int i = 0; i < 3; ++i)
#pragma unroll
    for (int k = 0; k < kOwn; ++k) others[i][k] = s_o[((i + (i >= wave)) * kPieces + wave * kOwn + k) * 64 + lane];
  const float m = fmaxf(fmaxf(ml[0][0], ml[1][0]), fmaxf(ml[2][0], ml[3][0]));
  float all = 0.f, factor[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float h = root_exp2(ml[w][0] - m);
    all = fmaf(ml[w][1] * h, h, all);
    factor[w] = h * h;
  }
  const float mine = wave < 2 ? (wave == 0 ? factor[0] : factor[1]) : (wave == 2 ? factor[2] : factor[3]);
  if (!r.real) return;
  const int64_t to = u.part < 0 ? row_address(a, u.s0 + row, head) : (int64_t)(u.part + row) * a.g.Hkv + head;
  const float inverse = inverse_of(all) * kLess;
#pragma unroll
  for (int k = 0; k < kOwn; ++k) {
    float4v o = own[k] * mine;
#pragma unroll
    for (int i = 0; i < 3; ++i) o += others[i][k] * (i >= wave ? factor[i + 1] : factor[i]);
    const int at = wave * kOwn + k;
    const int64_t dims = to * D + 32 * (at / 2) + 8 * part + 4 * (at % 2);
    if (u.part < 0) store_out(a, dims, o * inverse);
    else *(float4v*)(a.part_acc + dims) = o * kLess;
  }
  if (wave == 0 && part == 0) {
    if (u.part >= 0) a.part_ml[to] = float2v{m + kRoom, all};
    else if (a.lse) a.lse[to] = k4::lse_of(m, all);
  }
}

}  // namespace k4
