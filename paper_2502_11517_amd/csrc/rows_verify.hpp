// Drafted tokens against the target's probabilities.
//
// The vocabulary goes in segments of kLoads * 256 tokens, each a wave's: lane l holds four neighbouring tokens of every 256.  Sums are in fp64, where those of
// fp32 probabilities hardly round, and always in the same order.  Small vocabularies take one work-group a sequence, which keeps all of it in registers; larger
// ones a launch of as many waves as there are segments, which leave their sums, and one in which a work-group a sequence finds the segment that the draw falls
// into and reads that once more.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rows_rotate.hpp"

namespace rows {

struct VerifyArgs {
  int n_sequences, n_rows, vocab, segments;
  const int *row_offsets, *token;
  const void *target, *draft;
  int64_t target_stride, draft_stride;
  const float *draw, *last_draw;
  const int *length, *row_position;
  int *accepted, *next_token, *keep, *position_out;
  struct Sums* sums;  // workspace: [sequence][segment]
};

struct Sums {
  double rest, all;  // of max(p - q, 0), of p
};

constexpr int kSegment = 1024;  // tokens of a wave, where a sequence takes many

template <int CTRL, int ROWS = 0xf>
__device__ inline double dpp(double x) {  // of another lane; 0 where there is none
  const int64_t b = __double_as_longlong(x);
  const int lo = __builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
  return __longlong_as_double((int64_t)(uint32_t)lo | (int64_t)hi << 32);
}

// Sum over the lanes up to and including this one.
__device__ inline double upto(double x) {
  x += dpp<0x111>(x);  // row_shr: 1, 2, 4, 8
  x += dpp<0x112>(x);
  x += dpp<0x114>(x);
  x += dpp<0x118>(x);
  x += dpp<0x142, 0xa>(x);  // the end of a row of 16 lanes into the next, rows 1 and 3
  x += dpp<0x143, 0xc>(x);  // of half a wave into the other
  return x;
}

__device__ inline double of_lane(double x, int lane) {
  const int64_t b = __double_as_longlong(x);
  return __longlong_as_double((int64_t)(uint32_t)__builtin_amdgcn_readlane((int)b, lane) | (int64_t)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32);
}

template <int TYPE>
__device__ inline float value(const void* base, int64_t at) {
  using T = std::conditional_t<TYPE == kF32, uint32_t, uint16_t>;
  return to_float<TYPE>(((const T*)base)[at]);
}

// Four neighbouring values, wherever a row begins; beyond n they are 0.
template <int TYPE>
__device__ inline void four(const void* base, int64_t row, int at, int n, float (&x)[4]) {
  using T = std::conditional_t<TYPE == kF32, uint32_t, uint16_t>;
  struct __attribute__((packed, aligned(sizeof(T)))) Quad { T v[4]; };
  const T* p = (const T*)base + row + at;
  if (at + 4 <= n) {
    const Quad q = *(const Quad*)p;
    for (int i = 0; i < 4; ++i) x[i] = to_float<TYPE>(q.v[i]);
  } else {
    for (int i = 0; i < 4; ++i) x[i] = at + i < n ? to_float<TYPE>(p[i]) : 0.f;
  }
}

__device__ inline double weight(double x) { return x > 0.0 && x < __builtin_inf() ? x : 0.0; }

// What becomes of a sequence's drafts; every lane of the wave knows.
struct Verdict {
  int first, rows, accepted;
  int rejected;  // the token that was, -1: none
};

template <int TYPE>
__device__ inline Verdict judge(const VerifyArgs& a, int s) {
  const int lane = threadIdx.x & 63;
  const int end = min(max(a.row_offsets[a.n_sequences], 0), a.n_rows);
  Verdict v;
  v.first = min(max(a.row_offsets[s], 0), end);
  v.rows = min(max(a.row_offsets[s + 1], v.first), end) - v.first;
  v.accepted = max(v.rows - 1, 0), v.rejected = -1;
  for (int i0 = 1; i0 < v.rows; i0 += 64) {
    const int i = i0 + lane, row = v.first + min(i, v.rows - 1);
    const int t = a.token[row];
    const bool known = t >= 0 && t < a.vocab;
    const int at = known ? t : 0;
    const float u = fminf(fmaxf(a.draw[row], 0.f), 0x1.fffffep-1f);
    const double p = value<TYPE>(a.target, (row - 1) * a.target_stride + at);
    const double q = a.draft ? (double)value<TYPE>(a.draft, row * a.draft_stride + at) : 1.0;
    const uint64_t lost = __ballot(i < v.rows && !(known && (double)u * q < p));
    if (lost) {
      const int k = __builtin_ctzll(lost);
      v.accepted = i0 + k - 1, v.rejected = __builtin_amdgcn_readlane(t, k);
      break;
    }
  }
  return v;
}

// A wave's segment: weights of 4 * LOADS tokens in every lane.
template <int TYPE, int LOADS>
struct Segment {
  float p[LOADS][4], q[LOADS][4];

  __device__ void load(const VerifyArgs& a, const Verdict& v, int from) {
    const int lane = threadIdx.x & 63;
    const int64_t row = v.first + v.accepted;
    const bool both = a.draft && v.accepted + 1 < v.rows;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) four<TYPE>(a.target, row * a.target_stride, from + j * 256 + lane * 4, a.vocab, p[j]);
    if (both) {
#pragma unroll
      for (int j = 0; j < LOADS; ++j) four<TYPE>(a.draft, (row + 1) * a.draft_stride, from + j * 256 + lane * 4, a.vocab, q[j]);
    } else {
#pragma unroll
      for (int j = 0; j < LOADS; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) q[j][i] = !a.draft && from + j * 256 + lane * 4 + i == v.rejected ? __builtin_inff() : 0.f;
    }
  }

  // Weights are computed anew behind this: kept, as fp64, they take twice the registers that there are.
  __device__ void forget() {
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(p[j][i]), "+v"(q[j][i]));
  }

  __device__ double at(bool rest, int j, int i) const { return rest ? weight((double)p[j][i] - (double)q[j][i]) : weight((double)p[j][i]); }

  __device__ double lane_sum(bool rest, int j) const { return (at(rest, j, 0) + at(rest, j, 1)) + (at(rest, j, 2) + at(rest, j, 3)); }

  __device__ Sums sums() const {  // of the wave, in every lane
    Sums s{0.0, 0.0};
#pragma unroll
    for (int j = 0; j < LOADS; ++j) s.rest += lane_sum(true, j), s.all += lane_sum(false, j);
    return Sums{of_lane(upto(s.rest), 63), of_lane(upto(s.all), 63)};
  }

  // The first token whose sum, from `before` on, is above `mark`; where rounding leaves none, the last that has a weight.
  __device__ int find(bool rest, double before, double mark, int from) const {
    const int lane = threadIdx.x & 63;
    int found = -1, last = -1;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const double mine = lane_sum(rest, j), up = before + upto(mine);
      double here = up - mine;
      int hit = -1, some = -1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const double w = at(rest, j, i);
        here += w;
        if (w > 0.0) some = i;
        if (hit < 0 && w > 0.0 && here > mark) hit = i;
      }
      if (hit < 0 && some >= 0 && up > mark) hit = some;  // (its own sum was rounded otherwise)
      const uint64_t hits = __ballot(hit >= 0), any = __ballot(some >= 0);
      if (found < 0 && hits) {
        const int k = __builtin_ctzll(hits);
        found = from + j * 256 + k * 4 + __builtin_amdgcn_readlane(hit, k);
      }
      if (any) {
        const int k = 63 - __builtin_clzll(any);
        last = from + j * 256 + k * 4 + __builtin_amdgcn_readlane(some, k);
      }
      before = of_lane(up, 63);
    }
    return found >= 0 ? found : last;
  }
};

// Everything but next_token; the threads of a work-group.
__device__ inline void put_down(const VerifyArgs& a, int s, const Verdict& v) {
  if (threadIdx.x == 0) {
    a.accepted[s] = v.accepted;
    if (a.keep) a.keep[s] = v.rows ? max(a.length[s] - v.rows + 1 + v.accepted, 0) : a.length[s];
    if (v.rows == 0) a.next_token[s] = -1;
  }
  if (a.position_out)
    for (int i = threadIdx.x; i < v.rows; i += blockDim.x) a.position_out[v.first + i] = a.row_position[v.first + i] + 1 + v.accepted;
}

__device__ inline double mark_of(const VerifyArgs& a, int s, double total) {
  return (double)fminf(fmaxf(a.last_draw[s], 0.f), 0x1.fffffep-1f) * total;
}

// A sequence a work-group, the whole vocabulary in its registers.
template <int TYPE, int LOADS>
__global__ __launch_bounds__(1024) void rows_verify_whole(VerifyArgs a) {
  __shared__ Sums s_sums[16];
  const int s = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), from = wave * LOADS * 256;
  const Verdict v = judge<TYPE>(a, s);
  put_down(a, s, v);
  if (v.rows == 0) return;
  Segment<TYPE, LOADS> g;
  g.load(a, v, from);
  const Sums own = g.sums();
  g.forget();
  if ((threadIdx.x & 63) == 0) s_sums[wave] = own;
  __syncthreads();
  Sums total{0.0, 0.0}, before{0.0, 0.0};
  for (int w = 0; w < (int)blockDim.x >> 6; ++w) {
    if (w == wave) before = total;
    total.rest += s_sums[w].rest, total.all += s_sums[w].all;
  }
  const bool rest = v.accepted + 1 < v.rows && total.rest > 0.0;
  const double mark = mark_of(a, s, rest ? total.rest : total.all);
  if (!(total.all > 0.0) && !rest) {
    if (threadIdx.x == 0) a.next_token[s] = -1;
    return;
  }
  const double lower = rest ? before.rest : before.all, mine = rest ? own.rest : own.all;
  if (lower <= mark && lower + mine > mark) {  // (one wave, since sums go up by the same additions everywhere)
    const int t = g.find(rest, lower, mark, from);
    if ((threadIdx.x & 63) == 0) a.next_token[s] = t;
  }
}

// Sums of the segments; four of a sequence to a work-group.
template <int TYPE>
__global__ __launch_bounds__(256) void rows_verify_sums(VerifyArgs a) {
  const int s = blockIdx.y, segment = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (segment >= a.segments) return;
  const Verdict v = judge<TYPE>(a, s);
  if (v.rows == 0) return;
  Segment<TYPE, kSegment / 256> g;
  g.load(a, v, segment * kSegment);
  const Sums own = g.sums();
  if ((threadIdx.x & 63) == 0) a.sums[(int64_t)s * a.segments + segment] = own;
}

// The segment that the draw falls into, and the token; a sequence a work-group.
template <int TYPE>
__global__ __launch_bounds__(256) void rows_verify_pick(VerifyArgs a) {
  __shared__ Sums s_sums[4];
  const int s = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Sums* sums = a.sums + (int64_t)s * a.segments;
  const Verdict v = judge<TYPE>(a, s);
  put_down(a, s, v);
  if (v.rows == 0) return;
  const int each = (a.segments + 255) / 256, from = min((int)threadIdx.x * each, a.segments), to = min(from + each, a.segments);  // this thread's
  Sums own{0.0, 0.0};
  for (int i = from; i < to; ++i) own.rest += sums[i].rest, own.all += sums[i].all;
  const Sums up{upto(own.rest), upto(own.all)};
  if (lane == 63) s_sums[wave] = up;
  __syncthreads();
  Sums total{0.0, 0.0}, before{0.0, 0.0};
  for (int w = 0; w < 4; ++w) {
    if (w == wave) before = total;
    total.rest += s_sums[w].rest, total.all += s_sums[w].all;
  }
  const bool rest = v.accepted + 1 < v.rows && total.rest > 0.0;
  const double mark = mark_of(a, s, rest ? total.rest : total.all);
  if (!(total.all > 0.0) && !rest) {
    if (threadIdx.x == 0) a.next_token[s] = -1;
    return;
  }
  // the wave, the thread in it, the segment of that: each the first one whose sum is above the mark
  const double lower = rest ? before.rest : before.all, upper = lower + (rest ? s_sums[wave].rest : s_sums[wave].all);
  if (!(lower <= mark && upper > mark)) return;
  const double end = lower + (rest ? up.rest : up.all);
  const bool some = (rest ? own.rest : own.all) > 0.0;
  const uint64_t any = __ballot(some), past = __ballot(some && end > mark);  // (lanes' sums are rounded each in its own way)
  const int k = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any);
  double here = k ? of_lane(end, k - 1) : lower;
  const int first = __builtin_amdgcn_readlane(from, k), last = __builtin_amdgcn_readlane(to, k);
  int segment = -1;
  double base = here;
  for (int i = first; i < last; ++i) {
    const double w = rest ? sums[i].rest : sums[i].all;
    if (w > 0.0) segment = i, base = here;
    here += w;
    if (here > mark && w > 0.0) break;
  }
  Segment<TYPE, kSegment / 256> g;
  g.load(a, v, segment * kSegment);
  const int t = g.find(rest, base, mark, segment * kSegment);
  if (lane == 0) a.next_token[s] = t;
}

}  // namespace rows
