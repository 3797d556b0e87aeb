// Drafted tokens against the target's probabilities.
//
// The vocabulary goes in segments of kLoads * 256 tokens, each a wave's: lane l holds four neighbouring tokens of every 256.  Sums are in fp64, where those of
// fp32 probabilities hardly round, and always in the same order.  Small vocabularies take one work-group a sequence, which keeps all of it in registers; larger
// ones a launch of as many waves as there are segments, which leave their sums, and one in which a work-group a sequence finds the segment that the draw falls
// into and reads that once more.
//
// One sequence of 32000 tokens takes 7.3 us: positions, drafts and what becomes of them are reads behind one another, then one CU reads 256 KB.  64 sequences of 131072
// tokens, 67 MB, take 11.3 (sums, 5.9 TB/s: what is that small stays in the last-level cache) and 4.4 (the pick, a chain of reads).  Weights kept as fp64 took twice the
// registers and spilled (11.3 -> 7.6 for the one sequence, with its sums added once and the search by 256 tokens).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rows_rotate.hpp"

namespace rows {

struct VerifyArgs {
  int n_sequences, n_rows, vocab, segments;
  const int *row_offsets, *token, *slot;
  const void *target, *draft;
  int64_t target_stride, draft_stride;
  const float *draw, *last_draw;
  const int *length, *row_position;
  int *accepted, *next_token, *keep, *position_out;
  double* sums;     // workspace: [sequence][segment]
  int2* outcomes;   // workspace: [sequence] accepted, rejected
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

// What the target has beyond the draft's distribution; 0 for a NaN, too (the larger of a NaN and 0 is 0).
__device__ inline double weight(float p, float q) { return fmax((double)p - (double)q, 0.0); }

// What becomes of a sequence's drafts; every lane of the wave knows.
struct Outcome {
  int first, rows, accepted;
  int refused;   // rows of a sequence that has no place for them, whose `rows` are then 0
  int rejected;  // the token that was, -1: none
  __device__ bool left() const { return accepted + 1 < rows; }  // a draft was rejected: what the target has beyond the draft's distribution is left
};

__device__ inline Outcome rows_of(const VerifyArgs& a, int s) {
  const int end = min(max(a.row_offsets[a.n_sequences], 0), a.n_rows);
  Outcome v;
  v.first = min(max(a.row_offsets[s], 0), end);
  v.rows = min(max(a.row_offsets[s + 1], v.first), end) - v.first;
  v.refused = a.slot && v.rows && a.slot[v.first] < 0 ? v.rows : 0;
  if (v.refused) v.rows = 0;
  v.accepted = max(v.rows - 1, 0), v.rejected = -1;
  return v;
}

template <int TYPE>
__device__ inline Outcome decide(const VerifyArgs& a, int s) {
  const int lane = threadIdx.x & 63;
  Outcome v = rows_of(a, s);
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
  float p[LOADS][4], q[LOADS][4];  // q: 0 where the target alone counts, +inf where nothing is to count

  __device__ void load(const VerifyArgs& a, const Outcome& v, int from) {
    const int lane = threadIdx.x & 63;
    const int64_t row = v.first + v.accepted;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) four<TYPE>(a.target, row * a.target_stride, from + j * 256 + lane * 4, a.vocab, p[j]);
    if (a.draft && v.left()) {
#pragma unroll
      for (int j = 0; j < LOADS; ++j) four<TYPE>(a.draft, (row + 1) * a.draft_stride, from + j * 256 + lane * 4, a.vocab, q[j]);
    } else {
#pragma unroll
      for (int j = 0; j < LOADS; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) q[j][i] = !a.draft && v.left() && from + j * 256 + lane * 4 + i == v.rejected ? __builtin_inff() : 0.f;
    }
  }

  // Infinite weights count as 0: they are taken out here, and the sums need not look for them.  (p - q is that of an infinite p whatever a finite q, one below 0, too.)
  __device__ void hold() {
    float most = 0.f, least = 0.f;
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, p[j][i]), least = fminf(least, q[j][i]);
    if (__builtin_expect(!__any(most == __builtin_inff() || least == -__builtin_inff()), 1)) return;
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) p[j][i] = p[j][i] == __builtin_inff() ? -__builtin_inff() : p[j][i], q[j][i] = q[j][i] == -__builtin_inff() ? __builtin_inff() : q[j][i];
  }

  __device__ void target_alone() {
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) q[j][i] = 0.f;
  }

  // Weights are computed anew behind this: kept, as fp64, they take twice the registers that there are.
  __device__ void forget() {
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(p[j][i]), "+v"(q[j][i]));
  }

  __device__ double lane_sum(int j) const { return (weight(p[j][0], q[j][0]) + weight(p[j][1], q[j][1])) + (weight(p[j][2], q[j][2]) + weight(p[j][3], q[j][3])); }

  __device__ double sum() const {  // of the wave, in every lane
    double s = 0.0;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) s += lane_sum(j);
    return of_lane(upto(s), 63);
  }

  // The first token whose sum, from `before` on, is above `mark`; where rounding leaves none, the last that has a weight.
  __device__ int find(double before, double mark, int from) const {
    const int lane = threadIdx.x & 63;
    double up[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; ++j) up[j] = upto(lane_sum(j));
    int at = 0;  // which 256 tokens
    double base = before;
    bool found = false;
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const double all = of_lane(up[j], 63);
      if (!found && all > 0.0) at = j, base = before, found = before + all > mark;  // (the same for all lanes)
      before += all;
    }
    float x[4], y[4];
    double mine = 0.0;
#pragma unroll
    for (int j = 0; j < LOADS; ++j)
      if (j == at) {
        mine = base + up[j];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = p[j][i], y[i] = q[j][i];
      }
    double here = mine - ((weight(x[0], y[0]) + weight(x[1], y[1])) + (weight(x[2], y[2]) + weight(x[3], y[3])));
    int hit = -1, some = -1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const double w = weight(x[i], y[i]);
      here += w;
      if (w > 0.0) some = i;
      if (hit < 0 && w > 0.0 && here > mark) hit = i;
    }
    if (hit < 0 && some >= 0 && mine > mark) hit = some;  // (its own sum was rounded otherwise)
    const uint64_t hits = __ballot(hit >= 0), any = __ballot(some >= 0);
    const int k = hits ? __builtin_ctzll(hits) : any ? 63 - __builtin_clzll(any) : 0;
    return from + at * 256 + k * 4 + max(__builtin_amdgcn_readlane(hits ? hit : some, k), 0);
  }
};

// Everything but next_token; the threads of a work-group.
__device__ inline void put_down(const VerifyArgs& a, int s, const Outcome& v) {
  if (threadIdx.x == 0) {
    a.accepted[s] = v.accepted;
    if (a.keep) a.keep[s] = v.rows ? max(a.length[s] - v.rows + 1 + v.accepted, 0) : a.length[s];
    if (v.rows == 0) a.next_token[s] = -1;
  }
  if (a.position_out)
    for (int i = threadIdx.x; i < v.rows + v.refused; i += blockDim.x)
      a.position_out[v.first + i] = a.row_position[v.first + i] + (v.refused ? 0 : 1 + v.accepted);
}

__device__ inline double mark_of(const VerifyArgs& a, int s, double total) {
  return (double)fminf(fmaxf(a.last_draw[s], 0.f), 0x1.fffffep-1f) * total;
}

// A sequence a work-group, the whole vocabulary in its registers.
template <int TYPE, int LOADS>
__global__ __launch_bounds__(1024) void rows_verify_whole(VerifyArgs a) {
  __shared__ double s_sum[2][16];
  const int s = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), from = wave * LOADS * 256;
  const Outcome v = decide<TYPE>(a, s);
  if (v.rows == 0) return put_down(a, s, v);
  Segment<TYPE, LOADS> g;
  g.load(a, v, from);
  put_down(a, s, v);
  double own, total, before;
  g.hold();
  for (int turn = 0; turn < 2; ++turn) {  // where nothing is left of p - q, p alone
    own = g.sum();
    g.forget();
    if ((threadIdx.x & 63) == 0) s_sum[turn][wave] = own;
    __syncthreads();
    total = before = 0.0;
    for (int w = 0; w < (int)blockDim.x >> 6; ++w) {
      if (w == wave) before = total;
      total += s_sum[turn][w];
    }
    if (total > 0.0 || !v.left()) break;
    g.target_alone();
  }
  if (!(total > 0.0)) {
    if (threadIdx.x == 0) a.next_token[s] = -1;
    return;
  }
  const double mark = mark_of(a, s, total);
  if (before <= mark && before + own > mark) {  // (one wave, since sums go up by the same additions everywhere)
    const int t = g.find(before, mark, from);
    if ((threadIdx.x & 63) == 0) a.next_token[s] = t;
  }
}

// Sums of the segments; four of a sequence to a work-group.  What becomes of the drafts goes to the next launch.
template <int TYPE>
__global__ __launch_bounds__(256) void rows_verify_sums(VerifyArgs a) {
  const int s = blockIdx.y, segment = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (segment >= a.segments) return;
  const Outcome v = decide<TYPE>(a, s);
  if (segment == 0 && (threadIdx.x & 63) == 0) a.outcomes[s] = int2{v.accepted, v.rejected};
  if (v.rows == 0) return;
  Segment<TYPE, kSegment / 256> g;
  g.load(a, v, segment * kSegment);
  g.hold();
  const double own = g.sum();
  if ((threadIdx.x & 63) == 0) a.sums[(int64_t)s * a.segments + segment] = own;
}

// The segment that the draw falls into, and the token; a sequence a work-group.
template <int TYPE>
__global__ __launch_bounds__(256) void rows_verify_pick(VerifyArgs a) {
  __shared__ double s_sum[4];
  const int s = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  double* sums = a.sums + (int64_t)s * a.segments;
  const int each = (a.segments + 255) / 256, from = min((int)threadIdx.x * each, a.segments), to = min(from + each, a.segments);  // this thread's
  const double first = from < to ? sums[from] : 0.0;  // (asked for at once; of a sequence without rows it is nothing)
  const int2 known = a.outcomes[s];
  Outcome v = rows_of(a, s);
  v.accepted = known.x, v.rejected = known.y;
  put_down(a, s, v);
  if (v.rows == 0) return;
  Segment<TYPE, kSegment / 256> g;
  bool alone = false;  // nothing is left of p - q: p alone
  double own = first;
  for (int i = from + 1; i < to; ++i) own += sums[i];
  double up, total, before;
  auto add = [&] {
    up = upto(own);
    if (lane == 63) s_sum[wave] = up;
    __syncthreads();
    total = before = 0.0;
    for (int w = 0; w < 4; ++w) {
      if (w == wave) before = total;
      total += s_sum[w];
    }
  };
  add();
  if (!(total > 0.0) && v.left()) {
    alone = true;
    for (int i = wave; i < a.segments; i += 4) {
      g.load(a, v, i * kSegment);
      g.hold();
      g.target_alone();
      const double x = g.sum();
      if (lane == 0) sums[i] = x;
    }
    __syncthreads();
    own = 0.0;
    for (int i = from; i < to; ++i) own += sums[i];
    add();
  }
  if (!(total > 0.0)) {
    if (threadIdx.x == 0) a.next_token[s] = -1;
    return;
  }
  // the wave, the thread in it, the segment of that: each the first one whose sum is above the mark
  const double mark = mark_of(a, s, total);
  if (!(before <= mark && before + s_sum[wave] > mark)) return;
  const double end = before + up;
  const bool some = own > 0.0;
  const uint64_t any = __ballot(some), past = __ballot(some && end > mark);  // (lanes' sums are rounded each in its own way)
  const int k = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(any);
  double here = k ? of_lane(end, k - 1) : before;
  const int begin = __builtin_amdgcn_readlane(from, k), stop = __builtin_amdgcn_readlane(to, k);
  int segment = begin;
  double base = here;
  if (each > 1) {
    for (int i = begin; i < stop; ++i) {
      const double w = sums[i];
      if (w > 0.0) segment = i, base = here;
      here += w;
      if (here > mark && w > 0.0) break;
    }
  }
  g.load(a, v, segment * kSegment);
  g.hold();
  if (alone) g.target_alone();
  const int t = g.find(base, mark, segment * kSegment);
  if (lane == 0) a.next_token[s] = t;
}

}  // namespace rows
