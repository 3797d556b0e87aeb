// New rows of one layer into the 4-bit cache, and rows back out of it.
//
// A wave takes a run, at most 16 neighbouring rows that lie in one block, ascending, of one kv head, K or V.  A row's scales depend on that row
// alone, so nothing that was written before is rounded again.
//   K  a lane has 8 dims of a token, four neighbouring ones those under one scale
//   V  a lane has D / 64 neighbouring dims of all 16 tokens, whose codes lie together; a token's magnitudes are compared across the wave.  Codes of two
//      tokens share a byte, so those of the block's other tokens are read and put back.
//
// Long calls are bound by memory: 8192 rows of 8 heads of 128, bf16, 42 MB, in 11.9 us into the cache (3.6 TB/s) and in 9.6 out of it (4.4; a large copy 5.2);
// 32768 rows out of it, 169 MB, in 37 (4.6).  A step of eight rows takes 3.2 and 2.7 us, a launch and its two dependent reads (slots, then rows or codes).
// Tried and not taken for steps: rows asked for together with their slots, and V's codes set by atomics instead of read and put back (a step of eight rows, 8
// layers in and out, 51.4 -> 52.5 us; 128 single rows of as many requests 27 -> 35).
#pragma once
#include "k4_dev.hpp"
#include "k8_append.hpp"

namespace k4 {

struct RowArgs {
  Geometry g;
  int n_rows, group;  // rows that a work-group looks at
  const int* slot;
  int64_t k_stride, v_stride;    // of the rows, in values
  const void *k_new, *v_new;     // into the cache
  void *k_out, *v_out;           // out of it
  uint8_t *k, *v, *ks, *vs;
};

// Neighbouring rows that lie in one block, ascending.
struct Run {
  int row, n;       // the first, how many
  int offset;       // token of the first
  uint32_t tokens;  // theirs, a bit each
  int64_t block;
  int mine, lane;   // slots of the rows, from this lane on
  __device__ bool gaps() const { return (tokens >> offset) + 1 != 1u << n; }
  __device__ int token(int i) const { return gaps() ? __builtin_amdgcn_ds_bpermute(4 * (lane + min(i, n - 1)), mine) & 15 : offset + i; }  // of row i < n; for all lanes
  __device__ int rank(int t) const { return min(__builtin_popcount(tokens & ((1u << t) - 1u)), n - 1); }  // of token t's row; without one, of a near one's
};

// f(run) for every run that begins within the work-group's rows.  With GAPS it may leave slots out: what a wave puts back of a block's V codes has to be
// nobody else's to write.  Without, its slots are neighbours.
template <bool GAPS, class F>
__device__ inline void each_run(const RowArgs& a, int head, F f) {
  const int lane = threadIdx.x & 63, n_slots = a.g.n_pages << a.g.page_shift;
  const int first = blockIdx.x * a.group, last = min(first + a.group, a.n_rows);
  // lane k: the slot of row first + k - 1, and of the row ahead of it (read again, which is sooner than from lane to lane: a step's sixteen calls 49.9 / 50.7 us);
  // a run that begins within the group ends within 16 more rows
  const int row = first + lane - 1;
  const bool there = lane <= a.group + kBlock && row < a.n_rows;
  const int mine = there && row >= 0 ? a.slot[row] : -1, ahead = there && row > 0 ? a.slot[row - 1] : -1;
  const bool goes_on = ahead >= 0 && mine < n_slots && (GAPS ? mine > ahead : mine == ahead + 1) && (mine >> 4) == (ahead >> 4);
  const uint64_t joined = __ballot(goes_on);
  int i = first;
  while (i < last) {
    const int at = i - first + 1, slot = __builtin_amdgcn_readlane(mine, at);
    if (slot < 0 || slot >= n_slots) {
      ++i;
      continue;
    }
    const int n = 1 + __builtin_ctzll(~(joined >> (at + 1)));
    if (!(joined >> at & 1)) {  // the run begins here
      const int page = slot >> a.g.page_shift, b = (slot & (a.g.page_tokens - 1)) >> 4;
      uint32_t tokens = ((1u << n) - 1u) << (slot & 15);
      if (GAPS && __builtin_amdgcn_readlane(mine, at + n - 1) != slot + n - 1) {
        tokens = 0;
        for (int k = 0; k < n; ++k) tokens |= 1u << (__builtin_amdgcn_readlane(mine, at + k) & 15);
      }
      f(Run{i, n, slot & 15, tokens, ((int64_t)page * a.g.Hkv + head) * a.g.blocks_per_page + b, mine, at});
    }
    i += n;
  }
}

// K: a lane takes 8 dims of a token, D / 8 lanes a token; 512 / D tokens at a time.
template <int D>
struct KLane {
  static constexpr int kAtOnce = 512 / D, kTurns = kBlock / kAtOnce;
  int token, dim;
  __device__ KLane() : token((int)(threadIdx.x & 63) / (D / 8)), dim((int)(threadIdx.x & 63) % (D / 8) * 8) {}
  __device__ int64_t codes(int64_t block, int t) const { return block * kCodeBytes(D) + (dim / kGroup * kBlock + t) * 16 + dim % kGroup / 2; }
  __device__ int64_t scale(int64_t block, int t) const { return (block * kBlock + t) * (D / kGroup) + dim / kGroup; }
};

template <int D, int IN>
__device__ inline void append_k(const RowArgs& a, const Run& run, int head) {
  using L = KLane<D>;
  const L l;
  const int row = run.row, n = run.n;
  float x[L::kTurns][8];
  // Places without a row get the nearest one's and are dropped below: loads under branches wait for one another.
#pragma unroll
  for (int j = 0; j < L::kTurns; ++j)
    load_row<IN, 8>(a.k_new, (int64_t)(row + min(l.token + j * L::kAtOnce, n - 1)) * a.k_stride + head * D + l.dim, x[j]);
#pragma unroll
  for (int j = 0; j < L::kTurns; ++j) {
    uint32_t amax = magnitude(x[j], 0);
    amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0xb1, 0xf, 0xf, false));  // of lane ^ 1
    amax = max(amax, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)amax, 0x4e, 0xf, 0xf, false));  // of lane ^ 2
    const int byte = scale_byte(amax), i = l.token + j * L::kAtOnce;
    const float inverse = inverse_scale(byte);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[j][k] = byte == kNone ? 0.f : x[j][k] * inverse;
    const uint32_t w = encode8(x[j]);
    const int t = run.token(i);
    if (i >= n) continue;
    *(uint32_t*)(a.k + l.codes(run.block, t)) = w;
    if (l.dim % kGroup == 0) a.ks[l.scale(run.block, t)] = (uint8_t)byte;
  }
}

// 15 in the half byte of every token in `tokens`, of a dim's bytes 0 .. 7.
__device__ inline uint2v tokens_mask(uint32_t tokens) {
  uint64_t m = tokens & 0xffffu;
  m = (m | m << 24) & 0x000000ff000000ffull;
  m = (m | m << 12) & 0x000f000f000f000full;
  m = (m | m << 6) & 0x0303030303030303ull;
  m = (m | m << 3) & 0x1111111111111111ull;
  m *= 15;
  return uint2v{(uint32_t)m, (uint32_t)(m >> 32)};
}

template <int D, int IN>
__device__ inline void append_v(const RowArgs& a, const Run& run, int head) {
  constexpr int N = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t block = run.block;
  uint2v* codes = (uint2v*)(a.v + block * kCodeBytes(D)) + lane * N;
  float x[kBlock][N];
  // Places without a row get the nearest one's and are dropped below: loads under branches wait for one another.
#pragma unroll
  for (int t = 0; t < kBlock; ++t) load_row<IN, N>(a.v_new, (int64_t)(run.row + run.rank(t)) * a.v_stride + head * D + lane * N, x[t]);
  uint2v old[N];
#pragma unroll
  for (int j = 0; j < N; ++j) old[j] = uint2v{0, 0};
  if (run.n < kBlock)
#pragma unroll
    for (int j = 0; j < N; ++j) old[j] = codes[j];
  int byte = 0;  // lane t: of token t
#pragma unroll
  for (int t = 0; t < kBlock; ++t) {
    if (!(run.tokens >> t & 1)) continue;  // (the same for the whole wave)
    const int b = scale_byte(wave_max(magnitude(x[t], 0)));
    const float inverse = inverse_scale(b);
#pragma unroll
    for (int j = 0; j < N; ++j) x[t][j] = b == kNone ? 0.f : x[t][j] * inverse;
    byte = lane == t ? b : byte;
  }
  const uint2v mine = tokens_mask(run.tokens);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    uint2v w;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = x[8 * i + k][j];
      w[i] = (encode8(y) & mine[i]) | (old[j][i] & ~mine[i]);
    }
    codes[j] = w;
  }
  if (lane < kBlock && (run.tokens >> lane & 1)) a.vs[block * kBlock + lane] = (uint8_t)byte;
}

template <int D, int IN>
__global__ __launch_bounds__(256) void k4_append(RowArgs a) {
  const int task = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head = task >> 1;
  if (head >= a.g.Hkv) return;
  each_run<true>(a, head, [&](const Run& run) {
    if (task & 1)
      append_v<D, IN>(a, run, head);
    else
      append_k<D, IN>(a, run, head);
  });
}

// N neighbouring values of a row.
template <int OUT, int N>
__device__ inline void store_row(void* base, int64_t at, const float (&x)[N]) {
  if constexpr (OUT == kF32) {
    float* p = (float*)base + at;
    if constexpr (N >= 4) {
      for (int i = 0; i < N; i += 4) *(float4v*)(p + i) = float4v{x[i], x[i + 1], x[i + 2], x[i + 3]};
    } else if constexpr (N == 2) {
      *(float2v*)p = float2v{x[0], x[1]};
    } else {
      *p = x[0];
    }
  } else {
    // bf16 holds every code times a power of two: its upper half is the value, not a number included
    uint16_t b[N];
    for (int i = 0; i < N; ++i) {
      if constexpr (OUT == kBf16) {
        b[i] = (uint16_t)(__float_as_uint(x[i]) >> 16);
      } else {
        union { _Float16 h; uint16_t u; } c{(_Float16)x[i]};
        b[i] = c.u;
      }
    }
    uint16_t* p = (uint16_t*)base + at;
    if constexpr (N >= 8) {
      for (int i = 0; i < N; i += 8) {
        uint4v w;
        for (int k = 0; k < 4; ++k) w[k] = b[i + 2 * k] | (uint32_t)b[i + 2 * k + 1] << 16;
        *(uint4v*)(p + i) = w;
      }
    } else if constexpr (N == 2) {
      *(uint32_t*)p = b[0] | (uint32_t)b[1] << 16;
    } else {
      *p = b[0];
    }
  }
}

// A scale's byte as the conversions of codes take it: they go by the exponent alone, 0 is 2^-127 and 255 makes everything not a number.
__device__ inline float scale_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }

// n rows of a head that lie in LDS one behind the other, as OUT, to their places: 16 bytes a lane.  (V in bf16 by 4 bytes a lane, as its lanes have it, went at 3.2
// TB/s, this way at 3.9; fp32 K at 3.3 and 3.8.)  The wave's own LDS: its accesses are in order.
template <int D, int OUT>
__device__ inline void store_rows(const char* lds, void* base, int64_t row, int64_t stride, int n, int first) {
  constexpr int kSize = OUT == kF32 ? 4 : 2, kPieces = D * kSize / 16;  // of a row
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int j = 0; j < kBlock * kPieces / 64; ++j) {
    const int p = j * 64 + lane, i = p / kPieces, at = p % kPieces;
    const uint4v w = *(const uint4v*)(lds + p * 16);
    if (i < n) *(uint4v*)((char*)base + ((row + i) * stride + first) * kSize + at * 16) = w;
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

template <int D, int OUT>
__device__ inline void read_k(const RowArgs& a, int row, int n, int offset, int head, int64_t block, char* lds) {
  using L = KLane<D>;
  const L l;
  uint32_t w[L::kTurns];
  int byte[L::kTurns];
#pragma unroll
  for (int j = 0; j < L::kTurns; ++j) {
    const int t = offset + min(l.token + j * L::kAtOnce, n - 1);
    w[j] = *(const uint32_t*)(a.k + l.codes(block, t)), byte[j] = a.ks[l.scale(block, t)];
  }
#pragma unroll
  for (int j = 0; j < L::kTurns; ++j) {
    const int i = l.token + j * L::kAtOnce;
    float x[8];
    decode8(w[j], scale_of(byte[j]), x);
    if constexpr (OUT == kF32) store_row<OUT, 8>(lds, i * D + l.dim, x);
    else if (i < n) store_row<OUT, 8>(a.k_out, (int64_t)(row + i) * a.k_stride + head * D + l.dim, x);
  }
  if constexpr (OUT == kF32) store_rows<D, OUT>(lds, a.k_out, row, a.k_stride, n, head * D);
}

template <int D, int OUT>
__device__ inline void read_v(const RowArgs& a, int row, int n, int offset, int head, int64_t block, char* lds) {
  constexpr int N = D / 64;
  const int lane = threadIdx.x & 63;
  const uint2v* codes = (const uint2v*)(a.v + block * kCodeBytes(D)) + lane * N;
  uint2v w[N];
#pragma unroll
  for (int j = 0; j < N; ++j) w[j] = codes[j];
  const int bytes = a.vs[block * kBlock + (lane & 15)];
  float x[kBlock][N];
#pragma unroll
  for (int j = 0; j < N; ++j)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float y[8];
      decode8(w[j][i], 1.f, y);
#pragma unroll
      for (int k = 0; k < 8; ++k) x[8 * i + k][j] = y[k];
    }
#pragma unroll
  for (int t = 0; t < kBlock; ++t) {
    if (t < offset || t >= offset + n) continue;  // (the same for the whole wave)
    const int byte = __builtin_amdgcn_readlane(bytes, t);
    const float scale = byte == kNone ? __builtin_nanf("") : byte ? scale_of(byte) : 0x1p-127f;
#pragma unroll
    for (int j = 0; j < N; ++j) x[t][j] *= scale;
    store_row<OUT, N>(lds, (t - offset) * D + lane * N, x[t]);
  }
  store_rows<D, OUT>(lds, a.v_out, row, a.v_stride, n, head * D);
}

// Tasks: kv heads times K and V, or one of them where only that is wanted.
template <int D, int OUT>
__global__ __launch_bounds__(256) void k4_read(RowArgs a) {
  constexpr int kTile = kBlock * D * (OUT == kF32 ? 4 : 2);
  __shared__ __attribute__((aligned(16))) char tiles[4][kTile];
  char* lds = tiles[threadIdx.x >> 6];
  const bool both = a.k_out && a.v_out;
  const int task = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head = both ? task >> 1 : task;
  if (head >= a.g.Hkv) return;
  each_run<false>(a, head, [&](const Run& run) {
    if (both ? task & 1 : !a.k_out)
      read_v<D, OUT>(a, run.row, run.n, run.offset, head, run.block, lds);
    else
      read_k<D, OUT>(a, run.row, run.n, run.offset, head, run.block, lds);
  });
}

}  // namespace k4
