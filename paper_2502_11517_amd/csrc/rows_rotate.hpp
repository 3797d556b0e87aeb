// Rotary positions of a step's rows.
//
// A work-group takes some heads of one row: its threads find the row's cosines and sines, a plane apiece, while the values that they will turn are on their way.
// Angles are taken in 64 bits and reduced to a fraction of a revolution before they become fp32 (positions of 10^6 times a frequency near 1 are 10^5 turns);
// 16-bit rows then take the hardware's sine and cosine, which are off by 10^-6 or so, fp32 rows the library's.
//
// Bound by memory in long calls: 8192 rows of 32 + 8 heads of 128, bf16, 168 MB, in 34.9 us, 4.8 TB/s (a large copy 5.2).  A step of eight rows takes 2.9 us, its
// launch and one way to memory, positions and values at a time.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace rows {

enum { kF32 = 0, kBf16 = 1, kF16 = 2 };
constexpr int kMaxDim = 256;

using uint4v = __attribute__((ext_vector_type(4))) uint32_t;

struct Side {  // q or k
  const void* in;
  void* out;
  int64_t in_stride, out_stride;  // between rows, in values
};

struct RotateArgs {
  int n_rows, n_q, n_heads;  // heads 0 .. n_q - 1 are q's, the others k's
  int D, planes, interleaved;
  int pieces, at_once;       // pieces of a head, and heads that a work-group takes
  float magnitude, direction;
  const double* frequency;
  const int* position;
  Side q, k;
};

template <int TYPE>
__device__ inline float to_float(uint32_t b) {
  if constexpr (TYPE == kF32) return __uint_as_float(b);
  if constexpr (TYPE == kBf16) return __uint_as_float(b << 16);
  union { uint16_t u; _Float16 h; } c{(uint16_t)b};
  return (float)c.h;
}

template <int TYPE>
__device__ inline uint32_t from_float(float x) {  // rounded to the nearest, ties to even
  if constexpr (TYPE == kF32) return __float_as_uint(x);
  if constexpr (TYPE == kBf16) {
    union { __bf16 h; uint16_t u; } c{(__bf16)x};
    return c.u;
  }
  union { _Float16 h; uint16_t u; } c{(_Float16)x};
  return c.u;
}

// 16 bytes of a row as values, and back.
template <int TYPE>
struct Piece {
  static constexpr int N = TYPE == kF32 ? 4 : 8;
  float x[N];
  __device__ void load(const void* row, int at) {
    const uint4v w = *(const uint4v*)((const char*)row + (int64_t)at * (16 / N));
    for (int i = 0; i < N; ++i) x[i] = TYPE == kF32 ? __uint_as_float(w[i & 3]) : to_float<TYPE>(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu);
  }
  __device__ void store(void* row, int at) const {
    uint4v w;
    for (int i = 0; i < 4; ++i) {
      if constexpr (TYPE == kF32) w[i] = __float_as_uint(x[i]);
      else w[i] = from_float<TYPE>(x[2 * i]) | from_float<TYPE>(x[2 * i + 1]) << 16;
    }
    *(uint4v*)((char*)row + (int64_t)at * (16 / N)) = w;
  }
};

template <int TYPE>
__device__ inline void turn_of(double revolutions, float& c, float& s) {
  const float part = (float)(revolutions - __builtin_rint(revolutions));  // in [-1/2, 1/2]
  if constexpr (TYPE == kF32) {
    sincospif(2.f * part, &s, &c);
  } else {
    c = __builtin_amdgcn_cosf(part), s = __builtin_amdgcn_sinf(part);
  }
}

// WIDE: every piece of a head is 16 bytes, of one kind: half-split planes (then the piece is two, half the turned dims apart), interleaved ones, or dims that
// stay.  Else a piece is one plane or one dim that stays: rope_dims that are not whole 16-byte pieces.  A work-group turns ROWS rows.
// The narrow form is bound by its instructions and work-groups, two to four bytes to each: 8192 rows of 32 + 8 heads of 128 dims, of which 34 or 50 are turned, take 188 us,
// 100 128, against 35 of the wide one; a work-group has one row's two or three heads, and each finds the row's sines anew.
template <int TYPE, bool WIDE, int ROWS>
__global__ __launch_bounds__(256) void rows_rotate(RotateArgs a) {
  __shared__ float s_cos[ROWS][kMaxDim / 2], s_sin[ROWS][kMaxDim / 2];
  using T = std::conditional_t<TYPE == kF32, uint32_t, uint16_t>;
  constexpr int N = WIDE ? Piece<TYPE>::N : 1;
  const int row = blockIdx.x * ROWS, n_rows = min(ROWS, a.n_rows - row), slot = threadIdx.x / a.pieces, piece = threadIdx.x - slot * a.pieces;
  const int head = blockIdx.y * a.at_once + slot;
  const bool mine = slot < a.at_once && head < a.n_heads;
  const Side& side = head < a.n_q ? a.q : a.k;
  const int64_t at = (int64_t)(head < a.n_q ? head : head - a.n_q) * a.D;
  const char* in = (const char*)side.in + (row * side.in_stride + at) * sizeof(T);
  char* out = (char*)side.out + (row * side.out_stride + at) * sizeof(T);
  const int64_t in_step = side.in_stride * sizeof(T), out_step = side.out_stride * sizeof(T);
  // pieces of a head: the turned ones, then those that stay
  const int turned = a.interleaved && WIDE ? 2 * a.planes / N : a.planes / N;
  const bool turns = piece < turned;
  const int first = turns ? (a.interleaved ? (WIDE ? piece * N : 2 * piece) : piece * N) : 2 * a.planes + (piece - turned) * N;
  const int second = a.interleaved ? first + 1 : first + a.planes;  // of a half-split plane, or of one alone
  Piece<TYPE> x[ROWS], y[ROWS];
  if (mine) {
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
      const char* from = in + min(r, n_rows - 1) * in_step;  // (no branches around loads: they would wait for one another)
      if constexpr (WIDE) {
        x[r].load(from, first);
        if (turns && !a.interleaved) y[r].load(from, second);
      } else {
        x[r].x[0] = to_float<TYPE>(((const T*)from)[first]);
        if (turns) y[r].x[0] = to_float<TYPE>(((const T*)from)[second]);
      }
    }
  }
  for (int i = threadIdx.x; i < n_rows * a.planes; i += 256) {
    constexpr double kTurn = 0.15915494309189533577;  // 1 / (2 pi)
    const int r = ROWS == 1 ? 0 : i / a.planes, f = i - r * a.planes;
    float c, s;
    turn_of<TYPE>((double)a.position[row + r] * (a.frequency[f] * kTurn), c, s);
    s_cos[r][f] = c * a.magnitude, s_sin[r][f] = s * a.direction;
  }
  __syncthreads();
  if (!mine || (!turns && in == out)) return;
#pragma unroll
  for (int r = 0; r < ROWS; ++r) {
    if (r >= n_rows) break;
    char* to = out + r * out_step;
    if constexpr (WIDE) {
      if (turns && a.interleaved) {
        for (int i = 0; i < N; i += 2) {
          const float c = s_cos[r][(first + i) / 2], s = s_sin[r][(first + i) / 2], u = x[r].x[i], v = x[r].x[i + 1];
          x[r].x[i] = u * c - v * s, x[r].x[i + 1] = v * c + u * s;
        }
      } else if (turns) {
        for (int i = 0; i < N; ++i) {
          const float c = s_cos[r][first + i], s = s_sin[r][first + i], u = x[r].x[i], v = y[r].x[i];
          x[r].x[i] = u * c - v * s, y[r].x[i] = v * c + u * s;
        }
        y[r].store(to, second);
      }
      x[r].store(to, first);
    } else {
      float u = x[r].x[0];
      if (turns) {
        const float c = s_cos[r][piece], s = s_sin[r][piece], v = y[r].x[0];
        ((T*)to)[second] = (T)from_float<TYPE>(v * c + u * s);
        u = u * c - v * s;
      }
      ((T*)to)[first] = (T)from_float<TYPE>(u);
    }
  }
}

}  // namespace rows
