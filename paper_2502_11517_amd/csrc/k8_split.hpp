// How a tile's tokens go in pieces: plain arithmetic, in chunks of kChunkTokens.
#pragma once
#include <cstdint>

namespace k8 {

constexpr int kChunkTokens = 128;    // pieces of a tile's tokens begin at multiples of this (32 for each wave)
constexpr int kLeastTokens = 384;    // a tile goes in as many pieces as there would be of this, begun ones counted, or
constexpr int kLeastAlone = 256;     // of this where half as many work-groups as the chip holds do with pieces of
constexpr int kAloneTokens = 1024;   // at most this

// What a tile's tokens cost, in halves of kChunkTokens plain ones: behind the prefix of a request with few rows, where every token's tag has to be looked
// at, three for two.
struct Cost {
  int chunks, cheap;  // the first `cheap` of them plain
  __device__ int all() const { return 3 * chunks - cheap; }
  __device__ int chunk_at(int64_t cost) const { return (int)(cost <= 2 * cheap ? cost / 2 : cheap + (cost - 2 * cheap) / 3); }
};

// Into how many pieces a tile goes, for pieces that cost `most` or less before they are rounded to chunks.
__device__ inline int pieces_of(int cost, int most) {
  const int n = (cost + most - 1) / most;
  return n > 1 ? n : 1;
}

// First chunk of piece k of `parts` (of piece `parts`: behind the last).  Pieces cost alike, rounded down to chunks: each is a chunk at least, and on the
// mean more than half as long as `most` says.
__device__ inline int piece_at(const Cost& c, int k, int parts) { return c.chunk_at((int64_t)c.all() * k / parts); }

}  // namespace k8
