// How a tile's tokens go in pieces: plain arithmetic, in chunks of kChunkTokens.
#pragma once
#include <cstdint>

namespace k8 {

constexpr int kChunkTokens = 128;    // pieces of a tile's tokens begin at multiples of this (32 for each wave)
constexpr int kLeastTokens = 384;    // a tile goes in as many pieces as there would be of this, begun ones counted, or
constexpr int kLeastAlone = 256;     // of this (kLeastAlone4, in the 4-bit cache) where half as many work-groups as the chip holds do with pieces of
constexpr int kAloneTokens = 1024;   // at most this
constexpr int kLeastAlone4 = 128;    // two and eight rows over 1000 / 2000 / 3500 tokens, a layer: 10.4 and 11.1 / 10.5 and 11.5 / 10.7 and 11.8 us; by 256:
                                     // 10.9 and 11.9 / 10.8 and 11.9 / 11.1 and 12.1

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

// How many there may be at most, whatever `most` says, with none empty: on the mean a piece costs no less than the dearest chunk.  (From kLeastAlone on that
// is so without asking.)
__device__ inline int most_pieces(const Cost& c) {
  const int n = c.cheap < c.chunks ? c.all() / 3 : c.chunks;
  return n > 1 ? n : 1;
}

// First chunk of piece k of `parts` (of piece `parts`: behind the last).  Pieces cost alike, rounded down to chunks: each is a chunk at least, and on the
// mean more than half as long as `most` says.
__device__ inline int piece_at(const Cost& c, int k, int parts) { return c.chunk_at((int64_t)c.all() * k / parts); }

}  // namespace k8
