// Split of the attention's work: which stacked rows of which request over which tokens, a unit per (rows, tokens), times Hkv.
//
// Rows come in tiles of 32, or, in requests with more than 128 stacked rows, of 64 (a wave then turns its codes once for two groups; with fewer rows,
// fewer and longer pieces of the tokens are worth more: 128 rows over 49k tokens 60 us a layer in tiles of 32, 87 of 64).  A tile's tokens go in even
// pieces, and what they leave, partial rows, k8_merge joins.  How long pieces are:
//   * One work-group a CU where pieces of up to 1024 tokens do with that, no more of them than pieces of 256 would be.  Two on a CU take turns at its
//     SIMDs and gain a tenth; 328 of them take as long as 512 would.  Eight rows over 10k tokens in 224 / 328 pieces: 14.2 / 17.5 us a layer; 22 rows over
//     30k 134 / 148 us a pass.
//   * Else two, no more pieces than of 384 tokens.  The older one of a SIMD's two waves runs ahead, so the second half of the list stands in reverse:
//     a CU that starts with a dear piece (behind the prefix, where tags are looked at) gets a plain one with it.
//   * Even pieces of chunks of 128 tokens: what goes in n can come out at half of these lengths, a chunk at least (769 tokens: 128, 256, 256, 129).
//   * Where tables have room for at most 768 tokens (512 with tiles of 64) nothing is split, which saves the launch of k8_merge: two and eight rows over
//     300 / 500 / 700 tokens, a layer, 8.2 and 9.6 / 8.7 and 10.9 / 11.5 us; 11.1 and 12.4 / 11.2 and 12.2 / 12.1 in wide tables, as a server's are (the
//     table's width is all that the host knows of the lengths).
// What it takes, 3 to 5 us a step for all layers, is the launch and its chain of reads and sums.  From 256 requests or tiles on (k8_plan_long) 10 to 13.
#pragma once
#include "k8_dev.hpp"

namespace k8 {

struct PlanArgs {
  Geometry g;
  int n_requests, n_rows;
  int wide;       // requests with more than kManyRows stacked rows take tiles of 64
  int whole;      // no tile is split
  int capacity;   // units that the chip takes at once
  int max_units, max_tiles, max_part_rows;
  const int *length, *row_offsets, *prefix_len, *slot, *table;
  Unit* units;
  int* unit_blocks;  // [max_units][kUnitBlocks]
  Tile* tiles;
  int* w_tiles;   // workspace, n_requests + 1: tiles of the requests up to and including this one
};

struct RequestTiles {
  int row0, n, length, prefix, tile_rows, n_tiles;
};

// Request r, or (r == n_requests) the rows behind the last request, which see nothing.
__device__ inline RequestTiles request_tiles(const PlanArgs& a, int r) {
  RequestTiles q;
  const int here = max(min(r, a.n_requests - 1), 0);
  const int first = a.row_offsets[min(r, a.n_requests)], next = a.row_offsets[min(r + 1, a.n_requests)], all = a.row_offsets[a.n_requests];
  const int length = a.length[here], prefix = a.prefix_len ? a.prefix_len[here] : 0;
  const int end = min(max(all, 0), a.n_rows);
  if (r == a.n_requests) {
    q.row0 = end, q.n = a.n_rows - end, q.length = 0;
  } else {
    q.row0 = min(max(first, 0), end);
    q.n = min(max(next, q.row0), end) - q.row0;
    q.length = min(max(length, 0), a.g.table_width << a.g.page_shift);
    if (a.slot && q.n > 0 && a.slot[q.row0] < 0) q.length = 0;
  }
  q.prefix = min(max(prefix, 0), q.length);
  const int64_t stacked = (int64_t)q.n * a.g.G;
  q.tile_rows = a.wide && stacked > kManyRows ? kWideRows : kRows;
  q.n_tiles = (int)((stacked + q.tile_rows - 1) / q.tile_rows);
  return q;
}

// Tile t of request r, unsplit.
__device__ inline Unit tile_of(const PlanArgs& a, int r, const RequestTiles& q, int t) {
  Unit u{};
  const int first = t * q.tile_rows, stacked = q.n * a.g.G;
  u.request = max(min(r, a.n_requests - 1), 0);
  u.s0 = q.row0 * a.g.G + first;
  u.n_rows = min(stacked - first, q.tile_rows);
  u.pos0 = q.length - q.n + first / a.g.G;
  u.prefix = q.prefix;
  const int last = q.length - q.n + (first + u.n_rows - 1) / a.g.G;
  u.hi = min(q.length, max(max(last + 1, 0), u.prefix));
  return u;
}

__device__ inline int chunks_of(int tokens) { return (tokens + kChunkTokens - 1) / kChunkTokens; }

__device__ inline Cost cost_of(const Unit& u, const RequestTiles& q) {
  const int chunks = chunks_of(u.hi);
  return Cost{chunks, q.prefix > 0 && q.n <= kTaggedRows ? min(q.prefix / kChunkTokens, chunks) : chunks};
}

__device__ inline int parts_of(const PlanArgs& a, int cost, int most) { return a.whole ? 1 : pieces_of(cost, most); }

__device__ inline Unit part_of(Unit u, const Cost& c, int k, int parts, int row_at) {
  if (parts == 1) return u.lo = 0, u.part = -1, u;
  u.lo = piece_at(c, k, parts) * kChunkTokens;
  if (k + 1 < parts) u.hi = piece_at(c, k + 1, parts) * kChunkTokens;
  u.part = row_at + k * u.n_rows;
  return u;
}

// The first blocks of a unit, so that attention needs no page table on its way to them.
__device__ inline void list_blocks(const PlanArgs& a, const Unit& u, int unit, int k) {
  const int token = u.lo + k * kBlock;
  a.unit_blocks[unit * kUnitBlocks + k] = token < u.hi ? block_of(a.g, a.table, u.request, token, u.hi) : -1;
}

// Fewer requests than NT and at most NT tiles: a thread to a request, then a thread to a tile.  Every work-group finds out the same and
// writes down the unit of its own number, so that the whole plan is one launch whose way is no longer than one page's.
template <int NT>
__global__ __launch_bounds__(NT) void k8_plan(PlanArgs a) {
  __shared__ int2v s_tmp[NT / 64];
  __shared__ int s_upto[NT], s_chunks[NT], s_chunk[2];
  __shared__ RequestTiles s_request[NT];
  __shared__ Unit s_unit;
  const int tid = threadIdx.x;
  int mine = 0, n_tiles, work;
  if (tid <= a.n_requests) {
    s_request[tid] = request_tiles(a, tid);
    mine = s_request[tid].n_tiles;
  }
  const int upto = group_scan<NT>(mine, s_tmp, n_tiles);
  s_upto[tid] = upto;
  if (tid == 0) s_unit = Unit{};
  __syncthreads();
  n_tiles = min(n_tiles, a.max_tiles);
  Unit u{};
  Cost cost{};
  if (tid < n_tiles) {
    const int r = min(count_le(s_upto, a.n_requests + 1, tid), a.n_requests);
    const RequestTiles q = s_request[r];
    u = tile_of(a, r, q, tid - (s_upto[r] - q.n_tiles));
    cost = cost_of(u, q);
  }
  const int own = cost.all();
  s_chunks[tid] = own;
  group_scan<NT>(own, s_tmp, work);
  // The least chunk that makes at most `capacity` units, and the least that makes half as many: 64 candidates for each from the one without
  // remainders on, a lane for each.  Else one that does in any case: with one remainder per tile while there are few tiles; from half as many
  // tiles on, twice the mean load.
  if (tid < 128) {
    const int most = max(a.capacity >> (tid >> 6), 1), room = max(max(most - n_tiles, most / 2), 1);
    const int least = max(1, (work + most - 1) / most), c = least + (tid & 63);
    int units = n_tiles > most ? INT_MAX : 0;
    if (n_tiles <= most && n_tiles > 1)
      for (int j = 0; j < n_tiles; ++j) units += max(1, (s_chunks[j] + c - 1) / c);
    const uint64_t fits = __ballot(units <= most);
    const int any = max(1, (work + room - 1) / room);
    if ((tid & 63) == 0) s_chunk[tid >> 6] = min(any, fits ? least + __builtin_ctzll(fits) : any);
  }
  __syncthreads();
  const bool alone = 2 * n_tiles <= a.capacity && s_chunk[1] * (kChunkTokens / 2) <= kAloneTokens;
  const int chunk = alone ? max(s_chunk[1], 2 * kLeastAlone / kChunkTokens) : max(s_chunk[0], 2 * kLeastTokens / kChunkTokens);
  const int parts = tid < n_tiles ? parts_of(a, own, chunk) : 0;
  const int rows = parts > 1 ? parts * u.n_rows : 0;
  int2v all;
  const int2v upto_here = group_scan<NT>(int2v{parts, rows}, s_tmp, all);
  const int at = upto_here[0] - parts, row_at = upto_here[1] - rows, n_units = all[0];
  // the second half of what runs at once stands in reverse
  const int here = blockIdx.x, half = a.capacity / 2;
  const int unit = n_units <= a.capacity && here >= half && here < n_units ? half + n_units - 1 - here : here;
  const bool fits = at + parts <= a.max_units && row_at + rows <= a.max_part_rows;  // (the host's bounds hold: see pasta_kv8.hip)
  if (unit >= at && unit < at + parts && fits) s_unit = part_of(u, cost, unit - at, parts, row_at);
  if (blockIdx.x == 0 && tid < a.max_tiles) a.tiles[tid] = Tile{u.s0, u.n_rows, row_at, tid < n_tiles && fits ? parts : 0};
  __syncthreads();
  if (tid == 0) a.units[blockIdx.x] = s_unit;
  if (tid < kUnitBlocks && s_unit.n_rows) list_blocks(a, s_unit, blockIdx.x, tid);
}

// Any number of them, one work-group, NT at a time; the units' blocks follow in a launch of their own.
template <int NT>
__global__ __launch_bounds__(NT) void k8_plan_long(PlanArgs a) {
  __shared__ int2v s_tmp[NT / 64];
  const int tid = threadIdx.x;
  int n_tiles = 0;
  int64_t work = 0;
  for (int r0 = 0; r0 <= a.n_requests; r0 += NT) {
    const int r = r0 + tid;
    int mine = 0, all;
    if (r <= a.n_requests) mine = request_tiles(a, r).n_tiles;
    const int now = n_tiles + group_scan<NT>(mine, s_tmp, all);
    if (r <= a.n_requests) a.w_tiles[r] = now;
    n_tiles += all;
  }
  __syncthreads();
  n_tiles = min(n_tiles, a.max_tiles);
  auto tile = [&](int j) {
    const int r = min(count_le(a.w_tiles, a.n_requests + 1, j), a.n_requests);
    const RequestTiles q = request_tiles(a, r);
    return tile_of(a, r, q, j - (a.w_tiles[r] - q.n_tiles));
  };
  auto plain = [](const Unit& u) { return Cost{chunks_of(u.hi), chunks_of(u.hi)}; };
  for (int j0 = 0; j0 < n_tiles; j0 += NT) {
    int all;
    group_scan<NT>(j0 + tid < n_tiles ? chunks_of(tile(j0 + tid).hi) : 0, s_tmp, all);
    work += all;
  }
  const int room = max(max(a.capacity - n_tiles, a.capacity / 2), 1);
  const int chunk = max((int)min((2 * work + room - 1) / room, (int64_t)(2 * kMostTokens / kChunkTokens)), 2 * kLeastTokens / kChunkTokens);
  int n_units = 0, n_part_rows = 0;
  for (int j0 = 0; j0 < n_tiles; j0 += NT) {
    const int j = j0 + tid;
    Unit u{};
    int parts = 0, all, all_rows;
    if (j < n_tiles) {
      u = tile(j);
      parts = parts_of(a, plain(u).all(), chunk);
    }
    const int at = n_units + group_scan<NT>(parts, s_tmp, all) - parts;
    const int rows = parts > 1 ? parts * u.n_rows : 0;
    const int row_at = n_part_rows + group_scan<NT>(rows, s_tmp, all_rows) - rows;
    if (j < n_tiles) {
      const bool fits = at + parts <= a.max_units && row_at + rows <= a.max_part_rows;
      for (int k = 0; k < parts && fits; ++k) a.units[at + k] = part_of(u, plain(u), k, parts, row_at);
      a.tiles[j] = Tile{u.s0, u.n_rows, row_at, fits ? parts : 0};
    }
    n_units += all;
    n_part_rows += all_rows;
  }
  // what the launches of k8_attend and k8_merge go over beyond that is empty
  for (int j = min(n_units, a.max_units) + tid; j < a.max_units; j += NT) a.units[j] = Unit{};
  for (int j = n_tiles + tid; j < a.max_tiles; j += NT) a.tiles[j] = Tile{};
}

__global__ __launch_bounds__(256) void k8_unit_blocks(PlanArgs a) {
  const int unit = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= a.max_units) return;
  const Unit u = a.units[unit];
  if (u.n_rows) list_blocks(a, u, unit, threadIdx.x & 63);
}

}  // namespace k8
