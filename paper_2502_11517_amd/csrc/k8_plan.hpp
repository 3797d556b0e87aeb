// Split of the attention's work: which stacked rows of which request over which tokens, a unit per (rows, tokens), times Hkv.
//
// Rows come in tiles of 32 (a work-group whose waves split the tokens) or, in requests with more stacked rows than that, of 128 (four
// waves of 32 rows over the same tokens).  Tokens are split so that about as many work-groups run as the chip holds; a tile whose
// tokens are split leaves partial rows, which k8_merge joins.
#pragma once
#include "k8_dev.hpp"

namespace k8 {

struct PlanArgs {
  Geometry g;
  int n_requests, n_rows;
  int wide;       // requests with more than 32 stacked rows take tiles of 128
  int capacity;   // units that the chip takes at once
  int max_units, max_tiles, max_part_rows;
  const int *length, *row_offsets, *prefix_len, *slot;
  Unit* units;
  Tile* tiles;
  int* w_tiles;   // workspace, n_requests + 1: tiles of the requests up to and including this one
};

struct RequestTiles {
  int row0, n, length, tile_rows, n_tiles;
};

// Request r, or (r == n_requests) the rows behind the last request, which see nothing.
__device__ inline RequestTiles request_tiles(const PlanArgs& a, int r) {
  RequestTiles q;
  const int end = min(max(a.row_offsets[a.n_requests], 0), a.n_rows);
  if (r == a.n_requests) {
    q.row0 = end, q.n = a.n_rows - end, q.length = 0;
  } else {
    q.row0 = min(max(a.row_offsets[r], 0), end);
    q.n = min(max(a.row_offsets[r + 1], q.row0), end) - q.row0;
    q.length = min(max(a.length[r], 0), a.g.table_width << a.g.page_shift);
    if (a.slot && q.n > 0 && a.slot[q.row0] < 0) q.length = 0;
  }
  const int64_t stacked = (int64_t)q.n * a.g.G;
  q.tile_rows = a.wide && stacked > kRows ? kWideRows : kRows;
  q.n_tiles = (int)((stacked + q.tile_rows - 1) / q.tile_rows);
  return q;
}

__device__ inline Unit tile_of(const PlanArgs& a, int j) {
  const int r = count_le(a.w_tiles, a.n_requests + 1, j);
  Unit u{};
  if (r > a.n_requests) return u;
  const RequestTiles q = request_tiles(a, r);
  const int t = j - (a.w_tiles[r] - q.n_tiles);
  const int first = t * q.tile_rows, stacked = q.n * a.g.G;
  u.request = max(min(r, a.n_requests - 1), 0);
  u.s0 = q.row0 * a.g.G + first;
  u.n_rows = min(stacked - first, q.tile_rows);
  u.pos0 = q.length - q.n + first / a.g.G;
  if (q.length == 0) return u;
  u.prefix = a.prefix_len ? min(max(a.prefix_len[r], 0), q.length) : 0;
  const int last = q.length - q.n + (first + u.n_rows - 1) / a.g.G;
  u.hi = min(q.length, max(max(last + 1, 0), u.prefix));
  return u;
}

template <int NT>
__global__ __launch_bounds__(NT) void k8_plan(PlanArgs a) {
  __shared__ int s_tmp[NT / 64];
  const int tid = threadIdx.x;
  int n_tiles = 0;
  for (int r0 = 0; r0 <= a.n_requests; r0 += NT) {
    const int r = r0 + tid;
    int mine = 0, all;
    if (r <= a.n_requests) mine = request_tiles(a, r).n_tiles;
    const int upto = n_tiles + group_scan<NT>(mine, s_tmp, all);
    if (r <= a.n_requests) a.w_tiles[r] = upto;
    n_tiles += all;
  }
  __syncthreads();
  n_tiles = min(n_tiles, a.max_tiles);
  int work = 0;  // (in chunks of the least length: below 2^31 / 128 for a table's tokens, times the tiles)
  for (int j0 = 0; j0 < n_tiles; j0 += NT) {
    int all;
    const int j = j0 + tid;
    group_scan<NT>(j < n_tiles ? min((tile_of(a, j).hi + kChunkTokens - 1) / kChunkTokens, 1 << 20) : 0, s_tmp, all);
    work += all;
  }
  // Chunks of this many times 128 tokens: with one remainder per tile at most `capacity` units, while there are few tiles; from half as
  // many tiles on, chunks of twice the mean load.
  const int room = max(max(a.capacity - n_tiles, a.capacity / 2), 1);
  const int chunk = max(1, (work + room - 1) / room) * kChunkTokens;
  int n_units = 0, n_part_rows = 0;
  for (int j0 = 0; j0 < n_tiles; j0 += NT) {
    const int j = j0 + tid;
    Unit u{};
    int parts = 0, all, all_rows;
    if (j < n_tiles) {
      u = tile_of(a, j);
      parts = max(1, (u.hi + chunk - 1) / chunk);
    }
    const int at = n_units + group_scan<NT>(parts, s_tmp, all) - parts;
    const int rows = parts > 1 ? parts * u.n_rows : 0;
    const int row_at = n_part_rows + group_scan<NT>(rows, s_tmp, all_rows) - rows;
    if (j < n_tiles) {
      const bool fits = at + parts <= a.max_units && row_at + rows <= a.max_part_rows;  // (the host's bounds hold: see pasta_kv8_plan)
      const int hi = u.hi;
      for (int k = 0; k < parts && fits; ++k) {
        u.lo = k * chunk, u.hi = min(hi, (k + 1) * chunk), u.part = parts > 1 ? row_at + k * u.n_rows : -1;
        a.units[at + k] = u;
      }
      a.tiles[j] = Tile{u.s0, u.n_rows, row_at, fits ? parts : 0};
    }
    n_units += all;
    n_part_rows += all_rows;
  }
  // what the launches of k8_attend and k8_merge go over beyond that is empty
  for (int j = min(n_units, a.max_units) + tid; j < a.max_units; j += NT) a.units[j] = Unit{};
  for (int j = n_tiles + tid; j < a.max_tiles; j += NT) a.tiles[j] = Tile{};
}

}  // namespace k8
