// Host side of the attention, whatever the cache's codes: checks of arguments, how large a plan can get, its place in the workspace, its launches and that of
// the merge.
// `Config` is pasta_kv8_config or one with the same members.
#pragma once
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>

#include "../../include/pasta_kv8.h"
#include "k8_attend.hpp"
#include "k8_plan.hpp"

namespace k8 {

inline bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

inline int32_t launched() { return hipGetLastError() == hipSuccess ? PASTA_OK : PASTA_E_DEVICE; }

// Sizes that the kernels can do.
template <class Config>
bool sizes_hold(const Config& c) {
  if (c.n_kv_heads < 1 || c.n_kv_heads > 256 || c.n_q_heads < 1 || c.n_q_heads % c.n_kv_heads) return false;
  const int G = c.n_q_heads / c.n_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8) return false;
  if (c.head_dim != 64 && c.head_dim != 128) return false;
  if (c.n_layers < 1 || c.max_requests < 1 || c.max_rows < 1 || c.n_phys_pages < 1 || c.pages_per_request < 1) return false;
  if (c.page_tokens < 16 || c.page_tokens > 4096 || (c.page_tokens & (c.page_tokens - 1))) return false;
  if (!std::isfinite(c.softmax_scale)) return false;
  const int64_t most = INT32_MAX;
  if ((int64_t)c.n_phys_pages * c.page_tokens > most || (int64_t)c.pages_per_request * c.page_tokens > kMostTokens) return false;
  if ((int64_t)c.n_phys_pages * c.n_kv_heads * (c.page_tokens / 16) > most) return false;  // index of a scale within a layer
  if ((int64_t)c.max_requests * c.pages_per_request > most || c.max_requests > (1 << 20)) return false;
  if ((int64_t)c.max_rows * c.n_q_heads > most / 8) return false;
  return true;
}

// Work-groups of the attention: two per CU.  (256 / 384 / 768: eight streams over 8k tokens of the 4-bit cache, 8 layers, 118 / 110 / 124 us where these take 105, 16 ragged
// requests, 4 layers, 131 / 120 / 124 where they took 107, ahead of the weights in k8_plan.hpp.)
constexpr int kUnitsAtOnce = 512;

struct Bounds {
  int64_t capacity, units, tiles, part_rows, merge_rows;
};

// The last plan.
struct Planned {
  bool made = false;
  int n_rows = 0, wide = 0, whole = 0;
  Bounds most{};
};

// What a plan over n_rows rows of n_requests requests can come to (k8_plan.hpp: with R tiles, at most max(capacity, capacity / 2 + R, 1 + R)
// units, which a launch goes over one by one: 256 work-groups that find nothing cost 1.5 us; a tile is split only into pieces of more than half a chunk
// on the mean, so that at most twice max(capacity, 1) of them are partial).
template <class Config>
Bounds bounds(const Config& c, int64_t n_rows, int64_t n_requests, bool wide, bool whole, int least_alone) {
  const int64_t G = c.n_q_heads / c.n_kv_heads, stacked = n_rows * G;
  Bounds b;
  b.capacity = kUnitsAtOnce / c.n_kv_heads;
  b.tiles = (stacked + (n_requests + 1) * (kRows - 1)) / kRows;  // of requests, and of rows that none has, each rounded up
  // (with tiles of 64 a request has as many as that again rounds up to, or, being small, at most two more)
  if (wide) b.tiles = std::min(b.tiles, (stacked + (n_requests + 1) * (kWideRows - 1)) / kWideRows + 2 * (n_requests + 1));
  if (b.tiles > stacked) b.tiles = stacked;
  const int64_t chunks = ((int64_t)c.pages_per_request * c.page_tokens + kChunkTokens - 1) / kChunkTokens;
  b.units = std::min(std::max(b.capacity, std::max(b.capacity / 2, (int64_t)1) + b.tiles), b.tiles * (least_alone < kLeastAlone ? chunks : (3 * chunks + 3) / 4));
  if (whole) b.units = b.tiles;
  int64_t rows = wide ? kWideRows : kRows;
  b.merge_rows = rows < stacked ? rows : stacked;
  b.part_rows = 2 * b.capacity * b.merge_rows;
  return b;
}

// What a plan keeps in the workspace.
struct PlanSpace {
  int least_alone = kLeastAlone;  // (of the cache: the least length of pieces where a CU has one)
  int few_rows = 0;               // (of the cache: rows of a tile that costs less, k8_plan.hpp)
  int* tiles_upto = nullptr;
  Unit* units = nullptr;
  int* unit_blocks = nullptr;
  Tile* tiles = nullptr;
  float2v* part_ml = nullptr;
  float* part_acc = nullptr;

  template <class Config, class Take>
  void lay_out(const Config& c, Take take) {
    Bounds b = bounds(c, c.max_rows, c.max_requests, false, false, least_alone);
    if ((int64_t)c.max_rows * (c.n_q_heads / c.n_kv_heads) > kManyRows) b.part_rows = bounds(c, c.max_rows, c.max_requests, true, false, least_alone).part_rows;
    take(tiles_upto, c.max_requests + 1);
    take(units, b.units);
    take(unit_blocks, b.units * kUnitBlocks);
    take(tiles, b.tiles);
    take(part_ml, b.part_rows * c.n_kv_heads);
    take(part_acc, b.part_rows * c.n_kv_heads * c.head_dim);
  }
};

template <class Config>
int32_t check_plan(const Config& c, const pasta_kv8_plan_args* a) {
  if (!a || a->struct_size != sizeof(*a) || a->flags) return PASTA_E_INVAL;
  if (a->n_requests < 0 || a->n_rows < 0 || a->max_request_rows < 0) return PASTA_E_INVAL;
  if (a->n_requests > c.max_requests || a->n_rows > c.max_rows) return PASTA_E_CAPACITY;
  if (!a->row_offsets || !c.workspace || !c.page_table || (a->n_requests && !a->length)) return PASTA_E_INVAL;
  if (!aligned(a->length, 4) || !aligned(a->row_offsets, 4) || !aligned(a->prefix_len, 4) || !aligned(a->slot, 4)) return PASTA_E_INVAL;
  return PASTA_OK;
}

// The plan of checked arguments.  False: the launch failed, and there is no plan.
template <class Config>
bool launch_plan(const Config& c, const Geometry& g, const PlanSpace& space, const pasta_kv8_plan_args& a, Planned& plan) {
  plan.made = true;
  plan.n_rows = a.n_rows;
  if (a.n_rows == 0) return true;
  const int64_t most = a.max_request_rows < a.n_rows ? a.max_request_rows : a.n_rows;
  plan.wide = most * g.G > kManyRows;
  // where every tile is that short, splitting it costs more (a launch, partial rows) than it saves
  plan.whole = (int64_t)c.pages_per_request * c.page_tokens <= (plan.wide ? kWholeWide : kWholeTokens);
  plan.most = bounds(c, a.n_rows, a.n_requests, plan.wide, plan.whole, space.least_alone);
  PlanArgs k{};
  k.g = g, k.n_requests = a.n_requests, k.n_rows = a.n_rows, k.wide = plan.wide, k.whole = plan.whole, k.capacity = (int)plan.most.capacity, k.least_alone = space.least_alone, k.few_rows = space.few_rows;
  k.max_units = (int)plan.most.units, k.max_tiles = (int)plan.most.tiles, k.max_part_rows = (int)plan.most.part_rows;
  k.length = a.n_requests ? a.length : a.row_offsets;  // (read, not used, without a request)
  k.row_offsets = a.row_offsets, k.prefix_len = a.prefix_len, k.slot = a.slot;
  k.table = c.page_table;
  k.units = space.units, k.unit_blocks = space.unit_blocks, k.tiles = space.tiles, k.w_tiles = space.tiles_upto;
  hipStream_t s = (hipStream_t)c.hip_stream;
  if (plan.most.tiles <= 256 && a.n_requests < 256) {
    k8_plan<256><<<(unsigned)plan.most.units, 256, 0, s>>>(k);
  } else {
    k8_plan_long<1024><<<1, 1024, 0, s>>>(k);
    k8_unit_blocks<<<(unsigned)((plan.most.units + 3) / 4), 256, 0, s>>>(k);
  }
  return plan.made = hipGetLastError() == hipSuccess;
}

template <class Config>
int32_t check_attend(const Config& c, const pasta_kv8_attend_args* a, const Planned& plan) {
  if (!a || a->struct_size != sizeof(*a) || a->flags) return PASTA_E_INVAL;
  if (a->layer < 0 || a->layer >= c.n_layers || a->n_rows < 0) return PASTA_E_INVAL;
  if (!(a->logit_cap >= 0.f) || !std::isfinite(a->logit_cap)) return PASTA_E_INVAL;
  if (!plan.made || a->n_rows != plan.n_rows) return PASTA_E_STATE;
  if (!c.k_codes || !c.v_codes || !c.k_scale || !c.v_scale || !c.page_table) return PASTA_E_INVAL;
  if ((a->row_see && !c.slot_tag) || (a->row_position && (!c.slot_position || !a->slopes))) return PASTA_E_INVAL;
  if (a->n_rows == 0) return PASTA_OK;
  if (!a->q || !a->out || !aligned(a->q, 16) || !aligned(a->out, 16)) return PASTA_E_INVAL;
  if (!aligned(a->lse, 4) || !aligned(a->slopes, 4) || !aligned(a->row_see, 8) || !aligned(a->row_position, 4)) return PASTA_E_INVAL;
  return PASTA_OK;
}

// All but the codes and scales.
template <class Config>
void fill_attend(const Config& c, const Geometry& g, const PlanSpace& space, const pasta_kv8_attend_args& a, AttendArgs& k) {
  k.g = g, k.Hq = c.n_q_heads, k.dtype = c.dtype, k.n_rows = a.n_rows;
  while ((1 << k.g_shift) < k.g.G) k.g_shift++;
  k.scale_log2 = std::fabs(c.softmax_scale) * kLog2e;
  k.negate = c.softmax_scale < 0.f;
  // (below a cap of 2^-63 everything is the cap or less: how steeply it gets there no longer matters)
  if (a.logit_cap > 0.f) k.cap_log2 = std::fmax(std::fmin(a.logit_cap * kLog2e, FLT_MAX), FLT_MIN), k.cap_in = std::fmin(2.f / a.logit_cap, 0x1p64f);
  k.table = c.page_table, k.slot_tag = c.slot_tag, k.slot_position = c.slot_position;
  k.row_position = a.row_position, k.row_see = a.row_see, k.slopes = a.slopes;
  k.tagged = a.row_see, k.placed = a.row_position, k.lowered = a.slopes;
  // stand-ins: a slot has at least 32 bytes of K's codes, a row of q at least 128, and q has at least 128 a head
  if (!k.tagged) k.row_see = (const uint64_t*)a.q, k.slot_tag = (const uint8_t*)c.k_codes;
  if (!k.placed) k.row_position = (const int*)a.q, k.slot_position = (const int*)c.k_codes;
  if (!k.lowered) k.slopes = (const float*)a.q;
  k.units = space.units, k.unit_blocks = space.unit_blocks, k.tiles = space.tiles;
  while ((1 << k.block_shift) < k.g.blocks_per_page) k.block_shift++;
  k.q = a.q, k.out = a.out, k.lse = a.lse, k.part_ml = space.part_ml, k.part_acc = space.part_acc;
}

// f(whether tiles of 64 rows are wanted, what the call does to scores), as constants.
template <class F>
void by_kind(const AttendArgs& k, const Planned& plan, F f) {
  const int kind = k.tagged || k.placed ? kMarked : k.lowered || k.cap_log2 > 0.f ? kShaped : kPlain;
  auto with = [&](auto many) {
    if (kind == kMarked) f(many, std::integral_constant<int, kMarked>{});
    else if (kind == kShaped) f(many, std::integral_constant<int, kShaped>{});
    else f(many, std::integral_constant<int, kPlain>{});
  };
  plan.wide ? with(std::true_type{}) : with(std::false_type{});
}

inline void launch_merge(const AttendArgs& k, const Planned& plan, hipStream_t s) {
  if (plan.whole) return;
  const int64_t tiles = plan.most.tiles * k.g.Hkv;
  int64_t split = (2048 + tiles - 1) / tiles;  // work-groups to a tile: rows, one by one where there are so few tiles
  if (split > plan.most.merge_rows) split = plan.most.merge_rows;
  const dim3 grid((unsigned)tiles, (unsigned)split);
  if (k.g.D == 128)
    k8_merge<128><<<grid, 256, 0, s>>>(k);
  else
    k8_merge<64><<<grid, 256, 0, s>>>(k);
}

}  // namespace k8
