// Host side of the 8-bit paged KV cache (include/pasta_kv8.h): checks of arguments, layout of the workspace, launches.
// No call here depends on what a device array holds: grids go by the sizes that the caller gives, work-groups that find nothing to do end.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <new>

#include "../../include/pasta_kv8.h"
#include "k8_append.hpp"
#include "k8_attend.hpp"
#include "k8_plan.hpp"
#include "k8_rules.hpp"
#include "k8_slots.hpp"

namespace {

constexpr uint64_t kMagic = 0x3876'6b61'7473'6170ull;
constexpr int kUnitsAtOnce = 512;  // work-groups of the attention: two per CU

struct Bounds {
  int64_t capacity, units, tiles, part_rows, merge_rows;
};

}  // namespace

struct pasta_kv8 {
  uint64_t magic = kMagic;
  pasta_kv8_config cfg{};
  k8::Geometry g{};
  // workspace
  int *kept = nullptr, *old_pages = nullptr, *take = nullptr, *top = nullptr, *tiles_upto = nullptr;
  k8::Unit* units = nullptr;
  int* unit_blocks = nullptr;
  k8::Tile* tiles = nullptr;
  k8::float2v* part_ml = nullptr;
  float* part_acc = nullptr;
  // the last plan
  bool planned = false;
  int plan_rows = 0, plan_wide = 0, plan_whole = 0;
  Bounds plan{};
};

namespace {

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

int32_t check(const pasta_kv8_config* c) {
  if (!c || c->struct_size != sizeof(pasta_kv8_config)) return PASTA_E_INVAL;
  if (c->codes != PASTA_KV8_E4M3 && c->codes != PASTA_KV8_INT8) return PASTA_E_INVAL;
  if (c->dtype != PASTA_BF16 && c->dtype != PASTA_F16) return PASTA_E_INVAL;
  if (c->n_kv_heads < 1 || c->n_kv_heads > 256 || c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads) return PASTA_E_INVAL;
  const int G = c->n_q_heads / c->n_kv_heads;
  if (G != 1 && G != 2 && G != 4 && G != 8) return PASTA_E_INVAL;
  if (c->head_dim != 64 && c->head_dim != 128) return PASTA_E_INVAL;
  if (c->n_layers < 1 || c->max_requests < 1 || c->max_rows < 1 || c->n_phys_pages < 1 || c->pages_per_request < 1) return PASTA_E_INVAL;
  if (c->page_tokens < 16 || c->page_tokens > 4096 || (c->page_tokens & (c->page_tokens - 1))) return PASTA_E_INVAL;
  if (!std::isfinite(c->softmax_scale)) return PASTA_E_INVAL;
  const int64_t most = INT32_MAX;
  if ((int64_t)c->n_phys_pages * c->page_tokens > most || (int64_t)c->pages_per_request * c->page_tokens > k8::kMostTokens) return PASTA_E_INVAL;
  if ((int64_t)c->n_phys_pages * c->n_kv_heads * (c->page_tokens / 16) > most) return PASTA_E_INVAL;  // index of a scale within a layer
  if ((int64_t)c->max_requests * c->pages_per_request > most || c->max_requests > (1 << 20)) return PASTA_E_INVAL;
  if ((int64_t)c->max_rows * c->n_q_heads > most / 8) return PASTA_E_INVAL;
  return PASTA_OK;
}

// What a plan over n_rows rows of n_requests requests can come to (k8_plan.hpp: with R tiles, at most max(capacity, capacity / 2 + R, 1 + R)
// units, which a launch goes over one by one: 256 work-groups that find nothing cost 1.5 us; a tile is split only into pieces of more than half a chunk
// on the mean, so that at most twice max(capacity, 1) of them are partial).
Bounds bounds(const pasta_kv8_config& c, int64_t n_rows, int64_t n_requests, bool wide, bool whole) {
  const int64_t G = c.n_q_heads / c.n_kv_heads, stacked = n_rows * G;
  Bounds b;
  b.capacity = kUnitsAtOnce / c.n_kv_heads;
  b.tiles = (stacked + (n_requests + 1) * (k8::kRows - 1)) / k8::kRows;  // of requests, and of rows that none has, each rounded up
  // (with tiles of 64 a request has as many as that again rounds up to, or, being small, at most two more)
  if (wide) b.tiles = std::min(b.tiles, (stacked + (n_requests + 1) * (k8::kWideRows - 1)) / k8::kWideRows + 2 * (n_requests + 1));
  if (b.tiles > stacked) b.tiles = stacked;
  const int64_t chunks = ((int64_t)c.pages_per_request * c.page_tokens + k8::kChunkTokens - 1) / k8::kChunkTokens;
  b.units = std::min(std::max(b.capacity, std::max(b.capacity / 2, (int64_t)1) + b.tiles), b.tiles * ((3 * chunks + 3) / 4));
  if (whole) b.units = b.tiles;
  int64_t rows = wide ? k8::kWideRows : k8::kRows;
  b.merge_rows = rows < stacked ? rows : stacked;
  b.part_rows = 2 * b.capacity * b.merge_rows;
  return b;
}

uint64_t lay_out(const pasta_kv8_config& c, pasta_kv8* h) {
  Bounds b = bounds(c, c.max_rows, c.max_requests, false, false);
  if ((int64_t)c.max_rows * (c.n_q_heads / c.n_kv_heads) > k8::kManyRows) b.part_rows = bounds(c, c.max_rows, c.max_requests, true, false).part_rows;
  uint64_t at = 0;
  auto take = [&](auto*& p, uint64_t n) {
    p = reinterpret_cast<std::remove_reference_t<decltype(p)>>((uint8_t*)c.workspace + at);
    at += (n * sizeof(*p) + 255) / 256 * 256;
  };
  take(h->kept, c.max_requests);
  take(h->old_pages, c.max_requests);
  take(h->take, c.max_requests);
  take(h->top, 1);
  take(h->tiles_upto, c.max_requests + 1);
  take(h->units, b.units);
  take(h->unit_blocks, b.units * k8::kUnitBlocks);
  take(h->tiles, b.tiles);
  take(h->part_ml, b.part_rows * c.n_kv_heads);
  take(h->part_acc, b.part_rows * c.n_kv_heads * c.head_dim);
  return at;
}

bool overlap(const int32_t* a, int64_t n, const int32_t* b, int64_t m) { return (uintptr_t)a < (uintptr_t)(b + m) && (uintptr_t)b < (uintptr_t)(a + n); }

int32_t launched() { return hipGetLastError() == hipSuccess ? PASTA_OK : PASTA_E_DEVICE; }

}  // namespace

extern "C" int32_t pasta_kv8_create(pasta_kv8_config* cfg, pasta_kv8** out) {
  int32_t rc = check(cfg);
  if (rc != PASTA_OK) return rc;
  if (!out) {
    pasta_kv8 none;
    pasta_kv8_config c = *cfg;
    c.workspace = nullptr;
    cfg->workspace_bytes = lay_out(c, &none);
    return PASTA_OK;
  }
  *out = nullptr;
  if (!aligned(cfg->k_codes, 16) || !aligned(cfg->v_codes, 16) || !aligned(cfg->k_scale, 4) || !aligned(cfg->v_scale, 4)) return PASTA_E_INVAL;
  if (!aligned(cfg->page_table, 4) || !aligned(cfg->free_pages, 4) || !aligned(cfg->slot_tag, 16) || !aligned(cfg->slot_position, 16)) return PASTA_E_INVAL;
  if (!aligned(cfg->workspace, 256)) return PASTA_E_INVAL;
  pasta_kv8* h = new (std::nothrow) pasta_kv8();
  if (!h) return PASTA_E_NOMEM;
  h->cfg = *cfg;
  const uint64_t need = lay_out(*cfg, h);
  if (cfg->workspace && cfg->workspace_bytes < need) {
    delete h;
    return PASTA_E_CAPACITY;
  }
  k8::Geometry& g = h->g;
  g.Hkv = cfg->n_kv_heads, g.G = cfg->n_q_heads / cfg->n_kv_heads, g.D = cfg->head_dim;
  g.page_tokens = cfg->page_tokens, g.blocks_per_page = cfg->page_tokens / 16;
  while ((1 << g.page_shift) < cfg->page_tokens) g.page_shift++;
  g.n_pages = cfg->n_phys_pages, g.table_width = cfg->pages_per_request;
  *out = h;
  return PASTA_OK;
}

extern "C" int32_t pasta_kv8_destroy(pasta_kv8* h) {
  if (!h) return PASTA_OK;
  if (h->magic != kMagic) return PASTA_E_STATE;
  h->magic = 0;
  delete h;
  return PASTA_OK;
}

extern "C" int32_t pasta_kv8_slots(pasta_kv8* h, const pasta_kv8_slots_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  if (!a || a->struct_size != sizeof(*a) || a->flags) return PASTA_E_INVAL;
  const pasta_kv8_config& c = h->cfg;
  if (a->n_requests < 0 || a->n_rows < 0) return PASTA_E_INVAL;
  if (a->n_requests > c.max_requests || a->n_rows > c.max_rows) return PASTA_E_CAPACITY;
  if (!a->row_offsets || !a->free_count || !a->free_out || !c.page_table || !c.free_pages || !c.workspace) return PASTA_E_INVAL;
  if (a->n_requests && (!a->length || !a->length_out)) return PASTA_E_INVAL;
  if (a->n_rows && !a->slot) return PASTA_E_INVAL;
  if ((a->row_tag && !c.slot_tag) || (a->row_position && !c.slot_position)) return PASTA_E_INVAL;
  const void* words[] = {a->length, a->keep, a->row_offsets, a->row_position, a->free_count, a->slot, a->length_out, a->free_out};
  for (const void* p : words)
    if (!aligned(p, 4)) return PASTA_E_INVAL;
  k8::SlotsArgs k{};
  k.g = h->g, k.n_requests = a->n_requests, k.n_rows = a->n_rows;
  k.length = a->length, k.keep = a->keep, k.row_offsets = a->row_offsets, k.row_tag = a->row_tag, k.row_position = a->row_position;
  k.free_count = a->free_count, k.slot = a->slot, k.length_out = a->length_out, k.free_out = a->free_out;
  k.table = c.page_table, k.stack = c.free_pages, k.slot_tag = c.slot_tag, k.slot_position = c.slot_position;
  k.w_kept = h->kept, k.w_old = h->old_pages, k.w_take = h->take, k.w_top = h->top;
  hipStream_t s = (hipStream_t)c.hip_stream;
  const bool in_place = overlap(a->length, a->n_requests, a->length_out, a->n_requests) || overlap(a->free_count, 1, a->free_out, 1) ||
                        (a->keep && overlap(a->keep, a->n_requests, a->length_out, a->n_requests));
  const int rows = (a->n_rows + 255) / 256;
  if (a->n_requests <= 64 && a->n_rows <= 256) {
    k8::k8_slots<64><<<in_place || !rows ? 1 : (a->n_rows + 63) / 64, 64, 0, s>>>(k);
  } else if (a->n_requests <= 256 && (!in_place || a->n_rows <= k8::kSlotsHere)) {
    k8::k8_slots<256><<<in_place || !rows ? 1 : rows, 256, 0, s>>>(k);
  } else if (a->n_requests <= 512 && (!in_place || a->n_rows <= k8::kSlotsHere)) {
    k8::k8_slots<512><<<in_place || !rows ? 1 : (a->n_rows + 511) / 512, 512, 0, s>>>(k);
  } else if (a->n_requests <= 1024 && (!in_place || a->n_rows <= k8::kSlotsHere)) {
    k8::k8_slots<1024><<<in_place || !rows ? 1 : (a->n_rows + 1023) / 1024, 1024, 0, s>>>(k);
  } else {
    k8::k8_slots_long<1024><<<1, 1024, 0, s>>>(k);
    if (a->n_rows > k8::kSlotsHere) k8::k8_place<<<rows, 256, 0, s>>>(k);
  }
  return launched();
}

namespace {

template <int CODES, int D>
void launch_append(const k8::AppendArgs& k, int dtype, dim3 grid, hipStream_t s) {
  if (dtype == PASTA_F32)
    k8::k8_append<CODES, D, k8::kF32><<<grid, 256, 0, s>>>(k);
  else if (dtype == PASTA_BF16)
    k8::k8_append<CODES, D, k8::kBf16><<<grid, 256, 0, s>>>(k);
  else
    k8::k8_append<CODES, D, k8::kF16><<<grid, 256, 0, s>>>(k);
}

}  // namespace

extern "C" int32_t pasta_kv8_append(pasta_kv8* h, const pasta_kv8_append_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  if (!a || a->struct_size != sizeof(*a) || a->flags) return PASTA_E_INVAL;
  const pasta_kv8_config& c = h->cfg;
  if (a->layer < 0 || a->layer >= c.n_layers || a->n_rows < 0) return PASTA_E_INVAL;
  if (a->dtype != PASTA_F32 && a->dtype != PASTA_BF16 && a->dtype != PASTA_F16) return PASTA_E_INVAL;
  if (a->n_rows > c.max_rows) return PASTA_E_CAPACITY;
  if (!c.k_codes || !c.v_codes || !c.k_scale || !c.v_scale) return PASTA_E_INVAL;
  if (a->n_rows == 0) return PASTA_OK;
  if (!a->slot || !a->k_new || !a->v_new) return PASTA_E_INVAL;
  if (!aligned(a->slot, 4) || !aligned(a->k_new, 16) || !aligned(a->v_new, 16)) return PASTA_E_INVAL;
  const int64_t blocks = (int64_t)c.n_phys_pages * c.n_kv_heads * h->g.blocks_per_page, at = blocks * a->layer;
  k8::AppendArgs k{};
  k.g = h->g, k.n_rows = a->n_rows, k.slot = a->slot, k.k_new = a->k_new, k.v_new = a->v_new;
  k.k = (uint8_t*)c.k_codes + at * 16 * c.head_dim, k.v = (uint8_t*)c.v_codes + at * 16 * c.head_dim;
  k.ks = c.k_scale + at, k.vs = c.v_scale + at;
  k.group = k8::append_group(a->n_rows, c.n_kv_heads);
  const dim3 grid((a->n_rows + k.group - 1) / k.group, (2 * c.n_kv_heads + 3) / 4);
  hipStream_t s = (hipStream_t)c.hip_stream;
  if (c.codes == PASTA_KV8_E4M3)
    c.head_dim == 128 ? launch_append<k8::kE4m3, 128>(k, a->dtype, grid, s) : launch_append<k8::kE4m3, 64>(k, a->dtype, grid, s);
  else
    c.head_dim == 128 ? launch_append<k8::kInt8, 128>(k, a->dtype, grid, s) : launch_append<k8::kInt8, 64>(k, a->dtype, grid, s);
  return launched();
}

extern "C" int32_t pasta_kv8_plan(pasta_kv8* h, const pasta_kv8_plan_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  if (!a || a->struct_size != sizeof(*a) || a->flags) return PASTA_E_INVAL;
  const pasta_kv8_config& c = h->cfg;
  if (a->n_requests < 0 || a->n_rows < 0 || a->max_request_rows < 0) return PASTA_E_INVAL;
  if (a->n_requests > c.max_requests || a->n_rows > c.max_rows) return PASTA_E_CAPACITY;
  if (!a->row_offsets || !c.workspace || !c.page_table || (a->n_requests && !a->length)) return PASTA_E_INVAL;
  if (!aligned(a->length, 4) || !aligned(a->row_offsets, 4) || !aligned(a->prefix_len, 4) || !aligned(a->slot, 4)) return PASTA_E_INVAL;
  h->planned = true;
  h->plan_rows = a->n_rows;
  if (a->n_rows == 0) return PASTA_OK;
  const int64_t most = a->max_request_rows < a->n_rows ? a->max_request_rows : a->n_rows;
  h->plan_wide = most * h->g.G > k8::kManyRows;
  // where every tile is that short, splitting it costs more (a launch, partial rows) than it saves
  h->plan_whole = (int64_t)c.pages_per_request * c.page_tokens <= (h->plan_wide ? k8::kWholeWide : k8::kWholeTokens);
  h->plan = bounds(c, a->n_rows, a->n_requests, h->plan_wide, h->plan_whole);
  k8::PlanArgs k{};
  k.g = h->g, k.n_requests = a->n_requests, k.n_rows = a->n_rows, k.wide = h->plan_wide, k.whole = h->plan_whole, k.capacity = (int)h->plan.capacity;
  k.max_units = (int)h->plan.units, k.max_tiles = (int)h->plan.tiles, k.max_part_rows = (int)h->plan.part_rows;
  k.length = a->n_requests ? a->length : a->row_offsets;  // (read, not used, without a request)
  k.row_offsets = a->row_offsets, k.prefix_len = a->prefix_len, k.slot = a->slot;
  k.table = c.page_table;
  k.units = h->units, k.unit_blocks = h->unit_blocks, k.tiles = h->tiles, k.w_tiles = h->tiles_upto;
  hipStream_t s = (hipStream_t)c.hip_stream;
  if (h->plan.tiles <= 256 && a->n_requests < 256) {
    k8::k8_plan<256><<<(unsigned)h->plan.units, 256, 0, s>>>(k);
  } else {
    k8::k8_plan_long<1024><<<1, 1024, 0, s>>>(k);
    k8::k8_unit_blocks<<<(unsigned)((h->plan.units + 3) / 4), 256, 0, s>>>(k);
  }
  const int32_t rc = launched();
  if (rc != PASTA_OK) h->planned = false;
  return rc;
}

namespace {

template <int CODES, int D>
void launch_attend(const k8::AttendArgs& k, bool many, int64_t groups, hipStream_t s) {
  const int kind = k.tagged || k.placed ? k8::kMarked : k.lowered || k.cap_log2 > 0.f ? k8::kShaped : k8::kPlain;
  auto launch = [&](auto of, auto kind) {
    const dim3 grid((unsigned)groups, of.value && k8::kApart<CODES, D, kind.value> ? k8::kWideRows / k8::kRows : 1);
    k8::k8_attend<CODES, D, of.value, kind.value><<<grid, 256, 0, s>>>(k);
  };
  auto with = [&](auto of) {
    if (kind == k8::kMarked) launch(of, std::integral_constant<int, k8::kMarked>{});
    else if (kind == k8::kShaped) launch(of, std::integral_constant<int, k8::kShaped>{});
    else launch(of, std::integral_constant<int, k8::kPlain>{});
  };
  many ? with(std::true_type{}) : with(std::false_type{});
}

}  // namespace

extern "C" int32_t pasta_kv8_attend(pasta_kv8* h, const pasta_kv8_attend_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  if (!a || a->struct_size != sizeof(*a) || a->flags) return PASTA_E_INVAL;
  const pasta_kv8_config& c = h->cfg;
  if (a->layer < 0 || a->layer >= c.n_layers || a->n_rows < 0) return PASTA_E_INVAL;
  if (!(a->logit_cap >= 0.f) || !std::isfinite(a->logit_cap)) return PASTA_E_INVAL;
  if (!h->planned || a->n_rows != h->plan_rows) return PASTA_E_STATE;
  if (!c.k_codes || !c.v_codes || !c.k_scale || !c.v_scale || !c.page_table) return PASTA_E_INVAL;
  if ((a->row_see && !c.slot_tag) || (a->row_position && (!c.slot_position || !a->slopes))) return PASTA_E_INVAL;
  if (a->n_rows == 0) return PASTA_OK;
  if (!a->q || !a->out || !aligned(a->q, 16) || !aligned(a->out, 16)) return PASTA_E_INVAL;
  if (!aligned(a->lse, 4) || !aligned(a->slopes, 4) || !aligned(a->row_see, 8) || !aligned(a->row_position, 4)) return PASTA_E_INVAL;
  const float kLog2e = k8::kLog2e;
  k8::AttendArgs k{};
  k.g = h->g, k.Hq = c.n_q_heads, k.dtype = c.dtype, k.n_rows = a->n_rows;
  while ((1 << k.g_shift) < k.g.G) k.g_shift++;
  k.scale_log2 = std::fabs(c.softmax_scale) * kLog2e;
  k.negate = c.softmax_scale < 0.f;
  // (below a cap of 2^-63 everything is the cap or less: how steeply it gets there no longer matters)
  if (a->logit_cap > 0.f) k.cap_log2 = std::fmax(std::fmin(a->logit_cap * kLog2e, FLT_MAX), FLT_MIN), k.cap_in = std::fmin(2.f / a->logit_cap, 0x1p64f);
  const int64_t at = (int64_t)c.n_phys_pages * c.n_kv_heads * h->g.blocks_per_page * a->layer;
  k.k = (const uint8_t*)c.k_codes + at * 16 * c.head_dim, k.v = (const uint8_t*)c.v_codes + at * 16 * c.head_dim;
  k.ks = c.k_scale + at, k.vs = c.v_scale + at;
  k.table = c.page_table, k.slot_tag = c.slot_tag, k.slot_position = c.slot_position;
  k.row_position = a->row_position, k.row_see = a->row_see, k.slopes = a->slopes;
  k.tagged = a->row_see, k.placed = a->row_position, k.lowered = a->slopes;
  // stand-ins: a slot has at least 64 bytes of codes, a row of q at least 128, and q has at least 128 a head
  if (!k.tagged) k.row_see = (const uint64_t*)a->q, k.slot_tag = (const uint8_t*)c.k_codes;
  if (!k.placed) k.row_position = (const int*)a->q, k.slot_position = (const int*)c.k_codes;
  if (!k.lowered) k.slopes = (const float*)a->q;
  k.units = h->units, k.unit_blocks = h->unit_blocks, k.tiles = h->tiles;
  while ((1 << k.block_shift) < k.g.blocks_per_page) k.block_shift++;
  k.q = a->q, k.out = a->out, k.lse = a->lse, k.part_ml = h->part_ml, k.part_acc = h->part_acc;
  hipStream_t s = (hipStream_t)c.hip_stream;
  const int64_t groups = h->plan.units * c.n_kv_heads;
  const bool many = h->plan_wide;
  if (c.codes == PASTA_KV8_E4M3)
    c.head_dim == 128 ? launch_attend<k8::kE4m3, 128>(k, many, groups, s) : launch_attend<k8::kE4m3, 64>(k, many, groups, s);
  else
    c.head_dim == 128 ? launch_attend<k8::kInt8, 128>(k, many, groups, s) : launch_attend<k8::kInt8, 64>(k, many, groups, s);
  if (!h->plan_whole) {
    const int64_t tiles = h->plan.tiles * c.n_kv_heads;
    int64_t split = (2048 + tiles - 1) / tiles;  // work-groups to a tile: rows, one by one where there are so few tiles
    if (split > h->plan.merge_rows) split = h->plan.merge_rows;
    const dim3 grid((unsigned)tiles, (unsigned)split);
    if (c.head_dim == 128)
      k8::k8_merge<128><<<grid, 256, 0, s>>>(k);
    else
      k8::k8_merge<64><<<grid, 256, 0, s>>>(k);
  }
  return launched();
}
