// Host side of the 8-bit paged KV cache (include/pasta_kv8.h): checks of arguments, layout of the workspace, launches.
// No call here depends on what a device array holds: grids go by the sizes that the caller gives, work-groups that find nothing to do end.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>

#include "../../include/pasta_kv8.h"
#include "k8_append.hpp"
#include "k8_attend.hpp"
#include "k8_host.hpp"
#include "k8_rules.hpp"
#include "k8_slots.hpp"

namespace {

constexpr uint64_t kMagic = 0x3876'6b61'7473'6170ull;

}  // namespace

struct pasta_kv8 {
  uint64_t magic = kMagic;
  pasta_kv8_config cfg{};
  k8::Geometry g{};
  // workspace
  int *kept = nullptr, *old_pages = nullptr, *take = nullptr, *top = nullptr;
  k8::PlanSpace space;
  k8::Planned plan;  // the last one
};

namespace {

using k8::aligned;

int32_t check(const pasta_kv8_config* c) {
  if (!c || c->struct_size != sizeof(pasta_kv8_config)) return PASTA_E_INVAL;
  if (c->codes != PASTA_KV8_E4M3 && c->codes != PASTA_KV8_INT8) return PASTA_E_INVAL;
  if (c->dtype != PASTA_BF16 && c->dtype != PASTA_F16) return PASTA_E_INVAL;
  return k8::sizes_hold(*c) ? PASTA_OK : PASTA_E_INVAL;
}

uint64_t lay_out(const pasta_kv8_config& c, pasta_kv8* h) {
  uint64_t at = 0;
  auto take = [&](auto*& p, uint64_t n) {
    p = reinterpret_cast<std::remove_reference_t<decltype(p)>>((uint8_t*)c.workspace + at);
    at += (n * sizeof(*p) + 255) / 256 * 256;
  };
  take(h->kept, c.max_requests);
  take(h->old_pages, c.max_requests);
  take(h->take, c.max_requests);
  take(h->top, 1);
  h->space.lay_out(c, take);
  return at;
}

bool overlap(const int32_t* a, int64_t n, const int32_t* b, int64_t m) { return (uintptr_t)a < (uintptr_t)(b + m) && (uintptr_t)b < (uintptr_t)(a + n); }

using k8::launched;

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
  const int32_t rc = k8::check_plan(h->cfg, a);
  if (rc != PASTA_OK) return rc;
  return k8::launch_plan(h->cfg, h->g, h->space, *a, h->plan) ? PASTA_OK : PASTA_E_DEVICE;
}

namespace {

template <int CODES, int D>
void launch_attend(const k8::AttendArgs& k, const k8::Planned& plan, hipStream_t s) {
  const int64_t groups = plan.most.units * k.g.Hkv;
  k8::by_kind(k, plan, [&](auto many, auto kind) {
    const dim3 grid((unsigned)groups, many.value && k8::kApart<CODES, D, kind.value> ? k8::kWideRows / k8::kRows : 1);
    k8::k8_attend<CODES, D, many.value, kind.value><<<grid, 256, 0, s>>>(k);
  });
}

}  // namespace

extern "C" int32_t pasta_kv8_attend(pasta_kv8* h, const pasta_kv8_attend_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  const pasta_kv8_config& c = h->cfg;
  const int32_t rc = k8::check_attend(c, a, h->plan);
  if (rc != PASTA_OK || a->n_rows == 0) return rc;
  k8::AttendArgs k{};
  k8::fill_attend(c, h->g, h->space, *a, k);
  const int64_t at = (int64_t)c.n_phys_pages * c.n_kv_heads * h->g.blocks_per_page * a->layer;
  k.k = (const uint8_t*)c.k_codes + at * 16 * c.head_dim, k.v = (const uint8_t*)c.v_codes + at * 16 * c.head_dim;
  k.ks = c.k_scale + at, k.vs = c.v_scale + at;
  hipStream_t s = (hipStream_t)c.hip_stream;
  if (c.codes == PASTA_KV8_E4M3)
    c.head_dim == 128 ? launch_attend<k8::kE4m3, 128>(k, h->plan, s) : launch_attend<k8::kE4m3, 64>(k, h->plan, s);
  else
    c.head_dim == 128 ? launch_attend<k8::kInt8, 128>(k, h->plan, s) : launch_attend<k8::kInt8, 64>(k, h->plan, s);
  k8::launch_merge(k, h->plan, s);
  return launched();
}
