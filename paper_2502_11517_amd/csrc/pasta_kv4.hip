// Host side of the 4-bit paged KV cache (include/pasta_kv4.h): checks of arguments, launches.  The attention's plan is that of the 8-bit cache.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <new>

#include "../../include/pasta_kv4.h"
#include "k4_attend.hpp"
#include "k4_rows.hpp"
#include "k8_host.hpp"
#include "k8_rules.hpp"

namespace {

using k8::aligned;
using k8::launched;

constexpr int kMaxRead = 1 << 27;  // rows, 16 to a work-group in such calls: a launch has fewer than 2^32 threads
constexpr uint64_t kMagic = 0x3476'6b61'7473'6170ull;

}  // namespace

struct pasta_kv4 {
  uint64_t magic = kMagic;
  pasta_kv4_config cfg{};
  k8::Geometry g{};
  k8::PlanSpace space{k8::kLeastAlone4, k4::kFewRows};
  k8::Planned plan;  // the last one
};

namespace {

int32_t check(const pasta_kv4_config* c) {
  if (!c || c->struct_size != sizeof(pasta_kv4_config)) return PASTA_E_INVAL;
  if (c->dtype != PASTA_BF16 && c->dtype != PASTA_F16) return PASTA_E_INVAL;
  return k8::sizes_hold(*c) ? PASTA_OK : PASTA_E_INVAL;
}

uint64_t lay_out(const pasta_kv4_config& c, pasta_kv4* h) {
  uint64_t at = 0;
  h->space.lay_out(c, [&](auto*& p, uint64_t n) {
    p = reinterpret_cast<std::remove_reference_t<decltype(p)>>((uint8_t*)c.workspace + at);
    at += (n * sizeof(*p) + 255) / 256 * 256;
  });
  return at;
}

int64_t first_block(const pasta_kv4& h, int layer) { return (int64_t)h.cfg.n_phys_pages * h.cfg.n_kv_heads * h.g.blocks_per_page * layer; }

bool is_row_type(int32_t t) { return t == PASTA_F32 || t == PASTA_BF16 || t == PASTA_F16; }

// 0 becomes the row's own length; what is left has to hold a row and to keep rows aligned.
bool stride_of(const pasta_kv4_config& c, int32_t dtype, int64_t& stride) {
  const int64_t row = (int64_t)c.n_kv_heads * c.head_dim, unit = dtype == PASTA_F32 ? 4 : 8;
  if (stride == 0) stride = row;
  return stride >= row && stride % unit == 0 && stride < (int64_t)1 << 40;
}

// f(head dim, type of the rows), as constants.
template <class F>
void by_rows(int head_dim, int32_t dtype, F f) {
  auto with = [&](auto d) {
    if (dtype == PASTA_F32) f(d, std::integral_constant<int, k8::kF32>{});
    else if (dtype == PASTA_BF16) f(d, std::integral_constant<int, k8::kBf16>{});
    else f(d, std::integral_constant<int, k8::kF16>{});
  };
  head_dim == 128 ? with(std::integral_constant<int, 128>{}) : with(std::integral_constant<int, 64>{});
}

}  // namespace

extern "C" int32_t pasta_kv4_create(pasta_kv4_config* cfg, pasta_kv4** out) {
  const int32_t rc = check(cfg);
  if (rc != PASTA_OK) return rc;
  if (!out) {
    pasta_kv4 none;
    pasta_kv4_config c = *cfg;
    c.workspace = nullptr;
    cfg->workspace_bytes = lay_out(c, &none);
    return PASTA_OK;
  }
  *out = nullptr;
  if (!aligned(cfg->k_codes, 16) || !aligned(cfg->v_codes, 16) || !aligned(cfg->k_scale, 16) || !aligned(cfg->v_scale, 16)) return PASTA_E_INVAL;
  if (!aligned(cfg->page_table, 4) || !aligned(cfg->slot_tag, 16) || !aligned(cfg->slot_position, 16)) return PASTA_E_INVAL;
  if (!aligned(cfg->workspace, 256)) return PASTA_E_INVAL;
  pasta_kv4* h = new (std::nothrow) pasta_kv4();
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

extern "C" int32_t pasta_kv4_destroy(pasta_kv4* h) {
  if (!h) return PASTA_OK;
  if (h->magic != kMagic) return PASTA_E_STATE;
  h->magic = 0;
  delete h;
  return PASTA_OK;
}

extern "C" int32_t pasta_kv4_append(pasta_kv4* h, const pasta_kv4_append_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  if (!a || a->struct_size != sizeof(*a) || a->flags) return PASTA_E_INVAL;
  const pasta_kv4_config& c = h->cfg;
  if (a->layer < 0 || a->layer >= c.n_layers || a->n_rows < 0 || !is_row_type(a->dtype)) return PASTA_E_INVAL;
  if (a->n_rows > c.max_rows) return PASTA_E_CAPACITY;
  if (!c.k_codes || !c.v_codes || !c.k_scale || !c.v_scale) return PASTA_E_INVAL;
  k4::RowArgs k{};
  k.k_stride = a->k_stride, k.v_stride = a->v_stride;
  if (!stride_of(c, a->dtype, k.k_stride) || !stride_of(c, a->dtype, k.v_stride)) return PASTA_E_INVAL;
  if (a->n_rows == 0) return PASTA_OK;
  if (!a->slot || !a->k_new || !a->v_new) return PASTA_E_INVAL;
  if (!aligned(a->slot, 4) || !aligned(a->k_new, 16) || !aligned(a->v_new, 16)) return PASTA_E_INVAL;
  const int64_t at = first_block(*h, a->layer);
  k.g = h->g, k.n_rows = a->n_rows, k.slot = a->slot, k.k_new = a->k_new, k.v_new = a->v_new;
  k.k = (uint8_t*)c.k_codes + at * 8 * c.head_dim, k.v = (uint8_t*)c.v_codes + at * 8 * c.head_dim;
  k.ks = c.k_scale + at * 16 * (c.head_dim / 32), k.vs = c.v_scale + at * 16;
  k.group = k8::append_group(a->n_rows, c.n_kv_heads);
  const dim3 grid((a->n_rows + k.group - 1) / k.group, (2 * c.n_kv_heads + 3) / 4);
  by_rows(c.head_dim, a->dtype, [&](auto d, auto type) { k4::k4_append<d.value, type.value><<<grid, 256, 0, (hipStream_t)c.hip_stream>>>(k); });
  return launched();
}

extern "C" int32_t pasta_kv4_read(pasta_kv4* h, const pasta_kv4_read_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  if (!a || a->struct_size != sizeof(*a) || a->flags) return PASTA_E_INVAL;
  const pasta_kv4_config& c = h->cfg;
  if (a->layer < 0 || a->layer >= c.n_layers || a->n_rows < 0 || !is_row_type(a->dtype)) return PASTA_E_INVAL;
  if (a->n_rows > kMaxRead) return PASTA_E_CAPACITY;
  if ((a->k_out && (!c.k_codes || !c.k_scale)) || (a->v_out && (!c.v_codes || !c.v_scale))) return PASTA_E_INVAL;
  k4::RowArgs k{};
  k.k_stride = a->k_stride, k.v_stride = a->v_stride;
  if (!stride_of(c, a->dtype, k.k_stride) || !stride_of(c, a->dtype, k.v_stride)) return PASTA_E_INVAL;
  if (a->n_rows == 0) return PASTA_OK;
  if (!a->slot || (!a->k_out && !a->v_out)) return PASTA_E_INVAL;
  if (!aligned(a->slot, 4) || !aligned(a->k_out, 16) || !aligned(a->v_out, 16)) return PASTA_E_INVAL;
  const int64_t at = first_block(*h, a->layer);
  k.g = h->g, k.n_rows = a->n_rows, k.slot = a->slot, k.k_out = a->k_out, k.v_out = a->v_out;
  k.k = (uint8_t*)c.k_codes + at * 8 * c.head_dim, k.v = (uint8_t*)c.v_codes + at * 8 * c.head_dim;
  k.ks = c.k_scale + at * 16 * (c.head_dim / 32), k.vs = c.v_scale + at * 16;
  k.group = k8::append_group(a->n_rows, c.n_kv_heads);
  const int tasks = c.n_kv_heads * (a->k_out && a->v_out ? 2 : 1);
  const dim3 grid((a->n_rows + (int64_t)k.group - 1) / k.group, (tasks + 3) / 4);
  by_rows(c.head_dim, a->dtype, [&](auto d, auto type) { k4::k4_read<d.value, type.value><<<grid, 256, 0, (hipStream_t)c.hip_stream>>>(k); });
  return launched();
}

extern "C" int32_t pasta_kv4_plan(pasta_kv4* h, const pasta_kv8_plan_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  const int32_t rc = k8::check_plan(h->cfg, a);
  if (rc != PASTA_OK) return rc;
  return k8::launch_plan(h->cfg, h->g, h->space, *a, h->plan) ? PASTA_OK : PASTA_E_DEVICE;
}

namespace {

template <int D, bool F16>
void launch_attend(const k4::AttendArgs& k, const k8::Planned& plan, hipStream_t s) {
  const int64_t groups = plan.most.units * k.g.Hkv;
  k8::by_kind(k, plan, [&](auto many, auto kind) {
    const dim3 grid((unsigned)groups, many.value && k4::kApart<D, kind.value> ? k8::kWideRows / k8::kRows : 1);
    k4::k4_attend<D, F16, many.value, kind.value><<<grid, 256, 0, s>>>(k);
  });
}

}  // namespace

extern "C" int32_t pasta_kv4_attend(pasta_kv4* h, const pasta_kv8_attend_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  const pasta_kv4_config& c = h->cfg;
  const int32_t rc = k8::check_attend(c, a, h->plan);
  if (rc != PASTA_OK || a->n_rows == 0) return rc;
  k4::AttendArgs k{};
  k8::fill_attend(c, h->g, h->space, *a, k);
  const int64_t at = first_block(*h, a->layer);
  k.k = (const uint8_t*)c.k_codes + at * 8 * c.head_dim, k.v = (const uint8_t*)c.v_codes + at * 8 * c.head_dim;
  k.k_scale = c.k_scale + at * 16 * (c.head_dim / 32), k.v_scale = c.v_scale + at * 16;
  hipStream_t s = (hipStream_t)c.hip_stream;
  if (c.dtype == PASTA_BF16)
    c.head_dim == 128 ? launch_attend<128, false>(k, h->plan, s) : launch_attend<64, false>(k, h->plan, s);
  else
    c.head_dim == 128 ? launch_attend<128, true>(k, h->plan, s) : launch_attend<64, true>(k, h->plan, s);
  k8::launch_merge(k, h->plan, s);
  return launched();
}
