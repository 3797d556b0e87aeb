// Host side of the operators on a step's rows (include/pasta_rows.h): checks of arguments, launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <new>
#include <type_traits>

#include "../../include/pasta_rows.h"
#include "rows_rotate.hpp"
#include "rows_verify.hpp"

namespace {

constexpr uint64_t kMagic = 0x7277'6b61'7473'6170ull;
constexpr int kMaxRows = (1 << 24) - 1;  // of a work-group each: a launch has fewer than 2^32 threads
constexpr int kMaxVocab = 1 << 22, kWholeVocab = 16 * 8 * 256;  // the latter: 16 waves of 8 times 256 tokens

}  // namespace

struct pasta_rows {
  uint64_t magic = kMagic;
  pasta_rows_config cfg{};
  double* sums = nullptr;
  int2* outcomes = nullptr;
};

namespace {

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

int32_t launched() { return hipGetLastError() == hipSuccess ? PASTA_OK : PASTA_E_DEVICE; }

int segments_of(int vocab) { return vocab > kWholeVocab ? (vocab + rows::kSegment - 1) / rows::kSegment : 0; }

// Sums of every sequence's segments, then what became of its drafts.
uint64_t sums_of(const pasta_rows_config& c) { return (uint64_t)segments_of(c.vocab) * c.max_sequences; }
uint64_t workspace_of(const pasta_rows_config& c) { return segments_of(c.vocab) ? sums_of(c) * sizeof(double) + c.max_sequences * sizeof(int2) : 0; }

int32_t check(const pasta_rows_config* c) {
  if (!c || c->struct_size != sizeof(*c) || c->max_rows < 1 || c->max_rows > kMaxRows) return PASTA_E_INVAL;
  if (c->rope_dims == 0 && c->vocab == 0) return PASTA_E_INVAL;
  if (c->rope_dims) {
    if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_q_heads > 1024 || c->n_kv_heads > 1024 || c->n_q_heads + c->n_kv_heads > 1024) return PASTA_E_INVAL;
    if (c->head_dim < 8 || c->head_dim > rows::kMaxDim || c->head_dim % 8) return PASTA_E_INVAL;
    if (c->rope_dims < 2 || c->rope_dims > c->head_dim || c->rope_dims % 2) return PASTA_E_INVAL;
    if (c->rope_layout != PASTA_ROPE_HALF && c->rope_layout != PASTA_ROPE_INTERLEAVED) return PASTA_E_INVAL;
    if (!std::isfinite(c->rope_magnitude)) return PASTA_E_INVAL;
  } else if (c->n_q_heads || c->n_kv_heads || c->head_dim || c->rope_layout || c->rope_magnitude != 0.f || c->rope_frequency) {
    return PASTA_E_INVAL;
  }
  if (c->vocab) {
    if (c->vocab < 1 || c->vocab > kMaxVocab || c->max_sequences < 1 || c->max_sequences > 65535) return PASTA_E_INVAL;
  } else if (c->max_sequences) {
    return PASTA_E_INVAL;
  }
  return PASTA_OK;
}

bool is_row_type(int32_t t) { return t == PASTA_F32 || t == PASTA_BF16 || t == PASTA_F16; }

// f(type of the rows), as a constant.
template <class F>
void by_type(int32_t dtype, F f) {
  if (dtype == PASTA_F32) f(std::integral_constant<int, rows::kF32>{});
  else if (dtype == PASTA_BF16) f(std::integral_constant<int, rows::kBf16>{});
  else f(std::integral_constant<int, rows::kF16>{});
}

// Rows of `heads` heads from `in` to `out`; false: refused.
bool side_of(const pasta_rows_config& c, int32_t dtype, int heads, const void* in, void* out, int64_t in_stride, int64_t out_stride, rows::Side& s) {
  const int64_t row = (int64_t)heads * c.head_dim, unit = dtype == PASTA_F32 ? 4 : 8;
  s = rows::Side{in, out, in_stride ? in_stride : row, out_stride ? out_stride : row};
  for (const int64_t stride : {s.in_stride, s.out_stride})
    if (stride < row || stride % unit || stride >= (int64_t)1 << 40) return false;
  return !in == !out && aligned(in, 16) && aligned(out, 16) && (in != out || s.in_stride == s.out_stride);
}

}  // namespace

extern "C" int32_t pasta_rows_create(pasta_rows_config* cfg, pasta_rows** out) {
  const int32_t rc = check(cfg);
  if (rc != PASTA_OK) return rc;
  const uint64_t need = workspace_of(*cfg);
  if (!out) {
    cfg->workspace_bytes = need;
    return PASTA_OK;
  }
  *out = nullptr;
  if (!aligned(cfg->rope_frequency, 8) || !aligned(cfg->workspace, 256)) return PASTA_E_INVAL;
  if (cfg->workspace && cfg->workspace_bytes < need) return PASTA_E_CAPACITY;
  pasta_rows* h = new (std::nothrow) pasta_rows();
  if (!h) return PASTA_E_NOMEM;
  h->cfg = *cfg;
  h->sums = (double*)cfg->workspace, h->outcomes = (int2*)(h->sums + sums_of(*cfg));
  *out = h;
  return PASTA_OK;
}

extern "C" int32_t pasta_rows_destroy(pasta_rows* h) {
  if (!h) return PASTA_OK;
  if (h->magic != kMagic) return PASTA_E_STATE;
  h->magic = 0;
  delete h;
  return PASTA_OK;
}

extern "C" int32_t pasta_rows_rotate(pasta_rows* h, const pasta_rows_rotate_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  if (!a || a->struct_size != sizeof(*a) || (a->flags & ~(uint32_t)PASTA_ROWS_BACKWARD)) return PASTA_E_INVAL;
  const pasta_rows_config& c = h->cfg;
  if (!c.rope_dims || !c.rope_frequency || a->n_rows < 0 || !is_row_type(a->dtype)) return PASTA_E_INVAL;
  if (a->n_rows > c.max_rows) return PASTA_E_CAPACITY;
  rows::RotateArgs k{};
  if (!side_of(c, a->dtype, c.n_q_heads, a->q, a->q_out, a->q_stride, a->q_out_stride, k.q)) return PASTA_E_INVAL;
  if (!side_of(c, a->dtype, c.n_kv_heads, a->k, a->k_out, a->k_stride, a->k_out_stride, k.k)) return PASTA_E_INVAL;
  if (a->n_rows == 0) return PASTA_OK;
  if (!a->position || !aligned(a->position, 4) || (!a->q && !a->k)) return PASTA_E_INVAL;
  k.n_rows = a->n_rows, k.n_q = a->q ? c.n_q_heads : 0, k.n_heads = k.n_q + (a->k ? c.n_kv_heads : 0);
  k.D = c.head_dim, k.planes = c.rope_dims / 2, k.interleaved = c.rope_layout == PASTA_ROPE_INTERLEAVED;
  k.magnitude = c.rope_magnitude, k.direction = a->flags & PASTA_ROWS_BACKWARD ? -c.rope_magnitude : c.rope_magnitude;
  k.frequency = c.rope_frequency, k.position = a->position;
  const int unit = a->dtype == PASTA_F32 ? 4 : 8, stays = c.head_dim - c.rope_dims;
  const bool wide = (k.interleaved ? c.rope_dims : k.planes) % unit == 0;  // (head_dim is whole 16-byte pieces, and then so is what stays)
  k.pieces = wide ? (k.interleaved ? c.rope_dims : k.planes) / unit + stays / unit : k.planes + stays;
  k.at_once = 256 / k.pieces;
  // Two rows to a work-group where that leaves 2048 of them and more, since more has to be on its way then (8192 rows of 32 + 8 heads, interleaved / half: 36 /
  // 38 us instead of 43 / 40; 2048 rows 8.7 and 8.9; of 1024 rows 6.0 and 5.6; four rows to a work-group are no better).
  const unsigned parts = (unsigned)((k.n_heads + k.at_once - 1) / k.at_once);
  auto launch = [&](auto type, auto wide, auto rows) {
    const dim3 grid((unsigned)(((int64_t)a->n_rows + rows.value - 1) / rows.value), parts);
    rows::rows_rotate<type.value, wide.value, rows.value><<<grid, 256, 0, (hipStream_t)c.hip_stream>>>(k);
  };
  by_type(a->dtype, [&](auto type) {
    if (!wide) launch(type, std::false_type{}, std::integral_constant<int, 1>{});
    else if ((int64_t)a->n_rows * parts < 4096) launch(type, std::true_type{}, std::integral_constant<int, 1>{});
    else launch(type, std::true_type{}, std::integral_constant<int, 2>{});
  });
  return launched();
}

extern "C" int32_t pasta_rows_verify(pasta_rows* h, const pasta_rows_verify_args* a) {
  if (!h || h->magic != kMagic) return PASTA_E_STATE;
  if (!a || a->struct_size != sizeof(*a) || a->flags) return PASTA_E_INVAL;
  const pasta_rows_config& c = h->cfg;
  if (!c.vocab || a->n_sequences < 0 || a->n_rows < 0 || !is_row_type(a->dtype)) return PASTA_E_INVAL;
  if (a->n_sequences > c.max_sequences || a->n_rows > c.max_rows) return PASTA_E_CAPACITY;
  rows::VerifyArgs k{};
  k.segments = segments_of(c.vocab);
  k.target_stride = a->target_stride ? a->target_stride : c.vocab, k.draft_stride = a->draft_stride ? a->draft_stride : c.vocab;
  for (const int64_t stride : {k.target_stride, k.draft_stride})
    if (stride < c.vocab || stride >= (int64_t)1 << 40) return PASTA_E_INVAL;
  if (k.segments && !c.workspace) return PASTA_E_INVAL;
  if (!a->keep != !a->length || !a->position_out != !a->row_position) return PASTA_E_INVAL;
  if (a->n_sequences == 0) return PASTA_OK;
  if (!a->row_offsets || !a->accepted || !a->next_token || !a->last_draw || (a->n_rows && (!a->token || !a->target || !a->draw))) return PASTA_E_INVAL;
  const void* words[] = {a->row_offsets, a->token, a->slot, a->draw, a->last_draw, a->length, a->row_position, a->accepted, a->next_token, a->keep, a->position_out};
  for (const void* p : words)
    if (!aligned(p, 4)) return PASTA_E_INVAL;
  const uintptr_t size = a->dtype == PASTA_F32 ? 4 : 2;
  if (!aligned(a->target, size) || !aligned(a->draft, size)) return PASTA_E_INVAL;
  k.n_sequences = a->n_sequences, k.n_rows = a->n_rows, k.vocab = c.vocab;
  k.row_offsets = a->row_offsets, k.token = a->token, k.slot = a->slot, k.target = a->target, k.draft = a->draft, k.draw = a->draw, k.last_draw = a->last_draw;
  k.length = a->length, k.row_position = a->row_position, k.accepted = a->accepted, k.next_token = a->next_token, k.keep = a->keep;
  k.position_out = a->position_out, k.sums = h->sums, k.outcomes = h->outcomes;
  hipStream_t s = (hipStream_t)c.hip_stream;
  by_type(a->dtype, [&](auto type) {
    if (k.segments) {
      rows::rows_verify_sums<type.value><<<dim3((unsigned)(k.segments + 3) / 4, (unsigned)a->n_sequences), 256, 0, s>>>(k);
      rows::rows_verify_pick<type.value><<<(unsigned)a->n_sequences, 256, 0, s>>>(k);
      return;
    }
    auto whole = [&](auto loads) {
      const unsigned waves = (unsigned)(c.vocab + loads.value * 256 - 1) / (loads.value * 256);
      rows::rows_verify_whole<type.value, loads.value><<<(unsigned)a->n_sequences, 64 * waves, 0, s>>>(k);
    };
    if (c.vocab <= 4096) whole(std::integral_constant<int, 1>{});
    else if (c.vocab <= 8192) whole(std::integral_constant<int, 2>{});
    else if (c.vocab <= 16384) whole(std::integral_constant<int, 4>{});
    else whole(std::integral_constant<int, 8>{});
  });
  return launched();
}
