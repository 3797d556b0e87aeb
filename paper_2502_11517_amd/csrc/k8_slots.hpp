// Places of a step's rows: pages off and onto the stack, entries of the page tables, slots.
//
// One work-group does everything that goes in the order of the requests (two passes over them, NT at a time, with sums that carry
// over); the rows follow, each by itself: a new page has a first row, which writes its entry of the table.  Nothing here is bound
// by bandwidth; a step takes a handful of dependent reads and, per pass, two barriers for each sum.  Rows beyond kSlotsHere go to a
// second launch over the whole chip.
#pragma once
#include "k8_dev.hpp"

namespace k8 {

constexpr int kSlotsHere = 4096;  // rows that the one work-group places itself

struct SlotsArgs {
  Geometry g;
  int n_requests, n_rows;
  const int *length, *keep, *row_offsets;
  const uint8_t* row_tag;
  const int* row_position;
  const int* free_count;
  int *slot, *length_out, *free_out;
  int *table, *stack;
  uint8_t* slot_tag;
  int* slot_position;
  int *w_kept, *w_old, *w_take;  // workspace, one per request: tokens kept; pages it has; first page taken (in stack order), -1 refused
  int* w_top;                    // workspace: pages on the stack ahead of taking
};

struct RequestRows {
  int length, kept, n, old_pages, new_pages;
  bool fits;
};

__device__ inline RequestRows request_rows(const SlotsArgs& a, int r) {
  RequestRows q;
  const int cap = a.g.table_width << a.g.page_shift;
  q.length = min(max(a.length[r], 0), cap);
  q.kept = a.keep ? min(q.length, max(a.keep[r], 0)) : q.length;
  const int lo = min(max(a.row_offsets[r], 0), a.n_rows), hi = min(max(a.row_offsets[r + 1], lo), a.n_rows);
  q.n = hi - lo;
  const int64_t want = (int64_t)q.kept + q.n;
  q.fits = want <= cap;
  q.old_pages = (q.length + a.g.page_tokens - 1) >> a.g.page_shift;
  q.new_pages = (int)((want + a.g.page_tokens - 1) >> a.g.page_shift);
  return q;
}

__device__ inline void place_row(const SlotsArgs& a, int i) {
  int slot = -1;
  const int r = count_le(a.row_offsets + 1, a.n_requests, i);
  if (r < a.n_requests) {
    const int take = a.w_take[r];
    if (take >= 0) {
      const int p = a.w_kept[r] + i - max(a.row_offsets[r], 0);
      const int page_of = p >> a.g.page_shift, old = a.w_old[r];
      if (p >= 0 && page_of < a.g.table_width) {
        int* entry = a.table + (int64_t)r * a.g.table_width + page_of;
        int page;
        if (page_of < old) {
          page = *entry;
        } else {
          const int at = a.w_top[0] - 1 - (take + page_of - old);
          page = at >= 0 && at < a.g.n_pages ? a.stack[at] : -1;
          if ((p & (a.g.page_tokens - 1)) == 0) *entry = page;
        }
        if (page >= 0 && page < a.g.n_pages) slot = (page << a.g.page_shift) + (p & (a.g.page_tokens - 1));
      }
    }
  }
  a.slot[i] = slot;
  if (slot >= 0) {
    if (a.row_tag) a.slot_tag[slot] = a.row_tag[i];
    if (a.row_position) a.slot_position[slot] = a.row_position[i];
  }
}

template <int NT>
__global__ __launch_bounds__(NT) void k8_slots(SlotsArgs a) {
  __shared__ int s_tmp[NT / 64], s_first[NT], s_page[NT];
  const int tid = threadIdx.x;
  const int have = min(max(*a.free_count, 0), a.g.n_pages);
  // pages that go back
  int freed = 0;
  for (int r0 = 0; r0 < a.n_requests; r0 += NT) {
    const int r = r0 + tid;
    int mine = 0, first = 0;
    if (r < a.n_requests) {
      const RequestRows q = request_rows(a, r);
      mine = q.fits ? max(q.old_pages - q.new_pages, 0) : 0;
      first = q.new_pages;
    }
    int all;
    const int upto = group_scan<NT>(mine, s_tmp, all);
    if (all) {  // (the same for every thread)
      s_first[tid] = upto;
      s_page[tid] = first - (upto - mine);
      __syncthreads();
      for (int j = tid; j < all; j += NT) {
        const int q = count_le(s_first, NT, j);
        const int to = have + freed + j;
        if (to < a.g.n_pages) a.stack[to] = a.table[(int64_t)(r0 + q) * a.g.table_width + s_page[q] + j];
      }
      __syncthreads();
    }
    freed += all;
  }
  const int top = min(have + freed, a.g.n_pages);
  // pages that are taken
  int taken = 0, asked = 0;
  for (int r0 = 0; r0 < a.n_requests; r0 += NT) {
    const int r = r0 + tid;
    RequestRows q{};
    int need = 0;
    if (r < a.n_requests) {
      q = request_rows(a, r);
      need = q.fits ? max(q.new_pages - q.old_pages, 0) : 0;
    }
    int all;
    const int upto = asked + group_scan<NT>(need, s_tmp, all);  // (at most n_requests * table_width pages)
    const bool served = q.fits && (need == 0 || upto <= top);
    if (r < a.n_requests) {
      a.w_kept[r] = q.kept;
      a.w_old[r] = q.old_pages;
      a.w_take[r] = served ? upto - need : -1;
      a.length_out[r] = served ? q.kept + q.n : q.length;
    }
    int got;
    group_scan<NT>(served ? need : 0, s_tmp, got);
    taken += got;
    asked += all;
  }
  if (tid == 0) {
    *a.free_out = top - taken;
    *a.w_top = top;
  }
  if (a.n_rows > kSlotsHere) return;
  __syncthreads();
  for (int i = tid; i < a.n_rows; i += NT) place_row(a, i);
}

__global__ __launch_bounds__(256) void k8_place(SlotsArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < a.n_rows) place_row(a, i);
}

}  // namespace k8
