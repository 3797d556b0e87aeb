// Places of a step's rows: pages off and onto the stack, entries of the page tables, slots.
//
// Everything goes in the order of the requests, by sums over them; nothing is bound by bandwidth.  What a step takes is its dependent reads, one
// behind the other, so with up to a thread per request all of them are asked for at once, the sums stay in LDS, and every work-group finds out the
// same for itself: the first writes what belongs to the requests, all of them return pages and place rows, in one launch.  A page that comes back
// and is taken in the same step is looked up where it was, not on the stack.  Where lengths or the count are written in place that does not go (one work-group may write
// what another has still to read), and with more requests than threads neither: one work-group then does the requests, and rows beyond kSlotsHere
// follow in a second launch.  16 requests of up to eight rows 2.7 us, 512 requests with drafts taken back 5.8, 64 prompts with 259k rows 4.4 (3.7 MB):
// launch, three reads behind one another, two sums over the requests and a search per row.  In place, calls alone: the first 3.4 (3.5 apart), the second 6.8
// and 5.3 in two launches (6.2), the third 3.6 and 6.1 (5.3), 64 requests of 64 rows 12.3 (4.4).  1500 requests of a row, either way: 12.4.
#pragma once
#include "k8_dev.hpp"

namespace k8 {

constexpr int kSlotsHere = 4096;  // rows that one work-group places itself

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

__device__ inline RequestRows request_rows_of(const SlotsArgs& a, int r) {
  RequestRows q;
  const int length = a.length[r], keep = a.keep ? a.keep[r] : INT32_MAX, first = a.row_offsets[r], next = a.row_offsets[r + 1];
  const int cap = a.g.table_width << a.g.page_shift;
  q.length = min(max(length, 0), cap);
  q.kept = min(q.length, max(keep, 0));
  const int lo = min(max(first, 0), a.n_rows), hi = min(max(next, lo), a.n_rows);
  q.n = hi - lo;
  const int64_t want = (int64_t)q.kept + q.n;
  q.fits = want <= cap;
  q.old_pages = (q.length + a.g.page_tokens - 1) >> a.g.page_shift;
  q.new_pages = (int)((want + a.g.page_tokens - 1) >> a.g.page_shift);
  return q;
}

__device__ inline void give_slot(const SlotsArgs& a, int i, int page, int p) {
  const int slot = page >= 0 && page < a.g.n_pages ? (page << a.g.page_shift) + (p & (a.g.page_tokens - 1)) : -1;
  a.slot[i] = slot;
  if (slot >= 0) {
    if (a.row_tag) a.slot_tag[slot] = a.row_tag[i];
    if (a.row_position) a.slot_position[slot] = a.row_position[i];
  }
}

// At most NT requests.
template <int NT>
__global__ __launch_bounds__(NT) void k8_slots(SlotsArgs a) {
  __shared__ int2v s_tmp[NT / 64];
  __shared__ int s_next[NT], s_first[NT], s_kept[NT], s_old[NT], s_take[NT], s_freed[NT], s_page[NT];
  const int tid = threadIdx.x;
  const int have = min(max(*a.free_count, 0), a.g.n_pages);
  RequestRows q{};
  int first = 0, next = INT32_MAX;
  if (tid < a.n_requests) {
    q = request_rows_of(a, tid);
    first = max(a.row_offsets[tid], 0), next = a.row_offsets[tid + 1];
  }
  const int back = q.fits ? max(q.old_pages - q.new_pages, 0) : 0, need = q.fits ? max(q.new_pages - q.old_pages, 0) : 0;
  int2v all;
  int taken;
  const int2v upto = group_scan<NT>(int2v{back, need}, s_tmp, all);  // (at most n_requests * table_width pages)
  const int back_upto = upto[0], need_upto = upto[1], freed = all[0];
  const int top = min(have + freed, a.g.n_pages);
  const bool served = q.fits && (need == 0 || need_upto <= top);
  s_next[tid] = next, s_first[tid] = first, s_kept[tid] = q.kept, s_old[tid] = q.old_pages, s_take[tid] = served ? need_upto - need : -1;
  s_freed[tid] = back_upto, s_page[tid] = q.new_pages - (back_upto - back);
  group_scan<NT>(served ? need : 0, s_tmp, taken);  // (its barriers stand between the writes above and what follows)
  // page j of those that come back
  auto came_back = [&](int j) {
    const int r = min(count_le(s_freed, NT, j), max(a.n_requests - 1, 0));
    return a.table[(int64_t)r * a.g.table_width + s_page[r] + j];
  };
  if (blockIdx.x == 0) {
    if (tid < a.n_requests) a.length_out[tid] = served ? q.kept + q.n : q.length;
    if (tid == 0) *a.free_out = top - taken;
  }
  for (int j = blockIdx.x * NT + tid; j < freed; j += gridDim.x * NT)
    if (have + j < a.g.n_pages) a.stack[have + j] = came_back(j);
  for (int i = blockIdx.x * NT + tid; i < a.n_rows; i += gridDim.x * NT) {
    const int r = count_le(s_next, a.n_requests, i);
    int page = -1, p = 0;
    if (r < a.n_requests && s_take[r] >= 0) {
      p = s_kept[r] + i - s_first[r];
      const int of = p >> a.g.page_shift, old = s_old[r];
      if (p >= 0 && of < a.g.table_width) {
        int* entry = a.table + (int64_t)r * a.g.table_width + of;
        if (of < old) {
          page = *entry;
        } else {
          const int at = top - 1 - (s_take[r] + of - old);
          if (at >= 0) page = at < have ? a.stack[at] : came_back(at - have);
          if ((p & (a.g.page_tokens - 1)) == 0) *entry = page;
        }
      }
    }
    give_slot(a, i, page, p);
  }
}

__device__ inline void place_row(const SlotsArgs& a, int i) {
  const int r = count_le(a.row_offsets + 1, a.n_requests, i);
  int page = -1, p = 0;
  if (r < a.n_requests && a.w_take[r] >= 0) {
    p = a.w_kept[r] + i - max(a.row_offsets[r], 0);
    const int of = p >> a.g.page_shift, old = a.w_old[r];
    if (p >= 0 && of < a.g.table_width) {
      int* entry = a.table + (int64_t)r * a.g.table_width + of;
      if (of < old) {
        page = *entry;
      } else {
        const int at = a.w_top[0] - 1 - (a.w_take[r] + of - old);
        if (at >= 0 && at < a.g.n_pages) page = a.stack[at];
        if ((p & (a.g.page_tokens - 1)) == 0) *entry = page;
      }
    }
  }
  give_slot(a, i, page, p);
}

// Any number of requests, NT at a time, or lengths in place; one work-group.
template <int NT>
__global__ __launch_bounds__(NT) void k8_slots_long(SlotsArgs a) {
  __shared__ int2v s_tmp[NT / 64];
  __shared__ int s_first[NT], s_page[NT];
  const int tid = threadIdx.x;
  const int have = min(max(*a.free_count, 0), a.g.n_pages);
  // pages that go back
  int freed = 0;
  for (int r0 = 0; r0 < a.n_requests; r0 += NT) {
    const int r = r0 + tid;
    int mine = 0, first = 0;
    if (r < a.n_requests) {
      const RequestRows q = request_rows_of(a, r);
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
      q = request_rows_of(a, r);
      need = q.fits ? max(q.new_pages - q.old_pages, 0) : 0;
    }
    int all, got;
    const int upto = asked + group_scan<NT>(need, s_tmp, all);
    const bool served = q.fits && (need == 0 || upto <= top);
    if (r < a.n_requests) {
      a.w_kept[r] = q.kept;
      a.w_old[r] = q.old_pages;
      a.w_take[r] = served ? upto - need : -1;
      a.length_out[r] = served ? q.kept + q.n : q.length;
    }
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
