// The paged key/value cache: which pages and slots a step's tokens take (plan), and their keys and values into them (append).
#include <algorithm>

#include "pages.h"

using namespace vitenc;

namespace {

// ---- plan ---------------------------------------------------------------------------------
// Request r's new tokens i = 0 ... new - 1 are at = cached + i of it, in its page nth = at / page_size.  The first
// held = ceil(cached / page_size) pages are in its row of the block table; the others are the free list's entries
// first + nth - held, where `first` is *taken plus the pages that the requests before it take: a prefix sum, like the rows'.
//
// Nothing here but latencies, so one launch does it where it can: every workgroup adds up the lengths of all requests for
// itself, keeps the sums in LDS and gives some of the rows their slots; the first one writes the requests' numbers and
// counts what got no slot.  Above 1024 requests, and where results lie in place of what the other workgroups still read, the sums
// are a launch of their own and the rows another.  One token 3.0 us, 500 requests of one token 5.2, 96 requests of 363197
// tokens 6.0.  Sums of the launch are in 32 bits that stop at the largest number.
struct PlanArgs {
  const int32_t *cached, *fresh, *free, *taken;
  int32_t *table, *slots, *starts, *kv, *firsts, *counts;
  int64_t stride;
  int R, width, n_free, n_pages, shift, rows;
};

constexpr int PLAN_THREADS = 1024;
constexpr int MAX_LEN = 1 << 30;

// Sums of `v` and `w` over the threads below this one, and over all of them (`v_all`, `w_all`); `waves`: two words of LDS a wave.  In 32
// bits that stop at the largest number: rows end at n_rows, and there is no page of such a number.
__device__ void scan_below(uint32_t& v, uint32_t& w, uint32_t (*waves)[2], uint32_t& v_all, uint32_t& w_all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t v_sum = wave_scan(v), w_sum = wave_scan(w);
  if (lane == 63) {
    waves[wave][0] = v_sum;
    waves[wave][1] = w_sum;
  }
  // below this lane: the sums of the lane to the left
  v = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v_sum, 0x138, 0xF, 0xF, false);
  w = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w_sum, 0x138, 0xF, 0xF, false);
  __syncthreads();
  // each wave adds up the others' sums for itself: lane i those of wave i
  constexpr int WAVES = PLAN_THREADS / 64;
  const uint32_t v_up = wave_scan(lane < WAVES ? waves[lane][0] : 0u), w_up = wave_scan(lane < WAVES ? waves[lane][1] : 0u);
  v_all = (uint32_t)__builtin_amdgcn_readlane((int)v_up, WAVES - 1);
  w_all = (uint32_t)__builtin_amdgcn_readlane((int)w_up, WAVES - 1);
  if (wave > 0) {
    const int left = __builtin_amdgcn_readfirstlane(wave - 1);
    v = __builtin_elementwise_add_sat(v, (uint32_t)__builtin_amdgcn_readlane((int)v_up, left));
    w = __builtin_elementwise_add_sat(w, (uint32_t)__builtin_amdgcn_readlane((int)w_up, left));
  }
  __syncthreads();
}

__device__ __forceinline__ int pages_of(int64_t tokens, const PlanArgs& a) {  // that the table has room for
  return (int)min((tokens + (1 << a.shift) - 1) >> a.shift, (int64_t)a.width);
}

// The page of token `at` of a request whose first pages, `held` of them, are in its table, and whose next one is free[first]; -1: none.
__device__ __forceinline__ int page_of(const PlanArgs& a, int64_t entries, int nth, int held, int first) {
  if (nth >= a.width) return -1;
  const int64_t index = (int64_t)first + (nth - held);
  const int page = nth < held ? a.table[entries + nth] : index < a.n_free ? a.free[index] : -1;
  return (unsigned)page < (unsigned)a.n_pages ? page : -1;
}

constexpr int PLAN_MANY = 1024;   // requests whose numbers one workgroup keeps
constexpr int PLAN_ROWS = 4096;   // rows of a workgroup

__global__ __launch_bounds__(PLAN_THREADS) void plan_kernel(const PlanArgs a) {
  __shared__ uint32_t waves[PLAN_THREADS / 64][2];
  __shared__ int64_t lost_of[PLAN_THREADS / 64];
  __shared__ int starts[PLAN_MANY + 1], cacheds[PLAN_MANY], firsts[PLAN_MANY + 1];
  const int tid = threadIdx.x;
  const int taken = a.taken ? max(*a.taken, 0) : 0;
  const bool mine = tid < a.R;
  const int cached = mine ? min(max(a.cached[tid], 0), MAX_LEN) : 0;
  const int asked = mine ? min(max(a.fresh[tid], 0), MAX_LEN) : 0;
  uint32_t at = asked, page = pages_of((int64_t)cached + asked, a) - pages_of(cached, a), all_rows, all_pages;
  scan_below(at, page, waves, all_rows, all_pages);
  const int start = (int)min(at, (uint32_t)a.rows), end = (int)min((int64_t)at + asked, (int64_t)a.rows), total = cached + (end - start);
  if (all_rows > (uint32_t)a.rows) {  // rows for fewer: the pages of those again
    uint32_t none = 0;
    page = pages_of(total, a) - pages_of(cached, a);
    scan_below(none, page, waves, none, all_pages);
  }
  const int first = (int)min((int64_t)page + taken, (int64_t)INT32_MAX), rows = (int)min(all_rows, (uint32_t)a.rows);
  const int64_t end_pages = min((int64_t)all_pages + taken, (int64_t)INT32_MAX);
  if (mine) {
    starts[tid] = start;
    cacheds[tid] = cached;
    firsts[tid] = first;
  }
  if (tid == 0) {
    starts[a.R] = rows;
    firsts[a.R] = (int)end_pages;
  }
  __syncthreads();
  // rows: four at a time, of the request that holds the first one and the ones behind it
  const int from = blockIdx.x * PLAN_ROWS, to = (int)min((int64_t)from + PLAN_ROWS, (int64_t)a.rows);
  for (int t = from + tid * 4; t < to; t += PLAN_THREADS * 4) {
    int slot[4] = {-1, -1, -1, -1};
    if (t < rows) {
      int lo = 0, hi = a.R - 1;  // the last request that starts at t or below: of those that start there, the one with rows
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (starts[mid] <= t) lo = mid;
        else hi = mid - 1;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (t + i >= rows) break;
        while (starts[lo + 1] <= t + i) ++lo;
        const int place = cacheds[lo] + (t + i - starts[lo]), nth = place >> a.shift, held = pages_of(cacheds[lo], a), in_page = place & ((1 << a.shift) - 1);
        const int number = page_of(a, lo * a.stride, nth, held, firsts[lo]);
        if (number >= 0) slot[i] = (number << a.shift) + in_page;
        if (nth >= held && nth < a.width && in_page == 0) a.table[lo * a.stride + nth] = number;  // the token that opens the page
      }
    }
    if (t + 4 <= to && ((uintptr_t)(a.slots + t) & 15) == 0) {
      *(int4*)(a.slots + t) = int4{slot[0], slot[1], slot[2], slot[3]};
    } else {
      for (int i = 0; i < 4 && t + i < to; ++i) a.slots[t + i] = slot[i];
    }
  }
  if (blockIdx.x != 0) return;
  // tokens without a slot: page by page, those of the free list and each request's open one, and what the table has no room for
  int64_t lost = 0;
  if (mine) {
    const int held = pages_of(cached, a), room = (int)min((int64_t)total, (int64_t)a.width << a.shift);
    lost = asked - (end - start) + (total - max(room, cached));
    const int open = (int)min((int64_t)room, (int64_t)held << a.shift) - cached;  // tokens that go into the open page
    if (open > 0 && page_of(a, tid * a.stride, held - 1, held, 0) < 0) lost += open;
  }
  for (int64_t k = (int64_t)taken + tid; k < end_pages; k += PLAN_THREADS) {
    if (k < a.n_free && (unsigned)a.free[k] < (unsigned)a.n_pages) continue;
    int lo = 0, hi = a.R - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (firsts[mid] <= k) lo = mid;
      else hi = mid - 1;
    }
    const int64_t before = (pages_of(cacheds[lo], a) + (k - firsts[lo])) << a.shift;  // tokens that lie before the page
    lost += min((int64_t)1 << a.shift, (int64_t)cacheds[lo] + (starts[lo + 1] - starts[lo]) - before);
  }
  lost = (int64_t)wave_scan((uint64_t)lost);
  if ((tid & 63) == 63) lost_of[tid >> 6] = lost;
  __syncthreads();  // (everything read by now that lies in place of a result)
  if (mine) {
    a.starts[tid] = start;
    a.kv[tid] = total;
    a.firsts[tid] = first;
  }
  if (tid == 0) {
    a.starts[a.R] = rows;
    a.firsts[a.R] = firsts[a.R];
    lost = 0;
    for (int w = 0; w < PLAN_THREADS / 64; ++w) lost += lost_of[w];
    a.counts[0] = (int32_t)min(end_pages, (int64_t)a.n_free);
    a.counts[1] = (int32_t)min(lost, (int64_t)INT32_MAX);
  }
}

__global__ __launch_bounds__(PLAN_THREADS) void plan_sums_kernel(const PlanArgs a) {
  __shared__ uint32_t waves[PLAN_THREADS / 64][2];
  const int64_t taken = a.taken ? max(*a.taken, 0) : 0;
  int64_t row = 0, first = taken;
  for (int base = 0; base < a.R; base += PLAN_THREADS) {
    const int r = base + threadIdx.x;
    const bool mine = r < a.R;
    const int cached = mine ? min(max(a.cached[r], 0), MAX_LEN) : 0;
    const int asked = mine ? min(max(a.fresh[r], 0), MAX_LEN) : 0;
    uint32_t at = asked, none = 0, all_rows, all_pages;
    scan_below(at, none, waves, all_rows, all_pages);
    const int start = (int)min(row + at, (int64_t)a.rows), end = (int)min(row + at + asked, (int64_t)a.rows), total = cached + (end - start);
    uint32_t page = pages_of(total, a) - pages_of(cached, a);
    none = 0;
    uint32_t no_rows;
    scan_below(none, page, waves, no_rows, all_pages);
    if (mine) {
      a.starts[r] = start;
      a.kv[r] = total;
      a.firsts[r] = (int32_t)min(first + page, (int64_t)INT32_MAX);
    }
    row += all_rows;
    first += all_pages;
  }
  if (threadIdx.x == 0) {
    const int64_t end = min(row, (int64_t)a.rows);
    a.starts[a.R] = (int32_t)end;
    a.firsts[a.R] = (int32_t)min(first, (int64_t)INT32_MAX);
    a.counts[0] = (int32_t)min(first, (int64_t)a.n_free);
    a.counts[1] = (int32_t)min(row - end, (int64_t)INT32_MAX);  // the tokens without a slot are added by plan_slots_kernel
  }
}

// One thread a row.
__global__ __launch_bounds__(256) void plan_slots_kernel(const PlanArgs a) {
  const int t = blockIdx.x * 256 + threadIdx.x;
  const bool mine = t < a.rows, inside = mine && t < a.starts[a.R];
  int slot = -1;
  if (inside) {
    int lo = 0, hi = a.R - 1;  // the last request that starts at t or below: of those that start there, the one with rows
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.starts[mid] <= t) lo = mid;
      else hi = mid - 1;
    }
    const int start = a.starts[lo], cached = a.kv[lo] - (a.starts[lo + 1] - start);
    const int at = cached + (t - start), nth = at >> a.shift, held = pages_of(cached, a);
    const int page = page_of(a, lo * a.stride, nth, held, a.firsts[lo]), in_page = at & ((1 << a.shift) - 1);
    if (page >= 0) slot = (page << a.shift) + in_page;
    if (nth >= held && nth < a.width && in_page == 0) a.table[lo * a.stride + nth] = page;  // the token that opens the page
  }
  if (mine) a.slots[t] = slot;
  const int lost = __popcll(__builtin_amdgcn_ballot_w64(inside && slot < 0));
  if (lost && (threadIdx.x & 63) == 0) {
    // A sum of whole numbers: the order changes nothing.  It stops at the largest one: of the waves that find it above, each brings it
    // down behind its own addition, and all rows together are fewer than 2^30, so that it stays inside 32 bits meanwhile.
    uint32_t* const count = (uint32_t*)a.counts + 1;
    if (atomicAdd(count, (uint32_t)lost) + (uint32_t)lost > (uint32_t)INT32_MAX) atomicMin(count, (uint32_t)INT32_MAX);
  }
}

// ---- append -------------------------------------------------------------------------------
// A copy of rows to where their slots lie, 16 bytes a thread; bound by HBM (131 MB of bf16 rows read and written in 20.1 us, 6.5 TB/s, the
// inputs in a cache in part), or by latency where rows are few (24 rows 2.4 us).  Neighbouring threads take a head's row
// and then the next head's, so that reads run on; a page keeps heads apart, so that writes run on for a head's row, 128 bytes
// and more.
struct AppendArgs {
  const unsigned char *k, *v;
  unsigned char *kp, *vp;
  const int32_t* slots;
  int64_t k_row, v_row;  // bytes from a row to the next
  int rows, n_slots, shift, heads, per_head;  // per_head: 16-byte pieces of a head's row
};

__global__ __launch_bounds__(256) void append_kernel(const AppendArgs a) {
  const int pieces = a.heads * a.per_head;
  const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t row = item / pieces;
  if (row >= a.rows) return;
  const int piece = (int)(item - row * pieces), head = piece / a.per_head, c = piece - head * a.per_head;
  const int slot = a.slots[row];
  if ((unsigned)slot >= (unsigned)a.n_slots) return;
  const int page = slot >> a.shift, at = slot & ((1 << a.shift) - 1);
  const int64_t to = ((((int64_t)page * a.heads + head) << a.shift) + at) * a.per_head + c;
  const unsigned char* from = blockIdx.y ? a.v + row * a.v_row : a.k + row * a.k_row;
  ((u32x4*)(blockIdx.y ? a.vp : a.kp))[to] = *(const u32x4*)(from + (int64_t)piece * 16);
}

}  // namespace

extern "C" vit_status_t vit_pages_plan(const vit_pages_plan_t* p, void* stream) {
  if (!p) return set_error(VIT_EINVAL, "vit_pages_plan: NULL argument");
  if (p->n_requests < 0 || p->n_requests > 1 << 20 || p->table_width < 0 || p->n_free < 0 || p->n_rows < 0 || p->n_rows >= 1 << 30 ||
      p->table_stride < p->table_width)
    return set_error(VIT_EINVAL, "vit_pages_plan: sizes must not be negative, n_requests <= 2^20, n_rows < 2^30, table_stride >= table_width");
  if (const char* why = bad_pages(p->n_pages, p->page_size)) return set_error(VIT_EINVAL, "vit_pages_plan: %s", why);
  const bool some = p->n_requests > 0;
  if ((some && (!p->cached_lens || !p->new_lens || !p->kv_lens)) || (some && p->table_width > 0 && !p->block_table) ||
      (p->n_free > 0 && !p->free_pages) || (p->n_rows > 0 && !p->slots) || !p->query_offsets || !p->page_offsets || !p->counts)
    return set_error(VIT_EINVAL, "vit_pages_plan: NULL argument");
  PlanArgs a;
  a.cached = p->cached_lens; a.fresh = p->new_lens; a.free = p->free_pages; a.taken = p->taken;
  a.table = p->block_table; a.slots = p->slots; a.starts = p->query_offsets; a.kv = p->kv_lens;
  a.firsts = p->page_offsets; a.counts = p->counts;
  a.stride = p->table_stride; a.R = p->n_requests; a.width = p->table_width; a.n_free = p->n_free; a.n_pages = p->n_pages;
  a.shift = __builtin_ctz(p->page_size); a.rows = p->n_rows;
  hipStream_t s = (hipStream_t)stream;
  const bool in_place = a.kv == a.cached || a.counts == a.taken;
  if (a.R <= PLAN_MANY && (a.rows <= PLAN_ROWS || !in_place)) {
    hipLaunchKernelGGL(plan_kernel, dim3(std::max((a.rows + PLAN_ROWS - 1) / PLAN_ROWS, 1)), dim3(PLAN_THREADS), 0, s, a);
  } else {
    hipLaunchKernelGGL(plan_sums_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, a);
    if (a.rows > 0) hipLaunchKernelGGL(plan_slots_kernel, dim3((a.rows + 255) / 256), dim3(256), 0, s, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(VIT_EDEVICE, "vit_pages_plan: launch: %s", hipGetErrorString(e));
  return VIT_OK;
}

extern "C" vit_status_t vit_pages_append(const vit_pages_append_t* p, void* stream) {
  if (!p) return set_error(VIT_EINVAL, "vit_pages_append: NULL argument");
  if (const char* why = bad_pages(p->n_pages, p->page_size)) return set_error(VIT_EINVAL, "vit_pages_append: %s", why);
  if (const char* why = bad_heads(p->kv_heads, p->head_dim, p->dtype)) return set_error(VIT_EINVAL, "vit_pages_append: %s", why);
  const int es = p->dtype == VIT_DTYPE_FP32 ? 4 : 2, row = p->kv_heads * p->head_dim;
  if (p->n_rows < 0 || p->k_stride < row || p->v_stride < row || p->k_stride > (int64_t)1 << 32 || p->v_stride > (int64_t)1 << 32)
    return set_error(VIT_EINVAL, "vit_pages_append: n_rows must not be negative, strides kv_heads * head_dim to 2^32");
  if (p->n_rows == 0 || p->n_pages == 0) return VIT_OK;
  if (!p->k || !p->v || !p->slots || !p->key_pages || !p->value_pages) return set_error(VIT_EINVAL, "vit_pages_append: NULL argument");
  if ((((uintptr_t)p->k | (uintptr_t)p->v | (uintptr_t)p->key_pages | (uintptr_t)p->value_pages) & 15) || (p->k_stride * es & 15) ||
      (p->v_stride * es & 15))
    return set_error(VIT_EINVAL, "vit_pages_append: pointers and rows must be multiples of 16 bytes");
  AppendArgs a;
  a.k = (const unsigned char*)p->k; a.v = (const unsigned char*)p->v;
  a.kp = (unsigned char*)p->key_pages; a.vp = (unsigned char*)p->value_pages; a.slots = p->slots;
  a.k_row = p->k_stride * es; a.v_row = p->v_stride * es;
  a.rows = p->n_rows; a.n_slots = p->n_pages * p->page_size; a.shift = __builtin_ctz(p->page_size);
  a.heads = p->kv_heads; a.per_head = p->head_dim * es / 16;
  const int64_t groups = ((int64_t)a.rows * a.heads * a.per_head + 255) / 256;
  if (groups >= 1 << 24)  // (a launch has fewer than 2^32 threads)
    return set_error(VIT_EINVAL, "vit_pages_append: rows of k must be below 64 GiB together");
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)groups, 2), dim3(256), 0, (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(VIT_EDEVICE, "vit_pages_append: launch: %s", hipGetErrorString(e));
  return VIT_OK;
}
