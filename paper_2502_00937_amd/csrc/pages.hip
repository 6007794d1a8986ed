// The paged key/value cache: which pages and slots a step's tokens take (plan), and their keys and values into them (append).
#include "pages.h"

using namespace vitenc;

namespace {

// ---- plan ---------------------------------------------------------------------------------
// Request r's new tokens i = 0 ... new - 1 are at = cached + i of it, in its page nth = at / page_size.  The first
// held = ceil(cached / page_size) pages are in its row of the block table; the others are the free list's entries
// first + nth - held, where `first` is *taken plus the pages that the requests before it take: a prefix sum, like the rows'.
//
// Nothing here but latencies: the sums over the requests are one workgroup's, in 64 bits (lengths may add up past 32), and
// the tokens' slots follow from them token by token.
struct PlanArgs {
  const int32_t *cached, *fresh, *free, *taken;
  int32_t *table, *slots, *starts, *kv, *firsts, *counts;
  int64_t stride;
  int R, width, n_free, n_pages, shift, rows;
};

constexpr int PLAN_THREADS = 1024;
constexpr int MAX_LEN = 1 << 30;

// Sum of `v` over the threads below this one; *total over all of them.  `waves`: one word of LDS a wave.
__device__ int64_t scan_below(int64_t v, int64_t* waves, int64_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t sum = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t up = __shfl_up(sum, d, 64);
    if (lane >= d) sum += up;
  }
  if (lane == 63) waves[wave] = sum;
  __syncthreads();
  int64_t below = 0, all = 0;
#pragma unroll
  for (int w = 0; w < PLAN_THREADS / 64; ++w) {
    if (w < wave) below += waves[w];
    all += waves[w];
  }
  __syncthreads();
  *total = all;
  return below + sum - v;
}

__device__ __forceinline__ int pages_of(int tokens, const PlanArgs& a) {  // that the table has room for
  return min((int)(((int64_t)tokens + (1 << a.shift) - 1) >> a.shift), a.width);
}

__global__ __launch_bounds__(PLAN_THREADS) void plan_sums_kernel(const PlanArgs a) {
  __shared__ int64_t waves[PLAN_THREADS / 64];
  const int64_t taken = a.taken ? max(*a.taken, 0) : 0;
  int64_t row = 0, first = taken;
  for (int base = 0; base < a.R; base += PLAN_THREADS) {
    const int r = base + threadIdx.x;
    const bool mine = r < a.R;
    const int cached = mine ? min(max(a.cached[r], 0), MAX_LEN) : 0;
    const int64_t asked = mine ? min(max(a.fresh[r], 0), MAX_LEN) : 0;
    int64_t all_rows, all_pages;
    const int64_t at = row + scan_below(asked, waves, &all_rows);
    const int start = (int)min(at, (int64_t)a.rows), end = (int)min(at + asked, (int64_t)a.rows);
    const int total = cached + (end - start);
    const int64_t page = first + scan_below(pages_of(total, a) - pages_of(cached, a), waves, &all_pages);
    if (mine) {
      a.starts[r] = start;
      a.kv[r] = total;
      a.firsts[r] = (int32_t)min(page, (int64_t)INT32_MAX);
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
    if (nth < a.width) {
      int32_t* entry = a.table + (int64_t)lo * a.stride + nth;
      int page;
      if (nth < held) {
        page = *entry;
      } else {
        const int64_t index = (int64_t)a.firsts[lo] + (nth - held);
        page = index < a.n_free ? a.free[index] : -1;
        if ((unsigned)page >= (unsigned)a.n_pages) page = -1;
        if ((at & ((1 << a.shift) - 1)) == 0) *entry = page;  // the token that opens the page
      }
      if ((unsigned)page < (unsigned)a.n_pages) slot = (page << a.shift) + (at & ((1 << a.shift) - 1));
    }
  }
  if (mine) a.slots[t] = slot;
  const int lost = __popcll(__builtin_amdgcn_ballot_w64(inside && slot < 0));
  if (lost && (threadIdx.x & 63) == 0) atomicAdd(a.counts + 1, lost);  // (a sum of whole numbers: the order changes nothing)
}

// ---- append -------------------------------------------------------------------------------
// A copy of rows to where their slots lie, 16 bytes a thread; bound by HBM, or by latency where rows are few.
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
  hipLaunchKernelGGL(plan_sums_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, a);
  if (a.rows > 0) hipLaunchKernelGGL(plan_slots_kernel, dim3((a.rows + 255) / 256), dim3(256), 0, s, a);
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
  if (groups > INT32_MAX) return set_error(VIT_EINVAL, "vit_pages_append: too many rows");
  hipLaunchKernelGGL(append_kernel, dim3((unsigned)groups, 2), dim3(256), 0, (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(VIT_EDEVICE, "vit_pages_append: launch: %s", hipGetErrorString(e));
  return VIT_OK;
}
