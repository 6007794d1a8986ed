// Attention of new tokens over a paged cache, softmax(scale q k^T) v per row and head.
#include <cmath>

#include "pages.h"

using namespace vitenc;

namespace {

struct PagedArgs {
  const void *q, *kp, *vp;
  void* out;
  const int32_t *table, *starts, *kv;
  int64_t q_stride, out_stride, table_stride;
  int rows, R, max_new, width, n_pages, shift, heads, kv_heads, dh, causal;
  float scale;
};

// A workgroup of one wave a (row, head).  Each lane takes the logits of every 64th key with the online softmax's
// running maximum; the lanes' weights then multiply the values, a lane for every 64th column.
template <typename T>
__global__ __launch_bounds__(64) void paged_attention_simple_kernel(const PagedArgs a) {
  const int t = blockIdx.x, head = blockIdx.y, lane = threadIdx.x;
  if (t >= a.starts[a.R]) return;
  int lo = 0, hi = a.R - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.starts[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  const int start = a.starts[lo], fresh = a.starts[lo + 1] - start;
  if (t < start || t - start >= min(fresh, a.max_new)) return;
  const int kv = max(a.kv[lo], 0), all = (int)min((int64_t)kv, (int64_t)a.width << a.shift);
  const int keys = a.causal ? min(all, kv - fresh + (t - start) + 1) : all;
  const T* q = (const T*)a.q + (int64_t)t * a.q_stride + head * a.dh;
  const int kv_head = head / (a.heads / a.kv_heads), mask = (1 << a.shift) - 1;
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  for (int k0 = 0; k0 < keys; k0 += 64) {
    const int key = k0 + lane;
    int page = -1;
    float logit = -INFINITY;
    if (key < keys) page = a.table[(int64_t)lo * a.table_stride + (key >> a.shift)];
    if ((unsigned)page >= (unsigned)a.n_pages) page = -1;
    const int64_t at = ((((int64_t)page * a.kv_heads + kv_head) << a.shift) + (key & mask)) * a.dh;
    if (page >= 0) {
      logit = 0.f;
      for (int d = 0; d < a.dh; ++d) logit = fmaf(Elem<T>::load(q + d), Elem<T>::load((const T*)a.kp + at + d), logit);
      logit *= a.scale;
    }
    float up = logit;
    for (int d = 32; d; d >>= 1) up = fmaxf(up, __shfl_xor(up, d, 64));
    up = fmaxf(up, m);
    if (up == -INFINITY && !__any(page >= 0)) continue;
    const float shrink = m == -INFINITY ? 0.f : expf(m - up), w = page >= 0 ? expf(logit - up) : 0.f;
    float sum = w;
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d, 64);
    l = l * shrink + sum;
    o0 *= shrink;
    o1 *= shrink;
    m = up;
    for (int j = 0; j < 64; ++j) {
      if (__shfl(page, j, 64) < 0) continue;
      const int64_t base = __shfl(at, j, 64);
      const float wj = __shfl(w, j, 64);
      if (lane < a.dh) o0 = fmaf(wj, Elem<T>::load((const T*)a.vp + base + lane), o0);
      if (lane + 64 < a.dh) o1 = fmaf(wj, Elem<T>::load((const T*)a.vp + base + lane + 64), o1);
    }
  }
  T* out = (T*)a.out + (int64_t)t * a.out_stride + head * a.dh;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (lane < a.dh) Elem<T>::store(out + lane, o0 * inv);
  if (lane + 64 < a.dh) Elem<T>::store(out + lane + 64, o1 * inv);
}

vit_status_t check_sizes(const vit_pages_attend_t* p, const char* name) {
  if (const char* why = bad_pages(p->n_pages, p->page_size)) return set_error(VIT_EINVAL, "%s: %s", name, why);
  if (const char* why = bad_heads(p->kv_heads, p->head_dim, p->dtype)) return set_error(VIT_EINVAL, "%s: %s", name, why);
  if (p->q_heads <= 0 || p->q_heads > 1024 || p->q_heads % p->kv_heads != 0)
    return set_error(VIT_EINVAL, "%s: q_heads must be a multiple of kv_heads, at most 1024", name);
  if (p->n_rows < 0 || p->n_rows >= 1 << 30 || p->n_requests < 0 || p->n_requests > 1 << 20 || p->max_new < 0 || p->table_width < 0)
    return set_error(VIT_EINVAL, "%s: sizes must not be negative, n_rows < 2^30, n_requests <= 2^20", name);
  return VIT_OK;
}

}  // namespace

extern "C" vit_status_t vit_pages_attend_query(const vit_pages_attend_t* p, size_t* workspace_bytes) {
  if (!p || !workspace_bytes) return set_error(VIT_EINVAL, "vit_pages_attend_query: NULL argument");
  if (vit_status_t st = check_sizes(p, "vit_pages_attend_query"); st != VIT_OK) return st;
  *workspace_bytes = 0;
  return VIT_OK;
}

extern "C" vit_status_t vit_pages_attend(const vit_pages_attend_t* p, void* stream) {
  if (!p) return set_error(VIT_EINVAL, "vit_pages_attend: NULL argument");
  if (vit_status_t st = check_sizes(p, "vit_pages_attend"); st != VIT_OK) return st;
  const int es = p->dtype == VIT_DTYPE_FP32 ? 4 : 2, row = p->q_heads * p->head_dim;
  if (p->q_stride < row || p->out_stride < row || p->q_stride > (int64_t)1 << 32 || p->out_stride > (int64_t)1 << 32 ||
      p->table_stride < p->table_width || !std::isfinite(p->scale))
    return set_error(VIT_EINVAL, "vit_pages_attend: strides of q and out must be q_heads * head_dim to 2^32, table_stride >= table_width, "
                                 "scale finite");
  if (p->n_rows == 0 || p->n_requests == 0 || p->max_new == 0) return VIT_OK;
  if (!p->q || !p->out || !p->query_offsets || !p->kv_lens || (p->table_width > 0 && !p->block_table) ||
      (p->n_pages > 0 && (!p->key_pages || !p->value_pages)))
    return set_error(VIT_EINVAL, "vit_pages_attend: NULL argument");
  if ((((uintptr_t)p->q | (uintptr_t)p->out | (uintptr_t)p->key_pages | (uintptr_t)p->value_pages) & 15) || (p->q_stride * es & 15) ||
      (p->out_stride * es & 15) || ((uintptr_t)p->workspace & 255))
    return set_error(VIT_EINVAL, "vit_pages_attend: pointers and rows must be multiples of 16 bytes, the workspace 256-byte aligned");
  PagedArgs a;
  a.q = p->q; a.kp = p->key_pages; a.vp = p->value_pages; a.out = p->out;
  a.table = p->block_table; a.starts = p->query_offsets; a.kv = p->kv_lens;
  a.q_stride = p->q_stride; a.out_stride = p->out_stride; a.table_stride = p->table_stride;
  a.rows = p->n_rows; a.R = p->n_requests; a.max_new = p->max_new; a.width = p->table_width; a.n_pages = p->n_pages;
  a.shift = __builtin_ctz(p->page_size); a.heads = p->q_heads; a.kv_heads = p->kv_heads; a.dh = p->head_dim;
  a.causal = p->causal != 0; a.scale = p->scale;
  const dim3 grid(a.rows, a.heads);
  if (p->dtype == VIT_DTYPE_FP32) hipLaunchKernelGGL(paged_attention_simple_kernel<float>, grid, dim3(64), 0, (hipStream_t)stream, a);
  else hipLaunchKernelGGL(paged_attention_simple_kernel<bf16_t>, grid, dim3(64), 0, (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return set_error(VIT_EDEVICE, "vit_pages_attend: launch: %s", hipGetErrorString(e));
  return VIT_OK;
}
