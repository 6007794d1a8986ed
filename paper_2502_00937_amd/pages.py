"""The paged key/value cache that pulled image tokens and the text around them lie in, as torch tensors.

A layer's cache is two pools `[n_pages, kv_heads, page_size, head_dim]`, bf16 or fp32, that the caller owns; a request's row of
the block table names its pages in order.  `plan_pages` gives a step's new tokens their pages and slots (once a step, for
all layers), `append_pages` writes their keys and values, `attend_pages` lets their queries attend to the cache.  Every call is
queued on the current stream of the tensors' device, waits for nothing and may be captured into a graph.  The calls are for serving:
tensors that require a gradient are taken for their numbers alone, results carry no graph, and what is written (pools, tables,
`out`) is written without autograd's knowledge.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import NamedTuple

import torch

from .binding import VIT_DTYPE_BF16, VIT_DTYPE_FP32, VIT_EINVAL, VitError, _check, load_library

# the structs of include/vitenc.h, field by field
_PLAN = struct.Struct("10Qq6i")
_APPEND = struct.Struct("5Q2q6i")
_ATTEND = struct.Struct("8QQ3q11if")


class PagePlan(NamedTuple):
    """What `vit_pages_plan` writes (int32, on the GPU)."""
    slots: object          # [n_rows] slot of each row's token, -1: none
    query_offsets: object  # [n_requests + 1] first row of each request
    kv_lens: object        # [n_requests] tokens in the cache once the step's are
    page_offsets: object   # [n_requests + 1] first entry of the free list that each request takes
    counts: object         # [2] entries of the free list that are taken now; new tokens without a slot


def _refuse(why: str):
    raise VitError(VIT_EINVAL, why)


# A call of a few microseconds is as long as its checks: devices are compared by their number (`get_device`), shapes are
# read once, and the results of a plan share one allocation.
def _vector(name, t, device):
    """Checks an int32 vector on `device`; returns its length."""
    if t.dtype is not torch.int32 or t.dim() != 1 or t.get_device() != device or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous int32 vector on the other tensors' device")
    return t.numel()


def _table(t, device):
    """Checks a block table on `device`; returns (requests, width, entries from a row to the next)."""
    if t.dtype is not torch.int32 or t.dim() != 2 or t.get_device() != device:
        _refuse("block_table must be an int32 tensor [requests, width] on the other tensors' device")
    n, width = t.shape
    row, one = t.stride()
    if one != 1 and width > 1 and n:
        _refuse("block_table's rows must be contiguous")
    return n, width, row if n > 1 and width else width


def _pools(key_pages, value_pages):
    """Checks two pools; returns (VIT_DTYPE_*, device, pages, heads, page size, head dim)."""
    dt, shape, device = key_pages.dtype, key_pages.shape, key_pages.get_device()
    if dt not in (torch.bfloat16, torch.float32) or len(shape) != 4 or not key_pages.is_contiguous():
        _refuse("key_pages must be a contiguous bf16 or fp32 tensor [n_pages, kv_heads, page_size, head_dim]")
    if value_pages.dtype is not dt or value_pages.shape != shape or value_pages.get_device() != device or not value_pages.is_contiguous():
        _refuse("value_pages must be as key_pages is")
    return (VIT_DTYPE_BF16 if dt is torch.bfloat16 else VIT_DTYPE_FP32, device, *shape)


def _rows(name, t, dtype, device, dim, heads=None):
    """Checks `t`, [rows, heads, dim] with a row's heads next to each other; returns (rows, heads, elements from a row to the next)."""
    if t.dim() != 3 or t.dtype is not dtype or t.get_device() != device:
        _refuse(f"{name} must be a tensor [rows, heads, head_dim] of the pools' dtype and device")
    n, h, d = t.shape
    if (heads is not None and h != heads) or d != dim:
        _refuse(f"{name} is {tuple(t.shape)} where the pools ask for {heads or 'any number of'} heads of {dim}")
    row, head, one = t.stride()
    if (one != 1 and d > 1) or (head != d and h > 1):
        _refuse(f"{name}'s heads must lie next to each other in a row")
    return n, h, row if n > 1 else max(row, h * d)


def _pack(layout: struct.Struct, *fields) -> bytes:
    try:
        return layout.pack(*fields)
    except (struct.error, OverflowError) as e:  # a number that its field does not hold, or none at all
        _refuse(f"argument out of range: {e}")


def _call(function, packed: bytes, device: int) -> None:
    if device < 0:
        _refuse("the tensors must be on a GPU")
    if device == torch._C._cuda_getDevice():
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _check(function(packed, raw(device) if raw else torch.cuda.current_stream().cuda_stream))
    else:
        with torch.cuda.device(device):
            _check(function(packed, torch.cuda.current_stream().cuda_stream))


def plan_pages(cached_lens, new_lens, block_table, free_pages, taken, n_pages: int, page_size: int, n_rows: int, out=None) -> PagePlan:
    """Pages and slots of a step's tokens: see `vit_pages_plan`.  `cached_lens`, `new_lens` int32 [n_requests], `block_table` int32
    [n_requests, width] (the pages taken are entered), `free_pages` int32 [n], `taken` int32 [1] or more or None, all on one
    GPU.  `out`: a plan of the same sizes to write into, whose `kv_lens` may be `cached_lens` and `counts` `taken`."""
    device = cached_lens.get_device()
    n, width, stride = _table(block_table, device)
    if _vector("cached_lens", cached_lens, device) != n or _vector("new_lens", new_lens, device) != n:
        _refuse(f"cached_lens, new_lens and block_table are of {cached_lens.numel()}, {new_lens.numel()} and {n} requests")
    n_free = _vector("free_pages", free_pages, device)
    if taken is not None and _vector("taken", taken, device) < 1:
        _refuse("taken must hold a number")
    if not 0 <= n_rows < 1 << 30:
        _refuse("n_rows must be 0 to 2^30 - 1")
    sizes = (n_rows, n + 1, n, n + 1, 2)
    if out is None:
        both = cached_lens.new_empty(n_rows + 3 * n + 4)
        at = both.data_ptr()
        places = (at, at + 4 * n_rows, at + 4 * (n_rows + n + 1), at + 4 * (n_rows + 2 * n + 1), at + 4 * (n_rows + 3 * n + 2))
        out = PagePlan._make(both.split_with_sizes(sizes))
    else:
        for name, t, size in zip(PagePlan._fields, out, sizes):
            if _vector(name, t, device) != size:
                _refuse(f"the plan's {name} holds {t.numel()} numbers, {size} needed")
        places = tuple(t.data_ptr() for t in out)
    _call(load_library().vit_pages_plan,
          _pack(_PLAN, cached_lens.data_ptr(), new_lens.data_ptr(), block_table.data_ptr(), free_pages.data_ptr(),
                     0 if taken is None else taken.data_ptr(), *places, stride, n, width, n_free, n_pages, page_size, n_rows), device)
    return out


def append_pages(k, v, slots, key_pages, value_pages) -> None:
    """Rows of `k` and `v` ([rows, kv_heads, head_dim], a view of a fused product's rows for example) to their `slots` (int32
    [rows], -1: passed over) of the pools: see `vit_pages_append`."""
    dtype, device, n_pages, heads, page_size, dim = _pools(key_pages, value_pages)
    n, _, k_row = _rows("k", k, key_pages.dtype, device, dim, heads)
    n_v, _, v_row = _rows("v", v, key_pages.dtype, device, dim, heads)
    if not n == n_v == _vector("slots", slots, device):
        _refuse(f"k, v and slots have {n}, {n_v} and {slots.numel()} rows")
    _call(load_library().vit_pages_append,
          _pack(_APPEND, k.data_ptr(), v.data_ptr(), slots.data_ptr(), key_pages.data_ptr(), value_pages.data_ptr(), k_row, v_row, n,
                       n_pages, page_size, heads, dim, dtype), device)


def attend_pages(q, key_pages, value_pages, block_table, query_offsets, kv_lens, max_new: int, causal: bool = True, scale=None, out=None):
    """Attention of the rows of `q` ([rows, q_heads, head_dim]) over their requests' keys and values in the pools: see
    `vit_pages_attend`.  `scale` is 1 / sqrt(head_dim) if not given.  Returns `out`, [rows, q_heads, head_dim]; no gradient
    passes through it."""
    dtype, device, n_pages, kv_heads, page_size, dim = _pools(key_pages, value_pages)
    n, heads, q_row = _rows("q", q, key_pages.dtype, device, dim)
    requests, width, stride = _table(block_table, device)
    if _vector("query_offsets", query_offsets, device) != requests + 1 or _vector("kv_lens", kv_lens, device) != requests:
        _refuse(f"query_offsets, kv_lens and block_table are of {query_offsets.numel() - 1}, {kv_lens.numel()} and {requests} requests")
    if out is None:
        out, out_row = q.new_empty((n, heads, dim)), heads * dim
    else:
        out_n, _, out_row = _rows("out", out, key_pages.dtype, device, dim, heads)
        if out_n != n:
            _refuse(f"out has {out_n} rows, q {n}")
    lib, need = load_library(), C.c_size_t()
    pointers = (q.data_ptr(), key_pages.data_ptr(), value_pages.data_ptr(), block_table.data_ptr(), query_offsets.data_ptr(),
                kv_lens.data_ptr(), out.data_ptr())
    sizes = (q_row, out_row, stride, n, requests, max_new, width, n_pages, page_size, heads, kv_heads, dim, 1 if causal else 0, dtype,
             dim ** -0.5 if scale is None else scale)
    _check(lib.vit_pages_attend_query(_pack(_ATTEND, *pointers, 0, 0, *sizes), C.byref(need)))
    bytes_needed = need.value
    # from torch's allocator, call by call: another stream's or graph's calls have workspaces of their own
    workspace = query_offsets.new_empty(bytes_needed // 4) if bytes_needed else None
    _call(lib.vit_pages_attend, _pack(_ATTEND, *pointers, workspace.data_ptr() if bytes_needed else 0, bytes_needed, *sizes), device)
    return out
