"""The paged key/value cache that pulled image tokens and the text around them lie in, as torch tensors.

A layer's cache is two pools `[n_pages, kv_heads, page_size, head_dim]`, bf16 or fp32, that the caller owns; a request's row of
the block table names its pages in order.  `plan_pages` gives a step's new tokens their pages and slots (once a step, for
all layers), `append_pages` writes their keys and values, `attend_pages` lets their queries attend to the cache.  Every call is
queued on the current stream of the tensors' device, waits for nothing and may be captured into a graph.
"""
from __future__ import annotations

import ctypes as C
import struct
from typing import NamedTuple

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


def _int32(name, t, dims, device):
    import torch

    if t.dtype is not torch.int32 or t.dim() != dims or t.device != device or (
            t.numel() and not (t.is_contiguous() or (dims == 2 and t.stride(1) == 1))):
        _refuse(f"{name} must be an int32 tensor of {dims} dimensions, contiguous, on {device}")


def _pools(key_pages, value_pages):
    import torch

    if key_pages.dtype not in (torch.bfloat16, torch.float32) or key_pages.dim() != 4 or not key_pages.is_contiguous():
        _refuse("key_pages must be a contiguous bf16 or fp32 tensor [n_pages, kv_heads, page_size, head_dim]")
    if (value_pages.dtype is not key_pages.dtype or value_pages.shape != key_pages.shape or value_pages.device != key_pages.device or
            not value_pages.is_contiguous()):
        _refuse("value_pages must be as key_pages is")
    return VIT_DTYPE_BF16 if key_pages.dtype is torch.bfloat16 else VIT_DTYPE_FP32


def _rows(name, t, like, heads, dim):
    """Elements from a row of `t`, [rows, heads, dim] with a row's heads next to each other, to the next."""
    if t.dim() != 3 or t.dtype is not like.dtype or t.device != like.device:
        _refuse(f"{name} must be a tensor [rows, heads, head_dim] of the pools' dtype and device")
    n, h, d = t.shape
    if (heads is not None and h != heads) or d != dim:
        _refuse(f"{name} is {tuple(t.shape)} where the pools ask for {heads or 'any number of'} heads of {dim}")
    row, head, one = t.stride()
    if (d > 1 and one != 1) or (h > 1 and head != d):
        _refuse(f"{name}'s heads must lie next to each other in a row")
    return row if n > 1 else max(row, h * d)


def _call(function, packed: bytes, device) -> None:
    import torch

    index = device.index
    if device.type != "cuda":
        _refuse("the tensors must be on a GPU")
    if index == torch.cuda.current_device():
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _check(function(packed, raw(index) if raw else torch.cuda.current_stream().cuda_stream))
    else:
        with torch.cuda.device(device):
            _check(function(packed, torch.cuda.current_stream().cuda_stream))


def plan_pages(cached_lens, new_lens, block_table, free_pages, taken, n_pages: int, page_size: int, n_rows: int, out=None) -> PagePlan:
    """Pages and slots of a step's tokens: see `vit_pages_plan`.  `cached_lens`, `new_lens` int32 [n_requests], `block_table` int32
    [n_requests, width] (the pages taken are entered), `free_pages` int32 [n], `taken` int32 [1] or more or None, all on one
    GPU.  `out`: a plan of the same sizes to write into, whose `kv_lens` may be `cached_lens` and `counts` `taken`."""
    import torch

    device = cached_lens.device
    _int32("cached_lens", cached_lens, 1, device)
    _int32("new_lens", new_lens, 1, device)
    _int32("block_table", block_table, 2, device)
    _int32("free_pages", free_pages, 1, device)
    if taken is not None:
        _int32("taken", taken, 1, device)
        if taken.numel() < 1:
            _refuse("taken must hold a number")
    n, width = block_table.shape
    if new_lens.numel() != n or cached_lens.numel() != n:
        _refuse(f"cached_lens, new_lens and block_table are of {cached_lens.numel()}, {new_lens.numel()} and {n} requests")
    if not 0 <= n_rows < 1 << 30:
        _refuse("n_rows must be 0 to 2^30 - 1")
    sizes = (n_rows, n + 1, n, n + 1, 2)
    if out is None:
        out = PagePlan(*torch.empty(n_rows + 3 * n + 4, dtype=torch.int32, device=device).split_with_sizes(sizes))
    else:
        for name, t, size in zip(PagePlan._fields, out, sizes):
            _int32(name, t, 1, device)
            if t.numel() != size:
                _refuse(f"the plan's {name} holds {t.numel()} numbers, {size} needed")
    _call(load_library().vit_pages_plan,
          _PLAN.pack(cached_lens.data_ptr(), new_lens.data_ptr(), block_table.data_ptr(), free_pages.data_ptr(),
                     0 if taken is None else taken.data_ptr(), out[0].data_ptr(), out[1].data_ptr(), out[2].data_ptr(),
                     out[3].data_ptr(), out[4].data_ptr(), block_table.stride(0) if n > 1 else width, n, width,
                     free_pages.numel(), n_pages, page_size, n_rows), device)
    return out


def append_pages(k, v, slots, key_pages, value_pages) -> None:
    """Rows of `k` and `v` ([rows, kv_heads, head_dim], a view of a fused product's rows for example) to their `slots` (int32
    [rows], -1: passed over) of the pools: see `vit_pages_append`."""
    dtype = _pools(key_pages, value_pages)
    n_pages, heads, page_size, dim = key_pages.shape
    k_row, v_row = _rows("k", k, key_pages, heads, dim), _rows("v", v, key_pages, heads, dim)
    _int32("slots", slots, 1, key_pages.device)
    n = slots.numel()
    if k.shape[0] != n or v.shape[0] != n:
        _refuse(f"k, v and slots have {k.shape[0]}, {v.shape[0]} and {n} rows")
    _call(load_library().vit_pages_append,
          _APPEND.pack(k.data_ptr(), v.data_ptr(), slots.data_ptr(), key_pages.data_ptr(), value_pages.data_ptr(), k_row, v_row, n,
                       n_pages, page_size, heads, dim, dtype), key_pages.device)


def attend_pages(q, key_pages, value_pages, block_table, query_offsets, kv_lens, max_new: int, causal: bool = True, scale=None, out=None):
    """Attention of the rows of `q` ([rows, q_heads, head_dim]) over their requests' keys and values in the pools: see
    `vit_pages_attend`.  `scale` is 1 / sqrt(head_dim) if not given.  Returns `out`, [rows, q_heads, head_dim]."""
    import torch

    dtype = _pools(key_pages, value_pages)
    n_pages, kv_heads, page_size, dim = key_pages.shape
    device = key_pages.device
    q_row = _rows("q", q, key_pages, None, dim)
    n, heads, _ = q.shape
    _int32("block_table", block_table, 2, device)
    _int32("query_offsets", query_offsets, 1, device)
    _int32("kv_lens", kv_lens, 1, device)
    requests, width = block_table.shape
    if query_offsets.numel() != requests + 1 or kv_lens.numel() != requests:
        _refuse(f"query_offsets, kv_lens and block_table are of {query_offsets.numel() - 1}, {kv_lens.numel()} and {requests} requests")
    if out is None:
        out = torch.empty((n, heads, dim), dtype=q.dtype, device=device)
        out_row = heads * dim
    else:
        out_row = _rows("out", out, key_pages, heads, dim)
        if out.shape[0] != n:
            _refuse(f"out has {out.shape[0]} rows, q {n}")
    fields = [q.data_ptr(), key_pages.data_ptr(), value_pages.data_ptr(), block_table.data_ptr(), query_offsets.data_ptr(),
              kv_lens.data_ptr(), out.data_ptr(), 0, 0, q_row, out_row, block_table.stride(0) if requests > 1 else width, n, requests,
              max_new, width, n_pages, page_size, heads, kv_heads, dim, 1 if causal else 0, dtype,
              dim ** -0.5 if scale is None else scale]
    lib, need = load_library(), C.c_size_t()
    packed = _ATTEND.pack(*fields)
    _check(lib.vit_pages_attend_query(packed, C.byref(need)))
    if need.value:
        # from torch's allocator, call by call: another stream's or graph's calls have workspaces of their own
        workspace = torch.empty(need.value, dtype=torch.uint8, device=device)
        fields[7], fields[8] = workspace.data_ptr(), need.value
        packed = _ATTEND.pack(*fields)
    _call(lib.vit_pages_attend, packed, device)
    return out
