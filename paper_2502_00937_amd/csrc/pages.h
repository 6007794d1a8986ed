// What the paged key/value cache's sources share.
#pragma once
#include "../../include/vitenc.h"
#include "common.h"

namespace vitenc {

vit_status_t set_error(vit_status_t st, const char* fmt, ...);  // vitenc_api.hip: message for vit_last_error()

// nullptr, or what is wrong with the sizes of a pool of pages
inline const char* bad_pages(int32_t n_pages, int32_t page_size) {
  if (page_size < 8 || page_size > 4096 || (page_size & (page_size - 1))) return "page_size must be a power of two, 8 to 4096";
  if (n_pages < 0 || (int64_t)n_pages * page_size > INT32_MAX) return "n_pages must not be negative, n_pages * page_size below 2^31";
  return nullptr;
}

inline const char* bad_heads(int32_t kv_heads, int32_t head_dim, int32_t dtype) {
  if (kv_heads <= 0 || kv_heads > 1024) return "kv_heads must be 1 to 1024";
  if (head_dim <= 0 || head_dim % 8 != 0 || head_dim > 128) return "head_dim must be a multiple of 8, at most 128";
  if (dtype != VIT_DTYPE_FP32 && dtype != VIT_DTYPE_BF16) return "dtype must be VIT_DTYPE_FP32 or VIT_DTYPE_BF16";
  return nullptr;
}

// Sums over the lanes up to and with this one, by the vector unit's lane moves (through LDS each of the six steps costs a hundred
// clocks).  Saturating in 32 bits; whole in 64.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lane_move(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v = __builtin_elementwise_add_sat(v, lane_move<0x111, 0xF>(v));  // rows of 16 lanes: 1, 2, 4 and 8 to the right
  v = __builtin_elementwise_add_sat(v, lane_move<0x112, 0xF>(v));
  v = __builtin_elementwise_add_sat(v, lane_move<0x114, 0xF>(v));
  v = __builtin_elementwise_add_sat(v, lane_move<0x118, 0xF>(v));
  v = __builtin_elementwise_add_sat(v, lane_move<0x142, 0xA>(v));  // a row's last lane to the second and fourth row
  v = __builtin_elementwise_add_sat(v, lane_move<0x143, 0xC>(v));  // the second row's to the third and fourth
  return v;
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t lane_move(uint64_t v) {
  return (uint64_t)lane_move<CTRL, ROWS>((uint32_t)v) | (uint64_t)lane_move<CTRL, ROWS>((uint32_t)(v >> 32)) << 32;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {
  v += lane_move<0x111, 0xF>(v);
  v += lane_move<0x112, 0xF>(v);
  v += lane_move<0x114, 0xF>(v);
  v += lane_move<0x118, 0xF>(v);
  v += lane_move<0x142, 0xA>(v);
  v += lane_move<0x143, 0xC>(v);
  return v;
}

}  // namespace vitenc
