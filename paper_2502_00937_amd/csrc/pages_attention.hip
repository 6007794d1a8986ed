// Attention of new tokens over a paged cache: softmax(scale q k^T) v per row and head, the keys and values of a request
// spread over pages.
//
// The rows of a request that read the same keys are one operand: with `group` = q_heads / kv_heads query heads to a head of
// keys, row m of (request, head of keys) is head m % group of token m / group.  As in the encoder's attention everything is
// computed transposed, so that a lane owns one row for the whole kernel:
//   S^T[key, row] = K . Q^T          (K's tile from LDS, Q^T in registers)
//   O^T[d, row]  += V^T . P^T        (V^T from V's tile in LDS, P^T straight from the registers of S^T)
// in blocks of 32 keys x 32 rows: in bf16 on 32 x 32 x 16 matrix instructions, V^T by the transposing LDS read, in fp32 on
// 32 x 32 x 2 ones.
//
// Two forms.  WIDE: 128 rows a workgroup, 32 a wave, which share tiles of keys.  NARROW, where no request has more than 32
// rows (single tokens): the waves share the rows and each has keys of its own, so that four times as many loads are on
// their way and no barrier stands between them; their results are joined in LDS.
//
// Work is divided on the device, where the lengths are: every workgroup adds up the key tiles of all requests, which gives
// the share of a request's keys that one workgroup takes (all of them, where there are rows enough), and finds its own
// place in that order.  A request whose keys are divided leaves parts (sums without division, their reference maximum and
// sum of weights) in the workspace, which a second kernel joins, always in the same order.
//
// Keys and values go from their pages to LDS without passing registers (global_load_lds_dwordx4: 1 KiB of LDS a wave and
// instruction, each lane naming its 16 bytes).  Eight consecutive keys lie in one page, so that pages are looked up by
// scalar loads; LDS rows are swizzled by choosing which 16 bytes of its row a lane fetches.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "pages.h"

using namespace vitenc;

namespace {

struct PagedArgs {
  const void *q, *kp, *vp;
  void* out;
  const int32_t *table, *starts, *kv;
  // workspace, all nullptr if no request's keys are divided: (first part, parts) of every request, reference maximum and
  // sum of every part's rows, their unnormalised values
  int32_t* head;
  float *stats, *parts;
  int64_t max_parts;
  int64_t q_stride, out_stride, table_stride;
  int rows, R, max_new, width, n_pages, shift, heads, kv_heads, group, dh, causal;
  int target;    // workgroups to divide the keys for, 0: not at all
  int least;     // key tiles that are not divided further
  int part_rows; // rows of a part
  float scale;   // >= 0, times log2(e)
  int negative;  // the scale's sign, which goes to the queries
};

typedef const __attribute__((address_space(4))) int32_t* ScalarTable;  // read by scalar loads

constexpr int THREADS = 256;

template <typename T, int DB_, bool NARROW>
struct Shape {
  static constexpr int DB = DB_;                             // blocks of 32 columns
  static constexpr int ES = (int)sizeof(T);
  static constexpr int ROWB = DB * 32 * ES <= 128 ? 128 : DB * 32 * ES <= 256 ? 256 : 512;  // bytes of a row in LDS
  static constexpr int CPR = ROWB / 16, RPI = 64 / CPR;      // 16-byte pieces of a row; rows that a load instruction fills
  static constexpr int KS = DB * 32 * ES / 32;               // pairs of pieces that the first product runs over
  static constexpr int TK = ES == 2 ? 64 : 32;               // WIDE: keys of a tile
  static constexpr int KEYS = NARROW ? 32 : TK;              // keys that a wave works on at a time
  static constexpr int LOAD = NARROW ? 32 : TK / 4;          // of them, keys that it loads
  static constexpr int INSTR = LOAD / RPI;                   // load instructions for K, and for V
  static constexpr int PAGES = LOAD / 8;                     // pages it looks up
  static constexpr int STAGE = KEYS * ROWB * 2;              // bytes of LDS of a stage
  static constexpr int NS = NARROW && 8 * STAGE > 131072 ? 1 : 2;
  static constexpr int LDS = (NARROW ? 4 : 1) * NS * STAGE;
  static constexpr int ITEM_ROWS = NARROW ? 32 : 128;
  static constexpr int ITEM_KEYS = NARROW ? 128 : TK;        // keys of a step of the whole workgroup
};

// ---- a workgroup's place ------------------------------------------------------------------
struct Item {
  int r, tile, split, splits, part;  // request; which of its row tiles, which part of its keys and of how many; first part's place
  int start, fresh, kv, rows;        // its first row, rows, keys; rows of (request, head of keys)
};

struct Request {
  int start, fresh, kv, tiles, steps;
};

template <int ROWS, int KEYS>
__device__ __forceinline__ Request request(const PagedArgs& a, int r) {
  Request q{0, 0, 0, 0, 0};
  if (r < a.R) {
    q.start = a.starts[r];
    const int64_t n = (int64_t)a.starts[r + 1] - q.start;
    q.fresh = q.start < 0 || n < 0 || q.start + n > a.rows ? 0 : (int)n;
    q.kv = max(a.kv[r], 0);
    q.tiles = (int)(((int64_t)min(q.fresh, a.max_new) * a.group + ROWS - 1) / ROWS);
    q.steps = (int)((min((int64_t)q.kv, (int64_t)a.width << a.shift) + KEYS - 1) / KEYS);
  }
  return q;
}

__device__ __forceinline__ int64_t wave_scan(int64_t v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t up = __shfl_up(v, d, 64);
    if (lane >= d) v += up;
  }
  return v;
}

// Workgroup `at` of a head of keys, in the order of the requests; false if there are not so many.
template <int ROWS, int KEYS>
__device__ __forceinline__ bool find_item(const PagedArgs& a, int at, Item& it) {
  __shared__ int64_t sums[4];
  __shared__ Item found;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t share = INT32_MAX;
  if (a.target) {
    int64_t work = 0;
    for (int r = tid; r < a.R; r += THREADS) {
      const Request q = request<ROWS, KEYS>(a, r);
      work += (int64_t)q.tiles * q.steps;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) work += __shfl_xor(work, d, 64);
    if (lane == 0) sums[wave] = work;
    __syncthreads();
    work = (sums[0] + sums[1] + sums[2] + sums[3]) * a.kv_heads;
    __syncthreads();
    share = max((work + a.target - 1) / a.target, (int64_t)a.least);
  }
  if (tid == 0) found.r = -1;
  int64_t below = 0;  // places of the requests before, parts of those among them whose keys are divided in the upper half
  for (int base = 0; base < a.R; base += THREADS) {
    const Request q = request<ROWS, KEYS>(a, base + tid);
    const int splits = q.steps > share ? (int)((q.steps + share - 1) / share) : 1;
    const int64_t n = (int64_t)q.tiles * splits, mine = n + (splits > 1 ? n << 32 : 0);
    const int64_t incl = wave_scan(mine);
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    int64_t before = below + incl - mine;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) before += sums[w];
      below += sums[w];
    }
    const int64_t i = at - (before & 0xFFFFFFFF);
    if (i >= 0 && i < n) {
      // a request's longest row tile (the last one, if causal) first
      found = Item{base + tid, q.tiles - 1 - (int)(i / splits), (int)(i % splits), splits,
                   splits > 1 ? (int)(before >> 32) : -1, q.start, q.fresh, q.kv, min(q.fresh, a.max_new) * a.group};
    }
    __syncthreads();
    if (found.r >= 0) break;
  }
  it = found;
  return it.r >= 0;
}

// ---- matrix products of a block -----------------------------------------------------------
typedef short v4s __attribute__((ext_vector_type(4)));

// which values of four bytes (two bf16, one fp32) have an exponent of ones: infinities and NaN
template <typename T>
__device__ __forceinline__ uint32_t no_numbers(uint32_t w) {
  if constexpr (sizeof(T) == 2) return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
  else return ((w & 0x7F800000u) + 0x00800000u) & 0x80000000u;
}

template <typename T, int DB, bool NARROW>
__global__ __launch_bounds__(THREADS, NARROW || (sizeof(T) == 4 && DB > 2) ? 1 : 2) void paged_attention_kernel(const PagedArgs a) {
  using Sh = Shape<T, DB, NARROW>;
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int KS = Sh::KS, ROWB = Sh::ROWB;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  typedef typename std::conditional<BF16, bf16x8, f32x4>::type Piece;

  Item it;
  const int kv_head = blockIdx.x % a.kv_heads;
  if (!find_item<Sh::ITEM_ROWS, Sh::ITEM_KEYS>(a, blockIdx.x / a.kv_heads, it)) return;
  it.r = __builtin_amdgcn_readfirstlane(it.r);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, g = lane >> 5;
  if (a.head && tid == 0 && kv_head == 0 && it.tile == 0 && it.split == 0) {
    a.head[2 * it.r] = it.part;
    a.head[2 * it.r + 1] = it.splits;
  }

  // ---- rows: this lane's, and how many keys it sees
  const int all = __builtin_amdgcn_readfirstlane((int)min((int64_t)it.kv, (int64_t)a.width << a.shift));
  auto sees = [&](int row) __attribute__((always_inline)) {  // keys that a row of (request, head of keys) sees: the first ones
    if (!a.causal) return all;
    return max(min(all, it.kv - it.fresh + row / a.group + 1), 0);
  };
  const int row0 = it.tile * Sh::ITEM_ROWS + (NARROW ? 0 : wave * 32);
  const int row = min(row0 + lq, it.rows - 1);
  const bool active = __builtin_amdgcn_readfirstlane(row0 < it.rows);
  const int seen = sees(row);
  const int all_see = __builtin_amdgcn_readfirstlane(sees(min(row0, it.rows - 1)));          // keys that all rows of the wave see
  const int some_see = __builtin_amdgcn_readfirstlane(sees(min(row0 + 31, it.rows - 1)));    // ... that one of them does
  const int tile_sees = __builtin_amdgcn_readfirstlane(sees(min(it.tile * Sh::ITEM_ROWS + Sh::ITEM_ROWS - 1, it.rows - 1)));
  // this workgroup's steps of ITEM_KEYS keys
  const int steps = (tile_sees + Sh::ITEM_KEYS - 1) / Sh::ITEM_KEYS;
  const int first = __builtin_amdgcn_readfirstlane((int)((int64_t)steps * it.split / it.splits));
  const int last = __builtin_amdgcn_readfirstlane((int)((int64_t)steps * (it.split + 1) / it.splits));
  const int token = row / a.group, head = kv_head * a.group + (row - token * a.group);

  Piece qf[KS];
  const int pieces = a.dh * Sh::ES / 16;  // of a head's row
  {
    const T* q = (const T*)a.q + (int64_t)(it.start + token) * a.q_stride + (int64_t)head * a.dh;
    const uint32_t flip = !a.negative ? 0u : BF16 ? 0x80008000u : 0x80000000u;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      u32x4 x = {0u, 0u, 0u, 0u};
      if (2 * ks + g < pieces) x = *(const u32x4*)((const unsigned char*)q + (2 * ks + g) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] ^= flip;
      qf[ks] = __builtin_bit_cast(Piece, x);
    }
  }

  // ---- loads: rows of pages -> LDS
  // In LDS a row of K lies with its pieces swapped by an exclusive or with SWK, so that the same piece of 16 rows falls on all
  // banks; a row of V by one that spreads what the second product reads at a time: four rows' 64 bytes in bf16, the 128 bytes of two rows four apart in fp32.
  const bool full = pieces == Sh::CPR;
  const int row_bytes = a.dh * Sh::ES, in_row = lane % Sh::CPR, in_instr = lane / Sh::CPR;
  const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
  unsigned char* const mine = lds + (NARROW ? wave * Sh::NS * Sh::STAGE : 0);
  auto swk = [](int r) __attribute__((always_inline)) { return Sh::CPR == 8 ? (r >> 1) & 7 : r & 15; };
  auto swv = [](int r) __attribute__((always_inline)) { return !BF16 ? (r & 4) << 1 : Sh::CPR == 8 ? (r & 2) << 1 : (r & 3) << 2; };
  const ScalarTable table = (ScalarTable)(uintptr_t)(a.table + (int64_t)it.r * a.table_stride);
  const int last_entry = max(tile_sees - 1, 0) >> a.shift;
  struct Pages { int number[Sh::PAGES]; };
  auto step_key = [&](int step) __attribute__((always_inline)) { return step * Sh::ITEM_KEYS + wave * Sh::LOAD; };  // the first key that the wave loads
  auto look_up = [&](int step) __attribute__((always_inline)) {
    Pages p;
    const int key = step_key(step);
#pragma unroll
    for (int i = 0; i < Sh::PAGES; ++i) p.number[i] = table[min((key + 8 * i) >> a.shift, last_entry)];
    return p;
  };
  auto dma16 = [&](const unsigned char* page, uint32_t off, uint32_t to) __attribute__((always_inline)) {
    const uint64_t at = (uint64_t)(uintptr_t)page;
    // (the builtin's result is signed: as a half of an address it must not be extended)
    const uint64_t base = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)at) |
                          (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(at >> 32)) << 32;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
  };
  auto load = [&](int step, const Pages& p, int stage) __attribute__((always_inline)) {
    const int key = step_key(step);
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds0 + (uint32_t)(mine - lds) + stage * Sh::STAGE + (NARROW ? 0 : wave * Sh::LOAD * ROWB));
    auto group = [&](auto full_tag) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < Sh::INSTR; ++i) {
        const int r = i * Sh::RPI;  // first row of the instruction
        const int number = p.number[r / 8];
        const int64_t at = ((((int64_t)((unsigned)number < (unsigned)a.n_pages ? number : 0) * a.kv_heads + kv_head) << a.shift) +
                            ((key + r) & ((1 << a.shift) - 1))) * row_bytes;
        const int row_in = (NARROW ? 0 : wave * Sh::LOAD) + r + in_instr, ck = in_row ^ swk(row_in), cv = in_row ^ swv(row_in);
        if (decltype(full_tag)::value || ck < pieces) dma16((const unsigned char*)a.kp + at, in_instr * row_bytes + ck * 16, to + r * ROWB);
        if (decltype(full_tag)::value || cv < pieces) dma16((const unsigned char*)a.vp + at, in_instr * row_bytes + cv * 16, to + Sh::KEYS * ROWB + r * ROWB);
      }
    };
    if (full) group(std::true_type{});
    else group(std::false_type{});
  };
  auto bad_pages = [&](const Pages& p) __attribute__((always_inline)) {  // a bit for every eight keys
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < Sh::PAGES; ++i) bad |= (unsigned)p.number[i] < (unsigned)a.n_pages ? 0u : 1u << i;
    return bad;
  };

  // pieces that no load writes are zeros: they meet zeros of the queries
  if (!full) {
    for (int i = tid; i < Sh::LDS / 16; i += THREADS) ((u32x4*)lds)[i] = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();
  }

  // ---- one block of 32 keys
  f32x16 o[DB];
  float m = -INFINITY, l = 0.f;  // reference maximum in log2 units; sum of the weights
  f32x4 lsum = {0.f, 0.f, 0.f, 0.f};
  // In bf16 the sums of the weights come from two small products with ones: column n of a 16 x 16 x 32 product sums the eight
  // values of the lanes n, n + 16, n + 32 and n + 48, of the rows n and n + 16 that is; a first operand with ones for the
  // lanes of one in its even rows and for those of the other in its odd rows tells them apart.
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (__bf16)(((lane ^ (lane >> 4)) & 1) ? 0.0f : 1.0f);
  const uint32_t k_off = (uint32_t)(lq * ROWB + ((g ^ swk(lq)) << 4));
  // (the transposing read: lane j of 16 points at four columns of key j / 4 and receives column j of the four keys)
  const uint32_t v_row = BF16 ? 4 * g + ((lane & 15) >> 2) : 4 * g;
  const uint32_t v_off = BF16 ? v_row * ROWB + 32 * ((lane >> 4) & 1) + 8 * (lane & 3) : v_row * ROWB + (lq & 3) * 4;
  const uint32_t v_swap = BF16 ? (Sh::CPR == 8 ? (lane & 8) << 3 : ((lane & 15) >> 2) << 6) : 0;
  auto read_k = [&](const unsigned char* sK, int ks) __attribute__((always_inline)) { return *(const Piece*)(sK + (k_off ^ (uint32_t)(ks << 5))); };
  auto read_v16 = [&](const unsigned char* sV, int b, int s2) __attribute__((always_inline)) {  // bf16: keys 16 s2 + 4 g + (0 .. 3, 8 .. 11), column 32 b + lq
    const unsigned char* p = sV + s2 * 16 * ROWB + ((uint32_t)(b * 64) ^ v_swap) + v_off;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(p + 8 * ROWB)));
    return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
  };
  auto read_v32 = [&](const unsigned char* sV, int b, int v) __attribute__((always_inline)) {  // fp32: key 8 (v / 4) + 4 g + v % 4, column 32 b + lq
    return *(const float*)(sV + v_off + (8 * (v >> 2) + (v & 3)) * ROWB + (((8 * b + (lq >> 2)) ^ (g << 3)) << 4));
  };
  auto accumulate = [&](const unsigned char* sV, const uint32_t (&pw)[8], const f32x16& pf) __attribute__((always_inline)) {  // O^T += V^T P^T
    if constexpr (BF16) {
      bf16x8 p[2];
      p[0] = __builtin_bit_cast(bf16x8, u32x4{pw[0], pw[1], pw[2], pw[3]});
      p[1] = __builtin_bit_cast(bf16x8, u32x4{pw[4], pw[5], pw[6], pw[7]});
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_v16(sV, b, s2), p[s2], o[b], 0, 0, 0);
    } else {
#pragma unroll
      for (int v = 0; v < 16; ++v)
#pragma unroll
        for (int b = 0; b < DB; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(read_v32(sV, b, v), pf[v], o[b], 0, 0, 0);
    }
  };
  // Values that are no numbers, in a block in which not every row sees every key: a product would carry them, times a weight
  // of zero, into rows that do not see them.  The product takes zeros in their place, and rows that do see one
  // (counted by a product of ones) get what it makes of a sum.
  auto any_no_number = [&](const unsigned char* sV) __attribute__((always_inline)) {
    uint32_t any = 0;
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      if constexpr (BF16) {
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          const u32x4 w = __builtin_bit_cast(u32x4, read_v16(sV, b, s2));
#pragma unroll
          for (int e = 0; e < 4; ++e) any |= no_numbers<T>(w[e]);
        }
      } else {
#pragma unroll
        for (int v = 0; v < 16; ++v) any |= no_numbers<T>(__builtin_bit_cast(uint32_t, read_v32(sV, b, v)));
      }
    }
    return __builtin_amdgcn_ballot_w64(any != 0) != 0;
  };
  auto accumulate_around = [&](const unsigned char* sV, const uint32_t (&pw)[8], const f32x16& pf, const f32x16& st) __attribute__((always_inline)) {
    uint32_t sw[8];  // ones where a row sees a key
#pragma unroll
    for (int e = 0; e < 8; ++e)
      sw[e] = (st[2 * e] == -INFINITY ? 0u : 0x00003F80u) | (st[2 * e + 1] == -INFINITY ? 0u : 0x3F800000u);
    // kind 0: the product over numbers; 1 to 3: how many infinities, negative ones and NaN a row sees
#pragma unroll
    for (int b = 0; b < DB; ++b) {
#pragma unroll 1
      for (int kind = 0; kind < 4; ++kind) {
        f32x16 sum;
#pragma unroll
        for (int v = 0; v < 16; ++v) sum[v] = 0.f;
        auto pick = [&](uint32_t bits) __attribute__((always_inline)) {  // fp32 bits of a value -> those that the product takes
          const bool number = (bits & 0x7F800000u) != 0x7F800000u;
          if (kind == 0) return number ? bits : 0u;
          const bool is = kind == 1 ? bits == 0x7F800000u : kind == 2 ? bits == 0xFF800000u : !number && (bits & 0x007FFFFFu);
          return is ? 0x3F800000u : 0u;
        };
        if constexpr (BF16) {
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            u32x4 w = __builtin_bit_cast(u32x4, read_v16(sV, b, s2)), p;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              w[e] = (pick(w[e] << 16) >> 16) | pick(w[e] & 0xFFFF0000u);
              p[e] = kind == 0 ? pw[4 * s2 + e] : sw[4 * s2 + e];
            }
            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, p), sum, 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const float x = __builtin_bit_cast(float, pick(__builtin_bit_cast(uint32_t, read_v32(sV, b, v))));
            sum = __builtin_amdgcn_mfma_f32_32x32x2f32(x, kind == 0 ? pf[v] : st[v] == -INFINITY ? 0.f : 1.f, sum, 0, 0, 0);
          }
        }
        const float add = kind == 1 ? INFINITY : kind == 2 ? -INFINITY : NAN;
#pragma unroll
        for (int v = 0; v < 16; ++v) o[b][v] += kind == 0 ? sum[v] : sum[v] > 0.f ? add : 0.f;
      }
    }
  };

  // FAST: weights exp2(x - m) with the maximum m of the row's first block for all of its keys, which serves any row whose sum of
  // weights stays between 2^-100 and 2^100 (bf16 and fp32 have the same exponents, so nothing is lost); a wave with another row goes over its keys again with a running maximum.
  bool begun = false;
  auto block = [&](auto fast_tag, auto mask_tag, const unsigned char* sK, const unsigned char* sV, int key0, uint32_t bad) __attribute__((always_inline)) {
    constexpr bool FAST = decltype(fast_tag)::value, MASK = decltype(mask_tag)::value;
    f32x16 st;
#pragma unroll
    for (int v = 0; v < 16; ++v) st[v] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const Piece k = read_k(sK, ks);
      if constexpr (BF16) {
        st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[ks], st, 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) st = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], qf[ks][e], st, 0, 0, 0);
      }
    }
    if (MASK) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (key0 + 8 * (v >> 2) + 4 * g + (v & 3) >= seen || (bad >> (v >> 2) & 1)) st[v] = -INFINITY;
    }
    if (!FAST || !begun) {
      float up = st[0];
#pragma unroll
      for (int v = 1; v < 16; ++v) up = fmaxf(up, st[v]);
      up = fmaxf(up, __shfl_xor(up, 32, 64)) * a.scale;
      up = fmaxf(up, m);
      if (!FAST) {
        const float shrink = up == m ? 1.f : __builtin_amdgcn_exp2f(m - up);
        l *= shrink;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[b][v] *= shrink;
      }
      m = up;
      begun = true;
    }
    const float neg_m = m == -INFINITY ? 0.f : -m;
    uint32_t pw[8];
    f32x16 pf;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = __builtin_amdgcn_exp2f(fmaf(st[2 * e], a.scale, neg_m)), y = __builtin_amdgcn_exp2f(fmaf(st[2 * e + 1], a.scale, neg_m));
      if constexpr (BF16) {
        pw[e] = pack_bf16x2(x, y);
        if (!FAST) sum += __builtin_bit_cast(float, pw[e] << 16) + __builtin_bit_cast(float, pw[e] & 0xFFFF0000u);
      } else {
        pf[2 * e] = x;
        pf[2 * e + 1] = y;
        sum += x + y;
      }
    }
    if constexpr (FAST && BF16) {
#pragma unroll
      for (int s2 = 0; s2 < 2; ++s2)
        lsum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, __builtin_bit_cast(bf16x8, u32x4{pw[4 * s2], pw[4 * s2 + 1], pw[4 * s2 + 2], pw[4 * s2 + 3]}),
                                                       lsum, 0, 0, 0);
    } else {
      l += sum;
    }
    if (MASK && any_no_number(sV)) accumulate_around(sV, pw, pf, st);
    else accumulate(sV, pw, pf);
  };
  const std::true_type YES{};
  const std::false_type NO{};

  auto clear = [&]() __attribute__((always_inline)) {
    m = -INFINITY;
    l = 0.f;
    begun = false;
    lsum = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[b][v] = 0.f;
  };
  auto finish = [&](auto fast_tag) __attribute__((always_inline)) {  // the whole sum of a row, in both lanes that share it
    if constexpr (decltype(fast_tag)::value && BF16) l = lane & 16 ? lsum[1] : lsum[0];
    else l += __shfl_xor(l, 32, 64);
  };
  auto wait = []() __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };

  // WIDE: a tile is loaded while the one before it is worked on; one barrier a tile, behind which the tile is complete and
  // nobody reads the buffer that the next loads fill.
  bool careful = false;  // a page of the workgroup's keys lies outside the pool
  auto wide_pass = [&](auto fast_tag, const bool work) __attribute__((always_inline)) {
    if (work) clear();
    Pages next = look_up(first);
    load(first, next, first & 1);
    next = look_up(first + 1);
    for (int t = first; t < last; ++t) {
      wait();
      __syncthreads();
      if (t + 1 < last) {
        load(t + 1, next, (t + 1) & 1);
        next = look_up(t + 2);
      }
      if (!work) continue;
      const unsigned char* sK = lds + (t & 1) * Sh::STAGE;
      const unsigned char* sV = sK + Sh::KEYS * ROWB;
#pragma unroll
      for (int kb = 0; kb < Sh::KEYS / 32; ++kb) {
        const int key0 = t * Sh::ITEM_KEYS + kb * 32;
        if (key0 + 32 <= all_see && !careful) {
          block(fast_tag, NO, sK + kb * 32 * ROWB, sV + kb * 32 * ROWB, key0, 0);
        } else if (key0 < some_see) {
          uint32_t bad = 0;
          if (careful) {
            for (int i = 0; i < 4; ++i)
              bad |= (unsigned)table[min((key0 + 8 * i) >> a.shift, last_entry)] < (unsigned)a.n_pages ? 0u : 1u << i;
          }
          block(fast_tag, YES, sK + kb * 32 * ROWB, sV + kb * 32 * ROWB, key0, bad);
        }
      }
    }
    if (work) finish(fast_tag);
    __syncthreads();  // before the buffers are used again
  };
  // NARROW: a wave waits for its own loads alone, of which a stage more is on its way.
  auto narrow_pass = [&](auto fast_tag) __attribute__((always_inline)) {
    clear();
    constexpr int LOADS = 2 * Sh::INSTR;
    uint32_t bad[2] = {0u, 0u};
#pragma unroll
    for (int s = 0; s < Sh::NS; ++s)
      if (first + s < last) {
        const Pages p = look_up(first + s);
        bad[s] = bad_pages(p);
        load(first + s, p, s);
      }
    for (int t0 = first; t0 < last; t0 += Sh::NS) {
#pragma unroll
      for (int s = 0; s < Sh::NS; ++s) {
        const int t = t0 + s;
        if (t >= last) break;
        Pages p{};
        if (t + Sh::NS < last) p = look_up(t + Sh::NS);
        if (Sh::NS > 1 && t + 1 < last) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
        else wait();
        const unsigned char* sK = mine + s * Sh::STAGE;
        const unsigned char* sV = sK + Sh::KEYS * ROWB;
        const int key0 = step_key(t);
        if (key0 + 32 <= all_see && !bad[s]) block(fast_tag, NO, sK, sV, key0, 0);
        else if (key0 < some_see) block(fast_tag, YES, sK, sV, key0, bad[s]);
        if (t + Sh::NS < last) {
          bad[s] = bad_pages(p);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the block's reads of this stage are through
          load(t + Sh::NS, p, s);
        }
      }
    }
    finish(fast_tag);
  };

  // a row that sees keys of this part and whose sum is out of range
  auto out_of_range = [&]() __attribute__((always_inline)) {
    const bool sees_some = first * Sh::ITEM_KEYS < seen;
    return __builtin_amdgcn_ballot_w64(sees_some && !(l >= 0x1p-100f && l <= 0x1p100f)) != 0;
  };
  if constexpr (NARROW) {
    narrow_pass(YES);
    if (out_of_range()) narrow_pass(NO);
  } else if (first < last) {
    bool bad = false;
    for (int i = ((first * Sh::ITEM_KEYS) >> a.shift) + tid; i <= min((last * Sh::ITEM_KEYS - 1) >> a.shift, last_entry); i += THREADS)
      bad |= (unsigned)a.table[(int64_t)it.r * a.table_stride + i] >= (unsigned)a.n_pages;
    careful = __syncthreads_or(bad);
    wide_pass(YES, active);
    // rows of a wave that was in range stay as they are, whatever shares their workgroup
    const bool again = active && out_of_range();
    if (__syncthreads_or(again)) wide_pass(NO, again);
  } else {
    clear();
  }

  // ---- results: a lane owns a row; registers 4 j .. 4 j + 3 of block b are its columns 32 b + 8 j + 4 g .. + 3
  const int64_t part = it.part >= 0 ? ((int64_t)it.part + (int64_t)it.tile * it.splits + it.split) * a.kv_heads + kv_head : -1;
  if (part >= a.max_parts) return;  // (only if the offsets are none: requests that overlap)
  auto store = [&](int col, f32x4 v, int64_t at) __attribute__((always_inline)) {  // four columns of the row at element `at` of out
    if constexpr (BF16) *(u32x2*)((bf16_t*)a.out + at + col) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    else *(f32x4*)((float*)a.out + at + col) = v;
  };
  if constexpr (!NARROW) {
    if (!active || row0 + lq >= it.rows) return;
    const int64_t at = (int64_t)(it.start + token) * a.out_stride + (int64_t)head * a.dh;
    const float inv = part >= 0 ? 1.f : l == 0.f ? 0.f : 1.f / l;
    float* const po = a.parts + (part * a.part_rows + wave * 32 + lq) * (DB * 32);
    if (part >= 0 && g == 0) {
      a.stats[(part * a.part_rows + wave * 32 + lq) * 2] = m;
      a.stats[(part * a.part_rows + wave * 32 + lq) * 2 + 1] = l;
    }
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = 32 * b + 8 * j + 4 * g;
        const f32x4 v = {o[b][4 * j] * inv, o[b][4 * j + 1] * inv, o[b][4 * j + 2] * inv, o[b][4 * j + 3] * inv};
        if (part >= 0) *(f32x4*)(po + col) = v;
        else if (col < a.dh) store(col, v, at);
      }
  } else {
    // the four waves' sums are joined: each brought to the largest of their maxima
    __syncthreads();
    float* const ms = (float*)lds;              // [4][32] maxima, [4][32] sums
    float* const so = (float*)(lds + 1024);     // [4][32][32 DB + 4]: rows a bank apart
    constexpr int LD = DB * 32 + 4;
    const int rows = min(32, it.rows - row0);
    if (g == 0) {
      ms[wave * 32 + lq] = m;
      ms[128 + wave * 32 + lq] = l;
    }
    if (lq < rows) {
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *(f32x4*)(so + (wave * 32 + lq) * LD + 32 * b + 8 * j + 4 * g) = f32x4{o[b][4 * j], o[b][4 * j + 1], o[b][4 * j + 2], o[b][4 * j + 3]};
    }
    __syncthreads();
    constexpr int QUADS = DB * 8;
    for (int i = tid; i < rows * QUADS; i += THREADS) {
      const int r = i / QUADS, col = (i - r * QUADS) * 4;
      float top = ms[r];
#pragma unroll
      for (int w = 1; w < 4; ++w) top = fmaxf(top, ms[w * 32 + r]);
      const float ref = top == -INFINITY ? 0.f : top;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (ms[128 + w * 32 + r] == 0.f) continue;  // it saw nothing
        const float mw = ms[w * 32 + r], f = __builtin_amdgcn_exp2f((mw == -INFINITY ? 0.f : mw) - ref);
        const f32x4 x = *(const f32x4*)(so + (w * 32 + r) * LD + col);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(x[e], f, v[e]);
        sum = fmaf(ms[128 + w * 32 + r], f, sum);
      }
      const int tok = (row0 + r) / a.group, hd = kv_head * a.group + (row0 + r - tok * a.group);
      if (part >= 0) {
        *(f32x4*)(a.parts + (part * a.part_rows + r) * (DB * 32) + col) = v;
        if (col == 0) {
          a.stats[(part * a.part_rows + r) * 2] = top;
          a.stats[(part * a.part_rows + r) * 2 + 1] = sum;
        }
      } else if (col < a.dh) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        store(col, f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv}, (int64_t)(it.start + tok) * a.out_stride + (int64_t)hd * a.dh);
      }
    }
  }
}

// A wave for every row of a request whose keys were divided: its parts, in order.
template <typename T, int DB>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedArgs a, int item_rows) {
  const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int t = (int)(i / a.heads), head = (int)(i - (int64_t)t * a.heads);
  if (t >= a.rows) return;
  int lo = 0, hi = a.R;  // requests lo .. hi - 1 hold the one that starts at t or below last
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    const int n = __popcll(__builtin_amdgcn_ballot_w64(at < hi && a.starts[min(at, hi - 1)] <= t));
    if (n == 0) return;
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
  }
  const int start = a.starts[lo], fresh = a.starts[lo + 1] - start;
  if (t < start || t - start >= min(fresh, a.max_new)) return;
  const int first = a.head[2 * lo], splits = a.head[2 * lo + 1];
  if (first < 0) return;
  const int kv_head = head / a.group, row = (t - start) * a.group + (head - kv_head * a.group);
  const int tile = row / item_rows, in_tile = row - tile * item_rows;
  // the places of its parts lie kv_heads parts apart
  const int64_t part = ((int64_t)first + (int64_t)tile * splits) * a.kv_heads + kv_head;
  if (splits < 1 || part + (int64_t)(splits - 1) * a.kv_heads >= a.max_parts) return;  // (as above: nobody has written it)
  const float* const stats = a.stats + (part * a.part_rows + in_tile) * 2;
  const int64_t stats_step = (int64_t)a.kv_heads * a.part_rows * 2, step = (int64_t)a.kv_heads * a.part_rows * (DB * 32);
  float top = -INFINITY;
  for (int s = lane; s < splits; s += 64)
    if (stats[s * stats_step + 1] != 0.f) top = fmaxf(top, stats[s * stats_step]);
#pragma unroll
  for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
  const float ref = top == -INFINITY ? 0.f : top;
  const float* const values = a.parts + (part * a.part_rows + in_tile) * (DB * 32);
  float sum = 0.f, v[2] = {0.f, 0.f};
  for (int s0 = 0; s0 < splits; s0 += 64) {
    float f = 0.f, w = 0.f;
    if (s0 + lane < splits) {
      const float l = stats[(s0 + lane) * stats_step + 1], ml = stats[(s0 + lane) * stats_step];
      if (l != 0.f) f = __builtin_amdgcn_exp2f((ml == -INFINITY ? 0.f : ml) - ref);
      w = l;
    }
    for (int s = 0; s < min(64, splits - s0); ++s) {
      const float fs = __shfl(f, s, 64), ws = __shfl(w, s, 64);
      if (ws == 0.f) continue;
      sum = fmaf(ws, fs, sum);
      const float* p = values + (s0 + s) * step;
      if (lane < DB * 32) v[0] = fmaf(p[lane], fs, v[0]);
      if (lane + 64 < DB * 32) v[1] = fmaf(p[lane + 64], fs, v[1]);
    }
  }
  T* out = (T*)a.out + (int64_t)t * a.out_stride + (int64_t)head * a.dh;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (lane < a.dh) Elem<T>::store(out + lane, v[0] * inv);
  if (lane + 64 < a.dh) Elem<T>::store(out + lane + 64, v[1] * inv);
}

// ---- host ---------------------------------------------------------------------------------
// How a call is laid out: by the sizes that the host knows, upper bounds of what the device finds.
struct Layout {
  bool narrow;
  int target, part_rows, width;   // see PagedArgs; columns of a part's rows
  int64_t grid, parts;
  size_t head_bytes, stats_bytes, bytes;
};

constexpr int UNITS = 256;  // compute units of the device

Layout lay_out(const vit_pages_attend_t* p) {
  Layout y{};
  const int group = p->q_heads / p->kv_heads;
  const int64_t most = (int64_t)p->max_new * group;  // rows of a request and head of keys
  y.narrow = most <= 32;
  const int rows = y.narrow ? 32 : 128;
  const int64_t tiles = p->kv_heads * std::min<int64_t>((most + rows - 1) / rows * p->n_requests, (int64_t)p->n_rows * group / rows + p->n_requests);
  y.target = 2 * UNITS;
  // with rows for several rounds of the device there is nothing to divide
  if ((int64_t)p->n_rows * group / rows * p->kv_heads >= 4 * y.target || p->table_width == 0) y.target = 0;
  y.width = (p->head_dim <= 64 ? 2 : p->head_dim <= 96 ? 3 : 4) * 32;
  y.part_rows = (int)std::min<int64_t>(rows, most);
  y.grid = tiles + y.target;
  // divided requests have more than one share each, so at most twice as many parts as shares
  y.parts = y.target ? 2 * y.target + p->kv_heads : 0;
  if (y.target) {
    auto up = [](size_t n) __attribute__((always_inline)) { return (n + 255) / 256 * 256; };
    y.head_bytes = up((size_t)p->n_requests * 2 * sizeof(int32_t));
    y.stats_bytes = up((size_t)y.parts * y.part_rows * 2 * sizeof(float));
    y.bytes = y.head_bytes + y.stats_bytes + (size_t)y.parts * y.part_rows * y.width * sizeof(float);
  }
  return y;
}

template <typename T, int DB, bool NARROW>
hipError_t launch_as(const PagedArgs& a, int64_t grid, hipStream_t s) {
  using Sh = Shape<T, DB, NARROW>;
  constexpr int JOIN = NARROW ? 1024 + 4 * 32 * (DB * 32 + 4) * 4 : 0, smem = Sh::LDS > JOIN ? Sh::LDS : JOIN;
  auto kernel = paged_attention_kernel<T, DB, NARROW>;
  static LdsLimitOnce lds_limit;
  if (hipError_t e = lds_limit.ensure((const void*)kernel, smem); e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(THREADS), smem, s, a);
  if (a.target)
    hipLaunchKernelGGL((paged_join_kernel<T, DB>), dim3((unsigned)(((int64_t)a.rows * a.heads + 3) / 4)), dim3(256), 0, s, a, Sh::ITEM_ROWS);
  return hipGetLastError();
}

template <typename T>
hipError_t launch(const PagedArgs& a, const Layout& y, hipStream_t s) {
  switch (y.width / 32) {
    case 2: return y.narrow ? launch_as<T, 2, true>(a, y.grid, s) : launch_as<T, 2, false>(a, y.grid, s);
    case 3: return y.narrow ? launch_as<T, 3, true>(a, y.grid, s) : launch_as<T, 3, false>(a, y.grid, s);
    default: return y.narrow ? launch_as<T, 4, true>(a, y.grid, s) : launch_as<T, 4, false>(a, y.grid, s);
  }
}

vit_status_t check_sizes(const vit_pages_attend_t* p, const char* name) {
  if (const char* why = bad_pages(p->n_pages, p->page_size)) return set_error(VIT_EINVAL, "%s: %s", name, why);
  if (const char* why = bad_heads(p->kv_heads, p->head_dim, p->dtype)) return set_error(VIT_EINVAL, "%s: %s", name, why);
  if (p->q_heads <= 0 || p->q_heads > 1024 || p->q_heads % p->kv_heads != 0)
    return set_error(VIT_EINVAL, "%s: q_heads must be a multiple of kv_heads, at most 1024", name);
  if (p->n_rows < 0 || p->n_rows >= 1 << 30 || p->n_requests < 0 || p->n_requests > 1 << 20 || p->max_new < 0 || p->table_width < 0)
    return set_error(VIT_EINVAL, "%s: sizes must not be negative, n_rows < 2^30, n_requests <= 2^20", name);
  // so that numbers of rows, row tiles and workgroups stay inside 31 bits
  if ((int64_t)p->n_rows * p->q_heads >= (int64_t)1 << 31 || (int64_t)p->n_requests * p->kv_heads >= 1 << 30)
    return set_error(VIT_EINVAL, "%s: n_rows * q_heads must be below 2^31, n_requests * kv_heads below 2^30", name);
  return VIT_OK;
}

}  // namespace

extern "C" vit_status_t vit_pages_attend_query(const vit_pages_attend_t* p, size_t* workspace_bytes) {
  if (!p || !workspace_bytes) return set_error(VIT_EINVAL, "vit_pages_attend_query: NULL argument");
  if (vit_status_t st = check_sizes(p, "vit_pages_attend_query"); st != VIT_OK) return st;
  *workspace_bytes = p->n_rows == 0 || p->n_requests == 0 || p->max_new == 0 ? 0 : lay_out(p).bytes;
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
  const Layout y = lay_out(p);
  if (y.bytes && (!p->workspace || p->workspace_bytes < y.bytes))
    return set_error(VIT_ECAPACITY, "vit_pages_attend: workspace holds %zu bytes, %zu needed", p->workspace ? p->workspace_bytes : 0, y.bytes);
  PagedArgs a;
  a.q = p->q; a.kp = p->key_pages; a.vp = p->value_pages; a.out = p->out;
  a.table = p->block_table; a.starts = p->query_offsets; a.kv = p->kv_lens;
  unsigned char* ws = (unsigned char*)p->workspace;
  a.head = y.bytes ? (int32_t*)ws : nullptr;
  a.stats = y.bytes ? (float*)(ws + y.head_bytes) : nullptr;
  a.parts = y.bytes ? (float*)(ws + y.head_bytes + y.stats_bytes) : nullptr;
  a.q_stride = p->q_stride; a.out_stride = p->out_stride; a.table_stride = p->table_stride;
  a.rows = p->n_rows; a.R = p->n_requests; a.max_new = p->max_new; a.width = p->n_pages > 0 ? p->table_width : 0; a.n_pages = p->n_pages;
  a.shift = __builtin_ctz(p->page_size); a.heads = p->q_heads; a.kv_heads = p->kv_heads; a.group = p->q_heads / p->kv_heads;
  a.dh = p->head_dim; a.causal = p->causal != 0; a.target = y.target; a.least = 1; a.part_rows = y.part_rows; a.max_parts = y.parts;
  // (a scale of zero: all logits equal, and what no row sees still minus infinity)
  a.scale = std::max(std::fabs(p->scale) * 1.44269504088896340736f, 1e-35f); a.negative = p->scale < 0;
  const hipError_t e = p->dtype == VIT_DTYPE_FP32 ? launch<float>(a, y, (hipStream_t)stream) : launch<bf16_t>(a, y, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(VIT_EDEVICE, "vit_pages_attend: launch: %s", hipGetErrorString(e));
  return VIT_OK;
}
