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
// Two forms.  WIDE: 128 rows a workgroup, 32 a wave, which share tiles of 64 keys; bound by the matrix units at the device's power limit
// (4096 rows of 128 columns over 32768 keys 1.06 to 1.14 PFLOP/s, by the device; the causal half of 8192 tokens 0.91 to 0.97).  NARROW, where requests have few
// rows: the waves share 32 rows and each has keys of its own, so that four times as many loads are on their way and no
// barrier stands between them (fp32: of more than 32 rows two waves have 32 each and two pairs the same keys, whose second
// reader finds them in a cache: images 101.7 -> 97.4 us, with 128 columns 405 -> 358); bound by HBM (64 single tokens over 2.09 GB of keys and values 5.76 TB/s).
//
// Work is divided on the device, where the lengths are: every workgroup adds up the steps of all requests and finds its own
// place.  NARROW: the steps of all requests, one after the other, are dealt out evenly, one run of them a workgroup (a part of a
// request's keys each before: 8 tokens over 50000 keys 315 us, now 284).  WIDE: a workgroup is one row tile, whose
// keys are divided if they are longer than an even share of all work (runs as in NARROW are two starts and two parts a
// workgroup: 2048 tokens 97 us for 60).  What is divided leaves parts (sums without division, their reference maximum and sum of
// weights) in the workspace, which a second kernel joins, always in the same order.
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
  // workspace, all nullptr if no request's keys can be divided.  What the join needs to know (NARROW, int64: the steps of a head
  // of keys, then the steps before each request; WIDE, int32: whether anything was divided, nothing, then every request's
  // first part and parts); reference maximum and sum of every part's rows; their unnormalised values (and,
  // behind max_parts of them, those that a workgroup of WIDE has so far of more keys than a sum takes)
  int32_t* head;
  float *stats, *parts;
  int64_t max_parts;
  int64_t q_stride, out_stride, table_stride;
  int rows, R, max_new, width, n_pages, shift, heads, kv_heads, group, dh, causal;
  int divide;
  int slots;     // logarithm of the workgroups that the device holds at a time, which they are divided for
  int part_rows; // rows of a part
  float scale;   // > 0, times log2(e)
  int negative;  // the scale's sign, which goes to the queries
};

typedef const __attribute__((address_space(4))) int32_t* ScalarTable;  // read by scalar loads

constexpr int THREADS = 256;
constexpr int MOST_KEYS = INT32_MAX - 255;  // of a request: a few steps behind its last key, numbers of keys still fit 31 bits
// WIDE: a part of few steps is mostly its own start and its sums' way through memory, so it has 16 steps at the least (512 tokens 29.5
// us, 30.6 without the limit; 16 requests of 100 tokens 25.6 and 29; with 32 steps 256 tokens over 8000 keys take 67 us for 58).
constexpr int LEAST_STEPS = 16;
// Keys that one sum runs over, in fp32 and in bf16.  A sum of n terms of like size is off by n / 2 roundings of it at the most and stops at 2^24
// terms: 600 rows over 2^31 keys, all values one, came out as 0.8.  So longer runs are cut into sums that are joined as parts are:
// off by 2^-9 at the most, of itself (bf16's instruction adds several products before it rounds).
template <typename T>
constexpr int LONG_SUM = sizeof(T) == 4 ? 1 << 16 : 1 << 18;

template <typename T, int DB_, bool NARROW>
struct Shape {
  static constexpr int DB = DB_;                             // blocks of 32 columns
  static constexpr int ES = (int)sizeof(T);
  static constexpr int ROWB = DB * 32 * ES <= 128 ? 128 : DB * 32 * ES <= 256 ? 256 : 512;  // bytes of a row in LDS
  static constexpr int CPR = ROWB / 16, RPI = 64 / CPR;      // 16-byte pieces of a row; rows that a load instruction fills
  static constexpr int KS = DB * 32 * ES / 32;               // pairs of pieces that the first product runs over
  static constexpr int KEYS = NARROW ? 32 : 64;              // keys that a wave works on at a time
  static constexpr int LOAD = NARROW ? 32 : 16;              // of them, keys that it loads
  static constexpr int INSTR = LOAD / RPI;                   // load instructions for K, and for V
  static constexpr int PAGES = LOAD / 8;                     // pages it looks up
  static constexpr int TILE = KEYS * ROWB;                   // bytes of LDS of a tile of K or V
  // NARROW: tiles on their way at a time, of K and of V, for each wave: two in bf16; in fp32, twice the bytes, one, so that two workgroups
  // lie on a unit up to 64 columns (with two, text over images took 133 us where it took 109).  (WIDE: two of either.)
  static constexpr int NS = NARROW && ES == 4 ? 1 : 2;
  static constexpr int LDS = (NARROW ? 4 : 1) * NS * 2 * TILE;
  // NARROW in fp32: up to 64 rows, by two pairs of waves that have the same keys, half as many a step
  static constexpr int PAIRS = NARROW && ES == 4 ? 2 : 1;
  static constexpr int ITEM_ROWS = NARROW ? 32 * PAIRS : 128;
  static constexpr int ITEM_KEYS = NARROW ? 128 : 64;        // keys of a step of the whole workgroup, if its waves all have their own
  static constexpr int LONG = LONG_SUM<T> / (NARROW ? 32 : 64);  // steps that a wave adds up at a time
};

// ---- a workgroup's place ------------------------------------------------------------------
struct Item {
  int r, tile;                 // request, and which of its row tiles
  int split, splits;           // WIDE: which part of its keys, of how many
  int first, last;             // NARROW: which steps of its keys
  int part;                    // where its results go if they are a part (WIDE: the request's first part), else -1
  int start, fresh, kv, rows;  // the request's first row, rows, keys; rows of (request, head of keys)
  int stretch;                 // which Shape::LONG of its steps
};

struct Request {
  int start, fresh, kv, tiles;
  int steps, last;  // of a row tile's keys; of the last tile's
  __device__ __forceinline__ int64_t all() const { return tiles ? (int64_t)(tiles - 1) * steps + last : 0; }
  __device__ __forceinline__ int of(int tile) const { return tile == tiles - 1 ? last : steps; }
};

template <typename Sh>
__device__ __forceinline__ Request request(const PagedArgs& a, int r) {
  constexpr int ROWS = Sh::ITEM_ROWS, KEYS = Sh::ITEM_KEYS;
  Request q{0, 0, 0, 0, 0, 0};
  if (r < a.R) {
    q.start = a.starts[r];
    const int64_t n = (int64_t)a.starts[r + 1] - q.start;
    q.fresh = q.start < 0 || n < 0 || q.start + n > a.rows ? 0 : (int)n;
    q.kv = min(max(a.kv[r], 0), MOST_KEYS);
    const int64_t rows = (int64_t)min(q.fresh, a.max_new) * a.group, keys = min((int64_t)q.kv, (int64_t)a.width << a.shift);
    q.tiles = (int)((rows + ROWS - 1) / ROWS);
    // (at least one: rows that see nothing have to be written)
    q.steps = q.last = max((int)((keys + KEYS / Sh::PAIRS - 1) / (KEYS / Sh::PAIRS)), 1);
    if (Sh::PAIRS > 1 && rows - (int64_t)(q.tiles - 1) * ROWS <= 32) q.last = max((int)((keys + KEYS - 1) / KEYS), 1);
  }
  return q;
}

// a / b, of numbers that are small as a rule (a division in 64 bits is some hundred instructions)
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return (uint32_t)a / (uint32_t)b;
  return a / b;
}

// WIDE: workgroup `at` of a head of keys into `found` in LDS; false if there are not so many.  The requests whose rows are one wave's
// come first: beside the others they cost little, behind them they are the launch's end (a chunk of 2048 tokens as the first request
// and 24 single tokens behind it 349 us, in the requests' own order 385).
template <typename Sh>
__device__ __forceinline__ bool find_item(const PagedArgs& a, int at, Item& found) {
  __shared__ int64_t sums[4];
  __shared__ int most[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int share = INT32_MAX;
  const Request head = request<Sh>(a, tid);
  if (a.divide) {
    int64_t work = (int64_t)head.tiles * head.steps;
    int longest = head.tiles ? head.steps : 0;
    for (int r = tid + THREADS; r < a.R; r += THREADS) {
      const Request q = request<Sh>(a, r);
      work += (int64_t)q.tiles * q.steps;
      if (q.tiles) longest = max(longest, q.steps);
    }
    work = (int64_t)wave_scan((uint64_t)work);
#pragma unroll
    for (int d = 32; d; d >>= 1) longest = max(longest, __shfl_xor(longest, d, 64));
    if (lane == 63) {
      sums[wave] = work;
      most[wave] = longest;
    }
    __syncthreads();
    work = (sums[0] + sums[1] + sums[2] + sums[3]) * a.kv_heads;
    longest = max(max(most[0], most[1]), max(most[2], most[3]));
    __syncthreads();
    share = (int)min(max((work + (1 << a.slots) - 1) >> a.slots, (int64_t)LEAST_STEPS), (int64_t)INT32_MAX);
    if (blockIdx.x == 0 && tid == 0) a.head[0] = longest > share;  // whether there is anything to join
  }
  if (tid == 0) found.r = -1;
  int64_t below = 0;  // places of the requests before, parts of those among them whose keys are divided in the upper half
  for (int few = 1; few >= 0; --few) {
    for (int base = 0; base < a.R; base += THREADS) {
      const Request q = base == 0 ? head : request<Sh>(a, base + tid);
      const int rows = min(q.fresh, a.max_new) * a.group, splits = q.steps > share ? 1 + (q.steps - 1) / share : 1;
      const int64_t n = (rows <= 32) == (few != 0) ? (int64_t)q.tiles * splits : 0, mine = n + (splits > 1 ? n << 32 : 0);
      const int64_t incl = (int64_t)wave_scan((uint64_t)mine);
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
        found = Item{base + tid, q.tiles - 1 - (int)i / splits, (int)i % splits, splits, 0, 0, splits > 1 ? (int)(before >> 32) : -1,
                     q.start, q.fresh, q.kv, rows, 0};
      }
      __syncthreads();
      if (found.r >= 0) return true;
    }
  }
  return false;
}

__device__ __forceinline__ int64_t uniform(int64_t v) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)v) |
                   (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)v >> 32)) << 32);
}
__device__ __forceinline__ Item uniform(const Item& i) {  // the same for all threads, to the compiler too
  return Item{__builtin_amdgcn_readfirstlane(i.r), __builtin_amdgcn_readfirstlane(i.tile), __builtin_amdgcn_readfirstlane(i.split),
              __builtin_amdgcn_readfirstlane(i.splits), __builtin_amdgcn_readfirstlane(i.first), __builtin_amdgcn_readfirstlane(i.last),
              __builtin_amdgcn_readfirstlane(i.part), __builtin_amdgcn_readfirstlane(i.start), __builtin_amdgcn_readfirstlane(i.fresh),
              __builtin_amdgcn_readfirstlane(i.kv), __builtin_amdgcn_readfirstlane(i.rows), __builtin_amdgcn_readfirstlane(i.stretch)};
}

// NARROW: the steps of all heads, requests and row tiles, one after the other, are dealt out evenly: workgroup b of 2^slots takes
// those from first_step(b) up to first_step(b + 1), one at least if there are so few.
__device__ __forceinline__ int64_t first_step(int64_t total, int b, int slots) {
  return total >> slots ? (int64_t)(((unsigned __int128)total * (unsigned)b) >> slots) : min((int64_t)b, total);
}
__device__ __forceinline__ int workgroup_of(int64_t total, int64_t step, int slots) {  // the last whose first step is that one or before
  if (!(total >> slots)) return (int)step;
  int b = (int)((float)step / (float)total * (float)(1 << slots));
  b = min(max(b, 0), (1 << slots) - 1);
  while (first_step(total, b, slots) > step) --b;
  while (b + 1 < 1 << slots && first_step(total, b + 1, slots) <= step) ++b;
  return b;
}

// Where requests are many: the one among `from` and the ones behind it that holds step `at`, of which `below` lie before request `from`: its number,
// lengths and the steps before it, into LDS.  With `heads`, the steps before every request are written there.
struct Stretch { int64_t below; Request q; int r; };
template <typename Sh>
__device__ __forceinline__ void find_request(const PagedArgs& a, int from, int64_t below, int64_t at, int64_t* sums, Stretch& out, int64_t* heads) {
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // (nothing of this is kept through the loops over keys)
  const int lane = tid & 63, wave = tid >> 6;
  if (tid == 0) out.r = -1;
  __syncthreads();
  for (int base = from; base < a.R; base += THREADS) {
    const Request q = request<Sh>(a, base + tid);
    const int64_t n = q.all(), incl = (int64_t)wave_scan((uint64_t)n);
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    int64_t before = below + incl - n;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) before += sums[w];
      below += sums[w];
    }
    if (heads && base + tid < a.R) heads[base + tid] = before;
    if (before <= at && at < before + n) {
      out.below = before;
      out.q = q;
      out.r = base + tid;
    }
    __syncthreads();
    if (!heads && out.r >= 0) break;
  }
}

// ---- matrix products of a block -----------------------------------------------------------
typedef short v4s __attribute__((ext_vector_type(4)));

// which values of four bytes (two bf16, one fp32) have an exponent of ones: infinities and NaN
template <typename T>
__device__ __forceinline__ uint32_t no_numbers(uint32_t w) {
  if constexpr (sizeof(T) == 2) return ((w & 0x7F807F80u) + 0x00800080u) & 0x80008000u;
  else return ((w & 0x7F800000u) + 0x00800000u) & 0x80000000u;
}

// One item: a row tile of a request and a head of keys, and the steps of its keys that are this workgroup's (Shape::LONG of them: true if there
// are more behind those).
template <typename T, int DB, bool NARROW>
__device__ __forceinline__ bool work_on(const PagedArgs& args, const Item& found, const int kv_head, unsigned char* const lds) {
  using Sh = Shape<T, DB, NARROW>;
  constexpr bool BF16 = sizeof(T) == 2;
  constexpr int KS = Sh::KS, ROWB = Sh::ROWB;
  typedef typename std::conditional<BF16, bf16x8, f32x4>::type Piece;

  // WIDE: nothing is kept from one stretch to the next, as it would be registers that are not there: not what follows from the thread's
  // number, nor the arguments
  PagedArgs again;
  if (!NARROW) {
    typedef const __attribute__((address_space(4))) PagedArgs* ConstantArgs;
    ConstantArgs from = (ConstantArgs)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(from));
    __builtin_memcpy(&again, (const PagedArgs*)from, sizeof again);  // (the kernel's only argument)
  }
  const PagedArgs& a = NARROW ? args : again;
  const Item it = uniform(found);
  int tid = threadIdx.x;
  if (!NARROW) asm volatile("" : "+v"(tid));
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lq = lane & 31, g = lane >> 5;
  if (!NARROW && a.head && tid == 0 && kv_head == 0 && it.tile == 0 && it.split == 0) {
    a.head[2 + 2 * it.r] = it.part;
    a.head[3 + 2 * it.r] = it.splits;
  }

  // ---- rows: this lane's, and how many keys it sees
  const int all = __builtin_amdgcn_readfirstlane((int)min((int64_t)it.kv, (int64_t)a.width << a.shift));
  auto sees = [&](int row) __attribute__((always_inline)) {  // keys that a row of (request, head of keys) sees: the first ones
    if (!a.causal) return all;
    return max(min(all, it.kv - it.fresh + row / a.group + 1), 0);
  };
  const bool pairs = Sh::PAIRS > 1 && it.rows - it.tile * Sh::ITEM_ROWS > 32;  // NARROW: two pairs of waves have rows and keys in common
  const int item_keys = pairs ? Sh::ITEM_KEYS / Sh::PAIRS : Sh::ITEM_KEYS, keys_of = pairs ? wave & 1 : wave;
  const int row0 = it.tile * Sh::ITEM_ROWS + (!NARROW ? wave * 32 : pairs ? (wave >> 1) * 32 : 0);
  const int row = min(row0 + lq, it.rows - 1);
  const bool active = __builtin_amdgcn_readfirstlane(row0 < it.rows);
  const int seen = sees(row);
  const int seen_by_all = __builtin_amdgcn_readfirstlane(sees(min(it.tile * Sh::ITEM_ROWS, it.rows - 1)));  // ... of the workgroup
  const int all_see = __builtin_amdgcn_readfirstlane(sees(min(row0, it.rows - 1)));          // keys that all rows of the wave see
  const int some_see = __builtin_amdgcn_readfirstlane(sees(min(row0 + 31, it.rows - 1)));    // ... that one of them does
  const int tile_sees = __builtin_amdgcn_readfirstlane(sees(min(it.tile * Sh::ITEM_ROWS + Sh::ITEM_ROWS - 1, it.rows - 1)));
  // this workgroup's steps of ITEM_KEYS keys
  int first = it.first, last = it.last;
  const int steps = (tile_sees + item_keys - 1) / item_keys;
  if (NARROW) {  // (not those that no row of the tile sees, which are dealt out like the others)
    last = max(min(last, steps), first);
  } else {
    const int even = steps / it.splits, more = steps - even * it.splits;  // the first `more` parts have a step more
    first = __builtin_amdgcn_readfirstlane(it.split * even + min(it.split, more));
    last = __builtin_amdgcn_readfirstlane(first + even + (it.split < more ? 1 : 0));
  }
  first += it.stretch * Sh::LONG;  // (at most `last`: the stretch before had steps left)
  const bool unfinished = last - first > Sh::LONG;
  if (unfinished) last = first + Sh::LONG;

  Piece qf[KS];
  int pieces = a.dh * Sh::ES / 16;  // of a head's row
  asm volatile("" : "+s"(pieces));  // (what follows from it is worked out where it is used: kept from item to item it is more scalars than there are)
  {
    const int token = row / a.group, head = kv_head * a.group + (row - token * a.group);
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
  unsigned char* const mine = lds + (NARROW ? wave * Sh::NS * 2 * Sh::TILE : 0);  // K's tiles, then V's
  auto swk = [](int r) __attribute__((always_inline)) { return Sh::CPR == 8 ? (r >> 1) & 7 : r & 15; };
  auto swv = [](int r) __attribute__((always_inline)) { return !BF16 ? (r & 4) << 1 : Sh::CPR == 8 ? (r & 2) << 1 : (r & 3) << 2; };
  const ScalarTable table = (ScalarTable)(uintptr_t)(a.table + (int64_t)it.r * a.table_stride);
  const int last_entry = max(tile_sees - 1, 0) >> a.shift;
  struct Pages { int number[Sh::PAGES]; };
  auto step_key = [&](int step) __attribute__((always_inline)) { return step * item_keys + keys_of * Sh::LOAD; };  // the first key that the wave loads
  auto look_up = [&](int step) __attribute__((always_inline)) {
    Pages p;
    const int key = step_key(step);
#pragma unroll
    for (int i = 0; i < Sh::PAGES; ++i) p.number[i] = table[min((key + 8 * i) >> a.shift, last_entry)];
    return p;
  };
  // M0 holds the place in LDS, which the load takes one wait state behind the write at the least; five are what it needs behind
  // a vector instruction that writes its address (where the compiler has kept scalars in vector registers)
  auto dma16 = [&](const unsigned char* base, uint32_t off, uint32_t to) __attribute__((always_inline)) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
  };
  const uint32_t base = lds0 + (NARROW ? wave * Sh::NS * 2 * Sh::TILE : wave * Sh::LOAD * ROWB);  // of the wave's loads
  const uint32_t page_bytes = ((uint32_t)row_bytes << a.shift) * (uint32_t)a.kv_heads;  // (at most 4096 x 1024 x 512)
  const unsigned char* const keys0 = (const unsigned char*)a.kp + (((uint64_t)kv_head << a.shift) * (uint32_t)row_bytes);
  const int64_t to_values = (const unsigned char*)a.vp - (const unsigned char*)a.kp;
  // offsets inside the eight rows of a page look-up, the same for every tile
  uint32_t k_from[Sh::INSTR], v_from[Sh::INSTR];
#pragma unroll
  for (int i = 0; i < Sh::INSTR; ++i) {
    const int r = i * Sh::RPI + in_instr, row = (NARROW ? 0 : wave * Sh::LOAD) + r;
    k_from[i] = (r & 7) * row_bytes + ((in_row ^ swk(row)) << 4);
    v_from[i] = (r & 7) * row_bytes + ((in_row ^ swv(row)) << 4);
  }
  auto load = [&](auto values_tag, int step, const Pages& p, uint32_t tile) __attribute__((always_inline)) {
    constexpr bool VALUES = decltype(values_tag)::value;
    const int key = step_key(step);
    auto group = [&](auto full_tag) __attribute__((always_inline)) {
      constexpr bool FULL = decltype(full_tag)::value;
#pragma unroll
      for (int i = 0; i < Sh::INSTR; ++i) {
        const int eight = i * Sh::RPI / 8;
        const uint32_t number = (unsigned)p.number[eight] < (unsigned)a.n_pages ? p.number[eight] : 0;
        const unsigned char* const from = keys0 + (uint64_t)number * page_bytes + (uint32_t)((key + 8 * eight) & ((1 << a.shift) - 1)) * (uint32_t)row_bytes;
        const uint32_t to = base + tile + i * 1024;
        int piece = in_row, at = in_instr;
        if (!FULL) asm volatile("" : "+v"(piece), "+v"(at));  // compared again every time: kept, the lanes' masks are more scalars than there are
        const int row = (NARROW ? 0 : wave * Sh::LOAD) + i * Sh::RPI + at;
        if (FULL || (piece ^ (VALUES ? swv(row) : swk(row))) < pieces) dma16(VALUES ? from + to_values : from, VALUES ? v_from[i] : k_from[i], to);
        if (i % (8 / Sh::RPI) == 8 / Sh::RPI - 1) __builtin_amdgcn_sched_barrier(0);  // (all addresses at once are more scalars than there are)
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
    u32x4 zeros = {0u, 0u, 0u, 0u};
    asm volatile("" : "+v"(zeros));  // (not kept either)
    for (int i = tid; i < Sh::LDS / 16; i += THREADS) ((u32x4*)lds)[i] = zeros;
    __syncthreads();
  }

  // ---- one block of 32 keys
  f32x16 o[DB];
  float m = -INFINITY, l = 0.f;  // reference maximum in log2 units; sum of the weights
  f32x4 lsum = {0.f, 0.f, 0.f, 0.f};
  // In bf16 the sums of the weights come from two small products with ones: column n of a 16 x 16 x 32 product sums the eight
  // values of the lanes n, n + 16, n + 32 and n + 48, of the rows n and n + 16 that is; a first operand with ones for the
  // lanes of one in its even rows and for those of the other in its odd rows tells them apart.
  const uint32_t two_ones = ((lane ^ (lane >> 4)) & 1) ? 0u : 0x3F803F80u;
  uint32_t k_off = (uint32_t)(lq * ROWB + ((g ^ swk(lq)) << 4));
  // (the transposing read: lane j of 16 points at four columns of key j / 4 and receives column j of the four keys)
  const uint32_t v_row = BF16 ? 4 * g + ((lane & 15) >> 2) : 4 * g;
  uint32_t v_off = BF16 ? v_row * ROWB + 32 * ((lane >> 4) & 1) + 8 * (lane & 3) : v_row * ROWB + (lq & 3) * 4;
  uint32_t v_swap = BF16 ? (Sh::CPR == 8 ? (lane & 8) << 3 : ((lane & 15) >> 2) << 6) : 0;
  auto read_k = [&](const unsigned char* sK, int ks) __attribute__((always_inline)) { return *(const Piece*)(sK + (k_off ^ (uint32_t)(ks << 5))); };
  auto first_product = [&](f32x16& st, const Piece& k, int ks) __attribute__((always_inline)) {
    if constexpr (BF16) {
      st = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[ks], st, 0, 0, 0);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) st = __builtin_amdgcn_mfma_f32_32x32x2f32(k[e], qf[ks][e], st, 0, 0, 0);
    }
  };
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
#pragma unroll 1
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

  // Weights are exp2(x - m) with the maximum m of the row's first block for all of its keys, which serves any row whose sum of
  // weights stays between 2^-100 and 2^100 (bf16 and fp32 have the same exponents, so no weight is lost) and whose weighted values stay
  // below 2^100, so that joining them stays finite too (looked at where the weights' sum is above 2^10 alone: one token over
  // 1400 keys in a graph 13.5 us, always 13.7); a wave with another row goes over its keys again with a running maximum
  // (`fast` is false then): no weight is above one.
  bool fast = true, begun = false;
  float neg_m = 0.f;
  auto logits = [&](const unsigned char* sK) __attribute__((always_inline)) {
    f32x16 st;
#pragma unroll
    for (int v = 0; v < 16; ++v) st[v] = 0.f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) first_product(st, read_k(sK, ks), ks);
    return st;
  };
  // (In bf16 a weight is rounded to bf16, by half a step of itself at the most, as the second product takes no other.  The sum is of the
  // rounded ones, so that a row's weights still add up to one.  Against 64 bits the results are off by 0.0021 to 0.0023 of the values in
  // batches and prompts, where rounding the result alone makes 0.0016 to 0.0017; weights of two bf16 numbers each would double
  // the second product, on the units that bound prompts.)
  auto weight = [&](float x) __attribute__((always_inline)) { return __builtin_amdgcn_exp2f(fmaf(x, a.scale, neg_m)); };
  auto sum_ones = [&](const uint32_t (&pw)[8]) __attribute__((always_inline)) {
    uint32_t w = two_ones;
    asm volatile("" : "+v"(w));  // one register between two blocks, not four
    const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{w, w, w, w});
#pragma unroll
    for (int s2 = 0; s2 < 2; ++s2)
      lsum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, __builtin_bit_cast(bf16x8, u32x4{pw[4 * s2], pw[4 * s2 + 1], pw[4 * s2 + 2], pw[4 * s2 + 3]}),
                                                     lsum, 0, 0, 0);
  };
  // `between`: what is done once K's tile has been read and before V's is
  auto block = [&](auto mask_tag, const unsigned char* sK, const unsigned char* sV, int key0, uint32_t bad, auto&& between) __attribute__((always_inline)) {
    constexpr bool MASK = decltype(mask_tag)::value;
    // the general block works its places in LDS out again: kept for it, they would be registers that the others have not got
    const uint32_t keep[3] = {k_off, v_off, v_swap};
    if (MASK) asm volatile("" : "+v"(k_off), "+v"(v_off), "+v"(v_swap));
    f32x16 st = logits(sK);
    between();
    const bool hidden = MASK && (key0 + 32 > all_see || bad);  // some row does not see some key
    if (hidden) {
#pragma unroll
      for (int v = 0; v < 16; ++v)
        if (key0 + 8 * (v >> 2) + 4 * g + (v & 3) >= seen || (bad >> (v >> 2) & 1)) st[v] = -INFINITY;
    }
    if (MASK && (!begun || !fast)) {
      float up = st[0];
#pragma unroll
      for (int v = 1; v < 16; ++v) up = fmaxf(up, st[v]);
      up = fmaxf(up, __shfl_xor(up, 32, 64)) * a.scale;
      up = fmaxf(up, m);
      if (begun) {
        const float shrink = up == m ? 1.f : __builtin_amdgcn_exp2f(m - up);
        l *= shrink;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int v = 0; v < 16; ++v) o[b][v] *= shrink;
      }
      m = up;
      begun = true;
      neg_m = m == -INFINITY ? 0.f : -m;
    }
    uint32_t pw[8];
    f32x16 pf;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = weight(st[2 * e]), y = weight(st[2 * e + 1]);
      if constexpr (BF16) {
        pw[e] = pack_bf16x2(x, y);
        if (MASK && !fast) l += __builtin_bit_cast(float, pw[e] << 16) + __builtin_bit_cast(float, pw[e] & 0xFFFF0000u);
      } else {
        pf[2 * e] = x;
        pf[2 * e + 1] = y;
        l += x + y;
      }
    }
    if (BF16 && (!MASK || fast)) sum_ones(pw);
    if (hidden && any_no_number(sV)) accumulate_around(sV, pw, pf, st);
    else accumulate(sV, pw, pf);
    k_off = keep[0];
    v_off = keep[1];
    v_swap = keep[2];
  };
  const std::true_type YES{};
  const std::false_type NO{};
  // A block at key0, of which the wave's rows see all, some or none.  One whose pages all lie outside the pool is passed over, the first
  // one above all: it would leave its rows without a reference.
  constexpr uint32_t NOTHING = 15;
  auto any_block = [&](const unsigned char* sK, const unsigned char* sV, int key0, uint32_t bad, auto&& between) __attribute__((always_inline)) {
    if (fast && begun && key0 + 32 <= all_see && !bad) block(NO, sK, sV, key0, 0, between);
    else if (key0 < some_see && bad != NOTHING) block(YES, sK, sV, key0, bad, between);
    else between();
  };
  auto nothing = []() __attribute__((always_inline)) {};

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
  auto finish = [&]() __attribute__((always_inline)) {  // the whole sum of a row, in both lanes that share it
    int upper = lane & 16;
    asm volatile("" : "+v"(upper));
    if (BF16 && fast) l = upper ? lsum[1] : lsum[0];
    else l += __shfl_xor(l, 32, 64);
  };
  auto wait = []() __attribute__((always_inline)) { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };

  // WIDE: tiles that all rows see are worked on in pairs without branches.  A block's logits are formed while the exponentials of
  // the one before are, one or a few behind each matrix instruction, and every fragment is read a product ahead of its use.  A
  // tile's K is read for the last time a tile ahead of its V, so K's loads run a tile ahead of V's and one barrier a tile
  // does: behind it K of the next tile and V of this one are complete, and nobody reads the buffers that the next loads fill.
  bool careful = false;  // a page of the workgroup's keys lies outside the pool
  auto hot_block = [&](Piece (&kf)[KS], const unsigned char* sV, const unsigned char* next_k, f32x16& now, f32x16& next) __attribute__((always_inline)) {
    bf16x8 vf[DB][2];
    if constexpr (BF16) {
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) vf[b][s2] = read_v16(sV, b, s2);
    }
    __builtin_amdgcn_sched_barrier(0);
    uint32_t pw[8];
    f32x16 pf;
#pragma unroll
    for (int v = 0; v < 16; ++v) next[v] = 0.f;
    // behind each matrix instruction the arguments of a pair of weights, the exponentials of the pair before and the rounding of
    // the one before that: nothing waits for what was issued just ahead of it
    auto pair = [&](int e) __attribute__((always_inline)) {
      if (e < 8) {
        now[2 * e] = fmaf(now[2 * e], a.scale, neg_m);
        now[2 * e + 1] = fmaf(now[2 * e + 1], a.scale, neg_m);
      }
      if (e >= 1 && e < 9) {
        pf[2 * e - 2] = __builtin_amdgcn_exp2f(now[2 * e - 2]);
        pf[2 * e - 1] = __builtin_amdgcn_exp2f(now[2 * e - 1]);
      }
      if (e >= 2) {
        if constexpr (BF16) pw[e - 2] = pack_bf16x2(pf[2 * e - 4], pf[2 * e - 3]);
        else l += pf[2 * e - 4] + pf[2 * e - 3];
      }
    };
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      first_product(next, kf[ks], ks);
#pragma unroll
      for (int e = 10 * ks / KS; e < 10 * (ks + 1) / KS; ++e) pair(e);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kf[ks] = read_k(next_k, ks);
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (BF16) {
#pragma unroll
      for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2)
          o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[b][s2], __builtin_bit_cast(bf16x8, u32x4{pw[4 * s2], pw[4 * s2 + 1], pw[4 * s2 + 2], pw[4 * s2 + 3]}), o[b], 0, 0, 0);
      sum_ones(pw);
    } else {
      accumulate(sV, pw, pf);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto wide_pass = [&](const bool work) __attribute__((always_inline)) {
    auto k_at = [](int t) __attribute__((always_inline)) { return (t & 1) * Sh::TILE; };
    auto v_at = [](int t) __attribute__((always_inline)) { return (2 + (t & 1)) * Sh::TILE; };
    Pages p1 = look_up(first);
    load(NO, first, p1, k_at(first));
    load(YES, first, p1, v_at(first));
    p1 = look_up(first + 1);  // of the tile behind the present one, and of the one behind that
    if (first + 1 < last) load(NO, first + 1, p1, k_at(first + 1));
    Pages p2{};
    auto enter = [&](int t) __attribute__((always_inline)) {
      // (scalar loads come in any order: with one on its way, whoever waits for LDS waits for all of it.  The barrier does so anyway.)
      p2 = look_up(t + 2);
      wait();
      __syncthreads();
      if (t + 1 < last) load(YES, t + 1, p1, v_at(t + 1));
    };
    auto further = [&](int t) __attribute__((always_inline)) {
      if (t + 2 < last) load(NO, t + 2, p2, k_at(t));
      p1 = p2;
    };
    if (work) clear();
    const int hot_end = fast && !careful ? min(last, seen_by_all / Sh::ITEM_KEYS) : 0;
    int t = first;
#pragma unroll 1
    do {
      enter(t);
      if (work) {
#pragma unroll 1
        for (int kb = 0; kb < 2; ++kb) {
          const int key0 = t * Sh::ITEM_KEYS + kb * 32;
          uint32_t bad = 0;
          if (careful) {
            for (int i = 0; i < 4; ++i)
              bad |= (unsigned)table[min((key0 + 8 * i) >> a.shift, last_entry)] < (unsigned)a.n_pages ? 0u : 1u << i;
          }
          if (key0 < some_see && bad != NOTHING) block(YES, lds + k_at(t) + kb * 32 * ROWB, lds + v_at(t) + kb * 32 * ROWB, key0, bad, nothing);
        }
      }
      __syncthreads();
      further(t);
      ++t;
      if ((t & 1) || t + 1 >= hot_end) continue;
      if (work) {
        Piece kf[KS];
        f32x16 s0 = logits(lds), s1;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kf[ks] = read_k(lds + 32 * ROWB, ks);
#pragma unroll 1
        for (; t + 1 < hot_end; t += 2) {
          enter(t);
          further(t);
          hot_block(kf, lds + 2 * Sh::TILE, lds + Sh::TILE, s0, s1);
          hot_block(kf, lds + 2 * Sh::TILE + 32 * ROWB, lds + Sh::TILE + 32 * ROWB, s1, s0);
          enter(t + 1);
          further(t + 1);
          hot_block(kf, lds + 3 * Sh::TILE, lds, s0, s1);
          hot_block(kf, lds + 3 * Sh::TILE + 32 * ROWB, lds + 32 * ROWB, s1, s0);
        }
      } else {
#pragma unroll 1
        for (; t + 1 < hot_end; t += 2) {  // (as many barriers)
          enter(t);
          further(t);
          enter(t + 1);
          further(t + 1);
        }
      }
    } while (t < last);
    if (work) finish();
    __syncthreads();  // before the buffers are used again
  };
  // NARROW: a wave waits for its own loads alone, of which a stage more is on its way.  With one tile of K and of V, K's next one is
  // loaded as soon as K has been read, behind the first product, and V's behind the second: either has a product's time.
  auto narrow_pass = [&]() __attribute__((always_inline)) {
    clear();
    uint32_t bad[2] = {0u, 0u};
    auto load_both = [&](int t, const Pages& p, int s) __attribute__((always_inline)) {
      bad[s] = bad_pages(p);
      load(NO, t, p, s * 2 * Sh::TILE);
      load(YES, t, p, (s * 2 + 1) * Sh::TILE);
    };
    auto read = []() __attribute__((always_inline)) { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };  // reads of LDS are through
#pragma unroll
    for (int s = 0; s < Sh::NS; ++s)
      if (first + s < last) load_both(first + s, look_up(first + s), s);
    if constexpr (Sh::NS == 1) {
      for (int t = first; t < last; ++t) {
        Pages p{};
        if (t + 1 < last) p = look_up(t + 1);
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Sh::INSTR) : "memory");  // K is there, V perhaps not
        any_block(mine, mine + Sh::TILE, step_key(t), bad[0], [&]() __attribute__((always_inline)) {
          if (t + 1 < last) {
            read();
            load(NO, t + 1, p, 0);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Sh::INSTR) : "memory");  // V is there, the next K perhaps not
          } else {
            wait();
          }
        });
        if (t + 1 < last) {
          read();
          bad[0] = bad_pages(p);
          load(YES, t + 1, p, Sh::TILE);
        }
      }
    } else {
      for (int t0 = first; t0 < last; t0 += Sh::NS) {
#pragma unroll
        for (int s = 0; s < Sh::NS; ++s) {
          const int t = t0 + s;
          if (t >= last) break;
          Pages p{};
          if (t + Sh::NS < last) p = look_up(t + Sh::NS);
          if (t + 1 < last) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * Sh::INSTR) : "memory");
          else wait();
          any_block(mine + s * 2 * Sh::TILE, mine + (s * 2 + 1) * Sh::TILE, step_key(t), bad[s], nothing);
          if (t + Sh::NS < last) {
            read();
            load_both(t + Sh::NS, p, s);
          }
        }
      }
    }
    finish();
  };

  // A row that sees keys of this wave's (NARROW: they begin at its own place in a step; pages may hide them all) and whose sums are out of
  // range, or whose weights were measured against no maximum at all: its logits in the first block were minus infinity.  (So
  // that wherever sums are joined, one that is not zero has a reference.)
  auto out_of_range = [&]() __attribute__((always_inline)) {
    const bool sees_some = begun && (NARROW ? step_key(first) : first * item_keys) < seen;
    auto some_row = [](bool it) __attribute__((always_inline)) { return __builtin_amdgcn_ballot_w64(it) != 0; };
    const bool sees_without = sees_some && !(m > -INFINITY);
    if (!some_row(sees_without || (sees_some && !(l >= 0x1p-100f && l <= 0x1p10f)))) return false;
    f32x4 size = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
      for (int v = 0; v < 16; ++v) size[v & 3] += fabsf(o[b][v]);
    const bool in_range = l >= 0x1p-100f && l <= 0x1p100f && (size[0] + size[1]) + (size[2] + size[3]) < 0x1p100f;
    return some_row(sees_without || (sees_some && !in_range));
  };
  if constexpr (NARROW) {
    if (all == 0) {
      clear();
    } else {
#pragma unroll 1
      for (;;) {
        narrow_pass();
        if (!fast || !out_of_range()) break;
        fast = false;
      }
    }
  } else if (first < last) {
    bool bad = false;
    for (int i = ((first * Sh::ITEM_KEYS) >> a.shift) + tid; i <= min((last * Sh::ITEM_KEYS - 1) >> a.shift, last_entry); i += THREADS)
      bad |= (unsigned)a.table[(int64_t)it.r * a.table_stride + i] >= (unsigned)a.n_pages;
    careful = __syncthreads_or(bad);
    bool work = active;
#pragma unroll 1
    for (;;) {
      wide_pass(work);
      // rows of a wave that was in range stay as they are, whatever shares their workgroup
      work = work && out_of_range();
      if (!fast || !__syncthreads_or(work)) break;
      fast = false;
    }
  } else {
    clear();
  }

  // ---- results: a lane owns a row; registers 4 j .. 4 j + 3 of block b are its columns 32 b + 8 j + 4 g .. + 3
  const Item in = uniform(found);  // (read again: kept through the loops, it would be registers that they have not got)
  const int64_t part = NARROW ? in.part : in.part >= 0 ? ((int64_t)in.part + (int64_t)in.tile * in.splits + in.split) * a.kv_heads + kv_head : -1;
  if (part < a.max_parts) {  // (always, unless the offsets are none: requests that overlap)
    // Stretches are added up in the part's place, or in one of the workgroup's own: NARROW's second part, which is written last if at all
    const bool begun_before = in.stretch > 0, to_place = part >= 0 || unfinished;
    const int64_t place = part >= 0 ? part : NARROW ? 2 * (int64_t)blockIdx.x + 1 : a.max_parts + blockIdx.x;
    // sums so far (their reference and sum of weights) and this stretch's -> the factors of either, their common reference and sum
    struct Both { float before, now, top, sum; };
    auto both = [](float top0, float sum0, float top, float sum) __attribute__((always_inline)) {
      const float up = fmaxf(sum0 == 0.f ? -INFINITY : top0, sum == 0.f ? -INFINITY : top);
      const float f0 = sum0 == 0.f ? 0.f : __builtin_amdgcn_exp2f(top0 - up), f = sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(top - up);
      return Both{f0, f, up, fmaf(sum0, f0, sum * f)};
    };
    auto store = [&](int col, f32x4 v, int64_t at) __attribute__((always_inline)) {  // four columns of the row at element `at` of out
      if constexpr (BF16) *(u32x2*)((bf16_t*)a.out + at + col) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
      else *(f32x4*)((float*)a.out + at + col) = v;
    };
    if constexpr (!NARROW) {
      int thread = threadIdx.x;
      asm volatile("" : "+v"(thread));  // (what follows is worked out here, not ahead of the loops)
      const int lq = thread & 31, g = thread >> 5 & 1, wave = thread >> 6, own_row = in.tile * Sh::ITEM_ROWS + wave * 32 + lq;
      if (own_row < in.rows) {
        const int token = own_row / a.group, head = kv_head * a.group + (own_row - token * a.group);
        const int64_t at = (int64_t)(in.start + token) * a.out_stride + (int64_t)head * a.dh;
        float* const stats = a.stats + (place * a.part_rows + wave * 32 + lq) * 2;
        float* const po = a.parts + (place * a.part_rows + wave * 32 + lq) * (DB * 32);
        if (begun_before) {
          const Both x = both(stats[0], stats[1], m, l);
          m = x.top;
          l = x.sum;
#pragma unroll
          for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const f32x4 v = *(const f32x4*)(po + 32 * b + 8 * j + 4 * g);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[b][4 * j + e] = fmaf(v[e], x.before, o[b][4 * j + e] * x.now);
            }
        }
        const float inv = to_place ? 1.f : l == 0.f ? 0.f : 1.f / l;
        if (to_place && g == 0) {
          stats[0] = m;
          stats[1] = l;
        }
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int col = 32 * b + 8 * j + 4 * g;
            const f32x4 v = {o[b][4 * j] * inv, o[b][4 * j + 1] * inv, o[b][4 * j + 2] * inv, o[b][4 * j + 3] * inv};
            if (to_place) *(f32x4*)(po + col) = v;
            else if (col < a.dh) store(col, v, at);
          }
      }
    } else {
      // the four waves' sums are joined: each brought to the largest of their maxima
      __syncthreads();
      float* const ms = (float*)lds;              // [4][32] maxima, [4][32] sums
      float* const so = (float*)(lds + 1024);     // [4][32][32 DB + 4]: rows a bank apart
      constexpr int LD = DB * 32 + 4;
      const int rows = min(32, in.rows - row0), tile_row = in.tile * Sh::ITEM_ROWS, tile_rows = min(Sh::ITEM_ROWS, in.rows - tile_row);
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
      __shared__ float so_far[Sh::ITEM_ROWS][2];  // references and sums of the stretches before
      if (begun_before && tid < tile_rows) {
        so_far[tid][0] = a.stats[(place * a.part_rows + tid) * 2];
        so_far[tid][1] = a.stats[(place * a.part_rows + tid) * 2 + 1];
      }
      __syncthreads();
      constexpr int QUADS = DB * 8;
      for (int i = tid; i < tile_rows * QUADS; i += THREADS) {
        const int r = i / QUADS, col = (i - r * QUADS) * 4;
        const int at = pairs ? r + (r & 32) : r, waves = pairs ? 2 : 4;  // the first wave that has the row, its numbers' place; how many have
        float top = ms[at];
#pragma unroll
        for (int w = 1; w < 4; ++w)
          if (w < waves) top = fmaxf(top, ms[w * 32 + at]);
        const float ref = top == -INFINITY ? 0.f : top;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if (w >= waves || ms[128 + w * 32 + at] == 0.f) continue;  // (it saw nothing)
          const float mw = ms[w * 32 + at], f = __builtin_amdgcn_exp2f((mw == -INFINITY ? 0.f : mw) - ref);
          const f32x4 x = *(const f32x4*)(so + (w * 32 + at) * LD + col);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(x[e], f, v[e]);
          sum = fmaf(ms[128 + w * 32 + at], f, sum);
        }
        const int tok = (tile_row + r) / a.group, hd = kv_head * a.group + (tile_row + r - tok * a.group);
        float* const po = a.parts + (place * a.part_rows + r) * (DB * 32) + col;
        if (begun_before) {
          const Both x = both(so_far[r][0], so_far[r][1], top, sum);
          const f32x4 w = *(const f32x4*)po;
          top = x.top;
          sum = x.sum;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = fmaf(w[e], x.before, v[e] * x.now);
        }
        if (to_place) {
          *(f32x4*)po = v;
          if (col == 0) {
            a.stats[(place * a.part_rows + r) * 2] = top;
            a.stats[(place * a.part_rows + r) * 2 + 1] = sum;
          }
        } else if (col < a.dh) {
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          store(col, f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv}, (int64_t)(in.start + tok) * a.out_stride + (int64_t)hd * a.dh);
        }
      }
    }
  }
  return __builtin_amdgcn_readfirstlane(unfinished && part < a.max_parts);
}

template <typename T, int DB, bool NARROW>
__global__ __launch_bounds__(THREADS, (NARROW || sizeof(T) == 4) && DB > 2 ? 1 : 2) void paged_attention_kernel(const PagedArgs a) {
  using Sh = Shape<T, DB, NARROW>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  __shared__ Item found;
  if constexpr (!NARROW) {
    if (!find_item<Sh>(a, blockIdx.x / a.kv_heads, found)) return;
#pragma unroll 1
    while (work_on<T, DB, NARROW>(a, found, blockIdx.x % a.kv_heads, lds)) {
      __syncthreads();
      if (threadIdx.x == 0) ++found.stretch;
      __syncthreads();
    }
  } else {
    __shared__ int64_t sums[4], ahead[THREADS + 1];  // steps before each of the first requests, of a head of keys
    __shared__ Stretch stretch;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Request mine = request<Sh>(a, tid);
    int64_t more = 0;
    for (int r = tid + THREADS; r < a.R; r += THREADS) {
      const Request q = request<Sh>(a, r);
      more += q.all();
    }
    const int64_t own = mine.all(), incl = (int64_t)wave_scan((uint64_t)own);
    if (lane == 63) sums[wave] = incl;
    __syncthreads();
    int64_t before = incl - own;
#pragma unroll
    for (int w = 0; w < 3; ++w)
      if (w < wave) before += sums[w];
    ahead[tid] = before;
    if (tid == THREADS - 1) ahead[THREADS] = before + own;
    int64_t steps = sums[0] + sums[1] + sums[2] + sums[3];  // of a head of keys
    if (a.R > THREADS) {
      more = (int64_t)wave_scan((uint64_t)more);
      __syncthreads();
      if (lane == 63) sums[wave] = more;
      __syncthreads();
      steps += sums[0] + sums[1] + sums[2] + sums[3];
    }
    steps = uniform(steps);
    __syncthreads();
    if (blockIdx.x == 0) {  // for the kernel that joins the parts
      int64_t* const heads = (int64_t*)a.head;
      if (tid == 0) heads[0] = steps;
      if (tid < a.R) heads[1 + tid] = before;
      if (a.R > THREADS) find_request<Sh>(a, THREADS, ahead[THREADS], -1, sums, stretch, heads + 1);
    }
    const int64_t total = steps * a.kv_heads, from = first_step(total, blockIdx.x, a.slots), to = first_step(total, blockIdx.x + 1, a.slots);
    int kv_head = 0, r = -1;
    int64_t below = 0, at = from;
    if (from < to) {
      kv_head = (int)quotient(from, steps);
      at = from - kv_head * steps;
      if (before <= at && at < before + own) stretch = Stretch{before, mine, tid};
    }
    __syncthreads();
#pragma unroll 1
    for (int64_t done = from; done < to;) {
      if (r < 0 && at < ahead[THREADS]) {
        // (found above)
      } else if (at < ahead[THREADS]) {
        int mine = tid;
        asm volatile("" : "+v"(mine));  // (its addresses are worked out again)
        if (ahead[mine] <= at && at < ahead[mine + 1]) stretch = Stretch{ahead[mine], request<Sh>(a, mine), mine};
        __syncthreads();
      } else {
        if (r < THREADS) {
          r = THREADS;
          below = ahead[THREADS];
        }
        find_request<Sh>(a, r, below, at, sums, stretch, nullptr);
      }
      r = __builtin_amdgcn_readfirstlane(stretch.r);
      below = uniform(stretch.below);
      const Request q = stretch.q;
      const int tiles = __builtin_amdgcn_readfirstlane(q.tiles), its = __builtin_amdgcn_readfirstlane(q.steps), last_its = __builtin_amdgcn_readfirstlane(q.last);
      if (r < 0 || its < 1) return;  // (only if the lengths have changed meanwhile: nothing is right then, but it ends)
      int tile = min((int)quotient(at - below, its), tiles - 1), first = (int)(at - below - (int64_t)tile * its);
      if (tile < 0 || first >= (tile == tiles - 1 ? last_its : its)) return;  // (likewise)
#pragma unroll 1
      for (int stretch = 0; tile < tiles && done < to;) {
        const int end = tile == tiles - 1 ? last_its : its, last = (int)min((int64_t)end, first + (to - done));
        if (tid == 0) {
          // a workgroup leaves a part of its first item and one of its last at the most
          const int part = first == 0 && last == end ? -1 : 2 * (int)blockIdx.x + (done == from ? 0 : 1);
          found = Item{r, tile, 0, 1, first, last, part, q.start, q.fresh, q.kv, min(q.fresh, a.max_new) * a.group, stretch};
        }
        __syncthreads();
        const bool more = work_on<T, DB, NARROW>(a, found, kv_head, lds);
        __syncthreads();  // before LDS is used again
        if (more) {
          ++stretch;
          continue;
        }
        done += last - first;
        at += last - first;
        ++tile;
        first = stretch = 0;
      }
      below += (int64_t)(tiles - 1) * its + last_its;
      ++r;
      if (at == steps) {
        ++kv_head;
        at = below = 0;
        r = 0;
      }
    }
  }
}

// The parts of a row whose request's keys were divided, in order (one token over 131072 keys, 512 parts: 6.2 us).  Half a wave takes a part, 16 bytes a lane, four parts at a time: the
// loads' latencies are what this kernel is.  HALVES of them share a row: one where rows are many, all eight of a
// workgroup where they are few and may have many parts each.
template <typename T, int DB, bool NARROW, int HALVES>
__device__ __forceinline__ void join_row(const PagedArgs& a, uint32_t i) {
  using Sh = Shape<T, DB, NARROW>;
  const int half = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int t = (int)(i / (uint32_t)a.heads), head = (int)(i - (uint32_t)t * a.heads);
  int lo = 0, hi = a.R;  // of the requests lo .. hi - 1 one is the last to start at t or below
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, at = lo + lane * step;
    const uint64_t some = __builtin_amdgcn_ballot_w64(at < hi && a.starts[min(at, hi - 1)] <= t);
    const int n = __popc((uint32_t)(some >> (threadIdx.x & 32)));
    if (n == 0) return;
    lo += (n - 1) * step;
    hi = min(hi, lo + step);
  }
  const int start = a.starts[lo], fresh = a.starts[lo + 1] - start;
  if (t < start || t - start >= min(fresh, a.max_new)) return;
  const int kv_head = head / a.group, row = (t - start) * a.group + (head - kv_head * a.group);
  const int tile = row / Sh::ITEM_ROWS, in_tile = row - tile * Sh::ITEM_ROWS;
  int64_t part, next;  // the row's first part, and how far it is from the second one to the third
  int64_t second = 0;  // ... and to the second
  int splits;
  if constexpr (NARROW) {
    const int64_t* const heads = (const int64_t*)a.head;
    const int64_t steps = heads[0];
    const Request q = request<Sh>(a, lo);
    const int its = q.of(tile);
    const int64_t total = steps * a.kv_heads, at = kv_head * steps + heads[1 + lo] + (int64_t)tile * q.steps;
    const int b0 = workgroup_of(total, at, a.slots), b1 = workgroup_of(total, at + its - 1, a.slots);
    splits = b1 - b0 + 1;
    if (splits < 2) return;
    part = 2 * b0 + (first_step(total, b0, a.slots) == at ? 0 : 1);
    second = 2 * (b0 + 1) - part;
    next = 2;
  } else {
    const int first = a.head[2 + 2 * lo];
    splits = a.head[3 + 2 * lo];
    if (first < 0) return;
    part = ((int64_t)first + (int64_t)tile * splits) * a.kv_heads + kv_head;  // the others lie kv_heads parts apart
    second = next = a.kv_heads;
  }
  if (splits < 1 || part < 0 || part + second + (int64_t)(splits - 1) * next >= a.max_parts + next) return;  // (offsets that are none: nobody has written it)
  const float* const stats = a.stats + (part * a.part_rows + in_tile) * 2;
  const int64_t one_stats = (int64_t)a.part_rows * 2, one = (int64_t)a.part_rows * (DB * 32);
  const int col = lane * 4;
  const float* const values = a.parts + (part * a.part_rows + in_tile) * (DB * 32) + (col < DB * 32 ? col : 0);
  // a running maximum, as in the parts themselves
  float top = -INFINITY, sum = 0.f;
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](float top2, float sum2, f32x4 v2) __attribute__((always_inline)) {
    if (sum2 == 0.f) return;  // it saw nothing
    const float ref = top2 == -INFINITY ? 0.f : top2, up = fmaxf(top, ref);
    const float keep = __builtin_amdgcn_exp2f(top - up), f = __builtin_amdgcn_exp2f(ref - up);
    top = up;
    sum = fmaf(sum2, f, sum * keep);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = fmaf(v2[e], f, v[e] * keep);
  };
  for (int s0 = HALVES == 1 ? 0 : half; s0 < splits; s0 += 4 * HALVES) {
    f32x2 st[4];
    f32x4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = min(s0 + u * HALVES, splits - 1);
      const int64_t from = s == 0 ? 0 : second + (s - 1) * next;
      st[u] = *(const f32x2*)(stats + from * one_stats);
      x[u] = *(const f32x4*)(values + from * one);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (s0 + u * HALVES < splits) add(st[u][0], st[u][1], x[u]);
  }
  if constexpr (HALVES > 1) {
    __shared__ float tops[8], sums[8];
    __shared__ f32x4 all[8][32];
    if (lane == 0) {
      tops[half] = top;
      sums[half] = sum;
    }
    all[half][lane] = v;
    __syncthreads();
    if (threadIdx.x >= 32) return;
#pragma unroll
    for (int h = 1; h < 8; ++h) add(tops[h], sums[h], all[h][lane]);
  }
  if (col >= a.dh) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int64_t at = (int64_t)t * a.out_stride + (int64_t)head * a.dh + col;
  if constexpr (sizeof(T) == 2) *(u32x2*)((bf16_t*)a.out + at) = u32x2{pack_bf16x2(v[0] * inv, v[1] * inv), pack_bf16x2(v[2] * inv, v[3] * inv)};
  else *(f32x4*)((float*)a.out + at) = f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
}

template <typename T, int DB, bool NARROW, int HALVES>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedArgs a) {
  if (!NARROW && a.head[0] == 0) return;  // no request's keys were divided
  const uint32_t rows = (uint32_t)a.rows * a.heads, at_once = HALVES == 1 ? 8 : 1;  // (rows: below 2^31)
  for (uint32_t i = blockIdx.x * at_once + (HALVES == 1 ? threadIdx.x >> 5 : 0); i < rows; i += gridDim.x * at_once) {
    join_row<T, DB, NARROW, HALVES>(a, i);
    if constexpr (HALVES > 1) __syncthreads();  // before LDS is used again
  }
}

// ---- host ---------------------------------------------------------------------------------
// How a call is laid out: by the sizes that the host knows, upper bounds of what the device finds.
struct Layout {
  bool narrow;
  bool divide;
  int slots, part_rows, width;   // see PagedArgs; columns of a part's rows
  int64_t grid, parts, places;
  size_t head_bytes, stats_bytes, bytes;
};

constexpr int UNITS = 256;  // compute units of the device
constexpr float LOG2E = 1.44269504088896340736f;

Layout lay_out(const vit_pages_attend_t* p) {
  Layout y{};
  const int group = p->q_heads / p->kv_heads;
  const int64_t most = (int64_t)p->max_new * group;  // rows of a request and head of keys
  // NARROW reads keys once for every 32 rows (fp32: 64), WIDE for every 128 but with barriers and with idle waves where rows are fewer.
  // bf16: above 32 rows WIDE (8 requests of 64 rows 62 us, NARROW 101).  fp32's products take nine times as long, which hides the reads
  // for longer: 24 requests of 4 to 360 rows, 128 columns, over images in NARROW 354 us, in WIDE 517; 4 of 400 rows over 2000 keys 165
  // and 183; 1000 rows over 4000 keys 191 and 176.  (Prompts with nothing cached would be better off in WIDE, 8 of 200 tokens 28.6 us for
  // 41.8, 4 of 500 172 for 206: shares of a causal triangle are not even.  But only the device knows that they are.)
  y.narrow = most <= (p->dtype == VIT_DTYPE_FP32 ? 512 : 32);
  const int rows = !y.narrow ? 128 : p->dtype == VIT_DTYPE_FP32 ? 64 : 32;
  const int64_t tiles = p->kv_heads * std::min<int64_t>((most + rows - 1) / rows * p->n_requests, (int64_t)p->n_rows * group / rows + p->n_requests);
  // workgroups that LDS and registers let the device hold
  y.slots = (p->head_dim > 64 && (y.narrow || p->dtype == VIT_DTYPE_FP32) ? 1 : 2) * UNITS;
  y.width = (p->head_dim <= 64 ? 2 : p->head_dim <= 96 ? 3 : 4) * 32;
  y.part_rows = (int)std::min<int64_t>(rows, most);
  y.divide = y.narrow || (int64_t)p->table_width * p->page_size > LEAST_STEPS * 64;  // (there may be something to divide)
  y.grid = y.narrow ? y.slots : tiles + (y.divide ? y.slots : 0);
  // NARROW: two a workgroup.  WIDE: divided requests have more than one share each, so at most twice as many parts as shares.
  y.parts = !y.divide ? 0 : 2 * y.slots + (y.narrow ? 0 : p->kv_heads);
  // WIDE: where the table has room for more keys than a sum takes, each workgroup has a place for them (64 KiB at 128 columns)
  const bool longer = (int64_t)p->table_width * p->page_size > (p->dtype == VIT_DTYPE_FP32 ? LONG_SUM<float> : LONG_SUM<bf16_t>);
  y.places = y.parts + (!y.narrow && longer ? y.grid : 0);
  if (y.divide) {
    auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    y.head_bytes = up(((size_t)p->n_requests + 1) * sizeof(int64_t));
    y.stats_bytes = up((size_t)y.places * y.part_rows * 2 * sizeof(float));
    y.bytes = y.head_bytes + y.stats_bytes + (size_t)y.places * y.part_rows * y.width * sizeof(float);
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
  if (a.divide) {
    // few rows may have many parts each
    const int64_t rows = (int64_t)a.rows * a.heads;
    if (rows <= 16 * UNITS) hipLaunchKernelGGL((paged_join_kernel<T, DB, NARROW, 8>), dim3((unsigned)rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_join_kernel<T, DB, NARROW, 1>), dim3((unsigned)std::min<int64_t>((rows + 7) / 8, 8 * UNITS)), dim3(256), 0, s, a);
  }
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
  if (!std::isfinite(p->scale * LOG2E)) return set_error(VIT_EINVAL, "%s: scale must be finite, times log2(e) too", name);
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
      p->table_stride < p->table_width)
    return set_error(VIT_EINVAL, "vit_pages_attend: strides of q and out must be q_heads * head_dim to 2^32, table_stride >= table_width");
  if (p->n_rows == 0 || p->n_requests == 0 || p->max_new == 0) return VIT_OK;
  if (!p->q || !p->out || !p->query_offsets || !p->kv_lens || (p->table_width > 0 && !p->block_table) ||
      (p->n_pages > 0 && (!p->key_pages || !p->value_pages)))
    return set_error(VIT_EINVAL, "vit_pages_attend: NULL argument");
  if ((((uintptr_t)p->q | (uintptr_t)p->out | (uintptr_t)p->key_pages | (uintptr_t)p->value_pages) & 15) || (p->q_stride * es & 15) ||
      (p->out_stride * es & 15) || ((uintptr_t)p->workspace & 255))
    return set_error(VIT_EINVAL, "vit_pages_attend: pointers and rows must be multiples of 16 bytes, the workspace 256-byte aligned");
  const Layout y = lay_out(p);
  if (y.grid >= 1 << 24)  // (a launch has fewer than 2^32 threads)
    return set_error(VIT_EINVAL, "vit_pages_attend: more requests and rows than a launch has workgroups for");
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
  a.dh = p->head_dim; a.causal = p->causal != 0; a.divide = y.divide;  a.slots = __builtin_ctz(y.slots);  a.part_rows = y.part_rows; a.max_parts = y.parts;
  // (a scale of zero: the smallest number there is, so that what no row sees is still minus infinity; the largest product of queries and
  // keys times it is 2^-21)
  a.scale = std::max(std::fabs(p->scale) * LOG2E, 0x1p-149f); a.negative = p->scale < 0;
  const hipError_t e = p->dtype == VIT_DTYPE_FP32 ? launch<float>(a, y, (hipStream_t)stream) : launch<bf16_t>(a, y, (hipStream_t)stream);
  if (e != hipSuccess) return set_error(VIT_EDEVICE, "vit_pages_attend: launch: %s", hipGetErrorString(e));
  return VIT_OK;
}
