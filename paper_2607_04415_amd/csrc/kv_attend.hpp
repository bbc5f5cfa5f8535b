// Device code that the attention kernels of gorio_kv_attend share: the types
// of the matrix instructions, how a call's work is divided, and where keys and
// values lie.
//
// Transposed products.  A kernel computes S^T = K Q^T and O^T = V^T P^T on the
// matrix units.  In the result of a matrix instruction a lane holds several
// rows of ONE column, so with queries as columns everything the softmax needs
// of a query (its maximum, its sum, its rescaling factor, its position) is one
// value in its lanes, and the weights come out where the second product wants
// them: a lane holds the weights of its query for a set of keys, and that set
// may be any, as long as the values are loaded in the same order.
#pragma once

#include <hip/hip_runtime.h>

#include "kv.hpp"

namespace gorio {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Queries' element types.
struct KvBf16 {
  static constexpr bool kF16 = false;
  static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  }
  static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    const bf16x2 v = {(__bf16)x, (__bf16)y};
    return __builtin_bit_cast(uint32_t, v);
  }
  template <bool kHi>
  static __device__ __forceinline__ uint32_t widen(uint32_t w) {  // two 8-bit values, exactly
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, kHi));
  }
};

struct KvF16 {
  static constexpr bool kF16 = true;
  static __device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
  }
  static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0,
                                                  0);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    const f16x2 v = {(_Float16)x, (_Float16)y};
    return __builtin_bit_cast(uint32_t, v);
  }
  template <bool kHi>
  static __device__ __forceinline__ uint32_t widen(uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, kHi));
  }
};

// Eight elements as they lie in the pages -> eight of the queries' type.
template <typename Q>
__device__ __forceinline__ u32x4 widened(u32x4 r) {
  return r;
}
template <typename Q>
__device__ __forceinline__ u32x4 widened(u32x2 r) {
  return u32x4{Q::template widen<false>(r.x), Q::template widen<true>(r.x), Q::template widen<false>(r.y),
               Q::template widen<true>(r.y)};
}

// LDS by its 32-bit address: what is added to one as a constant goes into the instruction.
typedef __attribute__((address_space(3))) uint8_t LdsBytes;
template <typename T>
__device__ __forceinline__ __attribute__((address_space(3))) T *lds_at(uint32_t address) {
  return (__attribute__((address_space(3))) T *)(uintptr_t)address;
}

// Transposing LDS reads of two times sixteen keys' values at 32 kTiles elements: in each, lane l
// of 16 names the 8 bytes that hold elements 4 (l % 4) .. + 3 of a key l / 4, and gets element l
// of the four keys.  at[t][h]: address of elements 32 t.. and of the first (h = 0) or second eight
// of the sixteen; kFrom: offset of the first sixteen keys; kNext: how much further the others are.
// Written out, with the wait among them, because the compiler takes this read to depend on the
// loads into other parts of LDS that are on their way, and would wait for those.
template <int kTiles, uint32_t kFrom, uint32_t kNext>
__device__ __forceinline__ void read_transposed(const uint32_t (&at)[kTiles][2], u32x4 (&v)[2][kTiles]) {
  u32x2 x[2][kTiles][2];
  if constexpr (kTiles == 2)
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8 offset:%12\n"
        "ds_read_b64_tr_b16 %1, %9 offset:%12\n"
        "ds_read_b64_tr_b16 %2, %10 offset:%12\n"
        "ds_read_b64_tr_b16 %3, %11 offset:%12\n"
        "ds_read_b64_tr_b16 %4, %8 offset:%13\n"
        "ds_read_b64_tr_b16 %5, %9 offset:%13\n"
        "ds_read_b64_tr_b16 %6, %10 offset:%13\n"
        "ds_read_b64_tr_b16 %7, %11 offset:%13\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0][0]), "=&v"(x[0][0][1]), "=&v"(x[0][1][0]), "=&v"(x[0][1][1]), "=&v"(x[1][0][0]), "=&v"(x[1][0][1]), "=&v"(x[1][1][0]), "=&v"(x[1][1][1])
        : "v"(at[0][0]), "v"(at[0][1]), "v"(at[1][0]), "v"(at[1][1]), "n"(kFrom), "n"(kFrom + kNext)
        : "memory");
  else if constexpr (kTiles == 3)
    asm volatile(
        "ds_read_b64_tr_b16 %0, %12 offset:%18\n"
        "ds_read_b64_tr_b16 %1, %13 offset:%18\n"
        "ds_read_b64_tr_b16 %2, %14 offset:%18\n"
        "ds_read_b64_tr_b16 %3, %15 offset:%18\n"
        "ds_read_b64_tr_b16 %4, %16 offset:%18\n"
        "ds_read_b64_tr_b16 %5, %17 offset:%18\n"
        "ds_read_b64_tr_b16 %6, %12 offset:%19\n"
        "ds_read_b64_tr_b16 %7, %13 offset:%19\n"
        "ds_read_b64_tr_b16 %8, %14 offset:%19\n"
        "ds_read_b64_tr_b16 %9, %15 offset:%19\n"
        "ds_read_b64_tr_b16 %10, %16 offset:%19\n"
        "ds_read_b64_tr_b16 %11, %17 offset:%19\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0][0]), "=&v"(x[0][0][1]), "=&v"(x[0][1][0]), "=&v"(x[0][1][1]), "=&v"(x[0][2][0]), "=&v"(x[0][2][1]), "=&v"(x[1][0][0]), "=&v"(x[1][0][1]), "=&v"(x[1][1][0]), "=&v"(x[1][1][1]), "=&v"(x[1][2][0]), "=&v"(x[1][2][1])
        : "v"(at[0][0]), "v"(at[0][1]), "v"(at[1][0]), "v"(at[1][1]), "v"(at[2][0]), "v"(at[2][1]), "n"(kFrom), "n"(kFrom + kNext)
        : "memory");
  else if constexpr (kTiles == 4)
    asm volatile(
        "ds_read_b64_tr_b16 %0, %16 offset:%24\n"
        "ds_read_b64_tr_b16 %1, %17 offset:%24\n"
        "ds_read_b64_tr_b16 %2, %18 offset:%24\n"
        "ds_read_b64_tr_b16 %3, %19 offset:%24\n"
        "ds_read_b64_tr_b16 %4, %20 offset:%24\n"
        "ds_read_b64_tr_b16 %5, %21 offset:%24\n"
        "ds_read_b64_tr_b16 %6, %22 offset:%24\n"
        "ds_read_b64_tr_b16 %7, %23 offset:%24\n"
        "ds_read_b64_tr_b16 %8, %16 offset:%25\n"
        "ds_read_b64_tr_b16 %9, %17 offset:%25\n"
        "ds_read_b64_tr_b16 %10, %18 offset:%25\n"
        "ds_read_b64_tr_b16 %11, %19 offset:%25\n"
        "ds_read_b64_tr_b16 %12, %20 offset:%25\n"
        "ds_read_b64_tr_b16 %13, %21 offset:%25\n"
        "ds_read_b64_tr_b16 %14, %22 offset:%25\n"
        "ds_read_b64_tr_b16 %15, %23 offset:%25\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0][0]), "=&v"(x[0][0][1]), "=&v"(x[0][1][0]), "=&v"(x[0][1][1]), "=&v"(x[0][2][0]), "=&v"(x[0][2][1]), "=&v"(x[0][3][0]), "=&v"(x[0][3][1]), "=&v"(x[1][0][0]), "=&v"(x[1][0][1]), "=&v"(x[1][1][0]), "=&v"(x[1][1][1]), "=&v"(x[1][2][0]), "=&v"(x[1][2][1]), "=&v"(x[1][3][0]), "=&v"(x[1][3][1])
        : "v"(at[0][0]), "v"(at[0][1]), "v"(at[1][0]), "v"(at[1][1]), "v"(at[2][0]), "v"(at[2][1]), "v"(at[3][0]), "v"(at[3][1]), "n"(kFrom), "n"(kFrom + kNext)
        : "memory");
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int t = 0; t < kTiles; ++t) v[i][t] = u32x4{x[i][t][0].x, x[i][t][0].y, x[i][t][1].x, x[i][t][1].y};
}

struct AttendParams {
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  const uint8_t *keys, *values;
  const float *key_scale, *value_scale;
  const int32_t *starts, *lens, *tables, *fills, *prefix;
  const float *slopes;
  float *parts;  // workspace
  uint64_t q_stride, out_stride;                    // elements
  uint64_t page_stride, head_stride, token_stride;  // bytes
  uint32_t tokens, num_pages, requests, width, heads, kv_heads, D;
  FastDiv page_tokens, group, by_kv;
  float scale, cap;
  uint32_t window;  // 2^31 - 1: none
  // division of the work (see WorkItem)
  uint32_t rows;         // query rows of a tile
  uint32_t from, upto;   // requests with this many rows a key head, from <= rows < upto
  uint32_t least, most;  // key blocks of a part, at least; parts to aim at, all heads together
  uint32_t part_slots;   // parts that the workspace holds, of one head
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// A row of zeros that lanes without a key (or past a head's D) read instead of
// memory that is not theirs: a 0 from here, times any weight, adds nothing.
__device__ __align__(16) static uint32_t kv_zeros[128];

// A request as the kernels see it: every value clamped into its range.
struct Request {
  int32_t start, added, len, prefix;
};

__device__ __forceinline__ Request request_of(const AttendParams &p, uint32_t b) {
  Request r;
  r.start = min(max(p.starts[b], 0), (int32_t)p.tokens);
  r.added = max(min(max(p.starts[b + 1], 0), (int32_t)p.tokens) - r.start, 0);
  r.len = max(p.lens[b], 0);
  r.prefix = p.prefix ? max(p.prefix[b], 0) : 0;
  return r;
}

// The key blocks of kBlock keys that a run of tokens at positions first..last
// sees something of: `head` blocks from 0 (the prefix), then those from `near`
// on (the window), `count` in all.
struct KeyRange {
  int32_t head, near, count, end;  // end: no key from here on is seen
  __device__ __forceinline__ int32_t block(int32_t x) const { return x < head ? x : x - head + near; }
};

template <int kBlock>
__device__ __forceinline__ KeyRange key_range(const AttendParams &p, const Request &r, int32_t first, int32_t last) {
  KeyRange k;
  const int32_t held = (int32_t)min((int64_t)r.len, (int64_t)p.width * p.page_tokens.d);
  const int32_t prefix = min(r.prefix, held);
  k.end = min(held, max(last + 1, prefix));
  const int32_t from = (int32_t)max((int64_t)first - p.window + 1, (int64_t)0);
  k.head = (prefix + kBlock - 1) / kBlock;
  k.near = max(k.head, from / kBlock);
  const int32_t ends = (k.end + kBlock - 1) / kBlock;
  k.count = k.head + max(ends - k.near, 0);
  return k;
}

// ---------------------------------------------------------------------------
// Division of the work.  A tile is `rows` query rows (token x head of the
// group) of one request and key head; a part is a run of key blocks of a
// tile.  How long the requests are is known on the GPU only, so every block
// of threads finds its own part: it sums the key blocks of all tiles, takes
// from that the length c of a part (so that about `most` parts come out, none
// shorter than `least`), and walks the requests' numbers of parts up to its
// own index.  That is two passes over a few lengths in L2; a kernel that did
// it once before would cost a launch.
// ---------------------------------------------------------------------------
struct WorkItem {
  uint32_t request, tile, part;
  uint32_t parts;      // of each of the request's tiles, 1: undivided
  uint32_t slot;       // in the workspace, if divided
  uint32_t c;          // key blocks of a part
  Request r;
};

__device__ __forceinline__ uint32_t tiles_of(const AttendParams &p, const Request &r) {
  const uint32_t rows = (uint32_t)r.added * p.group.d;
  return (rows >= p.from) & (rows < p.upto) ? (rows + p.rows - 1) / p.rows : 0;
}

template <int kThreads>
__device__ __forceinline__ uint32_t scan_threads(uint32_t v, uint32_t *sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t up = __shfl_up(v, d);
    if (lane >= d) v += up;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w)
    if (w < wave) v += sums[w];
  return v;
}

// Item number `index` of the call, or false if there are not as many.  With
// kJoin the items are the divided tiles themselves (which a second kernel
// joins), and part is 0.  Every thread of the block gets the same answer.
template <int kThreads, int kBlock, bool kJoin>
__device__ bool find_item(const AttendParams &p, uint32_t index, WorkItem &item) {
  __shared__ uint32_t s_sums[kThreads / 64];
  __shared__ uint64_t s_work[kThreads / 64];
  __shared__ WorkItem s_item;
  __shared__ int s_found;
  uint64_t work = 0;
  for (uint32_t b = threadIdx.x; b < p.requests; b += kThreads) {
    const Request r = request_of(p, b);
    const uint32_t tiles = tiles_of(p, r);
    if (tiles) work += (uint64_t)tiles * key_range<kBlock>(p, r, r.len - r.added, r.len - 1).count;
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) work += __shfl_xor(work, d);
  if ((threadIdx.x & 63) == 0) s_work[threadIdx.x >> 6] = work;
  if (threadIdx.x == 0) s_found = 0;
  __syncthreads();
  work = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) work += s_work[w];
  const uint64_t each = (work * p.kv_heads + p.most - 1) / p.most;
  const uint32_t c = (uint32_t)min(max(each, (uint64_t)p.least), (uint64_t)1 << 30);
  uint32_t items0 = 0, slots0 = 0;
  for (uint32_t b0 = 0; b0 < p.requests; b0 += kThreads) {
    const uint32_t b = b0 + threadIdx.x;
    WorkItem mine;
    uint32_t tiles = 0, items = 0, slots = 0;
    mine.parts = 1;
    if (b < p.requests) {
      mine.r = request_of(p, b);
      tiles = tiles_of(p, mine.r);
      if (tiles) {
        const uint32_t blocks = key_range<kBlock>(p, mine.r, mine.r.len - mine.r.added, mine.r.len - 1).count;
        mine.parts = max((blocks + c - 1) / c, 1u);
        slots = mine.parts > 1 ? tiles * mine.parts : 0;
        items = kJoin ? (mine.parts > 1 ? tiles : 0) : tiles * mine.parts;
      }
    }
    const uint32_t items1 = items0 + scan_threads<kThreads>(items, s_sums);
    const uint32_t slots1 = slots0 + scan_threads<kThreads>(slots, s_sums);
    if (index < items1 && index >= items1 - items) {
      const uint32_t at = index - (items1 - items), per = kJoin ? 1 : mine.parts;
      mine.request = b;
      // the last tiles of a chunk see the most keys: they begin first
      const uint32_t from_end = at / per;
      mine.tile = tiles - 1 - from_end;
      mine.part = at - from_end * per;
      mine.slot = slots1 - slots + from_end * mine.parts + mine.part;
      mine.c = c;
      s_item = mine;
      s_found = 1;
    }
    __syncthreads();
    if (s_found) break;
    if (threadIdx.x == kThreads - 1) s_sums[0] = items1, s_work[0] = slots1;
    __syncthreads();
    items0 = s_sums[0];
    slots0 = (uint32_t)s_work[0];
    __syncthreads();
  }
  if (!s_found) return false;
  // the same for all: into scalar registers
  auto one = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
  item.request = one(s_item.request);
  item.tile = one(s_item.tile);
  item.part = one(s_item.part);
  item.parts = one(s_item.parts);
  item.slot = one(s_item.slot);
  item.c = one(s_item.c);
  item.r.start = (int32_t)one((uint32_t)s_item.r.start);
  item.r.added = (int32_t)one((uint32_t)s_item.r.added);
  item.r.len = (int32_t)one((uint32_t)s_item.r.len);
  item.r.prefix = (int32_t)one((uint32_t)s_item.r.prefix);
  return true;
}

// Rows of a tile: row n is token n / group of the request's new ones, head
// n % group of the key head's.
struct Tile {
  uint32_t row0, rows;    // first row, rows
  int32_t first, last;    // positions of its first and last token
};

__device__ __forceinline__ Tile tile_of(const AttendParams &p, const WorkItem &w) {
  Tile t;
  const uint32_t all = (uint32_t)w.r.added * p.group.d;
  t.row0 = w.tile * p.rows;
  t.rows = min(p.rows, all - t.row0);
  const int32_t base = w.r.len - w.r.added;
  t.first = base + (int32_t)fastdiv(t.row0, p.group);
  t.last = base + (int32_t)fastdiv(t.row0 + t.rows - 1, p.group);
  return t;
}

// One lane's look at a key's table entry.  What it loads is judged where it is needed, a block
// later: a comparison beside the load would wait for it, and for every load issued before.
struct KeyLook {
  int32_t page, fill;  // as the tables have them
  uint32_t place;
  bool seen;  // by some row of the tile: whatever other keys' values hold does not reach them
};

__device__ __forceinline__ KeyLook key_look(const AttendParams &p, const WorkItem &w, const Tile &t, bool in_part,
                                            int32_t j, int32_t end) {
  KeyLook k;
  const bool near = (j <= t.last) & ((int64_t)t.first - j < (int64_t)p.window);
  k.seen = in_part & (j < end) & (near | (j < w.r.prefix));
  const uint32_t at = (uint32_t)(k.seen ? j : 0), e = fastdiv(at, p.page_tokens);
  k.place = at - e * p.page_tokens.d;
  const uint64_t entry = (uint64_t)w.request * p.width + e;
  k.page = p.tables[entry];
  k.fill = p.fills ? p.fills[entry] : 0x7FFFFFFF;
  return k;
}

__device__ __forceinline__ bool key_there(const AttendParams &p, const KeyLook &k) {
  return k.seen & ((uint32_t)k.page < p.num_pages) & ((int32_t)k.place < k.fill);
}

__device__ __forceinline__ float xor32(float x, float (*op)(float, float)) {
  const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float xor16(float x, float (*op)(float, float)) {
  const u32x2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float sum_of(float a, float b) { return a + b; }

// The largest of three, NaN passed over.  Written out: fmaxf of values that may be signalling
// NaN quiets each of them first, an instruction a value.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// 2^x; -inf gives 0.
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

// Scores that are capped or biased, in log2: products x -> x * factor, or
// cap tanh(x scale / cap) log2 e, less slope * distance * log2 e.  With
// E = 2^(2 x scale / cap log2 e), tanh = 1 - 2 / (1 + E), which is right at
// both ends of E's range too; the quotient is below 1 and good to 2^-23, so the
// result to about 2^-22 of the cap.
struct ScoreChange {
  float factor, cap, twice, by, slope;
  __device__ __forceinline__ ScoreChange(float scale, float cap_, float slope_)
      : factor(scale * kLog2e), cap(cap_ * kLog2e), twice(-2.f * cap_ * kLog2e),
        by(cap_ > 0.f ? 2.f * kLog2e * scale / cap_ : 0.f), slope(-slope_ * kLog2e) {}
  __device__ __forceinline__ float capped(float x) const {
    return __builtin_fmaf(twice, __builtin_amdgcn_rcpf(1.f + pow2(x * by)), cap);
  }
  // y less the bias at this distance
  __device__ __forceinline__ float biased(float y, float distance) const {
    return __builtin_fmaf(slope, fabsf(distance), y);
  }
};

// Values that are NaN or inf, two 16-bit elements a word.
template <typename Q>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {  // all ones where an element is
  const uint32_t e = Q::kF16 ? 0x7C00u : 0x7F80u;
  return ((w & e) == e ? 0xFFFFu : 0u) | ((w >> 16 & e) == e ? 0xFFFF0000u : 0u);
}
template <typename Q>
__device__ __forceinline__ bool any_not_finite(uint32_t w) {
  return not_finite<Q>(w) != 0;
}
template <typename Q>
__device__ __forceinline__ bool any_not_finite4(u32x4 a) {
  return any_not_finite<Q>(a.x) | any_not_finite<Q>(a.y) | any_not_finite<Q>(a.z) | any_not_finite<Q>(a.w);
}
template <typename Q>
__device__ __forceinline__ u32x4 finite_only(u32x4 a) {
#pragma unroll
  for (int i = 0; i < 4; ++i) a[i] &= ~not_finite<Q>(a[i]);
  return a;
}
// What the NaN and inf among values `a` give a sum over the keys with a 1 in `seen`: the
// values of +inf or NaN and those of -inf or NaN are counted by two products, and a count
// stands for +inf, or -inf, whose sum is NaN where both are.
template <typename Q>
__device__ __forceinline__ u32x4 sign_ones(u32x4 a, bool negative) {
  u32x4 ones;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w = 0;
#pragma unroll
    for (int h = 0; h < 32; h += 16) {
      const uint32_t x = a[i] >> h & 0xFFFFu, e = Q::kF16 ? 0x7C00u : 0x7F80u;
      const bool nan = (x & 0x7FFFu) > e, inf = (x & 0x7FFFu) == e && (x >> 15) == (negative ? 1u : 0u);
      if (nan || inf) w |= (Q::kF16 ? 0x3C00u : 0x3F80u) << h;
    }
    ones[i] = w;
  }
  return ones;
}
__device__ __forceinline__ float not_finite_sum(float up, float down) {
  return (up > 0.f ? INFINITY : 0.f) + (down > 0.f ? -INFINITY : 0.f);
}
template <typename Q>
__device__ __forceinline__ f32x4 not_finite_part(u32x4 a, u32x4 seen) {
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  const f32x4 up = Q::mfma16(sign_ones<Q>(a, false), seen, zero), down = Q::mfma16(sign_ones<Q>(a, true), seen, zero);
  f32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = not_finite_sum(up[i], down[i]);
  return r;
}

// LDS written by some lanes of a wave and read by others of the same wave:
// the hardware keeps their order, the compiler has to.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

}  // namespace gorio
