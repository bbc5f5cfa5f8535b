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

#include <type_traits>

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
  // Two values of 8 bits, or of 4, times a power of two: the nearest of this type, exactly the
  // product where it has one.  `by` may be 0 for 2^-127 and inf for NaN: its exponent's bits count.
  template <bool kHi>
  static __device__ __forceinline__ uint32_t widen(uint32_t w, float by) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, by, kHi));
  }
  template <int kByte>
  static __device__ __forceinline__ uint32_t widen4(uint32_t w, float by) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, by, kByte));
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
  static __device__ __forceinline__ uint32_t widen(uint32_t w, float by) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, by, kHi));
  }
  template <int kByte>
  static __device__ __forceinline__ uint32_t widen4(uint32_t w, float by) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, by, kByte));
  }
};

// What pages hold: 16-bit elements, e4m3 by a factor a head, e4m3 and e2m1 by a power of two for
// each 32 of a row.
enum PageKind : int { kPages16, kPagesE4m3, kPagesMx8, kPagesMx4 };
template <int kPages>
struct PageOf {
  static constexpr bool kMx = kPages >= kPagesMx8;
  static constexpr uint32_t bytes(uint32_t elements) {
    return kPages == kPages16 ? elements * 2 : kPages == kPagesMx4 ? elements / 2 : elements;
  }
  // eight elements as they lie
  typedef typename std::conditional<kPages == kPages16, u32x4,
                                    typename std::conditional<kPages == kPagesMx4, uint32_t, u32x2>::type>::type Raw;
  // the offset of a row's powers, from that of its elements
  static __device__ __forceinline__ uint64_t powers(uint64_t bytes) { return bytes >> (kPages == kPagesMx4 ? 4 : 5); }
};

// Eight elements as they lie in the pages -> eight of the queries' type.
template <typename Q>
__device__ __forceinline__ u32x4 widened(u32x4 r, float = 1.f) {
  return r;
}
template <typename Q>
__device__ __forceinline__ u32x4 widened(u32x2 r, float by = 1.f) {
  return u32x4{Q::template widen<false>(r.x, by), Q::template widen<true>(r.x, by), Q::template widen<false>(r.y, by),
               Q::template widen<true>(r.y, by)};
}
template <typename Q>
__device__ __forceinline__ u32x4 widened(uint32_t r, float by) {
  return u32x4{Q::template widen4<0>(r, by), Q::template widen4<1>(r, by), Q::template widen4<2>(r, by),
               Q::template widen4<3>(r, by)};
}
// The first four of them.
template <typename Q>
__device__ __forceinline__ u32x4 widened_half(u32x2 r, float by) {
  return u32x4{Q::template widen<false>(r.x, by), Q::template widen<true>(r.x, by), 0, 0};
}
template <typename Q>
__device__ __forceinline__ u32x4 widened_half(uint32_t r, float by) {
  return u32x4{Q::template widen4<0>(r, by), Q::template widen4<1>(r, by), 0, 0};
}
template <typename Q>
__device__ __forceinline__ u32x4 widened_half(u32x4 r, float) {  // 16-bit pages have no halves
  return r;
}
// A power's byte as such a factor.
__device__ __forceinline__ float power_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Memory by its address.  Without the address space it would be read as what may be LDS, and every
// wait for LDS would wait for the loads that are on their way.
template <typename T>
__device__ __forceinline__ T load_at(uint64_t address) {
  return *(const __attribute__((address_space(1))) T *)(uintptr_t)address;
}

// LDS by its 32-bit address: what is added to one as a constant goes into the instruction.
typedef __attribute__((address_space(3))) uint8_t LdsBytes;
template <typename T>
__device__ __forceinline__ __attribute__((address_space(3))) T *lds_at(uint32_t address) {
  return (__attribute__((address_space(3))) T *)(uintptr_t)address;
}

// Transposing LDS reads of sixteen keys' values at 32 kTiles elements: in each, lane l of 16
// names the 8 bytes that hold elements 4 (l % 4) .. + 3 of a key l / 4, and gets element l of the
// four keys.  at[t][h]: address of elements 32 t.. of the first (h = 0) or second eight of the
// sixteen, less kFrom.
// Written out, with the wait among them, because the compiler takes this read to depend on the
// loads into other parts of LDS that are on their way, and would wait for those.
template <int kTiles, uint32_t kFrom>
__device__ __forceinline__ void read_transposed(const uint32_t (&at)[kTiles][2], u32x4 (&v)[kTiles]) {
  u32x2 x[kTiles][2];
  if constexpr (kTiles == 2)
    asm volatile(
        "ds_read_b64_tr_b16 %0, %4 offset:%8\n"
        "ds_read_b64_tr_b16 %1, %5 offset:%8\n"
        "ds_read_b64_tr_b16 %2, %6 offset:%8\n"
        "ds_read_b64_tr_b16 %3, %7 offset:%8\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1])
        : "v"(at[0][0]), "v"(at[0][1]), "v"(at[1][0]), "v"(at[1][1]), "n"(kFrom)
        : "memory");
  else if constexpr (kTiles == 3)
    asm volatile(
        "ds_read_b64_tr_b16 %0, %6 offset:%12\n"
        "ds_read_b64_tr_b16 %1, %7 offset:%12\n"
        "ds_read_b64_tr_b16 %2, %8 offset:%12\n"
        "ds_read_b64_tr_b16 %3, %9 offset:%12\n"
        "ds_read_b64_tr_b16 %4, %10 offset:%12\n"
        "ds_read_b64_tr_b16 %5, %11 offset:%12\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1])
        : "v"(at[0][0]), "v"(at[0][1]), "v"(at[1][0]), "v"(at[1][1]), "v"(at[2][0]), "v"(at[2][1]), "n"(kFrom)
        : "memory");
  else if constexpr (kTiles == 4)
    asm volatile(
        "ds_read_b64_tr_b16 %0, %8 offset:%16\n"
        "ds_read_b64_tr_b16 %1, %9 offset:%16\n"
        "ds_read_b64_tr_b16 %2, %10 offset:%16\n"
        "ds_read_b64_tr_b16 %3, %11 offset:%16\n"
        "ds_read_b64_tr_b16 %4, %12 offset:%16\n"
        "ds_read_b64_tr_b16 %5, %13 offset:%16\n"
        "ds_read_b64_tr_b16 %6, %14 offset:%16\n"
        "ds_read_b64_tr_b16 %7, %15 offset:%16\n"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(x[0][0]), "=&v"(x[0][1]), "=&v"(x[1][0]), "=&v"(x[1][1]), "=&v"(x[2][0]), "=&v"(x[2][1]), "=&v"(x[3][0]), "=&v"(x[3][1])
        : "v"(at[0][0]), "v"(at[0][1]), "v"(at[1][0]), "v"(at[1][1]), "v"(at[2][0]), "v"(at[2][1]), "v"(at[3][0]), "v"(at[3][1]), "n"(kFrom)
        : "memory");
#pragma unroll
  for (int t = 0; t < kTiles; ++t) v[t] = u32x4{x[t][0].x, x[t][0].y, x[t][1].x, x[t][1].y};
}

struct AttendParams {
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  const uint8_t *keys, *values;
  const float *key_scale, *value_scale;
  const uint8_t *key_powers, *value_powers;
  const int32_t *starts, *lens, *tables, *fills, *prefix;
  const float *slopes;
  float *parts;  // workspace
  // Shared prefixes (NULL without): group g is requests first[g]..first[g + 1], and request b's
  // positions below shared[b] lie in the pages of its group's first.  A launch of its own, in which
  // a group stands for a request, leaves of each row the sums over those positions in `carry`
  // (D floats a row, all rows, then their maximum and sum of weights); the launches after it
  // start behind them and add these.
  const int32_t *first, *shared;
  float *carry;
  uint32_t all_requests;
  bool grouped;  // this launch's requests are groups (the joining kernel asks; the others are made for it)
  uint64_t q_stride, out_stride;                    // elements
  uint64_t page_stride, head_stride, token_stride;  // bytes
  uint32_t tokens, num_pages, requests, width, heads, kv_heads, D;
  FastDiv page_tokens, group, by_kv;
  float scale, cap;
  uint32_t window;  // 2^31 - 1: none
  // division of the work (see WorkItem)
  uint32_t rows;         // query rows of a tile
  uint32_t from, upto;   // requests with this many rows a key head, from <= rows < upto
  uint32_t shares, least;  // workgroups of a key head, at most; key blocks of a share, at least
  uint32_t whole;          // key blocks of a tile that is not cut, at most
  uint32_t pad;            // of a tile on the line, at least
  bool cuts;               // a tile may be cut
};

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// 2^x; -inf gives 0.
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

// A row of zeros that lanes without a key (or past a head's D) read instead of
// memory that is not theirs: a 0 from here, times any weight, adds nothing.
__device__ __align__(16) static uint32_t kv_zeros[128];

// A request as the kernels see it: every value clamped into its range.
struct Request {
  int32_t start, added, len, prefix;
  int32_t skip;  // positions that were computed for the group
  uint32_t row;  // of the tables
};

// Shared positions that are computed for the group: whole blocks of either form, so that the
// requests' own blocks begin where the group's end.
constexpr int32_t kSharedBlock = 64;
__device__ __forceinline__ int32_t shared_of(const AttendParams &p, uint32_t b) {
  const int64_t held = (int64_t)p.width * p.page_tokens.d;  // below 2^31
  return (int32_t)min((int64_t)max(p.shared[b], 0), held) & -kSharedBlock;
}

// A group as a request: its requests' tokens, which follow one another, and the shared positions.
__device__ __forceinline__ uint32_t first_of(const AttendParams &p, uint32_t g) {
  return (uint32_t)min(max(p.first[g], 0), (int32_t)p.all_requests);
}
__device__ __forceinline__ Request group_of(const AttendParams &p, uint32_t g) {
  Request r{};
  r.row = first_of(p, g);
  const uint32_t end = first_of(p, g + 1);
  if (r.row >= end) return r;
  r.len = r.prefix = shared_of(p, r.row);
  r.start = min(max(p.starts[r.row], 0), (int32_t)p.tokens);
  r.added = r.len ? max(min(max(p.starts[end], 0), (int32_t)p.tokens) - r.start, 0) : 0;
  return r;
}

// kGroup: the launch's requests are groups.
template <bool kGroup>
__device__ __forceinline__ Request request_of(const AttendParams &p, uint32_t b) {
  if constexpr (kGroup) return group_of(p, b);
  Request r;
  r.row = b;
  r.skip = p.shared ? shared_of(p, b) : 0;
  r.start = min(max(p.starts[b], 0), (int32_t)p.tokens);
  r.added = max(min(max(p.starts[b + 1], 0), (int32_t)p.tokens) - r.start, 0);
  r.len = max(p.lens[b], 0);
  r.prefix = p.prefix ? max(p.prefix[b], 0) : 0;
  return r;
}

// The key blocks of kBlock keys that a run of tokens at positions first..last
// sees something of: `head` blocks from `skip` on (the prefix), then those from
// `near` on (the window), `count` in all.
struct KeyRange {
  int32_t skip, head, near, count, end;  // end: no key from here on is seen
  __device__ __forceinline__ int32_t block(int32_t x) const { return x < head ? x + skip : x - head + near; }
};

template <int kBlock>
__device__ __forceinline__ KeyRange key_range(const AttendParams &p, const Request &r, int32_t first, int32_t last) {
  KeyRange k;
  const int32_t held = (int32_t)min((int64_t)r.len, (int64_t)p.width * p.page_tokens.d);
  const int32_t prefix = min(r.prefix, held);
  k.end = min(held, max(last + 1, prefix));
  const int32_t from = (int32_t)max((int64_t)first - p.window + 1, (int64_t)0);
  k.skip = r.skip / kBlock;
  const int32_t seen = max((prefix + kBlock - 1) / kBlock, k.skip);
  k.head = seen - k.skip;
  k.near = max(seen, from / kBlock);
  const int32_t ends = (k.end + kBlock - 1) / kBlock;
  k.count = k.head + max(ends - k.near, 0);
  return k;
}

// ---------------------------------------------------------------------------
// Division of the work.  A tile is `rows` query rows (token x head of the
// group) of one request and key head.  Of each key head, the key blocks of all
// tiles, one tile after the other, make a line of W blocks, and workgroup i of
// the head takes an equal share of it: blocks i c .. (i + 1) c - 1, whatever
// tiles they belong to.  So all workgroups run equally long, however ragged the
// lengths (but for tiles of a few blocks, which cost more than their blocks),
// and a tile is cut only where a share ends in it.  A tile of up to
// `whole` blocks is not cut but goes to the share it begins in: parts of so few
// blocks would cost more than they save.  What a workgroup computes of a cut
// tile is a part: its sums go to the workspace, where it has two slots (a share
// cuts at most the tile it begins in and the one it ends in), and a second
// kernel joins them.
//
// How long the requests are is known on the GPU only, so every workgroup finds
// its share by itself: the tiles' blocks are counted and added up, in chunks of
// as many tiles as there are threads, from a few lengths in L2.  A kernel that
// did it once before would cost a launch.
// ---------------------------------------------------------------------------
struct WorkItem {
  uint32_t request, tile, tiles;  // tile of the request's tiles
  uint64_t begin;                 // of the tile on the line
  uint64_t share, line;           // c and W
  Request r;
};

__device__ __forceinline__ uint32_t tiles_of(const AttendParams &p, const Request &r) {
  const uint32_t rows = (uint32_t)r.added * p.group.d;
  return ((rows >= p.from) & (rows < p.upto)) ? (rows + p.rows - 1) / p.rows : 0;
}

// Rows of a tile: row n is token n / group of the request's new ones, head
// n % group of the key head's.
struct Tile {
  uint32_t row0, rows;  // first row, rows
  int32_t first, last;  // positions of its first and last token
};

__device__ __forceinline__ Tile tile_of(const AttendParams &p, const Request &r, uint32_t tile) {
  Tile t;
  const uint32_t all = (uint32_t)r.added * p.group.d;
  t.row0 = tile * p.rows;
  t.rows = min(p.rows, all - t.row0);
  const int32_t base = r.len - r.added;
  t.first = base + (int32_t)fastdiv(t.row0, p.group);
  t.last = base + (int32_t)fastdiv(t.row0 + t.rows - 1, p.group);
  return t;
}

// A tile's blocks on the line: one at least, so that a tile that sees nothing is written by someone.
template <int kBlock>
__device__ __forceinline__ uint32_t blocks_of(const AttendParams &p, const Request &r, uint32_t tile) {
  const Tile t = tile_of(p, r, tile);
  return max((uint32_t)max(key_range<kBlock>(p, r, t.first, t.last).count, 1), p.pad);
}

// Inclusive sum over the threads, in thread order.
template <int kThreads, typename T>
__device__ __forceinline__ T scan_threads(T v, T *sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const T up = __shfl_up(v, d);
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

// A value that is the same for all lanes, into scalar registers.
__device__ __forceinline__ uint64_t one(uint64_t v) {
  return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 |
         (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)v);
}
__device__ __forceinline__ Request one(const Request &r) {
  return Request{__builtin_amdgcn_readfirstlane(r.start), __builtin_amdgcn_readfirstlane(r.added),
                 __builtin_amdgcn_readfirstlane(r.len), __builtin_amdgcn_readfirstlane(r.prefix),
                 __builtin_amdgcn_readfirstlane(r.skip), (uint32_t)__builtin_amdgcn_readfirstlane((int)r.row)};
}

// The tile of the block that share number `index` begins with, or false if the line ends before.
// Every thread of the workgroup gets the same answer.
template <int kThreads, int kBlock, bool kGroup>
__device__ bool find_item(const AttendParams &p, uint32_t index, WorkItem &item) {
  __shared__ uint64_t s_sums[kThreads / 64], s_begin, s_line;
  __shared__ uint32_t s_tiles[kThreads], s_counts[kThreads / 64], s_found[2];  // request, tile
  __shared__ Request s_request;
  if (threadIdx.x == 0) s_found[0] = ~0u;
  uint64_t line = 0, share = 0;
  // this thread's tile, of the chunk last counted
  uint64_t begin = 0, end = 0;
  uint32_t request = 0, tile = 0;
  Request its{};
  bool once = true;  // there is one chunk only
  auto take = [&]() {
    const uint64_t at = (uint64_t)index * share;
    if (at >= begin && at < end) s_found[0] = request, s_found[1] = tile, s_begin = begin, s_request = its;
  };
  // twice over the tiles, unless they are few: W is known after the first pass
  for (int pass = 0; pass < 2; ++pass) {
    uint64_t at = 0;  // on the line, of the next tile
    for (uint32_t b0 = 0; b0 < p.requests; b0 += kThreads) {
      const uint32_t b = b0 + threadIdx.x;
      Request own{};
      if (b < p.requests) own = request_of<kGroup>(p, b);
      const uint32_t mine = b < p.requests ? tiles_of(p, own) : 0;
      if (!__syncthreads_or(mine > 1)) {  // single tokens: a thread's request is its tile
        request = b;
        tile = 0;
        its = own;
        const uint32_t blocks = mine ? blocks_of<kBlock>(p, own, 0) : 0;
        end = at + scan_threads<kThreads>((uint64_t)blocks, s_sums);
        begin = end - blocks;
        if (pass) take();
        if (threadIdx.x == kThreads - 1) s_line = end;
        __syncthreads();
        at = s_line;
        once &= p.requests <= kThreads;
        __syncthreads();
        if (pass && s_found[0] != ~0u) break;
        continue;
      }
      const uint32_t upto = scan_threads<kThreads>(mine, s_counts);
      s_tiles[threadIdx.x] = upto;
      __syncthreads();
      const uint32_t tiles = s_tiles[kThreads - 1];
      once &= p.requests <= kThreads && tiles <= kThreads;
      for (uint32_t f0 = 0; f0 < tiles; f0 += kThreads) {
        const uint32_t f = f0 + threadIdx.x;
        uint32_t blocks = 0, r = 0;
        if (f < tiles) {
          uint32_t hi = kThreads - 1;  // the first request whose tiles reach past f
          while (r < hi) {
            const uint32_t mid = (r + hi) / 2;
            if (s_tiles[mid] > f) hi = mid;
            else r = mid + 1;
          }
          tile = f - (r ? s_tiles[r - 1] : 0);
          request = b0 + r;
          its = request_of<kGroup>(p, request);
          blocks = blocks_of<kBlock>(p, its, tile);
        }
        end = at + scan_threads<kThreads>((uint64_t)blocks, s_sums);
        begin = end - blocks;
        if (pass) take();
        if (threadIdx.x == kThreads - 1) s_line = end;
        __syncthreads();
        at = s_line;
      }
      __syncthreads();
      if (pass && s_found[0] != ~0u) break;
    }
    if (pass == 0) {
      line = at;
      share = max((line + p.shares - 1) / p.shares, (uint64_t)p.least);
      if (once) {
        take();
        __syncthreads();
        break;
      }
    }
  }
  if (s_found[0] == ~0u) return false;
  item.request = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_found[0]);
  item.tile = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_found[1]);
  item.begin = one(s_begin);
  item.line = one(line);
  item.share = one(share);
  item.r = one(s_request);
  item.tiles = tiles_of(p, item.r);
  return true;
}

// The tile after w's on the line, if the line goes on.  Requests of the other form between two are
// passed one at a time, each a wait for its lengths: 4 prompts of 200 tokens spread among 2000
// single tokens take 803 us together, in front of them 683.
template <bool kGroup>
__device__ __forceinline__ bool next_item(const AttendParams &p, WorkItem &w, uint64_t begin) {
  w.begin = begin;
  if (++w.tile < w.tiles) return true;
  w.tile = 0;
  do {
    if (++w.request >= p.requests) return false;
    w.r = one(request_of<kGroup>(p, w.request));
    w.tiles = tiles_of(p, w.r);
  } while (w.tiles == 0);
  return true;
}

// What share number `index` computes of tile w: blocks from..upto - 1 of the tile, none if the
// tile begins in the share before and is not cut.
struct Part {
  uint32_t from, upto;
  uint32_t slot;
  bool divided, none;
};

__device__ __forceinline__ Part part_of(const AttendParams &p, const WorkItem &w, uint32_t blocks, uint32_t index) {
  // blocks: the tile's own, without what it is padded by; a tile that may be cut is not padded
  const uint64_t begin = index * w.share, end = min(begin + w.share, w.line);
  Part a{0, blocks, index * 2 + (w.begin > begin ? 1 : 0), false, false};
  if (blocks <= p.whole) {
    a.none = w.begin < begin;
  } else {
    a.from = (uint32_t)(max(begin, w.begin) - w.begin);
    a.upto = (uint32_t)(min(end, w.begin + blocks) - w.begin);
    a.divided = a.from > 0 || a.upto < blocks;
  }
  return a;
}

// Rows of a group's tile: each has its own request's position and prefix.
struct RowSees {
  int32_t pos, prefix;
};
struct TileSees {
  int32_t first, last, prefix;  // least and largest position, least prefix
};

// Fills in `rows` for the tile's rows and returns what all of them see, the same to all threads.
// Rows past the last repeat it.
template <int kThreads, int kRows>
__device__ TileSees place_rows(const AttendParams &p, const WorkItem &w, const Tile &tile, RowSees *rows) {
  static_assert(kRows <= kThreads, "a thread a row");
  __shared__ TileSees s_sees[kThreads / 64];
  __shared__ int32_t s_starts[kThreads];
  const uint32_t row = tile.row0 + min((uint32_t)threadIdx.x, tile.rows - 1);
  const int32_t token = w.r.start + (int32_t)fastdiv(row, p.group);
  RowSees mine{-1, 0};  // of no request: sees nothing
  // the group's request that has the token: the last that begins at or before it, by a bisection
  // in LDS of every so many-th request's start, and among those between in memory
  const uint32_t count = first_of(p, w.request + 1) - w.r.row, step = (count + kThreads - 1) / kThreads;
  if (threadIdx.x * step < count) s_starts[threadIdx.x] = p.starts[w.r.row + threadIdx.x * step];
  __syncthreads();
  if (threadIdx.x < kRows) {
    uint32_t lo = 0, hi = (count - 1) / step;
    while (lo < hi) {
      const uint32_t mid = (lo + hi + 1) / 2;
      if (s_starts[mid] <= token) lo = mid;
      else hi = mid - 1;
    }
    lo = w.r.row + lo * step;
    hi = min(lo + step, w.r.row + count) - 1;
    while (lo < hi) {
      const uint32_t mid = lo + (hi - lo + 1) / 2;
      if (p.starts[mid] <= token) lo = mid;
      else hi = mid - 1;
    }
    const int32_t from = min(max(p.starts[lo], 0), (int32_t)p.tokens), upto = min(max(p.starts[lo + 1], 0), (int32_t)p.tokens);
    const int32_t len = max(p.lens[lo], 0), prefix = p.prefix ? min(max(p.prefix[lo], 0), len) : 0;
    if (token >= from && token < upto) mine = RowSees{len - (upto - token), prefix};
    rows[threadIdx.x] = mine;
  }
  TileSees s{0x7FFFFFFF, -1, 0x7FFFFFFF};
  if (threadIdx.x < kRows) s = TileSees{mine.pos, mine.pos, mine.prefix};
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    s.first = min(s.first, __shfl_xor(s.first, d));
    s.last = max(s.last, __shfl_xor(s.last, d));
    s.prefix = min(s.prefix, __shfl_xor(s.prefix, d));
  }
  if ((threadIdx.x & 63) == 0) s_sees[threadIdx.x >> 6] = s;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) {
    s.first = min(s.first, s_sees[i].first);
    s.last = max(s.last, s_sees[i].last);
    s.prefix = min(s.prefix, s_sees[i].prefix);
  }
  return TileSees{__builtin_amdgcn_readfirstlane(s.first), __builtin_amdgcn_readfirstlane(s.last),
                  __builtin_amdgcn_readfirstlane(s.prefix)};
}

// A row's sums over its group's shared positions: where they lie, and how they count beside sums
// over others with the maximum `best`.
struct Carried {
  const float *o;
  float m, l, by;  // maximum, sum of weights, factor of both
};
__device__ __forceinline__ uint64_t carried_row(const AttendParams &p, uint64_t token, uint32_t head) {
  return token * p.heads + head;
}
__device__ __forceinline__ float *carried_sums(const AttendParams &p, uint64_t row) {
  return p.carry + (uint64_t)p.tokens * p.heads * p.D + row * 2;
}
// Takes them in: `best` becomes the larger maximum; returns the factor of the sums that had it.
__device__ __forceinline__ float take_carried(const AttendParams &p, uint64_t row, float &best, Carried &c) {
  const float *ml = carried_sums(p, row);
  c.o = p.carry + row * p.D;
  c.m = ml[0];
  c.l = ml[1];
  const float most = fmaxf(best, c.m), from = most == -INFINITY ? 0.f : most;
  const float keep = pow2(best - from);
  c.by = pow2(c.m - from);
  best = most;
  return keep;
}

// What the joining kernel needs of the tile that begins in a share and is cut at its end; parts
// is 0 if there is none.  Written by the share's workgroup behind the parts' sums: to find the
// tile again from the lengths took the joining kernel 12 us for 264 tiles.
struct Cut {
  int32_t start;         // of the request's tokens
  uint32_t row0, rows;   // of the tile
  uint32_t slot, parts;  // of its first part, and how many; the others begin their shares
};

template <int kRows>
__device__ __forceinline__ Cut *cuts_of(const AttendParams &p) {
  return reinterpret_cast<Cut *>(p.parts + (uint64_t)p.shares * 2 * p.kv_heads * kRows * (p.D + 2));
}

// At a workgroup's end: `part` of tile w is its last.  A call of which no tile is cut has no room for it.
template <int kRows>
__device__ __forceinline__ void note_cut(const AttendParams &p, uint32_t index, uint32_t head, const WorkItem &w,
                                         const Tile &tile, const Part &part, uint32_t blocks) {
  if (threadIdx.x != 0 || !p.cuts) return;
  const bool here = part.divided && part.from == 0;
  const uint32_t last = (uint32_t)((w.begin + blocks - 1) / w.share);
  cuts_of<kRows>(p)[index * p.kv_heads + head] = Cut{w.r.start, tile.row0, tile.rows, part.slot, here ? last - index + 1 : 0};
}
template <int kRows>
__device__ __forceinline__ void note_cut(const AttendParams &p, uint32_t index, uint32_t head) {
  if (threadIdx.x == 0 && p.cuts) cuts_of<kRows>(p)[index * p.kv_heads + head] = Cut{0, 0, 0, 0, 0};
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
  const uint64_t entry = (uint64_t)w.r.row * p.width + e;
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

// The largest, NaN passed over (where all of a pair are NaN, it may be +inf).  Written out: fmaxf
// of values that may be signalling NaN quiets each of them first, an instruction a value.  The
// first two are compared by the compiler, as the middle one of them and +inf: it then waits, if it
// has to, until the matrix instruction that gives the scores is done, which it does not do for
// registers that inline assembly reads.  kReciprocals: capped scores may come from a reciprocal
// right before the assembly, which waits a state for it itself.
template <bool kReciprocals>
__device__ __forceinline__ float max16(const f32x16 &s) {
  float inf = INFINITY;
  asm volatile("" : "+s"(inf));  // the middle of three with a constant inf would become fmaxf
  float r = __builtin_amdgcn_fmed3f(s[0], s[1], inf);
#define GORIO_MAX14(first)                                                                                            \
  asm(first "v_max3_f32 %0, %0, %1, %2\n"                                                                             \
            "v_max3_f32 %0, %0, %3, %4\n"                                                                             \
            "v_max3_f32 %0, %0, %5, %6\n"                                                                             \
            "v_max3_f32 %0, %0, %7, %8\n"                                                                             \
            "v_max3_f32 %0, %0, %9, %10\n"                                                                            \
            "v_max3_f32 %0, %0, %11, %12\n"                                                                           \
            "v_max3_f32 %0, %0, %13, %14"                                                                             \
      : "+&v"(r)                                                                                                      \
      : "v"(s[2]), "v"(s[3]), "v"(s[4]), "v"(s[5]), "v"(s[6]), "v"(s[7]), "v"(s[8]), "v"(s[9]), "v"(s[10]),           \
        "v"(s[11]), "v"(s[12]), "v"(s[13]), "v"(s[14]), "v"(s[15]))
  if constexpr (kReciprocals) GORIO_MAX14("s_nop 0\n");
  else GORIO_MAX14("");
#undef GORIO_MAX14
  return r;
}

// Caps up to this one go by one exponential and one reciprocal a score, which is good to 2^-21 of
// the cap then, 2^-15 at most.  Past it that error, which is as much of a weight, would grow with
// the cap, so a score is worked out to 2^-20 of itself, in twelve more instructions: 4 chunks of
// up to 500 tokens over 8192 take 171 us by a cap of 64 and 225 by one of 100, 4096 tokens over
// 32768 2561 and 3618, 64 single tokens over 16384, which HBM bounds, 453 and 456.
constexpr float kQuickCap = 64.f;

// Scores that are capped or biased, in log2: products x -> x * scale log2 e, or
// cap tanh(x scale / cap) log2 e, less slope * distance * log2 e.  With
// E = 2^a, a = 2 x scale / cap log2 e, tanh = 1 - 2 / (1 + E), which is right at
// both ends of E's range too; the quotient is below 1 and good to 2^-23, so the
// result to 2^-21 of the cap.  Where z = x scale / cap is below 1/2 that
// difference loses the score, the more the smaller z is, and
// z (1 - z^2 / 3 + 2 z^4 / 15 - ..) takes its place under a large cap.
struct ScoreChange {
  float to_log2, cap, twice, by, slope;
  __device__ __forceinline__ ScoreChange(float scale, float cap_, float slope_)
      : to_log2(scale * kLog2e), cap(cap_ * kLog2e), twice(-2.f * cap_ * kLog2e),
        // finite under a cap of no size too: a product of 0 stays one
        by(cap_ > 0.f ? fminf(fmaxf(2.f * kLog2e * scale / cap_, -3e38f), 3e38f) : 0.f), slope(-slope_ * kLog2e) {}
  // -1 / (1 + E): grows with the score, which is cap - twice * this
  __device__ __forceinline__ float quotient(float x) const { return __builtin_amdgcn_rcpf(-1.f - pow2(x * by)); }
  __device__ __forceinline__ float capped(float x) const { return __builtin_fmaf(quotient(x), -twice, cap); }
  // the same for any cap.  The series of tanh(z) / z in z^2 = a^2 c up to z^14: at 1/2 the next
  // term is 4e-9.
  __device__ __forceinline__ float capped_exactly(float x) const {
    constexpr float c = kLn2 / 2 * (kLn2 / 2);
    const float t = x * to_log2, a = x * by, z2 = a * a * c;
    float s = -929569.f / 638512875.f;
    s = __builtin_fmaf(s, z2, 21844.f / 6081075.f);
    s = __builtin_fmaf(s, z2, -1382.f / 155925.f);
    s = __builtin_fmaf(s, z2, 62.f / 2835.f);
    s = __builtin_fmaf(s, z2, -17.f / 315.f);
    s = __builtin_fmaf(s, z2, 2.f / 15.f);
    s = __builtin_fmaf(s, z2, -1.f / 3.f);
    return fabsf(a) < kLog2e ? __builtin_fmaf(t * z2, s, t) : capped(x);
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
  bool any = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) any |= any_not_finite<Q>(a[i]);
  return any;
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

// The low n bits, n of any size.
__device__ __forceinline__ uint64_t low_bits(int32_t n) {
  const uint64_t some = (1ull << (n & 63)) - 1;
  return n <= 0 ? 0 : n >= 64 ? ~0ull : some;
}

// x if the bit is set, or -inf.  On the bits: compares would hold a scalar pair for every score.
__device__ __forceinline__ float kept(float x, uint32_t bits, int bit) {
  const uint32_t mask = (uint32_t)((int32_t)(bits << (31 - bit)) >> 31);
  return __uint_as_float((__float_as_uint(x) & mask) | (0xFF800000u & ~mask));
}

// LDS written by some lanes of a wave and read by others of the same wave:
// the hardware keeps their order, the compiler has to.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

}  // namespace gorio
