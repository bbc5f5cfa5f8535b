// gorio_kv_attach and gorio_kv_plan: tables of pages from a search's ids, and
// a step's starts, positions, slots and new table entries from its lengths.
//
// Both are short prefix sums over small arrays followed by writes that no
// other write depends on, so each is one launch: what a block needs of the
// sums over all requests it computes by itself, in 256-request chunks, rather
// than wait for another kernel (a launch costs more than reading a few
// thousand lengths from L2).  What bounds them is latency, a chain of loads
// and barriers: attach takes 3.3 us for one request of 10 passages and 5.9 for
// 1000 with 512 entries each (4.1 MB written); plan 4.8 us for 64 single
// tokens and 5.6 for 256 prompts of up to 2047 (2.2 MB).
#include <algorithm>

#include "kv.hpp"

using namespace gorio;

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kMostFound = 1024;  // passages of a request

// Pages of x tokens, 0 <= x < 2^31.
__host__ __device__ __forceinline__ uint32_t pages_of(uint32_t x, FastDiv page_tokens) {
  return x ? fastdiv(x - 1, page_tokens) + 1 : 0;
}

// Inclusive sums of two values over the block's threads, in thread order; `sums` holds them a wave.
__device__ __forceinline__ void block_scan(uint64_t &a, uint64_t &b, uint64_t (*sums)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint64_t ua = __shfl_up(a, d), ub = __shfl_up(b, d);
    if (lane >= d) a += ua, b += ub;
  }
  __syncthreads();
  if (lane == 63) sums[wave][0] = a, sums[wave][1] = b;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w)
    if (w < wave) a += sums[w][0], b += sums[w][1];
}

// One block a request: the ends of its passages in the table, then every entry
// finds its passage by bisection.
__global__ __launch_bounds__(kThreads) void attach_kernel(const uint32_t *nodes, uint32_t k, const int32_t *first_page,
                                                          const int32_t *tokens, uint64_t n, FastDiv page_tokens,
                                                          uint32_t width, uint32_t limit, int32_t *tables,
                                                          int32_t *fills, int32_t *lens, int32_t *attached) {
  __shared__ uint64_t s_end[kMostFound];
  __shared__ int32_t s_first[kMostFound], s_held[kMostFound];
  __shared__ uint64_t s_sums[kThreads / 64][2];
  const uint64_t b = blockIdx.x;
  uint64_t carry = 0;
  uint64_t in_row = 0, passages = 0;  // of this thread's passages: the last end in the row, and how many
  for (uint32_t r0 = 0; r0 < k; r0 += kThreads) {
    const uint32_t r = r0 + threadIdx.x;
    uint64_t count = 0, nodes_so_far = 0;
    bool node = false;
    if (r < k) {
      const uint32_t v = nodes[b * k + r];
      const int32_t first = v < n ? first_page[v] : -1, all = v < n ? tokens[v] : 0;
      node = first >= 0;
      const int32_t held = node ? max(all, 0) : 0;
      s_first[r] = first;
      s_held[r] = held;
      count = pages_of(held, page_tokens);
    }
    block_scan(count, nodes_so_far, s_sums);
    const uint64_t end = carry + count;
    if (r < k) {
      s_end[r] = end;
      if (node && end <= limit) in_row = end, ++passages;
    }
    __syncthreads();
    carry = s_end[min(r0 + kThreads, k) - 1];
  }
  // the ends ascend, so the passages in the row are the first ones
  for (int d = 32; d; d >>= 1) {
    in_row = max(in_row, __shfl_xor(in_row, d));
    passages += __shfl_xor(passages, d);
  }
  __shared__ uint64_t s_row[kThreads / 64], s_count[kThreads / 64];
  if ((threadIdx.x & 63) == 0) s_row[threadIdx.x >> 6] = in_row, s_count[threadIdx.x >> 6] = passages;
  __syncthreads();
  in_row = passages = 0;
  for (int w = 0; w < kThreads / 64; ++w) in_row = max(in_row, s_row[w]), passages += s_count[w];
  if (threadIdx.x == 0) {
    lens[b] = (int32_t)min(in_row * page_tokens.d, kKvMost);
    if (attached) attached[b] = (int32_t)passages;
  }
  for (uint32_t e = threadIdx.x; e < width; e += kThreads) {
    int32_t page = -1, fill = (int32_t)page_tokens.d;
    if (e < in_row) {
      uint32_t lo = 0, hi = k - 1;  // the first passage that ends past e
      while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (s_end[mid] > e) hi = mid;
        else lo = mid + 1;
      }
      const uint32_t i = e - (uint32_t)(s_end[lo] - pages_of(s_held[lo], page_tokens));
      page = max((int32_t)((uint32_t)s_first[lo] + i), -1);  // past 2^31 - 1 there is none
      fill = min(s_held[lo] - (int32_t)(i * page_tokens.d), (int32_t)page_tokens.d);
    }
    tables[b * width + e] = page;
    fills[b * width + e] = fill;
  }
}

struct PlanParams {
  const int32_t *before, *added, *free_pages;
  int32_t *tables, *lens, *starts, *positions, *taken;
  int64_t *slots;
  uint64_t n_free, tokens;
  uint32_t requests, width;
  FastDiv page_tokens;
};

// Every block runs through the requests in chunks, with the sums so far; it
// writes the tokens of its own range (blockIdx.x of gridDim.x equal ones), the
// lengths of its own chunks and the table entries of its own requests.  A token
// finds its request by bisection of the chunk's starts in LDS; a page it needs
// is in the table if the request had it, and else in the free list, so nothing
// that another block writes is read.
__global__ __launch_bounds__(kThreads) void plan_kernel(PlanParams p) {
  __shared__ uint32_t s_start[kThreads];  // from the chunk's first token on
  __shared__ uint64_t s_off[kThreads];
  __shared__ uint32_t s_before[kThreads], s_had[kThreads], s_need[kThreads];
  __shared__ uint64_t s_sums[kThreads / 64][2], s_upto[2];
  const uint64_t span = (p.tokens + gridDim.x - 1) / gridDim.x;
  const uint64_t t0 = min(p.tokens, blockIdx.x * span), t1 = min(p.tokens, t0 + span);
  uint64_t start = 0, off = 0;  // of the chunk's first request
  for (uint32_t b0 = 0, chunk = 0; b0 < p.requests; b0 += kThreads, ++chunk) {
    const uint32_t b = b0 + threadIdx.x, count = min((uint32_t)kThreads, p.requests - b0);
    uint32_t before = 0, added = 0, had = 0, need = 0;
    if (b < p.requests) {
      before = max(p.before[b], 0);
      added = max(p.added[b], 0);
      had = min(pages_of(before, p.page_tokens), p.width);
      need = min(pages_of(min(before + added, (uint32_t)kKvMost), p.page_tokens), p.width) - had;
    }
    uint64_t end = added, off_end = need;
    block_scan(end, off_end, s_sums);
    s_start[threadIdx.x] = (uint32_t)min(end - added, (uint64_t)0xFFFFFFFFu);
    s_off[threadIdx.x] = off + off_end - need;
    s_before[threadIdx.x] = before;
    s_had[threadIdx.x] = had;
    s_need[threadIdx.x] = need;
    if (threadIdx.x == kThreads - 1) s_upto[0] = start + end, s_upto[1] = off + off_end;
    const bool mine = chunk % gridDim.x == blockIdx.x;
    if (mine && b < p.requests) {
      p.lens[b] = (int32_t)min(before + added, (uint32_t)kKvMost);
      p.starts[b] = (int32_t)min(start + end - added, kKvMost);
    }
    __syncthreads();
    const uint64_t upto = s_upto[0];
    // a wave a request, over all blocks: one block alone took 22 us for the entries of 182k tokens
    for (uint32_t r = blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); r < count; r += gridDim.x * (kThreads / 64))
      for (uint32_t i = threadIdx.x & 63; i < s_need[r]; i += 64) {
        const uint64_t at = s_off[r] + i;
        p.tables[(uint64_t)(b0 + r) * p.width + s_had[r] + i] = at < p.n_free ? p.free_pages[at] : -1;
      }
    for (uint64_t t = max(t0, start) + threadIdx.x; t < min(t1, upto); t += kThreads) {
      const uint32_t from = (uint32_t)(t - start);
      uint32_t lo = 0, hi = count - 1;  // the last request that starts at or before t
      while (lo < hi) {
        const uint32_t mid = (lo + hi + 1) / 2;
        if (s_start[mid] <= from) lo = mid;
        else hi = mid - 1;
      }
      const uint32_t pos = s_before[lo] + (from - s_start[lo]);  // below 2^32
      int32_t page = -1;
      uint32_t place = 0;
      if (pos < kKvMost) {
        const uint32_t entry = fastdiv(pos, p.page_tokens);
        place = pos - entry * p.page_tokens.d;
        if (entry < s_had[lo]) {
          page = p.tables[(uint64_t)(b0 + lo) * p.width + entry];
        } else if (entry < p.width) {
          const uint64_t at = s_off[lo] + (entry - s_had[lo]);
          if (at < p.n_free) page = p.free_pages[at];
        }
      }
      if (p.positions) p.positions[t] = (int32_t)min(pos, (uint32_t)kKvMost);
      if (p.slots) p.slots[t] = page < 0 ? -1 : (int64_t)page * p.page_tokens.d + place;
    }
    start = upto;
    off = s_upto[1];
    __syncthreads();
  }
  for (uint64_t t = max(t0, start) + threadIdx.x; t < t1; t += kThreads) {
    if (p.positions) p.positions[t] = -1;
    if (p.slots) p.slots[t] = -1;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.starts[p.requests] = (int32_t)min(start, kKvMost);
    if (p.taken) *p.taken = (int32_t)min(off, kKvMost);
  }
}

}  // namespace

extern "C" gorio_status gorio_kv_attach(const uint32_t *nodes, uint64_t requests, uint32_t k,
                                        const int32_t *first_page, const int32_t *tokens, uint64_t n,
                                        uint32_t page_tokens, uint32_t width, uint32_t limit, int32_t *tables,
                                        int32_t *fills, int32_t *lens, int32_t *attached, void *stream) {
  if (requests > kKvMost) return fail(GORIO_EINVAL, "requests=%llu too large", (unsigned long long)requests);
  if (k == 0 || k > kMostFound) return fail(GORIO_EINVAL, "k=%u, need 1..%u", k, kMostFound);
  if (page_tokens == 0 || page_tokens > 65536) return fail(GORIO_EINVAL, "page_tokens=%u, need 1..65536", page_tokens);
  if (width == 0 || width > kKvMost) return fail(GORIO_EINVAL, "width=%u, need 1..2^31-1", width);
  if (limit > width) return fail(GORIO_EINVAL, "limit=%u above width=%u", limit, width);
  if (requests == 0) return GORIO_OK;
  KvDevice dev;
  gorio_status st = dev.use({{"nodes", nodes, 4, false},
                             {"first_page", first_page, 4, n == 0},
                             {"tokens", tokens, 4, n == 0},
                             {"tables", tables, 4, false},
                             {"fills", fills, 4, false},
                             {"lens", lens, 4, false},
                             {"attached", attached, 4, true}});
  if (st != GORIO_OK) return st;
  st = kv_apart({{"nodes", nodes, 4 * requests * k, false},
                 {"first_page", first_page, 4 * n, false},
                 {"tokens", tokens, 4 * n, false},
                 {"tables", tables, 4 * requests * width, true},
                 {"fills", fills, 4 * requests * width, true},
                 {"lens", lens, 4 * requests, true},
                 {"attached", attached, 4 * requests, true}});
  if (st != GORIO_OK) return st;
  attach_kernel<<<(uint32_t)requests, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
      nodes, k, first_page, tokens, n, make_fastdiv(page_tokens), width, limit, tables, fills, lens, attached);
  return kv_launched("gorio_kv_attach");
}

extern "C" gorio_status gorio_kv_plan(const int32_t *before, const int32_t *added, uint64_t requests,
                                      uint32_t page_tokens, const int32_t *free_pages, uint64_t n_free,
                                      int32_t *tables, uint32_t width, uint64_t tokens, int32_t *lens,
                                      int32_t *starts, int32_t *positions, int64_t *slots, int32_t *taken,
                                      void *stream) {
  if (requests > kKvMost || tokens > kKvMost || n_free > kKvMost)
    return fail(GORIO_EINVAL, "requests, tokens and n_free must be below 2^31");
  if (page_tokens == 0 || page_tokens > 65536) return fail(GORIO_EINVAL, "page_tokens=%u, need 1..65536", page_tokens);
  if (width == 0 || width > kKvMost) return fail(GORIO_EINVAL, "width=%u, need 1..2^31-1", width);
  if (requests == 0) return GORIO_OK;
  if (lens == before) return fail(GORIO_EINVAL, "lens and before are the same array");
  KvDevice dev;
  gorio_status st = dev.use({{"before", before, 4, false},
                             {"added", added, 4, false},
                             {"free_pages", free_pages, 4, n_free == 0},
                             {"tables", tables, 4, false},
                             {"lens", lens, 4, false},
                             {"starts", starts, 4, false},
                             {"positions", positions, 4, true},
                             {"slots", slots, 8, true},
                             {"taken", taken, 4, true}});
  if (st != GORIO_OK) return st;
  st = kv_apart({{"before", before, 4 * requests, false},
                 {"added", added, 4 * requests, false},
                 {"free_pages", free_pages, 4 * n_free, false},
                 {"tables", tables, 4 * requests * width, true},
                 {"lens", lens, 4 * requests, true},
                 {"starts", starts, 4 * (requests + 1), true},
                 {"positions", positions, 4 * tokens, true},
                 {"slots", slots, 8 * tokens, true},
                 {"taken", taken, 4, true}});
  if (st != GORIO_OK) return st;
  PlanParams p;
  p.before = before;
  p.added = added;
  p.free_pages = free_pages;
  p.tables = tables;
  p.lens = lens;
  p.starts = starts;
  p.positions = positions;
  p.taken = taken;
  p.slots = slots;
  p.n_free = n_free;
  p.tokens = tokens;
  p.requests = (uint32_t)requests;
  p.width = width;
  p.page_tokens = make_fastdiv(page_tokens);
  // a token a thread, until more blocks than run at once would add up the requests again
  const uint64_t chunks = (requests + kThreads - 1) / kThreads, spans = (tokens + kThreads - 1) / kThreads;
  const uint32_t grid = (uint32_t)std::min<uint64_t>(std::max<uint64_t>({chunks, spans, 1}), 1024);
  plan_kernel<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(p);
  return kv_launched("gorio_kv_plan");
}
