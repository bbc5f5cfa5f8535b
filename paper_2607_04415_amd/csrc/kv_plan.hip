// gorio_kv_attach and gorio_kv_plan: tables of pages from a search's ids, and
// a step's starts, positions, slots and new table entries from its lengths.
//
// Both are short prefix sums over small arrays followed by writes that no
// other write depends on, so each is one launch: what a block needs of the
// sums over all requests it computes by itself, in 256-request chunks, rather
// than wait for another kernel (a launch costs more than reading a few
// thousand lengths from L2).
#include "kv.hpp"

using namespace gorio;

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kMostFound = 1024;  // passages of a request

__device__ __forceinline__ int64_t ceil_div(int64_t a, uint32_t b) { return (a + b - 1) / b; }

// Inclusive sum over the block's threads, in thread order; `sums` holds a value a wave.
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t *sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t up = __shfl_up(v, d);
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

// One block a request: the ends of its passages in the table, then every entry
// finds its passage by bisection.
__global__ __launch_bounds__(kThreads) void attach_kernel(const uint32_t *nodes, uint32_t k, const int32_t *first_page,
                                                          const int32_t *tokens, uint64_t n, uint32_t page_tokens,
                                                          uint32_t width, uint32_t limit, int32_t *tables,
                                                          int32_t *fills, int32_t *lens, int32_t *attached) {
  __shared__ int64_t s_end[kMostFound];
  __shared__ int32_t s_first[kMostFound], s_held[kMostFound];
  __shared__ int64_t s_sums[kThreads / 64];
  const uint64_t b = blockIdx.x;
  int64_t carry = 0;
  int64_t in_row = 0, passages = 0;  // of this thread's passages: the last end in the row, and how many
  for (uint32_t r0 = 0; r0 < k; r0 += kThreads) {
    const uint32_t r = r0 + threadIdx.x;
    int64_t count = 0;
    bool node = false;
    if (r < k) {
      const uint32_t v = nodes[b * k + r];
      node = v < n;
      const int32_t held = node ? max(tokens[v], 0) : 0;
      s_first[r] = node ? first_page[v] : -1;
      s_held[r] = held;
      count = ceil_div(held, page_tokens);
    }
    const int64_t end = carry + block_scan(count, s_sums);
    if (r < k) {
      s_end[r] = end;
      if (node && end <= limit) in_row = end, ++passages;
    }
    __syncthreads();
    carry = s_end[min(r0 + kThreads, k) - 1];
  }
  // the ends ascend, so the passages in the row are the first ones
  for (int d = 32; d; d >>= 1) {
    in_row = max(in_row, (int64_t)__shfl_xor(in_row, d));
    passages += __shfl_xor(passages, d);
  }
  __shared__ int64_t s_row[kThreads / 64], s_count[kThreads / 64];
  if ((threadIdx.x & 63) == 0) s_row[threadIdx.x >> 6] = in_row, s_count[threadIdx.x >> 6] = passages;
  __syncthreads();
  in_row = passages = 0;
  for (int w = 0; w < kThreads / 64; ++w) in_row = max(in_row, s_row[w]), passages += s_count[w];
  if (threadIdx.x == 0) {
    lens[b] = (int32_t)min(in_row * page_tokens, (int64_t)kKvMost);
    if (attached) attached[b] = (int32_t)passages;
  }
  for (uint32_t e = threadIdx.x; e < width; e += kThreads) {
    int32_t page = -1, fill = (int32_t)page_tokens;
    if (e < in_row) {
      uint32_t lo = 0, hi = k - 1;  // the first passage that ends past e
      while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (s_end[mid] > e) hi = mid;
        else lo = mid + 1;
      }
      const int64_t i = (int64_t)e - (s_end[lo] - ceil_div(s_held[lo], page_tokens));
      page = s_first[lo] + (int32_t)i;
      fill = (int32_t)min((int64_t)s_held[lo] - i * page_tokens, (int64_t)page_tokens);
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
  uint32_t requests, width, page_tokens;
};

// Every block runs through the requests in chunks, with the sums so far; it
// writes the tokens of its own range (blockIdx.x of gridDim.x equal ones) and
// the lengths and table entries of its own chunks.
__global__ __launch_bounds__(kThreads) void plan_kernel(PlanParams p) {
  __shared__ int64_t s_start[kThreads + 1], s_off[kThreads];
  __shared__ int32_t s_before[kThreads], s_had[kThreads], s_need[kThreads];
  __shared__ int64_t s_sums[kThreads / 64];
  const uint64_t span = (p.tokens + gridDim.x - 1) / gridDim.x;
  const uint64_t t0 = min(p.tokens, blockIdx.x * span), t1 = min(p.tokens, t0 + span);
  int64_t start = 0, off = 0;  // of the chunk's first request
  for (uint32_t b0 = 0, chunk = 0; b0 < p.requests; b0 += kThreads, ++chunk) {
    const uint32_t b = b0 + threadIdx.x, count = min((uint32_t)kThreads, p.requests - b0);
    int64_t before = 0, added = 0, had = 0, need = 0;
    if (b < p.requests) {
      before = max(p.before[b], 0);
      added = max(p.added[b], 0);
      had = min(ceil_div(before, p.page_tokens), (int64_t)p.width);
      need = min(ceil_div(before + added, p.page_tokens), (int64_t)p.width) - had;
    }
    const int64_t end = start + block_scan(added, s_sums);
    const int64_t off_end = off + block_scan(need, s_sums);
    s_start[threadIdx.x] = end - added;
    s_off[threadIdx.x] = off_end - need;
    s_before[threadIdx.x] = (int32_t)before;
    s_had[threadIdx.x] = (int32_t)had;
    s_need[threadIdx.x] = (int32_t)need;
    if (threadIdx.x == kThreads - 1) s_start[kThreads] = end;
    const bool mine = chunk % gridDim.x == blockIdx.x;
    if (mine && b < p.requests) {
      p.lens[b] = (int32_t)min(before + added, (int64_t)kKvMost);
      p.starts[b] = (int32_t)min(end - added, (int64_t)kKvMost);
    }
    __syncthreads();
    const int64_t chunk_start = start, chunk_end = s_start[kThreads];
    if (mine) {
      // a wave a request
      for (uint32_t r = threadIdx.x >> 6; r < count; r += kThreads / 64)
        for (int32_t i = threadIdx.x & 63; i < s_need[r]; i += 64) {
          const int64_t at = s_off[r] + i;
          p.tables[(uint64_t)(b0 + r) * p.width + s_had[r] + i] = (uint64_t)at < p.n_free ? p.free_pages[at] : -1;
        }
    }
    const int64_t lo_t = max((int64_t)t0, chunk_start), hi_t = min((int64_t)t1, chunk_end);
    for (int64_t t = lo_t + threadIdx.x; t < hi_t; t += kThreads) {
      uint32_t lo = 0, hi = count - 1;  // the last request that starts at or before t
      while (lo < hi) {
        const uint32_t mid = (lo + hi + 1) / 2;
        if (s_start[mid] <= t) lo = mid;
        else hi = mid - 1;
      }
      const int64_t pos = (int64_t)s_before[lo] + (t - s_start[lo]);
      const int64_t entry = pos / p.page_tokens;
      int64_t page = -1;
      if (entry < s_had[lo]) {
        page = p.tables[(uint64_t)(b0 + lo) * p.width + entry];
      } else if (entry < p.width) {
        const int64_t at = s_off[lo] + (entry - s_had[lo]);
        if ((uint64_t)at < p.n_free) page = p.free_pages[at];
      }
      if (p.positions) p.positions[t] = (int32_t)pos;
      if (p.slots) p.slots[t] = page < 0 ? -1 : page * p.page_tokens + pos % p.page_tokens;
    }
    start = chunk_end;
    __syncthreads();
    off = s_off[count - 1] + s_need[count - 1];
    __syncthreads();
  }
  for (int64_t t = max((int64_t)t0, start) + threadIdx.x; t < (int64_t)t1; t += kThreads) {
    if (p.positions) p.positions[t] = -1;
    if (p.slots) p.slots[t] = -1;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    p.starts[p.requests] = (int32_t)min(start, (int64_t)kKvMost);
    if (p.taken) *p.taken = (int32_t)min(off, (int64_t)kKvMost);
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
  const gorio_status st = dev.use({{"nodes", nodes, 4, false},
                                   {"first_page", first_page, 4, false},
                                   {"tokens", tokens, 4, false},
                                   {"tables", tables, 4, false},
                                   {"fills", fills, 4, false},
                                   {"lens", lens, 4, false},
                                   {"attached", attached, 4, true}});
  if (st != GORIO_OK) return st;
  attach_kernel<<<(uint32_t)requests, kThreads, 0, static_cast<hipStream_t>(stream)>>>(
      nodes, k, first_page, tokens, n, page_tokens, width, limit, tables, fills, lens, attached);
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
  const gorio_status st = dev.use({{"before", before, 4, false},
                                   {"added", added, 4, false},
                                   {"free_pages", free_pages, 4, n_free == 0},
                                   {"tables", tables, 4, false},
                                   {"lens", lens, 4, false},
                                   {"starts", starts, 4, false},
                                   {"positions", positions, 4, true},
                                   {"slots", slots, 8, true},
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
  p.page_tokens = page_tokens;
  const uint64_t chunks = (requests + kThreads - 1) / kThreads, spans = (tokens + 1023) / 1024;
  const uint32_t grid = (uint32_t)min(max(max(chunks, spans), (uint64_t)1), (uint64_t)512);
  plan_kernel<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(p);
  return kv_launched("gorio_kv_plan");
}
