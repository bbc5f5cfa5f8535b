// gorio_kv_share: groups of neighbouring requests whose tables begin with the
// same pages.
//
// Two launches: a block a request compares its row with the one before, up to
// the first difference; then one block makes groups of what they found.  Rows
// are read twice, the second time from L2; both kernels are chains of a few
// loads and barriers, and latency is what they cost: 2.9 and 3.0 us for 64 rows
// of 1060 entries, 3.5 and 3.2 for 1000 of 512 and their fills (4 MB).
#include "kv.hpp"

using namespace gorio;

namespace {

constexpr int kThreads = 256, kGroupThreads = 1024;
constexpr int kAhead = 4;  // entries of a thread whose loads are under way together

__global__ __launch_bounds__(kThreads) void common_kernel(const int32_t *tables, const int32_t *fills,
                                                          const int32_t *held, uint32_t width, FastDiv page_tokens,
                                                          int32_t *common) {
  __shared__ uint32_t s_first[kThreads / 64];
  const uint64_t b = blockIdx.x;
  if (b == 0) {
    if (threadIdx.x == 0) common[0] = 0;
    return;
  }
  const uint32_t whole = fastdiv((uint32_t)max(min(held[b - 1], held[b]), 0), page_tokens);
  const uint32_t upto = min(width, whole);
  const int32_t *mine = tables + b * width, *before = mine - width;
  const int32_t *my_fills = fills ? fills + b * width : mine, *fills_before = fills ? my_fills - width : before;
  uint32_t same = upto;  // leading entries without a difference
  for (uint64_t e0 = 0; e0 < upto; e0 += kThreads * kAhead) {
    bool differs[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const uint64_t e = min(e0 + i * kThreads + threadIdx.x, (uint64_t)upto - 1);
      differs[i] = (mine[e] != before[e]) | (my_fills[e] != fills_before[e]);
    }
    uint32_t first = upto;
#pragma unroll
    for (int i = kAhead - 1; i >= 0; --i)
      if (differs[i]) first = (uint32_t)min(e0 + i * kThreads + threadIdx.x, (uint64_t)upto - 1);
#pragma unroll
    for (int d = 32; d; d >>= 1) first = min(first, (uint32_t)__shfl_xor((int)first, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_first[threadIdx.x >> 6] = first;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) same = min(same, s_first[w]);
    if (same < upto) break;
  }
  if (threadIdx.x == 0) common[b] = (int32_t)(same * page_tokens.d);  // at most held
}

// Inclusive over the threads: sums of a, maxima of b.
__device__ __forceinline__ void scan(uint32_t &a, uint32_t &b, uint32_t (*sums)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t ua = __shfl_up(a, d), ub = __shfl_up(b, d);
    if (lane >= d) a += ua, b = max(b, ub);
  }
  __syncthreads();
  if (lane == 63) sums[wave][0] = a, sums[wave][1] = b;
  __syncthreads();
  for (int w = 0; w < wave; ++w) a += sums[w][0], b = max(b, sums[w][1]);
}

// A group is written when its end is known: the last one of a chunk stays open, with the smallest
// common so far, until a later chunk begins another.
__global__ __launch_bounds__(kGroupThreads) void group_kernel(const int32_t *common, uint32_t requests, int32_t least,
                                                              int32_t *first, int32_t *shared) {
  __shared__ uint32_t s_sums[kGroupThreads / 64][2], s_upto[2];
  __shared__ int32_t s_least[kGroupThreads + 1];  // of the open group, and of those that begin in the chunk
  constexpr int32_t kNone = 0x7FFFFFFF;           // a request alone
  auto put = [&](uint32_t b, int32_t of) { shared[b] = of == kNone ? 0 : of; };
  uint32_t groups = 0, open = 0;  // how many before the chunk; where the last one begins
  int32_t open_least = kNone;
  for (uint32_t b0 = 0; b0 < requests; b0 += kGroupThreads) {
    const uint32_t b = b0 + threadIdx.x;
    const bool in = b < requests;
    const int32_t mine = in ? common[b] : 0;
    const bool begin = in && (b == 0 || mine < least);
    uint32_t count = begin ? 1 : 0, at = begin ? b : open;
    s_least[threadIdx.x + 1] = kNone;
    if (threadIdx.x == 0) s_least[0] = open_least;
    scan(count, at, s_sums);
    if (begin) first[groups + count - 1] = (int32_t)b;
    if (in && !begin) atomicMin(&s_least[count], mine);
    if (threadIdx.x == kGroupThreads - 1) s_upto[0] = count, s_upto[1] = at;
    __syncthreads();
    const uint32_t here = s_upto[0];  // groups that begin in the chunk
    if (in && count < here) put(b, s_least[count]);
    if (here)
      for (uint32_t e = open + threadIdx.x; e < b0; e += kGroupThreads) put(e, s_least[0]);
    groups += here, open = s_upto[1], open_least = s_least[here];
    __syncthreads();
  }
  for (uint32_t b = open + threadIdx.x; b < requests; b += kGroupThreads) put(b, open_least);
  for (uint32_t g = groups + threadIdx.x; g <= requests; g += kGroupThreads) first[g] = (int32_t)requests;
}

}  // namespace

extern "C" gorio_status gorio_kv_share(const int32_t *tables, const int32_t *fills, const int32_t *held,
                                       uint64_t requests, uint32_t width, uint32_t page_tokens, uint32_t least,
                                       int32_t *common, int32_t *first, int32_t *shared, void *stream) {
  if (requests > 1u << 20) return fail(GORIO_EINVAL, "requests=%llu, need at most 2^20", (unsigned long long)requests);
  if (page_tokens == 0 || page_tokens > 65536) return fail(GORIO_EINVAL, "page_tokens=%u, need 1..65536", page_tokens);
  if (width == 0 || (uint64_t)width * page_tokens > kKvMost)
    return fail(GORIO_EINVAL, "width=%u: a row holds 1..2^31-1 positions", width);
  if (least > kKvMost) return fail(GORIO_EINVAL, "least=%u, need at most 2^31-1", least);
  if (requests == 0) return GORIO_OK;
  KvDevice dev;
  gorio_status st = dev.use({{"tables", tables, 4, false},
                             {"fills", fills, 4, true},
                             {"held", held, 4, false},
                             {"common", common, 4, false},
                             {"first", first, 4, false},
                             {"shared", shared, 4, false}});
  if (st != GORIO_OK) return st;
  st = kv_apart({{"tables", tables, 4 * requests * width, false},
                 {"fills", fills, 4 * requests * width, false},
                 {"held", held, 4 * requests, false},
                 {"common", common, 4 * requests, true},
                 {"first", first, 4 * (requests + 1), true},
                 {"shared", shared, 4 * requests, true}});
  if (st != GORIO_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  common_kernel<<<(uint32_t)requests, kThreads, 0, s>>>(tables, fills, held, width, make_fastdiv(page_tokens), common);
  st = kv_launched("gorio_kv_share");
  if (st != GORIO_OK) return st;
  group_kernel<<<1, kGroupThreads, 0, s>>>(common, (uint32_t)requests, (int32_t)(least ? least : 1), first, shared);
  return kv_launched("gorio_kv_share");
}
