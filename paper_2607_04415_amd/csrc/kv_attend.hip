// gorio_kv_attend: attention of new tokens over the pages of their requests.
#include <algorithm>

#include "kv.hpp"

using namespace gorio;

namespace {

struct AttendParams {
  const uint16_t *q;
  uint16_t *out;
  float *lse;
  const uint8_t *keys, *values;
  const float *key_scale, *value_scale;
  const int32_t *starts, *lens, *tables, *fills, *prefix;
  const float *slopes;
  uint64_t tokens, q_stride, out_stride;
  uint64_t page_stride, head_stride, token_stride;  // elements
  uint32_t num_pages, requests, width, heads, kv_heads, group, D;
  FastDiv page_tokens;
  float scale, cap;
  uint32_t window;
};

__device__ __forceinline__ float from_bits(uint16_t b, bool f16) {
  return f16 ? (float)__builtin_bit_cast(_Float16, b) : __uint_as_float((uint32_t)b << 16);
}

__device__ __forceinline__ uint16_t to_bits(float x, bool f16) {
  return f16 ? __builtin_bit_cast(uint16_t, (_Float16)x) : __builtin_bit_cast(uint16_t, (__bf16)x);
}

__device__ __forceinline__ float element(const uint8_t *pages, uint64_t at, bool e4m3, bool f16) {
  if (e4m3) return __builtin_amdgcn_cvt_f32_fp8((int)pages[at], 0);
  return from_bits(reinterpret_cast<const uint16_t *>(pages)[at], f16);
}

// A wave computes one row of one head, a key a lane and 64 keys at a time.
__global__ __launch_bounds__(64) void attend_rows(AttendParams p, bool e4m3, bool f16) {
  const uint32_t h = blockIdx.y, lane = threadIdx.x;
  const int64_t t = blockIdx.x;
  uint32_t lo = 0, hi = p.requests;  // the last request that starts at or before t
  while (lo < hi) {
    const uint32_t mid = (lo + hi + 1) / 2;
    if (p.starts[mid] <= t) lo = mid;
    else hi = mid - 1;
  }
  if (lo >= p.requests || t < p.starts[lo]) return;
  const uint32_t b = lo;
  const int64_t s0 = p.starts[b], s1 = min((int64_t)p.starts[b + 1], (int64_t)p.tokens);
  const int64_t len = max(p.lens[b], 0), pos = len - (s1 - s0) + (t - s0);
  const int64_t prefix = p.prefix ? p.prefix[b] : 0;
  const int64_t window = p.window ? p.window : (int64_t)1 << 40;
  const int64_t last = min(min(len, max(pos + 1, prefix)), (int64_t)p.width * p.page_tokens.d);
  const uint32_t kh = h / p.group;
  const uint16_t *q = p.q + t * p.q_stride + (uint64_t)h * p.D;
  const float scale = p.scale * (p.key_scale ? p.key_scale[kh] : 1.f);
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t j0 = 0; j0 < last; j0 += 64) {
    const int64_t j = j0 + lane;
    bool seen = j < last && ((j <= pos && pos - j < window) || j < prefix);
    uint64_t at = 0;
    if (seen) {
      const uint32_t e = fastdiv((uint32_t)j, p.page_tokens), place = (uint32_t)j - e * p.page_tokens.d;
      const int32_t page = p.tables[(uint64_t)b * p.width + e];
      seen = (uint32_t)page < p.num_pages && (!p.fills || (int32_t)place < p.fills[(uint64_t)b * p.width + e]);
      if (seen) at = (uint64_t)page * p.page_stride + kh * p.head_stride + place * p.token_stride;
    }
    float s = -INFINITY;
    if (seen) {
      float dot = 0.f;
      for (uint32_t d = 0; d < p.D; ++d) dot = fmaf(from_bits(q[d], f16), element(p.keys, at + d, e4m3, f16), dot);
      s = dot * scale;
      if (p.cap > 0.f) s = p.cap * tanhf(s / p.cap);
      if (p.slopes) s -= p.slopes[h] * fabsf((float)(pos - j));
    }
    float most = s;
    for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    const float to = fmaxf(m, most);
    const float by = to == -INFINITY ? 0.f : to;
    const float w = expf(s - by), keep = expf(m - by);
    float sum = w;
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    l = l * keep + sum;
    m = to;
    for (int i = 0; i < 4; ++i) o[i] *= keep;
    for (int src = 0; src < 64; ++src) {
      if (!__shfl((int)seen, src)) continue;
      const float ws = __shfl(w, src);
      const uint64_t row = __shfl(at, src);
      for (int i = 0; i < 4; ++i) {
        const uint32_t d = lane + 64 * i;
        if (d < p.D) o[i] = fmaf(ws, element(p.values, row + d, e4m3, f16), o[i]);
      }
    }
  }
  const float norm = l != 0.f ? (p.value_scale ? p.value_scale[kh] : 1.f) / l : 0.f;
  uint16_t *out = p.out + t * p.out_stride + (uint64_t)h * p.D;
  for (int i = 0; i < 4; ++i) {
    const uint32_t d = lane + 64 * i;
    if (d < p.D) out[d] = to_bits(o[i] * norm, f16);
  }
  if (p.lse && lane == 0) p.lse[t * p.heads + h] = l != 0.f ? m + logf(l) : -INFINITY;
}

// The sizes and types of a call, with the strides filled in.
gorio_status check(const gorio_kv_cache *cache, const gorio_kv_attention *a, gorio_kv_cache *c, gorio_kv_attention *out) {
  const gorio_status st = kv_check_cache(cache, c);
  if (st != GORIO_OK) return st;
  if (!a) return fail(GORIO_EINVAL, "attention is NULL");
  if (a->dtype != GORIO_KV_BF16 && a->dtype != GORIO_KV_F16)
    return fail(GORIO_EINVAL, "q must be bf16 or f16, not gorio_kv_dtype %u", a->dtype);
  if (c->dtype != GORIO_KV_E4M3 && c->dtype != a->dtype)
    return fail(GORIO_EUNSUPPORTED, "16-bit pages are read by queries of their own type");
  if (a->heads == 0 || a->heads % c->heads != 0 || a->heads > 65535)
    return fail(GORIO_EINVAL, "heads=%u, need a multiple of the cache's %u, at most 65535", a->heads, c->heads);
  if (a->requests > kKvMost || a->tokens > kKvMost) return fail(GORIO_EINVAL, "requests and tokens must be below 2^31");
  if (a->width == 0 || (uint64_t)a->width * c->page_tokens > kKvMost)
    return fail(GORIO_EINVAL, "width=%u: a row holds 1..2^31-1 positions", a->width);
  *out = *a;
  if (a->q_stride == 0) out->q_stride = (uint64_t)a->heads * c->D;
  if (a->out_stride == 0) out->out_stride = (uint64_t)a->heads * c->D;
  if (out->q_stride % 8 || out->out_stride % 8)
    return fail(GORIO_EINVAL, "q_stride and out_stride must be multiples of 8 elements");
  if (!(a->cap >= 0.f) || !(a->cap <= 3e38f)) return fail(GORIO_EINVAL, "cap=%g, need a number >= 0", (double)a->cap);
  if (!(a->scale <= 3e38f && a->scale >= -3e38f)) return fail(GORIO_EINVAL, "scale=%g", (double)a->scale);
  return GORIO_OK;
}

}  // namespace

extern "C" gorio_status gorio_kv_workspace(const gorio_kv_cache *cache, const gorio_kv_attention *a, uint64_t *bytes) {
  gorio_kv_cache c;
  gorio_kv_attention at;
  const gorio_status st = check(cache, a, &c, &at);
  if (st != GORIO_OK) return st;
  if (!bytes) return fail(GORIO_EINVAL, "bytes is NULL");
  *bytes = 0;
  return GORIO_OK;
}

extern "C" gorio_status gorio_kv_attend(const gorio_kv_cache *cache, const gorio_kv_attention *a, void *workspace,
                                        uint64_t workspace_bytes, void *stream) {
  gorio_kv_cache c;
  gorio_kv_attention at;
  gorio_status st = check(cache, a, &c, &at);
  if (st != GORIO_OK) return st;
  (void)workspace;
  (void)workspace_bytes;
  if (at.tokens == 0 || at.requests == 0) return GORIO_OK;
  KvDevice dev;
  st = dev.use({{"q", at.q, 16, false},
                {"out", at.out, 16, false},
                {"lse", at.lse, 4, true},
                {"starts", at.starts, 4, false},
                {"lens", at.lens, 4, false},
                {"tables", at.tables, 4, false},
                {"fills", at.fills, 4, true},
                {"prefix", at.prefix, 4, true},
                {"slopes", at.slopes, 4, true},
                {"cache keys", c.keys, 16, false},
                {"cache values", c.values, 16, false},
                {"key_scale", c.key_scale, 4, true},
                {"value_scale", c.value_scale, 4, true}});
  if (st != GORIO_OK) return st;
  AttendParams p;
  p.q = static_cast<const uint16_t *>(at.q);
  p.out = static_cast<uint16_t *>(at.out);
  p.lse = at.lse;
  p.keys = static_cast<const uint8_t *>(c.keys);
  p.values = static_cast<const uint8_t *>(c.values);
  p.key_scale = c.key_scale;
  p.value_scale = c.value_scale;
  p.starts = at.starts;
  p.lens = at.lens;
  p.tables = at.tables;
  p.fills = at.fills;
  p.prefix = at.prefix;
  p.slopes = at.slopes;
  p.tokens = at.tokens;
  p.q_stride = at.q_stride;
  p.out_stride = at.out_stride;
  p.page_stride = c.page_stride;
  p.head_stride = c.head_stride;
  p.token_stride = c.token_stride;
  p.num_pages = (uint32_t)c.num_pages;
  p.requests = at.requests;
  p.width = at.width;
  p.heads = at.heads;
  p.kv_heads = c.heads;
  p.group = at.heads / c.heads;
  p.D = c.D;
  p.page_tokens = make_fastdiv(c.page_tokens);
  p.scale = at.scale;
  p.cap = at.cap;
  p.window = at.window;
  const dim3 grid((uint32_t)at.tokens, at.heads);
  attend_rows<<<grid, 64, 0, static_cast<hipStream_t>(stream)>>>(p, c.dtype == GORIO_KV_E4M3, at.dtype == GORIO_KV_F16);
  return kv_launched("gorio_kv_attend");
}
