// gorio_kv_store: rows of new keys and values into their slots.
//
// A copy whose destination rows are scattered: a thread moves 8 elements (16
// bytes), neighbouring threads neighbouring parts of a row.
#include "kv.hpp"

using namespace gorio;

namespace {

struct StoreParams {
  const uint16_t *keys, *values;  // 16-bit elements, bf16 or f16
  uint8_t *to_keys, *to_values;
  const float *key_scale, *value_scale;
  const int64_t *slots;
  uint64_t key_stride, value_stride;  // elements
  uint64_t page_stride, head_stride, token_stride;
  uint64_t num_pages;
  uint64_t parts;  // 8-element parts of the keys: tokens * heads * D / 8
  FastDiv per_row, per_token;  // parts of a head's row, and of a token
  FastDiv page_tokens;
};

__device__ __forceinline__ float to_float(uint16_t bits, bool f16) {
  return f16 ? (float)__builtin_bit_cast(_Float16, bits) : __uint_as_float((uint32_t)bits << 16);
}

// +-448 is the largest value of the 8-bit type; a NaN stays one.
__device__ __forceinline__ float clamp_e4m3(float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; }

template <int kTo>  // 0: as it is; 1: bf16 to e4m3; 2: f16 to e4m3
__global__ __launch_bounds__(256) void store_kernel(StoreParams p) {
  const uint64_t part = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  if (part >= p.parts) return;
  const bool value = blockIdx.y != 0;
  // parts stay below 2^31 * 1024 * 32: the token by 64-bit division once per
  // thread, the rest by multiplication
  const uint64_t token = part / p.per_token.d;
  const uint32_t in = (uint32_t)(part - token * p.per_token.d);
  const uint32_t head = fastdiv(in, p.per_row), at = (in - head * p.per_row.d) * 8;
  const int64_t slot = p.slots[token];
  if (slot < 0) return;
  const uint64_t page = (uint64_t)slot / p.page_tokens.d;
  if (page >= p.num_pages) return;
  const uint32_t place = (uint32_t)((uint64_t)slot - page * p.page_tokens.d);
  const uint16_t *from = value ? p.values + token * p.value_stride : p.keys + token * p.key_stride;
  const uint4 x = *reinterpret_cast<const uint4 *>(from + (uint64_t)head * p.per_row.d * 8 + at);
  const uint64_t to = page * p.page_stride + head * p.head_stride + place * p.token_stride + at;
  uint8_t *pages = value ? p.to_values : p.to_keys;
  if constexpr (kTo == 0) {
    *reinterpret_cast<uint4 *>(pages + to * 2) = x;
  } else {
    const float *scales = value ? p.value_scale : p.key_scale;
    const float scale = scales ? scales[head] : 1.f;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    int packed[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        f[j] = clamp_e4m3(to_float((uint16_t)(w[2 * i + j / 2] >> (16 * (j & 1))), kTo == 2) / scale);
      packed[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
      packed[i] = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], packed[i], true);
    }
    *reinterpret_cast<int2 *>(pages + to) = make_int2(packed[0], packed[1]);
  }
}

}  // namespace

extern "C" gorio_status gorio_kv_store(const gorio_kv_cache *cache, gorio_kv_dtype dtype, const void *keys,
                                       const void *values, uint64_t tokens, uint64_t key_stride,
                                       uint64_t value_stride, const int64_t *slots, void *stream) {
  gorio_kv_cache c;
  gorio_status st = kv_check_cache(cache, &c);
  if (st != GORIO_OK) return st;
  if (dtype != GORIO_KV_BF16 && dtype != GORIO_KV_F16)
    return fail(GORIO_EINVAL, "keys and values must be bf16 or f16, not gorio_kv_dtype %d", (int)dtype);
  if (c.dtype != GORIO_KV_E4M3 && (gorio_kv_dtype)c.dtype != dtype)
    return fail(GORIO_EUNSUPPORTED, "16-bit pages take keys and values of their own type");
  if (tokens > kKvMost) return fail(GORIO_EINVAL, "tokens=%llu too large", (unsigned long long)tokens);
  if (key_stride == 0) key_stride = (uint64_t)c.heads * c.D;
  if (value_stride == 0) value_stride = (uint64_t)c.heads * c.D;
  if (key_stride % 8 || value_stride % 8)
    return fail(GORIO_EINVAL, "key_stride and value_stride must be multiples of 8 elements");
  if (tokens == 0) return GORIO_OK;
  KvDevice dev;
  st = dev.use({{"keys", keys, 16, false},
                {"values", values, 16, false},
                {"slots", slots, 8, false},
                {"cache keys", c.keys, 16, false},
                {"cache values", c.values, 16, false},
                {"key_scale", c.key_scale, 4, true},
                {"value_scale", c.value_scale, 4, true}});
  if (st != GORIO_OK) return st;
  StoreParams p;
  p.keys = static_cast<const uint16_t *>(keys);
  p.values = static_cast<const uint16_t *>(values);
  p.to_keys = static_cast<uint8_t *>(c.keys);
  p.to_values = static_cast<uint8_t *>(c.values);
  p.key_scale = c.key_scale;
  p.value_scale = c.value_scale;
  p.slots = slots;
  p.key_stride = key_stride;
  p.value_stride = value_stride;
  p.page_stride = c.page_stride;
  p.head_stride = c.head_stride;
  p.token_stride = c.token_stride;
  p.num_pages = c.num_pages;
  p.per_row = make_fastdiv(c.D / 8);
  p.per_token = make_fastdiv(c.heads * (c.D / 8));
  p.page_tokens = make_fastdiv(c.page_tokens);
  p.parts = tokens * p.per_token.d;
  const uint64_t blocks = (p.parts + 255) / 256;
  if (blocks > 0x7FFFFFFFull) return fail(GORIO_EINVAL, "tokens=%llu too large", (unsigned long long)tokens);
  const dim3 grid((uint32_t)blocks, 2);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (c.dtype != GORIO_KV_E4M3) store_kernel<0><<<grid, 256, 0, s>>>(p);
  else if (dtype == GORIO_KV_BF16) store_kernel<1><<<grid, 256, 0, s>>>(p);
  else store_kernel<2><<<grid, 256, 0, s>>>(p);
  return kv_launched("gorio_kv_store");
}
