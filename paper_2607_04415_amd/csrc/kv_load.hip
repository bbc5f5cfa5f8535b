// gorio_kv_load: rows of keys and values from their slots.
//
// The store's copy the other way: a thread moves 8 elements of a key and of its
// value, neighbouring threads neighbouring parts of a row, widened on the way.
// Bound by HBM where there are many: 16384 rows of 8 heads of 128 that no cache
// holds take 21.4 us from MX8 pages (102 MB, 4.75 TB/s; a large copy moves 4.85),
// 19.7 from MX4 (85 MB, 4.3), 25.2 from 16-bit pages (134 MB, 5.3) and 20.5 from
// e4m3 (101 MB, 4.9), 131072 rows 162, 143, 211 and 159 us (4.8 to 5.1 TB/s); 2000
// rows 5.8 us, the latency of a slot and then of a row.
#include "kv.hpp"
#include "kv_mx.hpp"

using namespace gorio;

namespace {

struct LoadParams {
  const uint8_t *keys, *values;
  const float *key_scale, *value_scale;
  const uint8_t *key_powers, *value_powers;
  uint16_t *to_keys, *to_values;
  const int64_t *slots;
  uint64_t key_stride, value_stride;  // elements
  uint64_t page_stride, head_stride, token_stride;
  uint64_t num_pages;
  uint64_t parts;  // 8-element parts of the keys: tokens * heads * D / 8, of which a block takes kParts
  FastDiv per_row, per_token;  // parts of a head's row, and of a token
  FastDiv page_tokens;
};

constexpr uint32_t kParts = 1024;

__device__ __forceinline__ uint32_t pack(float x, float y, bool f16) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  if (f16) {
    const f16x2 v = {(_Float16)x, (_Float16)y};
    return __builtin_bit_cast(uint32_t, v);
  }
  const bf16x2 v = {(__bf16)x, (__bf16)y};
  return __builtin_bit_cast(uint32_t, v);
}

// Eight elements from `at` elements behind the pages' start on: as they are (kFrom 0), or e4m3 by
// a factor (1), e4m3 (2) and e2m1 (3) by blocks.
template <int kFrom, bool kF16>
__device__ __forceinline__ uint4 get(const uint8_t *pages, const uint8_t *powers, uint64_t at, float by) {
  if constexpr (kFrom == 0) {
    return *reinterpret_cast<const uint4 *>(pages + at * 2);
  } else {
    float f[8];
    if constexpr (kFrom == 3) from_e2m1(*reinterpret_cast<const uint32_t *>(pages + at / 2), f);
    else from_e4m3(*reinterpret_cast<const uint2 *>(pages + at), f);
    if constexpr (kFrom > 1) by = mx_factor(powers[at / kMxBlock]);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= by;
    return make_uint4(pack(f[0], f[1], kF16), pack(f[2], f[3], kF16), pack(f[4], f[5], kF16), pack(f[6], f[7], kF16));
  }
}

template <int kFrom, bool kF16>
__global__ __launch_bounds__(256) void load_kernel(LoadParams p) {
  const uint64_t part0 = (uint64_t)blockIdx.x * kParts, token0 = part0 / p.per_token.d;
  const uint32_t in0 = (uint32_t)(part0 - token0 * p.per_token.d);
#pragma unroll
  for (uint32_t i = 0; i < kParts / 256; ++i) {
    const uint32_t at = i * 256 + threadIdx.x;
    if (part0 + at >= p.parts) return;
    const uint32_t n = fastdiv(in0 + at, p.per_token), in = in0 + at - n * p.per_token.d;
    const uint64_t token = token0 + n;
    const uint32_t head = fastdiv(in, p.per_row), d = (in - head * p.per_row.d) * 8;
    const int64_t slot = p.slots[token];
    const uint64_t page = slot < 0 ? ~0ull
                          : slot < (1ll << 31) ? fastdiv((uint32_t)slot, p.page_tokens) : (uint64_t)slot / p.page_tokens.d;
    uint4 k = make_uint4(0, 0, 0, 0), v = k;
    if (page < p.num_pages) {
      const uint32_t place = (uint32_t)((uint64_t)slot - page * p.page_tokens.d);
      const uint64_t from = page * p.page_stride + head * p.head_stride + place * p.token_stride + d;
      k = get<kFrom, kF16>(p.keys, p.key_powers, from, kFrom == 1 && p.key_scale ? p.key_scale[head] : 1.f);
      v = get<kFrom, kF16>(p.values, p.value_powers, from, kFrom == 1 && p.value_scale ? p.value_scale[head] : 1.f);
    }
    const uint32_t to = head * p.per_row.d * 8 + d;
    *reinterpret_cast<uint4 *>(p.to_keys + token * p.key_stride + to) = k;
    *reinterpret_cast<uint4 *>(p.to_values + token * p.value_stride + to) = v;
  }
}

// Whether a row of keys and one of values share a byte; rows of one array do not.  All in bytes.
bool rows_meet(uintptr_t keys, uint64_t key_step, uintptr_t values, uint64_t value_step, uint64_t row, uint64_t tokens) {
  if (keys >= values + (tokens - 1) * value_step + row || values >= keys + (tokens - 1) * key_step + row) return false;
  if (key_step == value_step) {  // parts of one wider row: how far behind a key's row the next value's begins
    const uint64_t behind = values >= keys ? (values - keys) % key_step : key_step - 1 - (keys - values - 1) % key_step;
    return behind < row || key_step - behind < row;
  }
  for (uint64_t i = 0, j = 0; i < tokens && j < tokens;) {
    const uintptr_t k = keys + i * key_step, v = values + j * value_step;
    if (k < v + row && v < k + row) return true;
    if (k < v) ++i;
    else ++j;
  }
  return false;
}

}  // namespace

extern "C" gorio_status gorio_kv_load(const gorio_kv_cache *cache, gorio_kv_dtype dtype, const int64_t *slots,
                                      uint64_t tokens, void *keys, void *values, uint64_t key_stride,
                                      uint64_t value_stride, void *stream) {
  gorio_kv_cache c;
  gorio_status st = kv_check_cache(cache, &c);
  if (st != GORIO_OK) return st;
  if (dtype != GORIO_KV_BF16 && dtype != GORIO_KV_F16)
    return fail(GORIO_EINVAL, "keys and values must be bf16 or f16, not gorio_kv_dtype %d", (int)dtype);
  if (c.dtype < GORIO_KV_E4M3 && (gorio_kv_dtype)c.dtype != dtype)
    return fail(GORIO_EUNSUPPORTED, "16-bit pages give keys and values of their own type");
  if (tokens > kKvMost) return fail(GORIO_EINVAL, "tokens=%llu too large", (unsigned long long)tokens);
  const uint64_t row = (uint64_t)c.heads * c.D;
  if (key_stride == 0) key_stride = row;
  if (value_stride == 0) value_stride = row;
  if (key_stride % 8 || value_stride % 8)
    return fail(GORIO_EINVAL, "key_stride and value_stride must be multiples of 8 elements");
  if (tokens > 1 && (key_stride < row || value_stride < row))
    return fail(GORIO_EINVAL, "key_stride and value_stride must be at least heads * D = %llu: rows are written",
                (unsigned long long)row);
  if (tokens == 0) return GORIO_OK;
  KvDevice dev;
  st = dev.use({{"keys", keys, 16, false},
                {"values", values, 16, false},
                {"slots", slots, 8, false},
                {"cache keys", c.keys, 16, false},
                {"cache values", c.values, 16, false},
                {"key_scale", c.key_scale, 4, true},
                {"value_scale", c.value_scale, 4, true},
                {"key_powers", c.key_powers, 1, !kv_is_mx(c.dtype)},
                {"value_powers", c.value_powers, 1, !kv_is_mx(c.dtype)}});
  if (st != GORIO_OK) return st;
  LoadParams p;
  p.keys = static_cast<const uint8_t *>(c.keys);
  p.values = static_cast<const uint8_t *>(c.values);
  p.key_scale = c.key_scale;
  p.value_scale = c.value_scale;
  p.key_powers = c.key_powers;
  p.value_powers = c.value_powers;
  p.to_keys = static_cast<uint16_t *>(keys);
  p.to_values = static_cast<uint16_t *>(values);
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
  const uint64_t grid = (p.parts + kParts - 1) / kParts;  // a launch has less than 2^32 threads
  if (grid >= 1ull << 24) return fail(GORIO_EINVAL, "tokens=%llu too large", (unsigned long long)tokens);
  // rows that are written overlap neither one another, though keys and values may alternate, nor the slots
  if (rows_meet((uintptr_t)keys, key_stride * 2, (uintptr_t)values, value_stride * 2, row * 2, tokens))
    return fail(GORIO_EINVAL, "keys and values overlap");
  st = kv_apart({{"keys", keys, key_stride == row ? tokens * row * 2 : 0, true},
                 {"values", values, value_stride == row ? tokens * row * 2 : 0, true},
                 {"slots", slots, tokens * 8, false}});
  if (st != GORIO_OK) return st;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool f16 = dtype == GORIO_KV_F16;
  auto launch = [&](void (*kernel)(LoadParams)) { kernel<<<(uint32_t)grid, 256, 0, s>>>(p); };
  switch (c.dtype) {
    case GORIO_KV_E4M3: launch(f16 ? load_kernel<1, true> : load_kernel<1, false>); break;
    case GORIO_KV_MX8: launch(f16 ? load_kernel<2, true> : load_kernel<2, false>); break;
    case GORIO_KV_MX4: launch(f16 ? load_kernel<3, true> : load_kernel<3, false>); break;
    default: launch(load_kernel<0, false>);
  }
  return kv_launched("gorio_kv_load");
}
