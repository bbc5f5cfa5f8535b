// gorio_kv_store: rows of new keys and values into their slots.
//
// A copy whose destination rows are scattered: a thread moves 8 elements (16
// bytes) of a key and of its value, neighbouring threads neighbouring parts of
// a row.  A block's first token is divided out once, so that the threads' own
// divisions are multiplications of 32 bits.  Bound by HBM where there are many
// tokens: 16384 of 8 heads of 128 into 8-bit pages, 101 MB in and out, take
// 24.7 us (4.1 TB/s; a large copy reaches 4.8), without factors 20.4, into
// 16-bit pages 24.3 (134 MB, 5.5 TB/s); 64 tokens take 3.9 us, the
// latency of a slot and then of a row.  An 8-bit element is rounded once, from
// the quotient in 32 bits.
// Blocks of 32 elements with a power lie in four neighbouring lanes: the largest
// size is found on the elements' bits, in two exchanges, and the power, its
// inverse and the products are exact, so an element is rounded once.  16384
// tokens of 8 heads of 128 take 18.6 us into MX8 pages (102 MB, 5.5 TB/s) and
// 15.6 into MX4 (85 MB, 5.4 TB/s); 64 tokens 5.1.
#include "kv.hpp"

#include "kv_mx.hpp"

using namespace gorio;

namespace {

struct StoreParams {
  const uint16_t *keys, *values;  // 16-bit elements, bf16 or f16
  uint8_t *to_keys, *to_values;
  const float *key_scale, *value_scale;
  uint8_t *key_powers, *value_powers;
  const int64_t *slots;
  uint64_t key_stride, value_stride;  // elements
  uint64_t page_stride, head_stride, token_stride;
  uint64_t num_pages;
  uint64_t parts;  // 8-element parts of the keys: tokens * heads * D / 8, of which a block takes kParts
  FastDiv per_row, per_token;  // parts of a head's row, and of a token
  FastDiv page_tokens;
};

// +-448 is the largest value of the 8-bit type; a NaN stays one.
__device__ __forceinline__ float clamp_e4m3(float x) { return x > 448.f ? 448.f : x < -448.f ? -448.f : x; }

// x / scale for the 8-bit type, x of 16 bits.  A division takes a dozen instructions, some of them
// slow, so there is one a row's part and not one an element (28 us in all then): with r the nearest
// value to 1 / scale, x r is off by at most two units in the last place, one correction by the
// remainder, which is exact, leaves it off by at most one, and after a second it is the nearest
// value to the quotient (Markstein's theorem), while nothing overflows or underflows: for factors
// of 2^-60 to 2^60, quotients up to 449 and those that are not 0 in 8 bits.  Others need no
// correction: they are clamped, or 0, or NaN.
struct Divisor {
  float scale, r;
  bool whole;  // divide after all
  __device__ __forceinline__ explicit Divisor(float s)
      : scale(s), r(1.f / s), whole(!(fabsf(s) >= 0x1p-60f && fabsf(s) <= 0x1p60f)) {}
  __device__ __forceinline__ float quotient(float x) const {
    const float q = x * r;
    float y = __builtin_fmaf(__builtin_fmaf(-q, scale, x), r, q);
    y = __builtin_fmaf(__builtin_fmaf(-y, scale, x), r, y);
    return fabsf(q) <= 449.f ? y : q;
  }
};

constexpr uint32_t kParts = 1024;

// Eight elements as they are (kTo 0), or bf16 (1) or f16 (2) to e4m3; 3 to 6: bf16 and f16 to
// e4m3 and to e2m1 by blocks.
template <int kTo>
__device__ __forceinline__ void put(uint8_t *pages, uint64_t to, const uint4 &x, bool scaled, float scale) {
  if constexpr (kTo == 0) {
    *reinterpret_cast<uint4 *>(pages + to * 2) = x;
  } else {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = to_float((uint16_t)(w[i / 2] >> (16 * (i & 1))), kTo == 2);
    if (scaled) {
      const Divisor by(scale);
      if (by.whole) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] /= by.scale;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = by.quotient(f[i]);
      }
    }
    int packed[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      packed[i] = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(f[i * 4]), clamp_e4m3(f[i * 4 + 1]), 0, false);
      packed[i] = __builtin_amdgcn_cvt_pk_fp8_f32(clamp_e4m3(f[i * 4 + 2]), clamp_e4m3(f[i * 4 + 3]), packed[i], true);
    }
    *reinterpret_cast<int2 *>(pages + to) = make_int2(packed[0], packed[1]);
  }
}

// Eight elements of a block of 32, whose other parts the quad's other lanes hold, to `to` elements
// from the pages' start on; `to` is of the block's first lane in the block's own.
template <bool kF16, bool k4>
__device__ __forceinline__ void put_mx(uint8_t *pages, uint8_t *powers, uint64_t to, const uint4 &x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t most = 0;  // sizes' bits, NaN and inf above all others
#pragma unroll
  for (int i = 0; i < 4; ++i) most = max(max(most, w[i] & 0x7FFFu), w[i] >> 16 & 0x7FFFu);
  most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xB1, 0xF, 0xF, true));  // lanes 1, 0, 3, 2
  most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4E, 0xF, 0xF, true));  // lanes 2, 3, 0, 1
  const uint32_t power = mx_power<k4>(to_float((uint16_t)most, kF16));
  const float by = mx_inverse(power);
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = to_float((uint16_t)(w[i / 2] >> (16 * (i & 1))), kF16) * by;
  if (power == 255) {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.f;
  }
  if constexpr (k4) {
    *reinterpret_cast<uint32_t *>(pages + to / 2) = to_e2m1(f);
  } else {
    *reinterpret_cast<uint2 *>(pages + to) = to_e4m3(f);
  }
  if (to % kMxBlock == 0) powers[to / kMxBlock] = (uint8_t)power;
}

template <int kTo>
__global__ __launch_bounds__(256) void store_kernel(StoreParams p) {
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
    if (slot < 0) continue;
    const uint64_t page = slot < (1ll << 31) ? fastdiv((uint32_t)slot, p.page_tokens) : (uint64_t)slot / p.page_tokens.d;
    if (page >= p.num_pages) continue;
    const uint32_t place = (uint32_t)((uint64_t)slot - page * p.page_tokens.d);
    const uint32_t from = head * p.per_row.d * 8 + d;
    const float by_key = kTo && kTo < 3 && p.key_scale ? p.key_scale[head] : 1.f;
    const float by_value = kTo && kTo < 3 && p.value_scale ? p.value_scale[head] : 1.f;
    const uint4 k = *reinterpret_cast<const uint4 *>(p.keys + token * p.key_stride + from);
    const uint4 v = *reinterpret_cast<const uint4 *>(p.values + token * p.value_stride + from);
    const uint64_t to = page * p.page_stride + head * p.head_stride + place * p.token_stride + d;
    if constexpr (kTo >= 3) {
      // the lanes of a block are in here together: its token's slot, and the end, are theirs alike
      put_mx<(kTo & 1) == 0, (kTo > 4)>(p.to_keys, p.key_powers, to, k);
      put_mx<(kTo & 1) == 0, (kTo > 4)>(p.to_values, p.value_powers, to, v);
    } else {
      put<kTo>(p.to_keys, to, k, p.key_scale, by_key);
      put<kTo>(p.to_values, to, v, p.value_scale, by_value);
    }
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
  if (c.dtype < GORIO_KV_E4M3 && (gorio_kv_dtype)c.dtype != dtype)
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
                {"value_scale", c.value_scale, 4, true},
                {"key_powers", c.key_powers, 1, !kv_is_mx(c.dtype)},
                {"value_powers", c.value_powers, 1, !kv_is_mx(c.dtype)}});
  if (st != GORIO_OK) return st;
  StoreParams p;
  p.keys = static_cast<const uint16_t *>(keys);
  p.values = static_cast<const uint16_t *>(values);
  p.to_keys = static_cast<uint8_t *>(c.keys);
  p.to_values = static_cast<uint8_t *>(c.values);
  p.key_scale = c.key_scale;
  p.value_scale = c.value_scale;
  p.key_powers = c.key_powers;
  p.value_powers = c.value_powers;
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
  // at most 2^31 tokens of 2^15 parts; a launch has less than 2^32 threads
  const uint64_t grid = (p.parts + kParts - 1) / kParts;
  if (grid >= 1ull << 24) return fail(GORIO_EINVAL, "tokens=%llu too large", (unsigned long long)tokens);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool f16 = dtype == GORIO_KV_F16;
  auto launch = [&](void (*kernel)(StoreParams)) { kernel<<<(uint32_t)grid, 256, 0, s>>>(p); };
  switch (c.dtype) {
    case GORIO_KV_E4M3: launch(f16 ? store_kernel<2> : store_kernel<1>); break;
    case GORIO_KV_MX8: launch(f16 ? store_kernel<4> : store_kernel<3>); break;
    case GORIO_KV_MX4: launch(f16 ? store_kernel<6> : store_kernel<5>); break;
    default: launch(store_kernel<0>);
  }
  return kv_launched("gorio_kv_store");
}
