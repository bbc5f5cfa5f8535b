// What the entry points of the paged key/value calls share: argument checks
// on the host, and the calling thread's device.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstring>
#include <initializer_list>

#include "../../include/gorio.h"
#include "common.hpp"

namespace gorio {

gorio_status fail(gorio_status st, const char *fmt, ...);

// Switches to the device that holds an array for the scope of a call.
class KvDevice {
 public:
  KvDevice() = default;
  KvDevice(const KvDevice &) = delete;
  ~KvDevice() {
    if (prev_ >= 0) (void)hipSetDevice(prev_);
  }

  // Each named array is device memory of one GPU, and starts at a multiple of
  // its alignment; NULL where `optional`.  Selects that GPU.
  struct Array {
    const char *name;
    const void *ptr;
    uint32_t align;
    bool optional;
  };
  gorio_status use(std::initializer_list<Array> arrays) {
    int dev = -1;
    for (const Array &a : arrays) {
      if (!a.ptr) {
        if (a.optional) continue;
        return fail(GORIO_EINVAL, "%s is NULL", a.name);
      }
      if ((uintptr_t)a.ptr % a.align != 0)
        return fail(GORIO_EINVAL, "%s must start at a multiple of %u bytes", a.name, a.align);
      hipPointerAttribute_t at;
      if (hipPointerGetAttributes(&at, a.ptr) != hipSuccess) {
        (void)hipGetLastError();
        return fail(GORIO_EINVAL, "%s is no device pointer", a.name);
      }
      if (at.type != hipMemoryTypeDevice && !at.isManaged)
        return fail(GORIO_EINVAL, "%s is no device pointer", a.name);
      if (dev >= 0 && at.device != dev)
        return fail(GORIO_EINVAL, "%s is on device %d, an earlier array on %d", a.name, at.device, dev);
      dev = at.device;
    }
    int now = -1;
    if (hipGetDevice(&now) != hipSuccess) return fail(GORIO_EDEVICE, "hipGetDevice failed");
    if (now != dev) {
      if (hipSetDevice(dev) != hipSuccess) return fail(GORIO_EDEVICE, "cannot select device %d", dev);
      prev_ = now;
    }
    return GORIO_OK;
  }

 private:
  int prev_ = -1;
};

// Arrays of a call whose blocks run in any order: one that is written shares no byte with another.
struct KvSpan {
  const char *name;
  const void *ptr;  // NULL: none
  uint64_t bytes;
  bool written;
};
inline gorio_status kv_apart(std::initializer_list<KvSpan> spans) {
  for (const KvSpan *a = spans.begin(); a != spans.end(); ++a)
    for (const KvSpan *b = a + 1; b != spans.end(); ++b) {
      const uintptr_t x = (uintptr_t)a->ptr, y = (uintptr_t)b->ptr;
      if ((a->written || b->written) && x && y && a->bytes && b->bytes && x < y + b->bytes && y < x + a->bytes)
        return fail(GORIO_EINVAL, "%s and %s overlap", a->name, b->name);
    }
  return GORIO_OK;
}

inline gorio_status kv_launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? GORIO_OK : fail(GORIO_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

constexpr uint64_t kKvMost = 0x7FFFFFFFull;  // tokens, pages, requests: below 2^31

// Elements of a block with a power of two of its own.
constexpr uint32_t kMxBlock = 32;
inline bool kv_is_mx(uint32_t dtype) { return dtype == GORIO_KV_MX8 || dtype == GORIO_KV_MX4; }
// Bytes of so many elements.
inline uint64_t kv_bytes(uint32_t dtype, uint64_t elements) {
  return dtype == GORIO_KV_MX4 ? elements / 2 : dtype == GORIO_KV_MX8 || dtype == GORIO_KV_E4M3 ? elements : elements * 2;
}

// The cache's sizes and strides, the strides filled in.
inline gorio_status kv_check_cache(const gorio_kv_cache *c, gorio_kv_cache *out) {
  if (!c) return fail(GORIO_EINVAL, "cache is NULL");
  if (c->dtype > GORIO_KV_E4M3 && !kv_is_mx(c->dtype))
    return fail(GORIO_EINVAL, "cache dtype %u is no gorio_kv_dtype", c->dtype);
  if (c->heads == 0 || c->heads > 1024) return fail(GORIO_EINVAL, "cache heads=%u, need 1..1024", c->heads);
  if (c->D == 0 || c->D % 8 != 0 || c->D > 256)
    return fail(GORIO_EINVAL, "D=%u, need a multiple of 8 in 8..256", c->D);
  if (c->page_tokens == 0 || c->page_tokens > 65536)
    return fail(GORIO_EINVAL, "page_tokens=%u, need 1..65536", c->page_tokens);
  if (c->num_pages == 0 || c->num_pages > kKvMost)
    return fail(GORIO_EINVAL, "num_pages=%llu, need 1..2^31-1", (unsigned long long)c->num_pages);
  const uint32_t whole = kv_is_mx(c->dtype) ? kMxBlock : 8;  // elements
  if (c->D % whole != 0) return fail(GORIO_EINVAL, "D=%u, need a multiple of %u for these pages", c->D, whole);
  // a caller that knows no powers may have a shorter struct
  memcpy(out, c, kv_is_mx(c->dtype) ? sizeof *c : offsetof(gorio_kv_cache, key_powers));
  if (!kv_is_mx(c->dtype)) out->key_powers = out->value_powers = nullptr;
  if (c->page_stride == 0 && c->head_stride == 0 && c->token_stride == 0) {
    out->token_stride = c->D;
    out->head_stride = (uint64_t)c->D * c->page_tokens;
    out->page_stride = out->head_stride * c->heads;
  }
  if (out->page_stride % whole || out->head_stride % whole || out->token_stride % whole)
    return fail(GORIO_EINVAL, "the cache's strides must be multiples of %u elements", whole);
  if (c->dtype != GORIO_KV_E4M3 && (c->key_scale || c->value_scale))
    return fail(GORIO_EINVAL, "key_scale and value_scale belong to GORIO_KV_E4M3 pages");
  return GORIO_OK;
}

}  // namespace gorio
