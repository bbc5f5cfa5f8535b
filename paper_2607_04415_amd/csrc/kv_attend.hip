// gorio_kv_attend: attention of new tokens over the pages of their requests.
#include <algorithm>

#include "kv_launch.hpp"

using namespace gorio;

namespace {

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
  if (a->tokens * (a->heads / c->heads) > kKvMost)
    return fail(GORIO_EINVAL, "tokens=%llu x %u heads a key head: need at most 2^31-1", (unsigned long long)a->tokens,
                a->heads / c->heads);
  *out = *a;
  if (a->q_stride == 0) out->q_stride = (uint64_t)a->heads * c->D;
  if (a->out_stride == 0) out->out_stride = (uint64_t)a->heads * c->D;
  if (out->q_stride % 8 || out->out_stride % 8)
    return fail(GORIO_EINVAL, "q_stride and out_stride must be multiples of 8 elements");
  // twice the cap, and the scale, are kept in log2: up to 1e38 neither overflows
  if (!(a->cap >= 0.f) || !(a->cap <= 1e38f))
    return fail(GORIO_EINVAL, "cap=%g, need a number in 0..1e38", (double)a->cap);
  if (!(a->scale <= 1e38f && a->scale >= -1e38f))
    return fail(GORIO_EINVAL, "scale=%g, need a number in -1e38..1e38", (double)a->scale);
  return GORIO_OK;
}

// Rows of a request and key head from which the form for many rows takes it.  The other form
// reads every key once per 16 rows.  16 requests of 12 rows over 4000 tokens: 56 us, by the form
// for many rows 70; of 20 rows 58 (its second reading is cached) and 72; but 64 requests over
// 16000 tokens, which no cache holds: of 16 rows 702 and 764 us, of 20 rows 1385 and 764.
constexpr uint32_t kFewUpto = 17;

// What a call launches and keeps, from the sizes that the host knows: the
// lengths are on the GPU, so these are bounds, and workgroups without work
// return.  `all`: workgroups that run at once on the GPU.  one_tile: no
// request that the form takes has more than one tile.
AttendForm divide(const gorio_kv_cache &c, const gorio_kv_attention &a, uint32_t rows, uint32_t block, uint32_t least,
                  uint32_t whole, uint32_t all, bool one_tile) {
  AttendForm f{};
  const uint64_t tiles = (one_tile ? 0 : a.tokens * (a.heads / c.heads) / rows) + std::min<uint64_t>(a.requests, a.tokens);
  const uint64_t blocks = ((uint64_t)a.width * c.page_tokens + block - 1) / block;
  f.rows = rows;
  f.from = 1;
  f.upto = 0xFFFFFFFFu;
  f.least = least;
  f.whole = whole;
  f.shares = (uint32_t)std::min<uint64_t>(std::max(all / c.heads, 1u), (tiles * blocks + least - 1) / least);
  f.cuts = f.shares > 1 && blocks > whole;
  return f;
}

// The forms that a call needs, and its workspace, which they use in turn.
AttendLaunch forms_of(const gorio_kv_cache &c, const gorio_kv_attention &a, uint64_t *bytes) {
  AttendLaunch l{};
  l.e4m3 = c.dtype == GORIO_KV_E4M3;
  l.more = a.cap > kQuickCap ? 3 : a.cap > 0.f ? 2 : a.slopes ? 1 : 0;
  const uint64_t group = a.heads / c.heads;
  // The most new tokens of a request, and the fewest of one that has any, as far as the host can
  // tell: rows of q may be padding, which counts as new tokens here, and max_new may be too small.
  // So they decide only which form is the faster one.  `fewest` is at most `most`, so that one form
  // is launched always, and a form launched alone takes requests of any number of rows.
  const uint64_t most = a.max_new ? std::min<uint64_t>(a.max_new, a.tokens) : a.tokens;
  const uint64_t others = (a.requests - 1) * most;
  const uint64_t fewest = a.tokens > others ? std::min(a.tokens - others, most) : 1;
  const bool few = fewest * group < kFewUpto, many = most * group >= kFewUpto;
  const int steps = steps_of(c.D);
  // The least share and the largest tile that is not cut, in blocks.  Few rows: 8 blocks are one
  // a wave; 8 requests of 250 tokens take 13 us, with shares of 16 blocks 19, of 32 31 us.  Tiles
  // of up to 16 are not cut: 8 requests of 500 tokens take 16 us, cut from 8 on 19; one of 1000
  // takes the same 20 us either way.  Tiles of fewer blocks than the least share are packed into
  // one, though, and run one after the other: 64 requests of 20 tokens take 41 us, of 60 25, of
  // 100 17, where 16 of 250 take 12.  Many rows: 128 new tokens over 500 take 33 us, with shares
  // of 8 blocks 54 us, 64 over 250 in 8 requests 23 and 40; of 2 blocks, over 2000, 68 instead of
  // 50 us.  Tiles of up to 8 are not cut: one of 500 keys takes 33 us, cut from 4 on 43; up to 16,
  // 8 requests of 64 over 1000 tokens take 47 instead of 42 us.
  // Workgroups: as many as run at once, a CU each for few rows, which has 128 KB of loads under way
  // then (64 requests of 16384 tokens take 451 us, and 454 with twice as many workgroups); for many
  // rows see attend_many.
  if (few) l.few = divide(c, a, kFewRows, kFewBlock, 8, 16, 256, many);
  if (many) l.many = divide(c, a, many_rows(steps), kManyBlock, 4, 8, steps == 2 ? 768 : steps == 3 ? 512 : 256, false);
  if (few && many) l.few.upto = l.many.from = kFewUpto;
  auto room = [&](const AttendForm &f) -> uint64_t {  // of a share and key head: two parts, and which tile is cut
    return f.cuts ? (uint64_t)f.shares * c.heads * (2 * (c.D + 2) * sizeof(float) * f.rows + sizeof(Cut)) : 0;
  };
  *bytes = std::max(room(l.few), room(l.many));
  return l;
}

}  // namespace

extern "C" gorio_status gorio_kv_workspace(const gorio_kv_cache *cache, const gorio_kv_attention *a, uint64_t *bytes) {
  gorio_kv_cache c;
  gorio_kv_attention at;
  const gorio_status st = check(cache, a, &c, &at);
  if (st != GORIO_OK) return st;
  if (!bytes) return fail(GORIO_EINVAL, "bytes is NULL");
  *bytes = 0;
  if (at.tokens && at.requests) (void)forms_of(c, at, bytes);
  return GORIO_OK;
}

extern "C" gorio_status gorio_kv_attend(const gorio_kv_cache *cache, const gorio_kv_attention *a, void *workspace,
                                        uint64_t workspace_bytes, void *stream) {
  gorio_kv_cache c;
  gorio_kv_attention at;
  gorio_status st = check(cache, a, &c, &at);
  if (st != GORIO_OK) return st;
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
                {"value_scale", c.value_scale, 4, true},
                {"workspace", workspace, 16, workspace_bytes == 0}});
  if (st != GORIO_OK) return st;
  uint64_t bytes = 0;
  const AttendLaunch l = forms_of(c, at, &bytes);
  if (bytes > workspace_bytes)
    return fail(GORIO_EINVAL, "workspace of %llu bytes, need %llu", (unsigned long long)workspace_bytes,
                (unsigned long long)bytes);
  const uint32_t group = at.heads / c.heads, element = c.dtype == GORIO_KV_E4M3 ? 1 : 2;
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
  p.parts = static_cast<float *>(workspace);
  p.q_stride = at.q_stride;
  p.out_stride = at.out_stride;
  p.page_stride = c.page_stride * element;
  p.head_stride = c.head_stride * element;
  p.token_stride = c.token_stride * element;
  p.tokens = (uint32_t)at.tokens;
  p.num_pages = (uint32_t)c.num_pages;
  p.requests = at.requests;
  p.width = at.width;
  p.heads = at.heads;
  p.kv_heads = c.heads;
  p.D = c.D;
  p.page_tokens = make_fastdiv(c.page_tokens);
  p.group = make_fastdiv(group);
  p.by_kv = make_fastdiv(c.heads);
  p.scale = at.scale;
  p.cap = at.cap;
  p.window = at.window ? at.window : (uint32_t)kKvMost;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool f16 = at.dtype == GORIO_KV_F16;
  const hipError_t e = l.e4m3 ? (f16 ? launch_attend_f16_e4m3(p, l, s) : launch_attend_bf16_e4m3(p, l, s))
                              : (f16 ? launch_attend_f16(p, l, s) : launch_attend_bf16(p, l, s));
  return e == hipSuccess ? GORIO_OK : fail(GORIO_EDEVICE, "gorio_kv_attend: %s", hipGetErrorString(e));
}
