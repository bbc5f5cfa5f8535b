// Attention of many query rows over many keys: the form for chunks.
//
// With 128 rows to a tile every key is used often enough that the matrix units
// are the bound, and next to them the vector units, which turn 2 x 32 x 32
// products into exponentials for every 16 matrix instructions.  Each of four
// waves owns 32 rows for the whole run; blocks of 64 keys and values pass
// through LDS, two buffers deep, so that a block's loads run during the
// products of the one before and a barrier a block suffices.  Two workgroups
// fit a CU, and one's exponentials run beside the other's products.  On
// 32x32x16 instructions:
//   S^T = K Q^T: lane (m, g) = (lane % 32, lane / 32) reads elements 16 s + 8 g
//     .. + 7 of key m; the result gives it, of query m, the scores of keys
//     8 i + 4 g .. + 3 for i = 0..3.
//   O^T = V^T P^T: sixteen keys at a time, of which the lane has the weights
//     of 4 g .. + 3 and 8 + 4 g .. + 3; the transposing LDS read gives it the
//     values of those keys at element m.
// Key rows are padded by 16 bytes, so that 16 neighbouring keys' 16-byte reads
// fall on different banks; value rows to 64 or 192 bytes past a multiple of
// 256, so that four keys' 64-byte reads do.
#pragma once

#include <type_traits>

#include "kv_attend.hpp"

namespace gorio {

constexpr int kManyWaves = 4;
constexpr int kManyThreads = kManyWaves * 64;
constexpr int kManyRows = kManyWaves * 32;
constexpr int kManyBlock = 64;  // keys

// A maximum is kept until a score passes it by 2^8 (weights stay far inside
// f16's range, and a sum of them loses nothing): most blocks then rescale nothing.
constexpr float kSlack = 8.f;

// The low n bits, n of any size.
__device__ __forceinline__ uint64_t low_bits(int32_t n) {
  const uint64_t some = (1ull << (n & 63)) - 1;
  return n <= 0 ? 0 : n >= 64 ? ~0ull : some;
}

// kSteps: D <= 32 kSteps.  k8: pages of 8-bit values.  kMore: scores are capped or biased.
template <typename Q, bool k8, int kSteps, bool kMore>
__global__ __launch_bounds__(kManyThreads, kSteps > 4 ? 1 : 2) void attend_many(AttendParams p) {
  constexpr int kDim = kSteps * 32, kChunks = kDim / 8;
  constexpr int kKeyRow = kDim + 8;                                                  // elements
  constexpr int kValueRow = (kDim * 2) % 256 == 192 ? kDim : kDim + 32;
  constexpr int kPasses = kManyBlock * kChunks / kManyThreads;                       // 16-byte pieces a thread
  static_assert(kPasses * kManyThreads == kManyBlock * kChunks, "pieces divide");
  constexpr int kElem = k8 ? 1 : 2;
  typedef typename std::conditional<k8, u32x2, u32x4>::type Raw;
  __shared__ __align__(16) uint16_t s_k[2][kManyBlock * kKeyRow];
  __shared__ __align__(16) uint16_t s_v[2][kManyBlock * kValueRow];
  __shared__ uint64_t s_row[2][2][kManyBlock];  // turn, keys or values
  __shared__ uint64_t s_there[4];
  // Values that are NaN or inf in a block that not all rows see: a weight of 0 would not keep
  // them out of a row.  They are 0 in s_v; here are the keys that have one at an element,
  // +inf (or NaN) and -inf (or NaN).
  __shared__ uint64_t s_odd[2][kDim];
  __shared__ uint32_t s_any_odd[2][kManyWaves];  // turn, wave that found one

  const uint32_t index = fastdiv(blockIdx.x, p.by_kv), head = blockIdx.x - index * p.kv_heads;
  WorkItem w;
  if (!find_item<kManyThreads, kManyBlock, false>(p, index, w)) return;
  const Tile tile = tile_of(p, w);
  const KeyRange range = key_range<kManyBlock>(p, w.r, tile.first, tile.last);
  const uint32_t parts = max(((uint32_t)range.count + w.c - 1) / w.c, 1u);
  if (w.part >= parts) return;
  const int32_t x0 = (int32_t)(w.part * w.c);
  const int32_t x_end = (int32_t)min((int64_t)range.count, (int64_t)x0 + w.c);

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int m = lane & 31, g = lane >> 5;
  const uint64_t zeros = (uint64_t)(uintptr_t)kv_zeros;

  // this lane's query; rows past the last repeat it
  const uint32_t wave_row = tile.row0 + min((uint32_t)wave * 32, tile.rows - 1);
  const uint32_t wave_end = min(tile.row0 + (uint32_t)wave * 32 + 31, tile.row0 + tile.rows - 1);
  const bool has_rows = (uint32_t)wave * 32 < tile.rows;
  const uint32_t row = min(tile.row0 + (uint32_t)wave * 32 + m, tile.row0 + tile.rows - 1);
  const uint32_t token = fastdiv(row, p.group), gh = row - token * p.group.d;
  const int32_t base = w.r.len - w.r.added;
  const int32_t pos = base + (int32_t)token;
  const int32_t oldest = (int32_t)max((int64_t)pos - p.window + 1, (int64_t)0);  // the window's first key
  const int32_t first = base + (int32_t)fastdiv(wave_row, p.group), last = base + (int32_t)fastdiv(wave_end, p.group);
  const uint32_t qhead = head * p.group.d + gh;
  const float scale = p.scale * (p.key_scale ? p.key_scale[head] : 1.f);
  // the running maximum is taken of the products as they are, so the factor has to be positive:
  // a negative one turns the queries' signs around
  const uint32_t flip = !kMore && scale < 0.f ? 0x80008000u : 0u;
  const float factor = scale == 0.f ? 1e-30f : fabsf(scale) * kLog2e;  // 0 times a masked score's -inf would be NaN
  u32x4 q[kSteps * 2];
  {
    const uint16_t *at = p.q + (uint64_t)(w.r.start + token) * p.q_stride + (uint64_t)qhead * p.D;
#pragma unroll
    for (int s = 0; s < kSteps * 2; ++s) {
      const uint32_t d = s * 16 + g * 8;
      q[s] = d < p.D ? *reinterpret_cast<const u32x4 *>(at + d) : u32x4{0, 0, 0, 0};
      q[s] ^= flip;
    }
  }
  const ScoreChange change(scale, p.cap, kMore && p.slopes ? p.slopes[qhead] : 0.f);

  // Where block x's keys lie: threads 0..63 look up a key each ...
  auto look_up = [&](int32_t x) {
    const int32_t j = x < x_end ? range.block(x) * kManyBlock + lane : range.end;
    return key_place(p, w, tile, j, range.end);
  };
  // ... and hand its rows to all.
  auto hand_out = [&](const KeyPlace &k, int32_t x) {
    const bool there = k.page >= 0;
    const uint64_t off = (uint64_t)(uint32_t)k.page * p.page_stride + head * p.head_stride + k.place * p.token_stride;
    s_row[x & 1][0][lane] = there ? (uint64_t)(uintptr_t)p.keys + off : 0;
    s_row[x & 1][1][lane] = there ? (uint64_t)(uintptr_t)p.values + off : 0;
    const uint64_t bits = __ballot(there);
    if (lane == 0) s_there[x & 3] = bits;
  };
  Raw stage[2][kPasses];
  auto load = [&](int32_t x) {
#pragma unroll
    for (int kv = 0; kv < 2; ++kv)
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const uint32_t piece = i * kManyThreads + threadIdx.x, key = piece / kChunks, d = piece % kChunks * 8;
        const uint64_t at = s_row[x & 1][kv][key];
        stage[kv][i] = *reinterpret_cast<const Raw *>(at && d < p.D ? at + d * kElem : zeros);
      }
  };
  // every row of the tile sees every key of block x
  auto all_see = [&](int32_t x) {
    const int32_t j0 = range.block(x) * kManyBlock;
    return s_there[x & 3] == ~0ull && ((j0 + kManyBlock - 1 <= tile.first && (int64_t)tile.last - j0 < p.window) ||
                                       j0 + kManyBlock <= w.r.prefix);
  };
  auto set_apart = [&](u32x4 v, uint32_t key, uint32_t d) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t x = v[i >> 1] >> (i & 1) * 16 & 0xFFFFu, size = x & 0x7FFFu, inf = Q::kF16 ? 0x7C00u : 0x7F80u;
      if (size > inf || x == inf) atomicOr((unsigned long long *)&s_odd[0][d + i], 1ull << key);
      if (size > inf || x == (inf | 0x8000u)) atomicOr((unsigned long long *)&s_odd[1][d + i], 1ull << key);
    }
  };
  auto put = [&](int32_t x) {
    const bool careful = !all_see(x);
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
      const uint32_t piece = i * kManyThreads + threadIdx.x, key = piece / kChunks, d = piece % kChunks * 8;
      *reinterpret_cast<u32x4 *>(&s_k[x & 1][key * kKeyRow + d]) = widened<Q>(stage[0][i]);
      u32x4 v = widened<Q>(stage[1][i]);
      if (careful && any_not_finite4<Q>(v)) {
        set_apart(v, key, d);
        v = finite_only<Q>(v);
        odd = 1;
      }
      *reinterpret_cast<u32x4 *>(&s_v[x & 1][key * kValueRow + d]) = v;
    }
    if (careful) {
      odd = __any(odd);
      if (lane == 0) s_any_odd[x & 1][wave] = odd;
    }
  };
  // block x, which not all rows see, holds such values
  auto is_odd = [&](int32_t x) {
    uint32_t odd = 0;
#pragma unroll
    for (int i = 0; i < kManyWaves; ++i) odd |= s_any_odd[x & 1][i];
    return odd != 0;
  };

  float best = -INFINITY, sum = 0.f;  // best: of scores in log2, as last rescaled to
  f32x16 o[kSteps];
#pragma unroll
  for (int t = 0; t < kSteps; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;

  // One block's products: `sees` are the keys that this lane's query sees, all of them if kWhole.
  auto block = [&](int32_t x, int32_t j0, uint64_t sees, bool odd, auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
    const uint16_t *keys = s_k[x & 1], *values = s_v[x & 1];
    f32x16 s[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
#pragma unroll
    for (int k = 0; k < kSteps * 2; ++k)
#pragma unroll
      for (int t = 0; t < 2; ++t)
        s[t] = Q::mfma32(*reinterpret_cast<const u32x4 *>(&keys[(t * 32 + m) * kKeyRow + k * 16 + g * 8]), q[k], s[t]);
    if constexpr (kMore) {
      if (p.cap > 0.f) {
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] = change.capped(s[i >> 4][i & 15]);
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i >> 4][i & 15] *= change.factor;
      }
      if (p.slopes) {
        const float distance = (float)(pos - j0 - g * 4);
#pragma unroll
        for (int i = 0; i < 32; ++i)
          s[i >> 4][i & 15] = change.biased(s[i >> 4][i & 15],
                                            distance - (float)((i >> 4) * 32 + ((i & 15) >> 2) * 8 + (i & 3)));
      }
    }
    const float to_log2 = kMore ? 1.f : factor;
    if constexpr (!kWhole) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t bits = (uint32_t)(sees >> (t * 32)) >> (g * 4);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = bits >> ((i >> 2) * 8 + (i & 3)) & 1u ? s[t][i] : -INFINITY;
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) top = fmaxf(top, s[i >> 4][i & 15]);
    top = xor32(top, max_of) * to_log2;
    if (__any(top > best + kSlack) || __any(best == -INFINITY)) {
      const float to = fmaxf(best, top);
      const float keep = to == -INFINITY ? 1.f : pow2(best - to);
      best = to;
      sum *= keep;
#pragma unroll
      for (int t = 0; t < kSteps; ++t) o[t] *= keep;
    }
    const float from = best == -INFINITY ? 0.f : best;
    u32x4 weights[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int e = (i & 1) * 8 + c * 2;
        const float w0 = pow2(__builtin_fmaf(s[i >> 1][e], to_log2, -from));
        const float w1 = pow2(__builtin_fmaf(s[i >> 1][e + 1], to_log2, -from));
        sum += w0 + w1;
        weights[i][c] = Q::pack(w0, w1);
      }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < kSteps; ++t) {
        // sixteen keys' values at elements 32 t + m
        const uint16_t *at = &values[(i * 16 + g * 4 + ((lane & 15) >> 2)) * kValueRow + t * 32 + (lane & 16) + (lane & 3) * 4];
        o[t] = Q::mfma32(transposed(at, at + 8 * kValueRow), weights[i], o[t]);
      }
    if constexpr (!kWhole) {
      if (odd) {
#pragma unroll
        for (int t = 0; t < kSteps; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t d = t * 32 + (i >> 2) * 8 + g * 4 + (i & 3);
            o[t][i] += ((s_odd[0][d] & sees) ? INFINITY : 0.f) + ((s_odd[1][d] & sees) ? -INFINITY : 0.f);
          }
      }
    }
  };

  for (uint32_t i = threadIdx.x; i < 2 * kDim; i += kManyThreads) (&s_odd[0][0])[i] = 0;
  KeyPlace ahead{-1, 0};
  if (wave == 0) {
    hand_out(look_up(x0), x0);
    hand_out(look_up(x0 + 1), x0 + 1);
    ahead = look_up(x0 + 2);
  }
  __syncthreads();
  load(x0);
  put(x0);
  __syncthreads();
  for (int32_t x = x0; x < x_end; ++x) {
    const bool more = x + 1 < x_end;
    if (more) load(x + 1);
    if (wave == 0) {
      hand_out(ahead, x + 2);
      ahead = look_up(x + 3);
    }
    const int32_t j0 = range.block(x) * kManyBlock;
    const uint64_t there = s_there[x & 3];
    const bool odd = !all_see(x) && is_odd(x);  // all waves agree
    const bool whole = !odd && there == ~0ull &&
                       ((j0 + kManyBlock - 1 <= first && (int64_t)last - j0 < p.window) || j0 + kManyBlock <= w.r.prefix);
    const bool any = (j0 <= last && (int64_t)j0 + kManyBlock - 1 > (int64_t)first - p.window) || j0 < w.r.prefix;
    if (has_rows && any) {
      if (whole) {
        block(x, j0, ~0ull, false, std::true_type{});
      } else {
        block(x, j0, there & ((low_bits(pos - j0 + 1) & ~low_bits(oldest - j0)) | low_bits(w.r.prefix - j0)),
              odd, std::false_type{});
      }
    }
    if (odd) {  // the next such block starts with no keys
      __syncthreads();
      for (uint32_t i = threadIdx.x; i < 2 * kDim; i += kManyThreads) (&s_odd[0][0])[i] = 0;
      __syncthreads();
    }
    if (more) put(x + 1);
    __syncthreads();
  }

  sum = xor32(sum, sum_of);
  if ((uint32_t)wave * 32 + m >= tile.rows) return;
  const bool divided = parts > 1;
  const uint64_t t_out = (uint64_t)(w.r.start + token);
  const float vs = p.value_scale ? p.value_scale[head] : 1.f;
  const float norm = divided ? 1.f : sum != 0.f ? vs / sum : 0.f;
  const uint64_t slot = ((uint64_t)w.slot * p.kv_heads + head) * kManyRows + wave * 32 + m;
#pragma unroll
  for (int t = 0; t < kSteps; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t d = t * 32 + i * 8 + g * 4;
      if (d >= p.D) continue;
      const f32x4 y = {o[t][i * 4] * norm, o[t][i * 4 + 1] * norm, o[t][i * 4 + 2] * norm, o[t][i * 4 + 3] * norm};
      if (divided)
        *reinterpret_cast<f32x4 *>(p.parts + slot * p.D + d) = y;
      else
        *reinterpret_cast<u32x2 *>(p.out + t_out * p.out_stride + (uint64_t)qhead * p.D + d) =
            u32x2{Q::pack(y.x, y.y), Q::pack(y.z, y.w)};
    }
  if (g == 0) {
    if (divided) {
      float *ml = p.parts + (uint64_t)p.part_slots * p.kv_heads * kManyRows * p.D + slot * 2;
      ml[0] = best;
      ml[1] = sum;
    } else if (p.lse) {
      p.lse[t_out * p.heads + qhead] = sum != 0.f ? (best + __log2f(sum)) * kLn2 : -INFINITY;
    }
  }
}

}  // namespace gorio
