// Attention of few query rows (up to 16 of a request and key head) over many
// keys: the form for single tokens.
//
// Every key and value is read once for 16 rows or fewer, far below what the
// matrix units could do with it, so the rate at which HBM gives them is the
// bound.  Eight waves share a part of the keys, 32 at a time each; a wave keeps
// its own running maximum, sum and output, joined in LDS at the end, so no
// wave waits for another in between.  Keys and values go from memory straight
// into the operands of the matrix instructions (16x16x32), a block ahead of
// their use:
//   S^T = K Q^T: lane (m, g) = (lane % 16, lane / 16) holds elements 32 s + 8 g
//     .. + 7 of key m, one 16-byte load; the result gives it the scores of
//     query m for keys 4 g .. + 3 of each 16.
//   O^T = V^T P^T: the lane's eight weights are those of keys 4 g .. + 3 and
//     16 + 4 g .. + 3, so it loads elements 8 m .. + 7 of these eight values
//     (one 16-byte load each) and transposes 8 x 8 in registers, a byte
//     permutation a pair: product t then yields elements 8 m + t.
// Where a key's row lies (table entry, page, place) is worked out by one lane
// a key, a block before the loads, and handed to the others through LDS.
// Weights are rounded to q's type for the second product, the sum adds them
// before that rounding.
//
// Measured, 64 requests of up to 16384 tokens, 8 key heads: 5.8 TB/s of keys
// and values at D = 128 (449 us), 5.6 at 64, 5.9 at 256; from 8-bit pages 5.4
// at 128 and 4.1 at 64, where a row is 64 bytes.
// A copy on the same card moves 4.8 TB/s.  One request: 10 us for 64 tokens,
// 16 for 1000, 42 for 32000 (59 with two key heads, whose 125 parts the join
// adds up one after the other), of which the first 10 are the wait for
// lengths, table and keys, one after the other, and of the longer ones 3 to 5
// the joining kernel.
#pragma once

#include <type_traits>

#include "kv_attend.hpp"

namespace gorio {

// Waves of a workgroup: 64 requests of 16384 tokens take 235 us at D = 64 and 451 at 128 with
// eight, 256 and 456 with four.  256 elements take the registers of twice as many.
__host__ __device__ constexpr int few_waves(int steps) { return steps > 4 ? 4 : 8; }
constexpr int kFewRows = 16;
constexpr int kFewBlock = 32;  // keys

// kSteps: 32-element steps of a head, D <= 32 kSteps.  k8: pages of 8-bit values.
// kMore: scores are capped or biased.
template <typename Q, bool k8, int kSteps, bool kMore>
__device__ __forceinline__ void few_part(const AttendParams &p, const WorkItem &w, const Tile &tile,
                                         const KeyRange &range, const Part &part, uint32_t head) {
  constexpr int kFewWaves = few_waves(kSteps), kFewThreads = kFewWaves * 64;
  constexpr int kHalves = (kSteps + 3) / 4;  // 128 elements of a value
  constexpr int kDim = kHalves * 128;
  constexpr int kPad = kDim + 4;
  typedef typename std::conditional<k8, u32x2, u32x4>::type Raw;  // 8 elements as they lie
  __shared__ uint64_t s_row[kFewWaves][2][2][kFewBlock];  // wave, turn, keys or values
  __shared__ float s_o[kFewWaves][kFewRows][kPad];
  __shared__ float s_m[kFewWaves][kFewRows], s_l[kFewWaves][kFewRows];

  const int32_t x_end = min(range.count, (int32_t)part.upto);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;
  const uint64_t zeros = (uint64_t)(uintptr_t)kv_zeros;
  constexpr int kElem = k8 ? 1 : 2;

  // this lane's query
  const uint32_t n = min((uint32_t)m, tile.rows - 1);  // rows past the last repeat it
  const uint32_t token = fastdiv(tile.row0 + n, p.group), gh = tile.row0 + n - token * p.group.d;
  const int32_t pos = w.r.len - w.r.added + (int32_t)token;
  const int32_t oldest = (int32_t)max((int64_t)pos - p.window + 1, (int64_t)0);  // the window's first key
  const uint32_t qhead = head * p.group.d + gh;
  u32x4 q[kSteps];
  {
    const uint16_t *row = p.q + (uint64_t)(w.r.start + token) * p.q_stride + (uint64_t)qhead * p.D;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const uint32_t d = s * 32 + g * 8;
      q[s] = d < p.D ? *reinterpret_cast<const u32x4 *>(row + d) : u32x4{0, 0, 0, 0};
    }
  }
  const float scale = p.scale * (p.key_scale ? p.key_scale[head] : 1.f);
  const float to_log2 = scale * kLog2e;
  const ScoreChange change(scale, p.cap, kMore && p.slopes ? p.slopes[qhead] : 0.f);

  float best = -INFINITY, sum = 0.f;
  f32x4 o[kHalves * 8];
#pragma unroll
  for (int t = 0; t < kHalves * 8; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Rows of block x into LDS, and its keys' bits: lanes 0..31 a key each.
  auto place_of = [&](int32_t x) __attribute__((always_inline)) {
    return key_look(p, w, tile, (x < x_end) & (lane < kFewBlock), range.block(x) * kFewBlock + (lane & 31), range.end);
  };
  auto hand_out = [&](const KeyLook &k, int turn) __attribute__((always_inline)) -> uint32_t {
    const bool there = key_there(p, k);
    if (lane < kFewBlock) {
      const uint64_t off = (uint64_t)(uint32_t)k.page * p.page_stride + head * p.head_stride + k.place * p.token_stride;
      s_row[wave][turn][0][lane] = there ? (uint64_t)(uintptr_t)p.keys + off : 0;
      s_row[wave][turn][1][lane] = there ? (uint64_t)(uintptr_t)p.values + off : 0;
    }
    wave_lds_order();
    return (uint32_t)__ballot(there);
  };
  auto load_keys = [&](Raw (&k)[2][kSteps], int turn) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint64_t row = s_row[wave][turn][0][i * 16 + m];
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const uint32_t d = s * 32 + g * 8;
        const uint64_t at = row && d < p.D ? row + d * kElem : zeros;
        k[i][s] = *reinterpret_cast<const Raw *>(at);
      }
    }
  };
  auto load_values = [&](Raw (&v)[8], int half, int turn) __attribute__((always_inline)) {
    const uint32_t d = half * 128 + m * 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint64_t row = s_row[wave][turn][1][(i >> 2) * 16 + g * 4 + (i & 3)];
      const uint64_t at = row && d < p.D ? row + d * kElem : zeros;
      v[i] = *reinterpret_cast<const Raw *>(at);
    }
  };
  // Block x, with the next one's keys and values on their way; the registers alternate.
  Raw k[2][2][kSteps], v[2][kHalves][8];
  uint32_t there[2];
  KeyLook next;
  auto load = [&](auto turn) __attribute__((always_inline)) {
    constexpr int t = decltype(turn)::value;
    load_keys(k[t], t);
#pragma unroll
    for (int h = 0; h < kHalves; ++h) load_values(v[t][h], h, t);
  };
  auto step = [&](int32_t x, auto turn) __attribute__((always_inline)) {
    constexpr int t0 = decltype(turn)::value, t1 = 1 - t0;
    const int32_t j0 = range.block(x) * kFewBlock;
    const uint32_t there_now = there[t0];
    there[t1] = hand_out(next, t1);
    next = place_of(x + 2 * kFewWaves);
    load(std::integral_constant<int, t1>{});

    f32x4 s2[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s2[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) s2[i] = Q::mfma16(widened<Q>(k[t0][i][s]), q[s], s2[i]);
    }
    float e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float y = s2[i >> 2][i & 3];
      if constexpr (kMore) {
        y = p.cap > kQuickCap ? change.capped_exactly(y) : p.cap > 0.f ? change.capped(y) : y * change.to_log2;
        if (p.slopes) y = change.biased(y, (float)(pos - j0 - g * 4) - (float)((i >> 2) * 16 + (i & 3)));
      } else {
        y *= to_log2;
      }
      e[i] = y;
    }
    // all rows see all of these keys, or each row is asked for each key
    const bool whole = there_now == 0xFFFFFFFFu &&
                       ((j0 + kFewBlock - 1 <= tile.first && tile.last - j0 < (int64_t)p.window) ||
                        j0 + kFewBlock <= w.r.prefix);
    uint32_t sees = ~0u;  // this lane's keys: bits 0..3 and 16..19
    if (!whole) {
      const uint64_t seen = (low_bits(pos - j0 + 1) & ~low_bits(oldest - j0)) | low_bits(w.r.prefix - j0);
      sees = (there_now & (uint32_t)seen) >> (g * 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = kept(e[i], sees, (i >> 2) * 16 + (i & 3));
    }
    float top = fmaxf(fmaxf(fmaxf(e[0], e[1]), fmaxf(e[2], e[3])), fmaxf(fmaxf(e[4], e[5]), fmaxf(e[6], e[7])));
    top = xor16(xor32(top, max_of), max_of);
    if (__any(top > best)) {
      const float to = fmaxf(best, top);
      const float keep = to == -INFINITY ? 1.f : pow2(best - to);
      best = to;
      sum *= keep;
#pragma unroll
      for (int t = 0; t < kHalves * 8; ++t) o[t] *= keep;
    }
    const float base = best == -INFINITY ? 0.f : best;
    float part = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      e[i] = pow2(e[i] - base);
      part += e[i];
    }
    sum += part;
    const u32x4 weights = {Q::pack(e[0], e[1]), Q::pack(e[2], e[3]), Q::pack(e[4], e[5]), Q::pack(e[6], e[7])};
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      u32x4 vw[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) vw[i] = widened<Q>(v[t0][h][i]);
      // A weight of 0 keeps a value out of a row, unless the value is NaN or inf.  Such
      // values in a block that some rows see only in part go in apart from the others.
      bool odd = false;
      if (!whole && tile.first != tile.last) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) odd |= any_not_finite<Q>(vw[i][c]);
        odd = __any(odd);
      }
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const uint32_t sel = t & 1 ? 0x07060302u : 0x05040100u;
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(vw[2 * i + 1][t >> 1], vw[2 * i][t >> 1], sel);
        if (__builtin_expect(odd, 0)) {
          u32x4 seen;  // 1 where the row sees the key
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int at = (i >> 1) * 16 + (i & 1) * 2;
            seen[i] = Q::pack((float)(sees >> at & 1u), (float)(sees >> (at + 1) & 1u));
          }
          o[h * 8 + t] += not_finite_part<Q>(a, seen);
          a = finite_only<Q>(a);
        }
        o[h * 8 + t] = Q::mfma16(a, weights, o[h * 8 + t]);
      }
    }
  };
  int32_t x = (int32_t)part.from + wave;
  there[0] = hand_out(place_of(x), 0);
  next = place_of(x + kFewWaves);
  load(std::integral_constant<int, 0>{});
  while (x < x_end) {
    step(x, std::integral_constant<int, 0>{});
    if ((x += kFewWaves) >= x_end) break;
    step(x, std::integral_constant<int, 1>{});
    x += kFewWaves;
  }

  // the waves' results, joined
  sum = xor16(xor32(sum, sum_of), sum_of);
  if (g == 0) s_m[wave][m] = best, s_l[wave][m] = sum;
#pragma unroll
  for (int h = 0; h < kHalves; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float *to = &s_o[wave][m][h * 128 + (g * 4 + r) * 8];
#pragma unroll
      for (int t = 0; t < 8; t += 4)
        *reinterpret_cast<f32x4 *>(to + t) =
            f32x4{o[h * 8 + t][r], o[h * 8 + t + 1][r], o[h * 8 + t + 2][r], o[h * 8 + t + 3][r]};
    }
  __syncthreads();
  constexpr int kRowThreads = kFewThreads / kFewRows, kOwn = 128 / kRowThreads;  // elements of each 128
  const uint32_t row = threadIdx.x / kRowThreads, at = threadIdx.x % kRowThreads;
  if (row >= tile.rows) return;
  float most = s_m[0][row];
#pragma unroll
  for (int i = 1; i < kFewWaves; ++i) most = fmaxf(most, s_m[i][row]);
  const float base = most == -INFINITY ? 0.f : most;
  float by[kFewWaves], all = 0.f;
#pragma unroll
  for (int i = 0; i < kFewWaves; ++i) {
    by[i] = pow2(s_m[i][row] - base);
    all += s_l[i][row] * by[i];
  }
  const uint32_t tk = fastdiv(tile.row0 + row, p.group), hq = head * p.group.d + (tile.row0 + row - tk * p.group.d);
  const uint64_t t_out = (uint64_t)(w.r.start + tk);
  const float vs = p.value_scale ? p.value_scale[head] : 1.f;
  const bool divided = part.divided;
  const float norm = divided ? 1.f : all != 0.f ? vs / all : 0.f;
  const uint64_t slot = ((uint64_t)part.slot * p.kv_heads + head) * kFewRows + row;
#pragma unroll
  for (int h = 0; h < kHalves; ++h) {
    const uint32_t d = h * 128 + at * kOwn;
    if (d >= p.D) break;
#pragma unroll
    for (int i = 0; i < kOwn; i += 4) {
      f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kFewWaves; ++j) {
        const f32x4 o4 = *reinterpret_cast<const f32x4 *>(&s_o[j][row][d + i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = fmaf(o4[e], by[j], y[e]);
      }
      y *= norm;
      if (divided)
        *reinterpret_cast<f32x4 *>(p.parts + slot * p.D + d + i) = y;
      else
        *reinterpret_cast<u32x2 *>(p.out + t_out * p.out_stride + (uint64_t)hq * p.D + d + i) =
            u32x2{Q::pack(y.x, y.y), Q::pack(y.z, y.w)};
    }
  }
  if (at == 0) {
    if (divided) {
      float *ml = p.parts + (uint64_t)p.shares * 2 * p.kv_heads * kFewRows * p.D + slot * 2;
      ml[0] = most;
      ml[1] = all;
    } else if (p.lse) {
      p.lse[t_out * p.heads + hq] = all != 0.f ? (base + __log2f(all)) * kLn2 : -INFINITY;
    }
  }
}

template <typename Q, bool k8, int kSteps, bool kMore>
__global__ __launch_bounds__(few_waves(kSteps) * 64) void attend_few(AttendParams p) {
  const uint32_t index = fastdiv(blockIdx.x, p.by_kv), head = blockIdx.x - index * p.kv_heads;
  WorkItem w;
  if (!find_item<few_waves(kSteps) * 64, kFewBlock>(p, index, w)) return note_cut<kFewRows>(p, index, head);
  for (;;) {
    const Tile tile = tile_of(p, w.r, w.tile);
    const KeyRange range = key_range<kFewBlock>(p, w.r, tile.first, tile.last);
    const uint32_t blocks = (uint32_t)max(range.count, 1);
    const Part part = part_of(p, w, blocks, index);
    if (!part.none) few_part<Q, k8, kSteps, kMore>(p, w, tile, range, part, head);
    const uint64_t end = w.begin + blocks;
    if (end >= (index + 1) * w.share || end >= w.line || !next_item(p, w, end))
      return note_cut<kFewRows>(p, index, head, w, tile, part, blocks);
    __syncthreads();  // the next tile's sums go where this one's are read
  }
}

// Joins the parts of divided tiles: a workgroup a share and head, for the tile that begins in the
// share and is cut at its end; 16 rows, 16 threads a row (64 rows a workgroup, four after the other:
// 128 new tokens over 2000 took 54 us in all, now 41).  A row's parts are added one after the
// other, and each waits for its loads.
//   out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i over the parts i
// Bound by the latency of two dependent loads, 4 us, and for many tiles by reading the parts
// (750 cut tiles of 128 rows, 64 elements: 50 MB in 14 us).
template <typename Q, int kRows>
__global__ __launch_bounds__(256) void attend_join(AttendParams p) {
  const uint32_t s0 = fastdiv(blockIdx.x, p.by_kv), head = blockIdx.x - s0 * p.kv_heads;
  const Cut cut = cuts_of<kRows>(p)[blockIdx.x];
  const uint32_t parts = cut.parts, slot0 = cut.slot, lane = threadIdx.x & 15;  // slot0: of the first part
  const float *ml = p.parts + (uint64_t)p.shares * 2 * p.kv_heads * kRows * p.D;
  const float vs = p.value_scale ? p.value_scale[head] : 1.f;
  const uint32_t row = blockIdx.y * 16 + (threadIdx.x >> 4);
  if (parts && row < cut.rows) {
    auto slot = [&](uint32_t i) {
      return ((uint64_t)(i ? (s0 + i) * 2 : slot0) * p.kv_heads + head) * kRows + row;
    };
    float most = -INFINITY;
    for (uint32_t i = lane; i < parts; i += 16) most = fmaxf(most, ml[slot(i) * 2]);
#pragma unroll
    for (int d = 8; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    const float from = most == -INFINITY ? 0.f : most;
    f32x4 y[4];  // 8 elements, and 8 more of a head past 128
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float all = 0.f;
    const uint32_t d0 = lane * 8, d1 = d0 + 128;
    for (uint32_t i0 = 0; i0 < parts; i0 += 16) {
      float by = 0.f;  // of part i0 + lane
      if (i0 + lane < parts) {
        const uint64_t at = slot(i0 + lane) * 2;
        by = pow2(ml[at] - from);
        all = fmaf(ml[at + 1], by, all);
      }
      const uint32_t some = min(parts - i0, 16u);
      for (uint32_t i = 0; i < some; ++i) {
        const float one = __shfl(by, (int)i, 16);
        const float *o = p.parts + slot(i0 + i) * p.D;
        if (d0 < p.D) {
          y[0] += *reinterpret_cast<const f32x4 *>(o + d0) * one;
          y[1] += *reinterpret_cast<const f32x4 *>(o + d0 + 4) * one;
        }
        if (d1 < p.D) {
          y[2] += *reinterpret_cast<const f32x4 *>(o + d1) * one;
          y[3] += *reinterpret_cast<const f32x4 *>(o + d1 + 4) * one;
        }
      }
    }
#pragma unroll
    for (int d = 8; d; d >>= 1) all += __shfl_xor(all, d);
    const float norm = all != 0.f ? vs / all : 0.f;
    const uint32_t tk = fastdiv(cut.row0 + row, p.group), hq = head * p.group.d + (cut.row0 + row - tk * p.group.d);
    const uint64_t t_out = (uint64_t)(cut.start + tk);
    uint16_t *out = p.out + t_out * p.out_stride + (uint64_t)hq * p.D;
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const uint32_t d = i ? d1 : d0;
      if (d >= p.D) continue;
      const f32x4 a = y[i] * norm, b = y[i + 1] * norm;
      *reinterpret_cast<u32x4 *>(out + d) = u32x4{Q::pack(a.x, a.y), Q::pack(a.z, a.w), Q::pack(b.x, b.y), Q::pack(b.z, b.w)};
    }
    if (p.lse && lane == 0) p.lse[t_out * p.heads + hq] = all != 0.f ? (from + __log2f(all)) * kLn2 : -INFINITY;
  }
}

}  // namespace gorio
