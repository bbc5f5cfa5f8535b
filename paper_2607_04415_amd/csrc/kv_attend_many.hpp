// Attention of many query rows over many keys: the form for chunks.
//
// With 128 or 256 rows to a tile every key is used often enough that what the
// waves issue is the bound: matrix instructions for 4 D flops of a row and key
// (half of a SIMD's time at D = 128, a quarter at D = 64) and, on the same
// issue slots, the score's way to a weight (an exponential of 9 clocks, a
// fused multiply, an add, half a conversion and half a maximum of 4.5 each).
// Each wave owns 32 rows for the whole run, so softmax, rescaling and output
// never leave its registers; blocks of 64 keys and values pass through LDS for
// all of them, two buffers deep, so that a block's loads run during the
// products of the one before and a barrier a block suffices.  S^T of the next
// 32 keys is computed between the exponentials of these, because a wave issues
// other work while its matrix instruction runs.  On 32x32x16 instructions:
//   S^T = K Q^T: lane (m, g) = (lane % 32, lane / 32) reads elements 16 s + 8 g
//     .. + 7 of key m; the result gives it, of query m, the scores of keys
//     8 i + 4 g .. + 3 for i = 0..3.
//   O^T = V^T P^T: sixteen keys at a time, of which the lane has the weights
//     of 4 g .. + 3 and 8 + 4 g .. + 3; the transposing LDS read gives it the
//     values of those keys at element m.
// Keys and values of 16 bits go straight from memory into LDS, where a wave's
// 64 pieces of 16 bytes lie one after the other; which piece a lane asks for is
// turned by its key (see `turned`), so that neighbouring keys' reads fall on
// different banks.  Pages of 8 bits are widened in registers on the way, and
// rows of 96 elements padded by 16 bytes instead.
//
// Weights are rounded to q's type for the second product, the nearest value
// that the matrix units take; the sum adds them before that rounding.
//
// Measured, 4096 new tokens after 12288, two heads of queries to each of 8:
// 689 TF at D = 64, 723 at 96, 913 at 128, 485 at 192, 648 at 256 (heads past
// 128 are computed as 256 elements); from 8-bit pages 671, 747, 900, 359 and
// 479; with a cap, an exponential and a reciprocal more a score, 752 at 128,
// with one past 64 550.  A large matrix product reaches 1210.
// Vector registers are spilled at D <= 64 from 8-bit pages (10 to 13 of them)
// and under caps (9 to 33), at D <= 128 from 8-bit pages under caps (14, 15)
// and under caps past 64 (2), at 96 under these (1), and past 128 (5 to 14, from
// 8-bit pages 54 to 62).
// Counters at D = 128: the matrix units work 43% of the time, and a SIMD
// issues 72% of it, 6.7 vector instructions beside each matrix instruction.
#pragma once

#include <type_traits>

#include "kv_attend.hpp"

namespace gorio {

// Waves of a workgroup, 32 rows each.  Eight for heads of 97..128, which is one workgroup a CU:
// 4096 tokens over 8192 take 470 us, with four waves and two workgroups 505 (but 128 tokens over
// 2000 took 43 us with four, 51 with eight).  Four for smaller heads: at D = 64 three workgroups
// fit a CU, and 33 requests of 1000 tokens take 207 us, with eight waves 232.  Four for larger
// ones, whose blocks fill LDS.
__host__ __device__ constexpr int many_waves(int steps) { return steps == 4 ? 8 : 4; }
__host__ __device__ constexpr int many_rows(int steps) { return many_waves(steps) * 32; }
constexpr int kManyBlock = 64;  // keys

// A maximum is kept until a score passes it by 2^8 (weights stay far inside
// f16's range, and a sum of them loses nothing): most blocks then rescale nothing.
constexpr float kSlack = 8.f;

// kSteps: D <= 32 kSteps.  k8: pages of 8-bit values.  kMore: 1 if scores are biased, 2 if they
// are capped, and biased if there are slopes, 3 the same by a cap past kQuickCap (kernels of their
// own: a branch in those of 2 made these spill up to 40 registers more, for caps of any size).
template <typename Q, bool k8, int kSteps, int kMore>
__device__ __forceinline__ void many_part(const AttendParams &p, const WorkItem &w, const Tile &tile,
                                          const KeyRange &range, const Part &part, uint32_t head) {
  constexpr int kManyWaves = many_waves(kSteps), kManyThreads = kManyWaves * 64, kManyRows = kManyWaves * 32;
  constexpr int kDim = kSteps * 32, kChunks = kDim / 8;                              // 16-byte pieces of a row
  constexpr int kPasses = kManyBlock * kChunks / kManyThreads;                       // pieces a thread
  static_assert(kPasses * kManyThreads == kManyBlock * kChunks, "pieces divide");
  constexpr bool kTurned = (kChunks & (kChunks - 1)) == 0, kDirect = kTurned && !k8;  // see `turned`
  constexpr int kKeyRow = kTurned ? kDim : kDim + 8;                                 // elements
  constexpr int kValueRow = kDim;
  static_assert(kTurned || (kDim * 2) % 256 == 192, "rows of values fall on different banks");
  constexpr int kElem = k8 ? 1 : 2;
  typedef typename std::conditional<k8, u32x2, u32x4>::type Raw;
  constexpr uint32_t kKeyBytes = kManyBlock * kKeyRow * 2, kValueBytes = kManyBlock * kValueRow * 2;
  __shared__ __align__(1024) uint8_t s_kv[2 * (kKeyBytes + kValueBytes)];  // keys, keys, values, values
  constexpr int kRing = kManyWaves * 2;                 // blocks
  __shared__ uint64_t s_row[kRing][2][kManyBlock];      // block, keys or values
  __shared__ uint64_t s_there[kRing];
  // Values that are NaN or inf in a block that not all rows see: a weight of 0 would not keep
  // them out of a row.  They are 0 in s_kv; here are the keys that have one at an element,
  // +inf (or NaN) and -inf (or NaN).
  __shared__ uint64_t s_odd[2][kDim];
  __shared__ uint32_t s_any_odd[kManyWaves];

  const int32_t x0 = (int32_t)part.from, x_end = min(range.count, (int32_t)part.upto);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  const int32_t first = base + (int32_t)fastdiv(wave_row, p.group), last = base + (int32_t)fastdiv(wave_end, p.group);
  const uint32_t qhead = head * p.group.d + gh;
  const float scale = p.scale * (p.key_scale ? p.key_scale[head] : 1.f);
  // the running maximum is taken of the products as they are, so the factor has to be positive:
  // a negative one turns the queries' signs around
  constexpr bool capped = kMore >= 2, large = kMore == 3;
  const bool biased = kMore == 1 || (capped && p.slopes);
  const uint32_t flip = !capped && scale < 0.f ? 0x80008000u : 0u;
  // 0 times a masked score's -inf would be NaN, and a bias is divided by it
  const float factor = scale == 0.f || (biased && fabsf(scale) < 1e-30f) ? 1e-30f : fabsf(scale) * kLog2e;
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
  const ScoreChange change(scale, p.cap, biased ? p.slopes[qhead] : 0.f);

  // Where block x's keys lie: wave 0 looks up a key a lane ...
  auto look_up = [&](int32_t x) __attribute__((always_inline)) {
    return key_look(p, w, tile, (x >= x0) & (x < x_end), range.block(x) * kManyBlock + lane, range.end);
  };
  // ... and hands its rows to all.
  auto hand_out = [&](const KeyLook &k, int32_t x) __attribute__((always_inline)) {
    const bool there = key_there(p, k);
    const uint64_t off = (uint64_t)(uint32_t)k.page * p.page_stride + head * p.head_stride + k.place * p.token_stride;
    s_row[x & (kRing - 1)][0][lane] = there ? (uint64_t)(uintptr_t)p.keys + off : zeros;
    s_row[x & (kRing - 1)][1][lane] = there ? (uint64_t)(uintptr_t)p.values + off : zeros;
    const uint64_t bits = __ballot(there);
    if (lane == 0) s_there[x & (kRing - 1)] = bits;
  };
  // Every row of the tile sees every key of block x that is there, by its position.
  auto all_see = [&](int32_t x) __attribute__((always_inline)) {
    const int32_t j0 = range.block(x) * kManyBlock;
    return (j0 + kManyBlock - 1 <= tile.first && (int64_t)tile.last - j0 < p.window) || j0 + kManyBlock <= w.r.prefix;
  };

  // A thread's pieces of a block.  Straight from memory into LDS, a wave's 64 pieces lie one
  // after the other there, so the banks are spread by which piece a lane asks for: piece c of
  // key j lies at c ^ turned(j), which sets 16 neighbouring keys' equal pieces, and 4 keys' 64
  // bytes, on different banks.
  auto turned = [](uint32_t key) __attribute__((always_inline)) -> uint32_t {
    return kChunks == 8 ? (key >> 1 & 1u) << 2 | (key >> 2 & 3u) : (key & 3u) << 2 | (key >> 2 & 3u);
  };
  Raw stage[2][kDirect ? 1 : kPasses];
  const uint32_t lds = (uint32_t)(uintptr_t)(LdsBytes *)s_kv;
  constexpr uint32_t kKeys[2] = {0, kKeyBytes}, kValues[2] = {2 * kKeyBytes, 2 * kKeyBytes + kValueBytes};
  // The values of block x and the keys half a block later: 32.. of block x, ..31 of x + 1.
  auto row_of = [&](int32_t x, int kv, int i) __attribute__((always_inline)) -> uint64_t {
    const uint32_t key = ((i * kManyWaves + wave) * 64 + lane) / kChunks;
    return kv ? s_row[x & (kRing - 1)][1][key] : s_row[(x + (key >> 5)) & (kRing - 1)][0][key ^ 32];
  };
  const bool whole_rows = p.D == kDim;
  auto load_row = [&](uint64_t row, int kv, int i, uint32_t to, bool whole) __attribute__((always_inline)) {
    const uint32_t piece = (i * kManyWaves + wave) * 64 + lane, c = piece % kChunks;
    const uint32_t d = (kDirect ? c ^ turned(piece / kChunks) : c) * 8;
    const uint64_t at = whole || d < p.D ? row + d * kElem : zeros;
    if constexpr (kDirect) {
      typedef __attribute__((address_space(1))) const uint32_t global_u32;
      __builtin_amdgcn_global_load_lds((global_u32 *)at, (LdsBytes *)(uintptr_t)(lds + to + (i * kManyWaves + wave) * 1024),
                                       16, 0, 0);
    } else {
      stage[kv][i] = *reinterpret_cast<const Raw *>(at);
    }
  };
  auto load = [&](int32_t x, int kv, uint32_t to) __attribute__((always_inline)) {
    uint64_t row[kPasses];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) row[i] = row_of(x, kv, i);
    __builtin_amdgcn_sched_barrier(0);  // all rows are read before the first is waited for
    if (whole_rows) {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) load_row(row[i], kv, i, to, true);
    } else {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) load_row(row[i], kv, i, to, false);
    }
  };
  auto put = [&](int kv, uint32_t to) __attribute__((always_inline)) {
    if constexpr (!kDirect) {
#pragma unroll
      for (int i = 0; i < kPasses; ++i) {
        const uint32_t piece = (i * kManyWaves + wave) * 64 + lane, key = piece / kChunks, c = piece % kChunks;
        *lds_at<u32x4>(lds + to + key * (kv ? kValueRow : kKeyRow) * 2 + (kTurned ? c ^ turned(key) : c) * 16) = widened<Q>(stage[kv][i]);
      }
    }
  };
  // Takes the NaN and inf out of a block of values in LDS; true if there were any.  All threads.
  auto set_apart = [&](uint32_t values) __attribute__((always_inline)) -> bool {
    uint32_t odd = 0;
#pragma unroll 1
    for (uint32_t piece = threadIdx.x; piece < kManyBlock * kChunks; piece += kManyThreads) {
      const uint32_t key = piece / kChunks, c = piece % kChunks;
      auto at = lds_at<u32x4>(lds + values + key * kValueRow * 2 + (kTurned ? c ^ turned(key) : c) * 16);
      const u32x4 v = *at;
      if (!any_not_finite4<Q>(v)) continue;
      odd = 1;
      *at = finite_only<Q>(v);
#pragma unroll 1
      for (int i = 0; i < 8; ++i) {
        const uint32_t pair = i < 2 ? v.x : i < 4 ? v.y : i < 6 ? v.z : v.w;
        const uint32_t x = pair >> (i & 1) * 16 & 0xFFFFu, size = x & 0x7FFFu, inf = Q::kF16 ? 0x7C00u : 0x7F80u;
        if (size > inf || x == inf) atomicOr((unsigned long long *)&s_odd[0][c * 8 + i], 1ull << key);
        if (size > inf || x == (inf | 0x8000u)) atomicOr((unsigned long long *)&s_odd[1][c * 8 + i], 1ull << key);
      }
    }
    odd = __any(odd);
    if (lane == 0) s_any_odd[wave] = odd;
    __syncthreads();
    odd = 0;
#pragma unroll
    for (int i = 0; i < kManyWaves; ++i) odd |= s_any_odd[i];
    return __builtin_amdgcn_readfirstlane(odd) != 0;
  };

  float best = -INFINITY, sum = 0.f;  // best: of scores in log2, as last rescaled to
  f32x16 o[kSteps];
#pragma unroll
  for (int t = 0; t < kSteps; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;

  // Where this lane reads, in block 0 of each buffer's keys and values: a step of 16 elements
  // (or 32) turns a bit of the address, or adds to it, and all else is a constant offset.
  auto beside = [](uint32_t at, uint32_t bytes) __attribute__((always_inline)) { return kTurned ? at ^ bytes : at + bytes; };
  uint32_t key_at = lds + m * kKeyRow * 2 + (kTurned ? g ^ turned(m) : (uint32_t)g) * 16;
  uint32_t value_at[2];
  {
    const uint32_t key = g * 4 + ((lane & 15) >> 2);
    const uint32_t c = (lane & 16) >> 3 | (lane & 3) >> 1;  // piece of the 64 bytes of 32 elements
    value_at[0] = lds + key * kValueRow * 2 + (kTurned ? c ^ turned(key) : c) * 16 + (lane & 1) * 8;
    value_at[1] = lds + (key + 8) * kValueRow * 2 + (kTurned ? c ^ turned(key + 8) : c) * 16 + (lane & 1) * 8;
  }
  // A score in log2 is s * mul + add.  Without a cap s is the product, to which the bias is
  // added as what the product starts from.  With a cap s is -1 / (1 + E) (see ScoreChange), or,
  // if the cap is large or there is a bias as well, the score itself.
  const float mul = !capped ? factor : biased || large ? 1.f : -change.twice;
  const float add = capped && !biased && !large ? change.cap : 0.f;
  const float start_slope = biased && !capped ? change.slope / factor : 0.f;
  auto start = [&](f32x16 &s, int32_t j) __attribute__((always_inline)) {
    if constexpr (kMore == 1) {
      const float distance = (float)(pos - j - g * 4);
      if (j < w.r.prefix && j + 31 > first) {  // keys after a row's position that it sees
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = start_slope * fabsf(distance - (float)((i >> 2) * 8 + (i & 3)));
      } else {
        const float here = start_slope * distance;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = __builtin_fmaf(-start_slope, (float)((i >> 2) * 8 + (i & 3)), here);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 0.f;
    }
  };
  auto changed = [&](f32x16 &s, int32_t j0) __attribute__((always_inline)) {
    if constexpr (capped) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (large) {
          s[i] = change.capped_exactly(s[i]);
          __builtin_amdgcn_sched_barrier(0);  // one score's registers at a time
        } else {
          s[i] = change.quotient(s[i]);
        }
      }
      if (biased) {
        const float distance = (float)(pos - j0 - g * 4);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if constexpr (!large) s[i] = __builtin_fmaf(s[i], -change.twice, change.cap);
          s[i] = change.biased(s[i], distance - (float)((i >> 2) * 8 + (i & 3)));
        }
      }
    }
  };
  // The running maximum takes in 32 keys' scores; the sums are rescaled to it.
  auto rescale = [&](const f32x16 &s) __attribute__((always_inline)) {
    float top = max16<capped>(s);
    top = __builtin_fmaf(xor32(top, max_of), mul, add);
    if (__any((top > best + kSlack) | (best == -INFINITY))) {
      const float to = fmaxf(best, top);
      const float keep = to == -INFINITY ? 1.f : pow2(best - to);
      best = to;
      sum *= keep;
#pragma unroll
      for (int t = 0; t < kSteps; ++t) o[t] *= keep;
    }
  };
  // 32 keys' scores to weights and O^T of their values, with the scores of the 32 keys after
  // them computed beside (S^T from `keys`): a matrix instruction takes as long as eight others,
  // so the exponentials go between those of S^T.  LDS is read first, all at once, while the
  // products of the 32 keys before are still under way and the maximum is looked for.
  auto both = [&](f32x16 &s, f32x16 &next, int32_t j_next, auto keys, auto values, auto &&prepare) __attribute__((always_inline)) {
    constexpr int kTiles = kSteps > 4 ? 4 : kSteps, kTurns = kSteps / kTiles;
    constexpr uint32_t kFrom = decltype(values)::value, kSixteen = 16 * kValueRow * 2;
    constexpr uint32_t kFar = kFrom + kSixteen > 65535 ? kFrom : 0;  // an instruction's offset has 16 bits
    // held as they are: the addresses made of them would cost registers
    asm volatile("" : "+v"(key_at), "+v"(value_at[0]), "+v"(value_at[1]));
    u32x4 kf[4], vf[2][kTiles];  // keys: four steps ahead; values: sixteen keys ahead
    __builtin_amdgcn_sched_barrier(0);
    auto read_keys = [&](int k) __attribute__((always_inline)) {
      kf[k & 3] = *lds_at<u32x4>(beside(key_at, k * 32) + decltype(keys)::value);
    };
    auto read_values = [&](auto turn) __attribute__((always_inline)) {  // elements outside, keys inside
      constexpr int u = decltype(turn)::value / 2, i = decltype(turn)::value % 2;
      uint32_t at[kTiles][2];
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) at[t][h] = beside(value_at[h], (u * kTiles + t) * 64) + kFar;
      read_transposed<kTiles, kFrom - kFar + i * kSixteen>(at, vf[i]);
    };
#pragma unroll
    for (int k = 0; k < 4; ++k) read_keys(k);
    read_values(std::integral_constant<int, 0>{});
    __builtin_amdgcn_sched_barrier(0);
    prepare(s);
    const float less = add - (best == -INFINITY ? 0.f : best);
    u32x4 weights[2];
    start(next, j_next);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int k = 0; k < kSteps * 2; ++k) {
      next = Q::mfma32(kf[k & 3], q[k], next);
      if (k + 4 < kSteps * 2) read_keys(k + 4);
#pragma unroll
      for (int e = 8 * k / (kSteps * 2); e < 8 * (k + 1) / (kSteps * 2); ++e) {  // pairs of scores
        const float w0 = pow2(__builtin_fmaf(s[e * 2], mul, less));
        const float w1 = pow2(__builtin_fmaf(s[e * 2 + 1], mul, less));
        weights[e >> 2][e & 3] = Q::pack(w0, w1);
        sum += w0 + w1;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    auto values_turn = [&](auto turn) __attribute__((always_inline)) {
      constexpr int u = decltype(turn)::value / 2, i = decltype(turn)::value % 2;
#pragma unroll
      for (int t = 0; t < kTiles; ++t) o[u * kTiles + t] = Q::mfma32(vf[i][t], weights[i], o[u * kTiles + t]);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (decltype(turn)::value + 1 < 2 * kTurns)
        read_values(std::integral_constant<int, decltype(turn)::value + 1>{});
    };
    values_turn(std::integral_constant<int, 0>{});
    values_turn(std::integral_constant<int, 1>{});
    if constexpr (kTurns > 1) {
      values_turn(std::integral_constant<int, 2>{});
      values_turn(std::integral_constant<int, 3>{});
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  // Block x, the scores of whose first 32 keys are in `now`, up to those of block x + 1.  The
  // buffers alternate, and two steps make a round, so that which one is read is known when this
  // is compiled.
  constexpr uint32_t kHalfKeys = 32 * kKeyRow * 2, kHalfValues = 32 * kValueRow * 2;
  f32x16 now, next;
  KeyLook ahead{};
  auto step = [&](int32_t x, auto turn, auto computes) __attribute__((always_inline)) {
    constexpr int kNow = decltype(turn)::value, kNext = 1 - kNow;
    constexpr uint32_t k_now = kKeys[kNow], k_next = kKeys[kNext], v_now = kValues[kNow], v_next = kValues[kNext];
    const bool more = x + 1 < x_end;
    if (((x - x0) & (kManyWaves - 1)) == 0) {  // a block a wave, for the steps up to the next such
      hand_out(ahead, x + 3 + wave);
      ahead = look_up(x + 3 + kManyWaves + wave);
    }
    if (more) {
      load(x + 1, 0, k_next);
      load(x + 1, 1, v_next);
    }
    const int32_t j0 = range.block(x) * kManyBlock;
    const uint64_t bits = s_there[x & (kRing - 1)];  // the same for all
    const uint64_t there = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(bits >> 32)) << 32 |
                           (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)bits);
    bool odd = false;
    if (__builtin_expect(!all_see(x), 0)) odd = set_apart(v_now);
    const bool near = (j0 + kManyBlock - 1 <= first && (int64_t)last - j0 < p.window) || j0 + kManyBlock <= w.r.prefix;
    const bool any = (j0 <= last && (int64_t)j0 + kManyBlock - 1 > (int64_t)first - p.window) || j0 < w.r.prefix;
    const bool masked = !near | odd | (there != ~0ull);
    uint64_t sees = ~0ull;
    if (masked) {
      int32_t here = pos;
      asm("" : "+v"(here));  // what follows from it is worked out here, not kept in registers
      const int32_t oldest = (int32_t)max((int64_t)here - p.window + 1, (int64_t)0);  // the window's first key
      sees = !any ? 0 : there & ((low_bits(here - j0 + 1) & ~low_bits(oldest - j0)) | low_bits(w.r.prefix - j0));
    }
    auto mask = [&](f32x16 &s, uint32_t seen) __attribute__((always_inline)) {
      if (masked) {
        seen >>= g * 4;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = kept(s[i], seen, (i >> 2) * 8 + (i & 3));
      }
    };
    if constexpr (decltype(computes)::value) {
      both(now, next, j0 + 32, std::integral_constant<uint32_t, k_now>{}, std::integral_constant<uint32_t, v_now>{},
           [&](f32x16 &s) __attribute__((always_inline)) {
             changed(s, j0);
             mask(s, (uint32_t)sees);
             rescale(s);
           });
      both(next, now, range.block(x + 1) * kManyBlock, std::integral_constant<uint32_t, k_now + kHalfKeys>{},
           std::integral_constant<uint32_t, v_now + kHalfValues>{}, [&](f32x16 &s) __attribute__((always_inline)) {
             changed(s, j0 + 32);
             mask(s, (uint32_t)(sees >> 32));
             rescale(s);
           });
      if (__builtin_expect(odd, 0)) {
#pragma unroll
        for (int t = 0; t < kSteps; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint32_t d = t * 32 + (i >> 2) * 8 + g * 4 + (i & 3);
            o[t][i] += ((s_odd[0][d] & sees) ? INFINITY : 0.f) + ((s_odd[1][d] & sees) ? -INFINITY : 0.f);
            __builtin_amdgcn_sched_barrier(0);
          }
      }
    }
    if (odd) {  // the next such block starts with no keys
      __syncthreads();
      for (uint32_t i = threadIdx.x; i < 2 * kDim; i += kManyThreads) (&s_odd[0][0])[i] = 0;
    }
    if (more) {
      put(0, k_next);
      put(1, v_next);
    }
    __syncthreads();
  };

  for (uint32_t i = threadIdx.x; i < 2 * kDim; i += kManyThreads) (&s_odd[0][0])[i] = 0;
  for (int i = wave; i < 4; i += kManyWaves) hand_out(look_up(x0 - 1 + i), x0 - 1 + i);
  ahead = look_up(x0 + 3 + wave);
  __syncthreads();
  if (x0 < x_end) {
    load(x0 - 1, 0, kKeys[1]);
    put(0, kKeys[1]);
    load(x0, 0, kKeys[0]);
    load(x0, 1, kValues[0]);
    put(0, kKeys[0]);
    put(1, kValues[0]);
    __syncthreads();
    start(now, range.block(x0) * kManyBlock);
#pragma unroll
    for (int k = 0; k < kSteps * 2; ++k)
      now = Q::mfma32(*lds_at<u32x4>(beside(key_at, k * 32) + kKeys[1] + kHalfKeys), q[k], now);
    // the first step loads into the buffer that these products read
    __syncthreads();
    auto steps = [&](auto computes) __attribute__((always_inline)) {
      for (int32_t x = x0;;) {
        step(x, std::integral_constant<int, 0>{}, computes);
        if (++x >= x_end) break;
        step(x, std::integral_constant<int, 1>{}, computes);
        if (++x >= x_end) break;
      }
    };
    if (has_rows) steps(std::true_type{});
    else steps(std::false_type{});  // loads for the others
  }

  sum = xor32(sum, sum_of);
  if ((uint32_t)wave * 32 + m >= tile.rows) return;
  // the row again, which was not kept in registers
  uint32_t n = m;
  asm("" : "+v"(n));
  n += tile.row0 + wave * 32;
  const uint32_t token_out = fastdiv(n, p.group), head_out = head * p.group.d + (n - token_out * p.group.d);
  const bool divided = part.divided;
  const uint64_t t_out = (uint64_t)(w.r.start + token_out);
  const float vs = p.value_scale ? p.value_scale[head] : 1.f;
  const float norm = divided ? 1.f : sum != 0.f ? vs / sum : 0.f;
  const uint64_t slot = ((uint64_t)part.slot * p.kv_heads + head) * kManyRows + wave * 32 + m;
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
        *reinterpret_cast<u32x2 *>(p.out + t_out * p.out_stride + (uint64_t)head_out * p.D + d) =
            u32x2{Q::pack(y.x, y.y), Q::pack(y.z, y.w)};
    }
  if (g == 0) {
    if (divided) {
      float *ml = p.parts + (uint64_t)p.shares * 2 * p.kv_heads * kManyRows * p.D + slot * 2;
      ml[0] = best;
      ml[1] = sum;
    } else if (p.lse) {
      p.lse[t_out * p.heads + head_out] = sum != 0.f ? (best + __log2f(sum)) * kLn2 : -INFINITY;
    }
  }
}

// Workgroups a CU: three for D <= 64, in 168 registers (8 requests of 1000 tokens over 8000: 127
// us; two workgroups, with room for more registers, 137), two for 96.
template <typename Q, bool k8, int kSteps, int kMore>
__global__ __launch_bounds__(many_waves(kSteps) * 64, kSteps >= 4 ? 1 : kSteps > 2 ? 2 : 3) void attend_many(AttendParams p) {
  const uint32_t index = fastdiv(blockIdx.x, p.by_kv), head = blockIdx.x - index * p.kv_heads;
  WorkItem w;
  if (!find_item<many_waves(kSteps) * 64, kManyBlock>(p, index, w)) return note_cut<many_rows(kSteps)>(p, index, head);
  for (;;) {
    const Tile tile = tile_of(p, w.r, w.tile);
    const KeyRange range = key_range<kManyBlock>(p, w.r, tile.first, tile.last);
    const uint32_t blocks = (uint32_t)max(range.count, 1);
    const Part part = part_of(p, w, blocks, index);
    if (!part.none) many_part<Q, k8, kSteps, kMore>(p, w, tile, range, part, head);
    const uint64_t end = w.begin + blocks;
    if (end >= (index + 1) * w.share || end >= w.line || !next_item(p, w, end))
      return note_cut<many_rows(kSteps)>(p, index, head, w, tile, part, blocks);
    __syncthreads();
  }
}

}  // namespace gorio
