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
// Elements with powers (MX8, MX4) are widened by the conversions that take a
// power of two, so it costs nothing there; but the powers are a byte for 32
// elements, and to have them where they are needed is what costs.  The lane
// that looks a key up loads its powers, all in two loads, and the lanes get
// them through LDS a block later.  A lane's elements of a key follow one
// another: one 16-byte load of 4-bit ones, one power.
// Loads are written as loads of memory (load_at) and without tests among them:
// else waits for LDS, or for a table entry, wait for keys and values as well
// (4-bit pages 300 us in the first form, byte by byte; 195; 155 now).
//
// Measured, 64 requests of up to 16384 tokens, 8 key heads: 5.8 TB/s of keys
// and values at D = 128 (449 us), 5.6 at 64, 5.9 at 256; from 8-bit pages 5.4
// at 128 and 4.1 at 64, where a row is 64 bytes; from MX8 pages 5.4 at 128, 5.0
// at 96, 4.8 at 64, 4.9 at 160, 5.6 at 256; from MX4 pages, 0.53 bytes an
// element, 4.5 at 128 (155 us, 2.9 times as fast as from 16 bits), 3.1 at 96
// and 64, 2.7 at 160, 4.2 at 256: latency, 0.12 to 0.13 TB/s for each KB that a
// CU has under way (a block a wave: 35, 26, 22 and 35 KB; from MX8 pages 42 to 68,
// which HBM bounds).  Beside it 20 vector instructions to a matrix instruction:
// a wave issues 43% of its time and waits 41%.
// A copy on the same card moves 4.8 TB/s.  One request: 10 us for 64 tokens,
// 16 for 1000, 35 for 32000, of which the first 10 are the wait for
// lengths, table and keys, one after the other, and of the longer ones 3 to 5
// the joining kernel.
#pragma once

#include "kv_attend.hpp"

namespace gorio {

// Waves of a workgroup: 64 requests of 16384 tokens take 235 us at D = 64 and 451 at 128 with
// eight, 256 and 456 with four.  256 elements take the registers of twice as many.  brief: behind a
// shared prefix a request's own keys are few, and two workgroups of four waves a CU, a tile each, wait
// for them together (64 requests of 125 to 500 own keys: 24 us, with one of eight 35).
__host__ __device__ constexpr int few_waves(int steps, bool brief) { return steps > 4 || brief ? 4 : 8; }
// Small heads from pages with powers take the registers and the LDS for three workgroups of four waves a
// CU: 64 requests of 16384 tokens at D = 64 from MX4 pages take 114 us, as one of eight 131.
__host__ __device__ constexpr bool few_small(int pages, int steps) { return pages >= kPagesMx8 && steps == 2; }
constexpr int kFewRows = 16;
constexpr int kFewBlock = 32;  // keys

// Memory at any byte: a struct keeps its alignment as a template's argument, a typedef does not.
template <typename T>
struct __attribute__((packed)) Anywhere {
  T value;
};
template <typename T>
__device__ __forceinline__ uint32_t load_anywhere(uint64_t address) {
  return ((const __attribute__((address_space(1))) Anywhere<T> *)(uintptr_t)address)->value;
}

// The powers of a row's blocks, of which there are `count`: kBlocks or one less.  Two loads, the
// second up to the last of them.
template <int kBlocks, typename Powers>
__device__ __forceinline__ Powers load_powers(uint64_t from, uint32_t count) {
  static_assert(kBlocks == 2 || kBlocks == 4 || kBlocks == 6 || kBlocks == 8, "pairs of blocks");
  const uint32_t less = kBlocks - count;
  if constexpr (kBlocks == 2) return load_at<uint8_t>(from) | (uint32_t)load_at<uint8_t>(from + count - 1) << (count - 1) * 8;
  else if constexpr (kBlocks == 4) return load_anywhere<uint16_t>(from) | load_anywhere<uint16_t>(from + count - 2) << (count - 2) * 8;
  else if constexpr (kBlocks == 6) return Powers{load_anywhere<uint32_t>(from), load_anywhere<uint16_t>(from + count - 2) >> less * 8};
  else return Powers{load_anywhere<uint32_t>(from), load_anywhere<uint32_t>(from + count - 4) >> less * 8};
}

// kSteps: 32-element steps of a head, D <= 32 kSteps (2, 4, 6 or 8 with powers).  kPages: a PageKind.
// kMore: scores are capped or biased.
template <typename Q, int kPages, int kSteps, bool kMore, int kFewWaves>
__device__ __forceinline__ void few_part(const AttendParams &p, const WorkItem &w, const Tile &tile,
                                         const KeyRange &range, const Part &part, uint32_t head) {
  constexpr int kFewThreads = kFewWaves * 64;
  typedef PageOf<kPages> Page;
  typedef typename Page::Raw Raw;
  constexpr bool kMx = Page::kMx;
  // A value in runs of 128 elements, eight to a lane, of which as many products come; with powers the
  // last run may be 64, four to a lane.  (16-bit pages of 64 elements are read as if they had 128, which
  // costs them nothing while HBM is the bound.)
  constexpr int kRuns = (kSteps + 3) / 4, kFull = kMx ? kSteps / 4 : kRuns;
  constexpr auto per = [](int h) { return h < kFull ? 8 : 4; };
  constexpr int kProducts = kFull * 8 + (kRuns - kFull) * 4, kDim = kProducts * 16;
  constexpr int kPad = kDim + 4;
  // Powers of a row's blocks, a byte each; the lanes that look a key up load them and hand them
  // out a block later.
  constexpr int kBlocks = kSteps;
  typedef typename std::conditional<(kSteps > 4), u32x2, uint32_t>::type Powers;
  __shared__ __align__(16) Powers s_power[kMx ? kFewWaves : 1][2][kFewBlock];  // keys, values
  // Elements of a key in a lane, which need not be every fourth eight of them: with powers they
  // follow one another, so that they are one load, or few, and their powers one or two.
  constexpr int kWords = kPages == kPagesMx4 ? kSteps : kSteps * 2, kLoad = kWords % 4 ? 2 : 4;
  typedef typename std::conditional<kLoad == 2, u32x2, u32x4>::type Load;
  auto element = [](int s, int g) __attribute__((always_inline)) -> uint32_t { return kMx ? g * 8 * kSteps + s * 8 : s * 32 + g * 8; };
  __shared__ uint64_t s_row[kFewWaves][2][2][kFewBlock];  // wave, turn, keys or values
  __shared__ float s_o[kFewWaves][kFewRows][kPad];
  __shared__ float s_m[kFewWaves][kFewRows], s_l[kFewWaves][kFewRows];

  const int32_t x_end = min(range.count, (int32_t)part.upto);

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m = lane & 15, g = lane >> 4;
  const uint64_t zeros = (uint64_t)(uintptr_t)kv_zeros;

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
      const uint32_t d = element(s, g);
      q[s] = d < p.D ? *reinterpret_cast<const u32x4 *>(row + d) : u32x4{0, 0, 0, 0};
    }
  }
  const float scale = p.scale * (p.key_scale ? p.key_scale[head] : 1.f);
  const float to_log2 = scale * kLog2e;
  const ScoreChange change(scale, p.cap, kMore && p.slopes ? p.slopes[qhead] : 0.f);

  float best = -INFINITY, sum = 0.f;
  f32x4 o[kProducts];
#pragma unroll
  for (int t = 0; t < kProducts; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  // Rows of block x into LDS, and its keys' bits: lanes 0..31 a key each, with powers the others too.
  auto place_of = [&](int32_t x) __attribute__((always_inline)) {
    return key_look(p, w, tile, (x < x_end) & (kMx || lane < kFewBlock), range.block(x) * kFewBlock + (lane & 31), range.end);
  };
  uint64_t all_powers = 0;  // worked out once: a choice between two arguments would pass through memory
  if constexpr (kMx) {
    const uint64_t of_keys = (uint64_t)(uintptr_t)p.key_powers, of_values = (uint64_t)(uintptr_t)p.value_powers;
    all_powers = lane < kFewBlock ? of_keys : of_values;
    asm("" : "+v"(all_powers));
  }
  Powers powers{};  // of a key (lanes 0..31) or value (32..63) of the block whose rows were handed out last
  auto hand_out = [&](const KeyLook &k, int turn) __attribute__((always_inline)) -> uint32_t {
    const bool there = key_there(p, k);
    const uint64_t off = (uint64_t)(uint32_t)k.page * p.page_stride + head * p.head_stride + k.place * p.token_stride;
    if (lane < kFewBlock) {
      s_row[wave][turn][0][lane] = there ? (uint64_t)(uintptr_t)p.keys + off : zeros;
      s_row[wave][turn][1][lane] = there ? (uint64_t)(uintptr_t)p.values + off : zeros;
    }
    if constexpr (kMx) {
      const uint64_t from = there ? all_powers + Page::powers(off) : zeros;
      powers = load_powers<kBlocks, Powers>(from, p.D / kMxBlock);
    }
    wave_lds_order();
    return (uint32_t)__ballot(there);
  };
  auto load_keys = [&](Raw (&k)[2][kSteps], int turn, auto whole_rows) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      uint64_t row = s_row[wave][turn][0][i * 16 + m];
      asm("" : "+v"(row));  // read by all lanes, also by those whose elements end before: no branch
      if constexpr (kMx) {
        uint32_t words[kWords];
#pragma unroll
        for (int u = 0; u < kWords / kLoad; ++u) {
          const uint32_t d = element(u * kLoad * kSteps / kWords, g);
          const Load some = load_at<Load>(decltype(whole_rows)::value || d < p.D ? row + Page::bytes(d) : zeros);
#pragma unroll
          for (int c = 0; c < kLoad; ++c) words[u * kLoad + c] = some[c];
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          if constexpr (kPages == kPagesMx4) k[i][s] = words[s];
          else if constexpr (kPages == kPagesMx8) k[i][s] = u32x2{words[2 * s], words[2 * s + 1]};
        }
      } else {
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const uint32_t d = element(s, g);
          k[i][s] = load_at<Raw>(decltype(whole_rows)::value || d < p.D ? row + Page::bytes(d) : zeros);
        }
      }
    }
  };
  auto load_values = [&](Raw (&v)[8], int h, int turn, auto whole_rows) __attribute__((always_inline)) {
    const uint32_t d = h * 128 + m * per(h);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint64_t row = s_row[wave][turn][1][(i >> 2) * 16 + g * 4 + (i & 3)];
      asm("" : "+v"(row));
      const uint64_t at = decltype(whole_rows)::value || d < p.D ? row + Page::bytes(d) : zeros;
      if (h < kFull) v[i] = load_at<Raw>(at);
      else if constexpr (kPages == kPagesMx4) v[i] = load_at<uint16_t>(at);
      else if constexpr (kPages == kPagesMx8) v[i] = u32x2{load_at<uint32_t>(at), 0};
    }
  };
  // What the powers of step s of a key, and of a value's run, multiply by, from LDS.
  auto key_factor = [&](int i, int s) __attribute__((always_inline)) -> float {
    if constexpr (!kMx) return 1.f;
    const Powers all = s_power[kMx ? wave : 0][0][i * 16 + m];
    const uint32_t block = element(s, g) / kMxBlock;
    if constexpr (kSteps > 4) return power_of((block < 4 ? all.x : all.y) >> (block & 3) * 8 & 255);
    else return power_of(all >> block * 8 & 255);
  };
  auto value_factor = [&](int i, int h) __attribute__((always_inline)) -> float {
    if constexpr (!kMx) return 1.f;
    const Powers all = s_power[kMx ? wave : 0][1][(i >> 2) * 16 + g * 4 + (i & 3)];
    const uint32_t block = m * per(h) / kMxBlock;
    if constexpr (kSteps > 4) return power_of((h ? all.y : all.x) >> block * 8 & 255);
    else return power_of(all >> block * 8 & 255);
  };
  // Block x, with the next one's keys and values on their way; the registers alternate.
  Raw k[2][2][kSteps];
  Raw v[2][kRuns][8];
  uint32_t there[2];
  KeyLook next;
  auto load = [&](auto turn, auto whole_rows) __attribute__((always_inline)) {
    constexpr int t = decltype(turn)::value;
    load_keys(k[t], t, whole_rows);
#pragma unroll
    for (int h = 0; h < kRuns; ++h) load_values(v[t][h], h, t, whole_rows);
  };
  auto step = [&](int32_t x, auto turn, auto whole_rows) __attribute__((always_inline)) {
    constexpr int t0 = decltype(turn)::value, t1 = 1 - t0;
    const int32_t j0 = range.block(x) * kFewBlock;
    const uint32_t there_now = there[t0];
    if constexpr (kMx) {
      s_power[wave][lane >> 5][lane & 31] = powers;
      wave_lds_order();
    }
    there[t1] = hand_out(next, t1);
    next = place_of(x + 2 * kFewWaves);
    load(std::integral_constant<int, t1>{}, whole_rows);

    f32x4 s2[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s2[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) s2[i] = Q::mfma16(widened<Q>(k[t0][i][s], key_factor(i, s)), q[s], s2[i]);
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
      for (int t = 0; t < kProducts; ++t) o[t] *= keep;
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
    for (int h = 0; h < kRuns; ++h) {
      u32x4 vw[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (h < kFull) vw[i] = widened<Q>(v[t0][h][i], value_factor(i, h));
        else vw[i] = widened_half<Q>(v[t0][h][i], value_factor(i, h));
      }
      // A weight of 0 keeps a value out of a row, unless the value is NaN or inf.  Such
      // values in a block that some rows see only in part go in apart from the others.
      bool odd = false;
      if (!whole && tile.first != tile.last) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int c = 0; c < per(h) / 2; ++c) odd |= any_not_finite<Q>(vw[i][c]);
        odd = __any(odd);
      }
      auto products = [&](auto test) __attribute__((always_inline)) {
#pragma unroll
        for (int t = 0; t < per(h); ++t) {
          const uint32_t sel = t & 1 ? 0x07060302u : 0x05040100u;
          u32x4 a;
#pragma unroll
          for (int i = 0; i < 4; ++i) a[i] = __builtin_amdgcn_perm(vw[2 * i + 1][t >> 1], vw[2 * i][t >> 1], sel);
          if constexpr (decltype(test)::value) {
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
          }
          o[h * 8 + t] = Q::mfma16(a, weights, o[h * 8 + t]);
        }
      };
      // One test is better than eight, but 16-bit pages' registers do not hold the products twice.
      if (kMx && __builtin_expect(!odd, 1)) products(std::false_type{});
      else products(std::true_type{});
    }
  };
  auto steps = [&](auto whole_rows) __attribute__((always_inline)) {
    int32_t x = (int32_t)part.from + wave;
    there[0] = hand_out(place_of(x), 0);
    next = place_of(x + kFewWaves);
    load(std::integral_constant<int, 0>{}, whole_rows);
    while (x < x_end) {
      step(x, std::integral_constant<int, 0>{}, whole_rows);
      if ((x += kFewWaves) >= x_end) break;
      step(x, std::integral_constant<int, 1>{}, whole_rows);
      x += kFewWaves;
    }
  };
  // A loop of its own where lanes have no elements past D: tests among the loads would make the
  // compiler wait for all of them.
  if (kMx && p.D == kSteps * 32) steps(std::true_type{});
  else steps(std::false_type{});

  // the waves' results, joined
  sum = xor16(xor32(sum, sum_of), sum_of);
  if (g == 0) s_m[wave][m] = best, s_l[wave][m] = sum;
#pragma unroll
  for (int h = 0; h < kRuns; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float *to = &s_o[wave][m][h * 128 + (g * 4 + r) * per(h)];
#pragma unroll
      for (int t = 0; t < per(h); t += 4)
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
  float base = most == -INFINITY ? 0.f : most;
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
  const bool carries = w.r.skip > 0 && part.from == 0;  // the group's sums join as those of one wave more
  Carried carried{nullptr, 0.f, 0.f, 0.f};
  if (carries) {
    const float keep = take_carried(p, carried_row(p, t_out, hq), most, carried);
    base = most == -INFINITY ? 0.f : most;
    all = all * keep + carried.l * carried.by;
#pragma unroll
    for (int i = 0; i < kFewWaves; ++i) by[i] *= keep;
  }
  const float norm = divided ? 1.f : all != 0.f ? vs / all : 0.f;
  const uint64_t slot = ((uint64_t)part.slot * p.kv_heads + head) * kFewRows + row;
#pragma unroll
  for (int h = 0; h < kRuns; ++h) {
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
      if (carries) y += *reinterpret_cast<const f32x4 *>(carried.o + d + i) * carried.by;
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

template <typename Q, int kPages, int kSteps, bool kMore, int kWaves>
__global__ __launch_bounds__(kWaves * 64, kWaves == 4 && kSteps <= 4 ? (few_small(kPages, kSteps) ? 3 : 2) : 1) void attend_few(AttendParams p) {
  const uint32_t index = fastdiv(blockIdx.x, p.by_kv), head = blockIdx.x - index * p.kv_heads;
  WorkItem w;
  if (!find_item<kWaves * 64, kFewBlock, false>(p, index, w)) return note_cut<kFewRows>(p, index, head);
  for (;;) {
    const Tile tile = tile_of(p, w.r, w.tile);
    const KeyRange range = key_range<kFewBlock>(p, w.r, tile.first, tile.last);
    const uint32_t blocks = (uint32_t)max(range.count, 1);
    const Part part = part_of(p, w, blocks, index);
    if (!part.none) few_part<Q, kPages, kSteps, kMore, kWaves>(p, w, tile, range, part, head);
    const uint64_t end = w.begin + max(blocks, p.pad);
    if (end >= (index + 1) * w.share || end >= w.line || !next_item<false>(p, w, end))
      return note_cut<kFewRows>(p, index, head, w, tile, part, blocks);
    __syncthreads();  // the next tile's sums go where this one's are read
  }
}

// Joins the parts of divided tiles, of a group's into what its rows carry: a workgroup a share and
// head, for the tile that begins in the share and is cut at its end; 16 rows, 16 threads a row (64 rows
// a workgroup, four after the other: 128 new tokens over 2000 took 54 us in all, now 41).  A row's
// parts are added in order, and eight are loaded together: 31 parts of 2048 rows take 10 us, one after
// the other 18, sixteen together 14, a wave a row 13.  A tile's workgroups are neighbours in the
// launch, so that the few that have work begin together.  kWide: heads of more than 128 elements.
//   out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i over the parts i
// Bound by the latency of two dependent loads, 4 us, and for many tiles by reading the parts
// (750 cut tiles of 128 rows, 64 elements: 50 MB in 14 us).
template <typename Q, int kRows, bool kWide>
__global__ __launch_bounds__(256) void attend_join(AttendParams p) {
  const uint32_t s0 = fastdiv(blockIdx.y, p.by_kv), head = blockIdx.y - s0 * p.kv_heads;
  const Cut cut = cuts_of<kRows>(p)[blockIdx.y];
  const uint32_t parts = cut.parts, slot0 = cut.slot, lane = threadIdx.x & 15;  // slot0: of the first part
  const float *ml = p.parts + (uint64_t)p.shares * 2 * p.kv_heads * kRows * p.D;
  const float vs = p.value_scale ? p.value_scale[head] : 1.f;
  const uint32_t row = blockIdx.x * 16 + (threadIdx.x >> 4);
  if (parts && row < cut.rows) {
    auto slot = [&](uint32_t i) {
      return ((uint64_t)(i ? (s0 + i) * 2 : slot0) * p.kv_heads + head) * kRows + row;
    };
    float most = -INFINITY;
    for (uint32_t i = lane; i < parts; i += 16) most = fmaxf(most, ml[slot(i) * 2]);
#pragma unroll
    for (int d = 8; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    const float from = most == -INFINITY ? 0.f : most;
    constexpr int kEights = kWide ? 2 : 1, kTogether = 8;
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
      for (uint32_t i = 0; i < some; i += kTogether) {
        f32x4 o[kTogether][2 * kEights];
#pragma unroll
        for (uint32_t u = 0; u < kTogether; ++u)
#pragma unroll
          for (int h = 0; h < kEights; ++h) {
            const uint32_t d = d0 + h * 128;
            o[u][2 * h] = o[u][2 * h + 1] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (i + u < some && d < p.D) {
              const float *at = p.parts + slot(i0 + i + u) * p.D + d;
              o[u][2 * h] = *reinterpret_cast<const f32x4 *>(at);
              o[u][2 * h + 1] = *reinterpret_cast<const f32x4 *>(at + 4);
            }
          }
#pragma unroll
        for (uint32_t u = 0; u < kTogether; ++u) {
          const float one = __shfl(by, (int)(i + u), 16);  // 0 past the last part
#pragma unroll
          for (int h = 0; h < 2 * kEights; ++h) y[h] += o[u][h] * one;
        }
      }
    }
#pragma unroll
    for (int d = 8; d; d >>= 1) all += __shfl_xor(all, d);
    const float norm = all != 0.f ? vs / all : 0.f;
    const uint32_t tk = fastdiv(cut.row0 + row, p.group), hq = head * p.group.d + (cut.row0 + row - tk * p.group.d);
    const uint64_t t_out = (uint64_t)(cut.start + tk);
    if (p.grouped) {
      const uint64_t at = carried_row(p, t_out, hq);
#pragma unroll
      for (int i = 0; i < 4; i += 2) {
        const uint32_t d = i ? d1 : d0;
        if (d >= p.D) continue;
        *reinterpret_cast<f32x4 *>(p.carry + at * p.D + d) = y[i];
        *reinterpret_cast<f32x4 *>(p.carry + at * p.D + d + 4) = y[i + 1];
      }
      if (lane == 0) {
        float *sums = carried_sums(p, at);
        sums[0] = most;
        sums[1] = all;
      }
      return;
    }
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
