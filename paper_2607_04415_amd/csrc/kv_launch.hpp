// Which attention kernels run: by the pages' type, the head's size, whether
// scores are changed, and the form.
#pragma once

#include "kv_attend_few.hpp"
#include "kv_attend_many.hpp"

namespace gorio {

// Whether the form for many rows has workgroups of four waves where it has eight: with powers, two of
// them would not fit LDS.
constexpr bool brief_many(int pages) { return pages < kPagesMx8; }

// One form's launch: AttendParams' fields for the division of its work.
struct AttendForm {
  uint32_t rows, from, upto, shares, least, whole, pad;
  bool cuts;  // a tile may be cut
};

struct AttendLaunch {
  int pages;  // a PageKind
  int more;   // 1 if scores are biased, 2 if they are capped, 3 if by a cap past kQuickCap
  AttendForm few, many;
  AttendForm group;  // the form for many rows over the groups' shared positions, before the others
  uint32_t groups;
};

template <typename Q, int kPages, int kSteps, int kMore>
hipError_t launch_forms(AttendParams p, const AttendLaunch &l, hipStream_t s) {
  auto divide = [&](const AttendForm &f) {
    p.rows = f.rows;
    p.from = f.from;
    p.upto = f.upto;
    p.shares = f.shares;
    p.least = f.least;
    p.whole = f.whole;
    p.pad = f.pad;
    p.cuts = f.cuts;
  };
  auto run_many = [&](const AttendForm &f, void (*kernel)(AttendParams), auto waves) {
    constexpr int kWaves = decltype(waves)::value;
    divide(f);
    kernel<<<f.shares * p.kv_heads, kWaves * 64, 0, s>>>(p);
    if (f.cuts)
      attend_join<Q, kWaves * 32, (kSteps > 4)><<<dim3(kWaves * 2, (f.shares - 1) * p.kv_heads), 256, 0, s>>>(p);
  };
  constexpr int kLong = many_waves(kSteps, false);
  constexpr int kBrief = many_waves(kSteps, brief_many(kPages));
  if (l.group.shares) {
    p.grouped = true;
    p.requests = l.groups;
    run_many(l.group, attend_many<Q, kPages, kSteps, kMore == 1 ? 3 : kMore, true, kLong>, std::integral_constant<int, kLong>{});
    p.grouped = false;
    p.requests = p.all_requests;
  }
  if (l.few.shares) {
    divide(l.few);
    // a key's lanes take equal numbers of eights
    constexpr int kFew = PageOf<kPages>::kMx && kSteps == 3 ? 4 : kSteps;
    constexpr int kWaves = few_waves(kFew, false), kShort = few_waves(kFew, true);
    if (l.group.shares || few_small(kPages, kFew))
      attend_few<Q, kPages, kFew, (kMore > 0), kShort><<<l.few.shares * p.kv_heads, kShort * 64, 0, s>>>(p);
    else
      attend_few<Q, kPages, kFew, (kMore > 0), kWaves><<<l.few.shares * p.kv_heads, kWaves * 64, 0, s>>>(p);
    if (l.few.cuts) attend_join<Q, kFewRows, (kSteps > 4)><<<dim3(1, (l.few.shares - 1) * p.kv_heads), 256, 0, s>>>(p);
  }
  if (l.many.shares) {
    if (l.group.shares) run_many(l.many, attend_many<Q, kPages, kSteps, kMore, false, kBrief>, std::integral_constant<int, kBrief>{});
    else run_many(l.many, attend_many<Q, kPages, kSteps, kMore, false, kLong>, std::integral_constant<int, kLong>{});
  }
  return hipGetLastError();
}

template <typename Q, int kPages, int kSteps>
hipError_t launch_steps(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  if constexpr (!PageOf<kPages>::kMx)
    if (l.more == 1) return launch_forms<Q, kPages, kSteps, 1>(p, l, s);
  switch (l.more) {
    case 0: return launch_forms<Q, kPages, kSteps, 0>(p, l, s);
    case 2: return launch_forms<Q, kPages, kSteps, 2>(p, l, s);
    default: return launch_forms<Q, kPages, kSteps, 3>(p, l, s);
  }
}

// 32-element steps of the kernels for a head of D elements.  Heads of 129..192 have kernels of their
// own where elements have powers, which take registers on their way into LDS: 4096 tokens of 160
// elements over 16384 took 2981 us from MX8 pages as 256 elements.
inline int steps_of(uint32_t D, int pages) {
  return D <= 64 ? 2 : D <= 96 ? 3 : D <= 128 ? 4 : D <= 192 && pages >= kPagesMx8 ? 6 : 8;
}

template <typename Q, int kPages>
hipError_t launch_pages(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  if constexpr (PageOf<kPages>::kMx)
    if (steps_of(p.D, kPages) == 6) return launch_steps<Q, kPages, 6>(p, l, s);
  switch (steps_of(p.D, kPages)) {
    case 2: return launch_steps<Q, kPages, 2>(p, l, s);
    case 3: return launch_steps<Q, kPages, 3>(p, l, s);
    case 4: return launch_steps<Q, kPages, 4>(p, l, s);
    default: return launch_steps<Q, kPages, 8>(p, l, s);
  }
}

hipError_t launch_attend_bf16(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_bf16_e4m3(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_bf16_mx8(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_bf16_mx4(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_f16(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_f16_e4m3(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_f16_mx8(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_f16_mx4(const AttendParams &p, const AttendLaunch &l, hipStream_t s);

}  // namespace gorio
