// Which attention kernels run: by the pages' type, the head's size, whether
// scores are changed, and the form.
#pragma once

#include "kv_attend_few.hpp"
#include "kv_attend_many.hpp"

namespace gorio {

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
  auto run_many = [&](const AttendForm &f, void (*kernel)(AttendParams)) {
    divide(f);
    kernel<<<f.shares * p.kv_heads, many_waves(kSteps) * 64, 0, s>>>(p);
    if (f.cuts)
      attend_join<Q, many_rows(kSteps), (kSteps > 4)><<<dim3((f.shares - 1) * p.kv_heads, many_rows(kSteps) / 16), 256, 0, s>>>(p);
  };
  if (l.group.shares) {
    p.grouped = true;
    p.requests = l.groups;
    run_many(l.group, attend_many<Q, kPages, kSteps, kMore == 1 ? 3 : kMore, true>);
    p.grouped = false;
    p.requests = p.all_requests;
  }
  if (l.few.shares) {
    divide(l.few);
    constexpr int kFew = PageOf<kPages>::kMx && kSteps == 3 ? 4 : kSteps;  // a key's lanes take equal numbers of eights
    constexpr int kWaves = few_waves(kFew, false), kShort = few_waves(kFew, true);
    if (l.group.shares)
      attend_few<Q, kPages, kFew, (kMore > 0), kShort><<<l.few.shares * p.kv_heads, kShort * 64, 0, s>>>(p);
    else
      attend_few<Q, kPages, kFew, (kMore > 0), kWaves><<<l.few.shares * p.kv_heads, kWaves * 64, 0, s>>>(p);
    if (l.few.cuts) attend_join<Q, kFewRows, (kSteps > 4)><<<(l.few.shares - 1) * p.kv_heads, 256, 0, s>>>(p);
  }
  if (l.many.shares) run_many(l.many, attend_many<Q, kPages, kSteps, kMore, false>);
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

// 32-element steps of the kernels for a head of D elements.
inline int steps_of(uint32_t D) { return D <= 64 ? 2 : D <= 96 ? 3 : D <= 128 ? 4 : 8; }

template <typename Q, int kPages>
hipError_t launch_pages(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  switch (steps_of(p.D)) {
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
