// Which attention kernels run: by the pages' type, the head's size, whether
// scores are changed, and the form.
#pragma once

#include "kv_attend_few.hpp"
#include "kv_attend_many.hpp"

namespace gorio {

// One form's launch: AttendParams' fields for the division of its work.
struct AttendForm {
  uint32_t rows, from, upto, shares, least, whole;
  bool cuts;  // a tile may be cut
};

struct AttendLaunch {
  bool e4m3;  // 8-bit pages
  int more;   // 1 if scores are biased, 2 if they are capped, 3 if by a cap past kQuickCap
  AttendForm few, many;
};

template <typename Q, bool k8, int kSteps, int kMore>
hipError_t launch_forms(AttendParams p, const AttendLaunch &l, hipStream_t s) {
  auto divide = [&](const AttendForm &f) {
    p.rows = f.rows;
    p.from = f.from;
    p.upto = f.upto;
    p.shares = f.shares;
    p.least = f.least;
    p.whole = f.whole;
    p.cuts = f.cuts;
  };
  if (l.few.shares) {
    divide(l.few);
    attend_few<Q, k8, kSteps, (kMore > 0)><<<l.few.shares * p.kv_heads, few_waves(kSteps) * 64, 0, s>>>(p);
    if (l.few.cuts) attend_join<Q, kFewRows><<<(l.few.shares - 1) * p.kv_heads, 256, 0, s>>>(p);
  }
  if (l.many.shares) {
    divide(l.many);
    attend_many<Q, k8, kSteps, kMore><<<l.many.shares * p.kv_heads, many_waves(kSteps) * 64, 0, s>>>(p);
    if (l.many.cuts)
      attend_join<Q, many_rows(kSteps)><<<dim3((l.many.shares - 1) * p.kv_heads, many_rows(kSteps) / 16), 256, 0, s>>>(p);
  }
  return hipGetLastError();
}

template <typename Q, bool k8, int kSteps>
hipError_t launch_steps(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  switch (l.more) {
    case 0: return launch_forms<Q, k8, kSteps, 0>(p, l, s);
    case 1: return launch_forms<Q, k8, kSteps, 1>(p, l, s);
    case 2: return launch_forms<Q, k8, kSteps, 2>(p, l, s);
    default: return launch_forms<Q, k8, kSteps, 3>(p, l, s);
  }
}

// 32-element steps of the kernels for a head of D elements.
inline int steps_of(uint32_t D) { return D <= 64 ? 2 : D <= 96 ? 3 : D <= 128 ? 4 : 8; }

template <typename Q, bool k8>
hipError_t launch_pages(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  switch (steps_of(p.D)) {
    case 2: return launch_steps<Q, k8, 2>(p, l, s);
    case 3: return launch_steps<Q, k8, 3>(p, l, s);
    case 4: return launch_steps<Q, k8, 4>(p, l, s);
    default: return launch_steps<Q, k8, 8>(p, l, s);
  }
}

hipError_t launch_attend_bf16(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_bf16_e4m3(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_f16(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_f16_e4m3(const AttendParams &p, const AttendLaunch &l, hipStream_t s);

}  // namespace gorio
