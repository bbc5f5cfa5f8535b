// Which attention kernels run: by the pages' type, the head's size, whether
// scores are changed, and the form.
#pragma once

#include "kv_attend_few.hpp"
#include "kv_attend_many.hpp"

namespace gorio {

// One form's launch: AttendParams' fields for the division of its work, blocks, and blocks
// that join divided tiles (0: none are).
struct AttendForm {
  uint32_t rows, from, upto, least, most, part_slots;
  uint32_t grid, join;
};

struct AttendLaunch {
  bool e4m3, more;  // 8-bit pages; scores capped or biased
  AttendForm few, many;
};

template <typename Q, bool k8, int kSteps, bool kMore>
hipError_t launch_forms(AttendParams p, const AttendLaunch &l, hipStream_t s) {
  auto divide = [&](const AttendForm &f) {
    p.rows = f.rows;
    p.from = f.from;
    p.upto = f.upto;
    p.least = f.least;
    p.most = f.most;
    p.part_slots = f.part_slots;
  };
  if (l.few.grid) {
    divide(l.few);
    attend_few<Q, k8, kSteps, kMore><<<l.few.grid, kFewThreads, 0, s>>>(p);
    if (l.few.join) attend_join<Q, kFewRows, kFewBlock><<<l.few.join, 256, 0, s>>>(p);
  }
  if (l.many.grid) {
    divide(l.many);
    attend_many<Q, k8, kSteps, kMore><<<l.many.grid, kManyThreads, 0, s>>>(p);
    if (l.many.join) attend_join<Q, kManyRows, kManyBlock><<<l.many.join, 256, 0, s>>>(p);
  }
  return hipGetLastError();
}

template <typename Q, bool k8, int kSteps>
hipError_t launch_steps(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  return l.more ? launch_forms<Q, k8, kSteps, true>(p, l, s) : launch_forms<Q, k8, kSteps, false>(p, l, s);
}

template <typename Q, bool k8>
hipError_t launch_pages(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  if (p.D <= 64) return launch_steps<Q, k8, 2>(p, l, s);
  if (p.D <= 96) return launch_steps<Q, k8, 3>(p, l, s);
  if (p.D <= 128) return launch_steps<Q, k8, 4>(p, l, s);
  return launch_steps<Q, k8, 8>(p, l, s);
}

hipError_t launch_attend_bf16(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_bf16_e4m3(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_f16(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_f16_e4m3(const AttendParams &p, const AttendLaunch &l, hipStream_t s);

}  // namespace gorio
