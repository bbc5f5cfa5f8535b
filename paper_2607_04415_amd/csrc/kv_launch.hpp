// Which attention kernel runs: by the pages' type, the head's size and whether
// scores are changed.
#pragma once

#include "kv_attend.hpp"

namespace gorio {

struct AttendLaunch {
  bool e4m3, more;  // 8-bit pages; scores capped or biased
  uint32_t few_grid, join_grid;  // blocks; no join: 0
};

template <typename Q, bool k8, int kSteps>
void launch_few(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  if (l.more) attend_few<Q, k8, kSteps, true><<<l.few_grid, kFewThreads, 0, s>>>(p);
  else attend_few<Q, k8, kSteps, false><<<l.few_grid, kFewThreads, 0, s>>>(p);
}

template <typename Q, bool k8>
void launch_few(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  if (p.D <= 64) launch_few<Q, k8, 2>(p, l, s);
  else if (p.D <= 96) launch_few<Q, k8, 3>(p, l, s);
  else if (p.D <= 128) launch_few<Q, k8, 4>(p, l, s);
  else launch_few<Q, k8, 8>(p, l, s);
}

template <typename Q>
hipError_t launch_attend(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  if (l.e4m3) launch_few<Q, true>(p, l, s);
  else launch_few<Q, false>(p, l, s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || l.join_grid == 0) return e;
  attend_join<Q, kFewRows, kFewBlock><<<l.join_grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

hipError_t launch_attend_bf16(const AttendParams &p, const AttendLaunch &l, hipStream_t s);
hipError_t launch_attend_f16(const AttendParams &p, const AttendLaunch &l, hipStream_t s);

}  // namespace gorio
