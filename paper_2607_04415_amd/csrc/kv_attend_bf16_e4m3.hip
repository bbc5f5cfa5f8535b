// Attention kernels of bf16 queries over 8-bit pages.
#include "kv_launch.hpp"

namespace gorio {

hipError_t launch_attend_bf16_e4m3(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  return launch_pages<KvBf16, true>(p, l, s);
}

}  // namespace gorio
