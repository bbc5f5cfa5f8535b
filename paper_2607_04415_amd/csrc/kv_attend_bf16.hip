// Attention kernels of bf16 queries over bf16 pages.
#include "kv_launch.hpp"

namespace gorio {

hipError_t launch_attend_bf16(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  return launch_pages<KvBf16, false>(p, l, s);
}

}  // namespace gorio
