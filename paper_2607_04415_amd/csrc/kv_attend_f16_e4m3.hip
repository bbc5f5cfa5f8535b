// Attention kernels of f16 queries over 8-bit pages.
#include "kv_launch.hpp"

namespace gorio {

hipError_t launch_attend_f16_e4m3(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  return launch_pages<KvF16, kPagesE4m3>(p, l, s);
}

}  // namespace gorio
