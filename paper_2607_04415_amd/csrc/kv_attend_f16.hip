// Attention kernels of f16 queries over f16 pages.
#include "kv_launch.hpp"

namespace gorio {

hipError_t launch_attend_f16(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  return launch_pages<KvF16, false>(p, l, s);
}

}  // namespace gorio
