// Attention kernels of f16 queries over 4-bit pages of blocks with a power.
#include "kv_launch.hpp"

namespace gorio {

hipError_t launch_attend_f16_mx4(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  return launch_pages<KvF16, kPagesMx4>(p, l, s);
}

}  // namespace gorio
