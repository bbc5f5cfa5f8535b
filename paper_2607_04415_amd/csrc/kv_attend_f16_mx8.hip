// Attention kernels of f16 queries over 8-bit pages of blocks with a power.
#include "kv_launch.hpp"

namespace gorio {

hipError_t launch_attend_f16_mx8(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  return launch_pages<KvF16, kPagesMx8>(p, l, s);
}

}  // namespace gorio
