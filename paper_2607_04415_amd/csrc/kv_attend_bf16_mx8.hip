// Attention kernels of bf16 queries over 8-bit pages of blocks with a power.
#include "kv_launch.hpp"

namespace gorio {

hipError_t launch_attend_bf16_mx8(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  return launch_pages<KvBf16, kPagesMx8>(p, l, s);
}

}  // namespace gorio
