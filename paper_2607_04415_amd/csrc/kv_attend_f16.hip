// Attention kernels for f16 queries.
#include "kv_attend_few.hpp"
#include "kv_launch.hpp"

namespace gorio {

hipError_t launch_attend_f16(const AttendParams &p, const AttendLaunch &l, hipStream_t s) {
  return launch_attend<KvF16>(p, l, s);
}

}  // namespace gorio
