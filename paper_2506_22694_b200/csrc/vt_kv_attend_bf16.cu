// Instances of the paged attention for caches of bf16.
#include "vt_kv_attend.cuh"

namespace vt {

cudaError_t launch_kv_attend_bf16(const KvAttendArgs& a, int& ctas, cudaStream_t s) { return attend_any<false>(a, ctas, s); }

}  // namespace vt
