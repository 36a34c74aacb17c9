// Instances of the paged attention for caches of e4m3.
#include "vt_kv_attend.cuh"

namespace vt {

cudaError_t launch_kv_attend_e4m3(const KvAttendArgs& a, int& ctas, cudaStream_t s) { return attend_any<true>(a, ctas, s); }

}  // namespace vt
