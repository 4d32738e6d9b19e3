// Attention over 8-bit caches on the tensor cores (kvx_attend_tc.cuh).
#include "kvx_attend_tc.cuh"

namespace kvx {

cudaError_t launch_attend_tc_codes(const AttendParams& P, int num_sms, cudaStream_t stream) { return run_attend_tc<false, true>(P, num_sms, stream); }

}  // namespace kvx
