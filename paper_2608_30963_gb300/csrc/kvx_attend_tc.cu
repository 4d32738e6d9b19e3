// kvx_attend_tc.cu -- the attention kernels on the tensor cores, plain scores.
#include "kvx_attend_tc.cuh"

namespace kvx {

cudaError_t launch_attend_tc(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    return P.cap > 0.0f ? launch_attend_tc_capped(P, num_sms, stream) : run_attend_tc<false>(P, num_sms, stream);
}

}  // namespace kvx
