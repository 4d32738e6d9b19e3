// kvx_attend_tc_cap.cu -- the attention kernels on the tensor cores, scores capped by a tanh.
#include "kvx_attend_tc.cuh"

namespace kvx {

cudaError_t launch_attend_tc_capped(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    return run_attend_tc<true>(P, num_sms, stream);
}

}  // namespace kvx
