// Attention of few tokens over 8-bit caches, scores capped (kvx_attend_few.cuh).
#include "kvx_attend_few.cuh"

namespace kvx {

cudaError_t launch_attend_few_capped(const AttendParams& P, int rows, int num_sms, cudaStream_t stream)
{
    constexpr bool CAP = true;
    if (P.d == 128)
        return rows <= 8 ? run_few<128, 8, CAP>(P, num_sms, stream) : rows <= 16 ? run_few<128, 16, CAP>(P, num_sms, stream) : run_few<128, 32, CAP>(P, num_sms, stream);
    return rows <= 8 ? run_few<256, 8, CAP>(P, num_sms, stream) : rows <= 16 ? run_few<256, 16, CAP>(P, num_sms, stream) : run_few<256, 32, CAP>(P, num_sms, stream);
}

}  // namespace kvx
