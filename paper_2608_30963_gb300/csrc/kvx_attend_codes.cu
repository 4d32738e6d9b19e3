// kvx_attend_codes.cu -- attention of new tokens over an 8-bit cache: the choice of the kernels.
#include "kvx_attend_simt.cuh"

namespace kvx {
namespace {

template <typename T, int D, bool CAP> cudaError_t run_codes(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    // few rows: 16-row tiles, as over fp32 caches
    const bool few = (long long)P.T * P.G <= 16ll * P.batch;
    return few ? run_simt<T, D, 16, CAP, true>(P, num_sms, stream) : run_simt<T, D, D == 256 ? 32 : 64, CAP, true>(P, num_sms, stream);
}
template <typename T, bool CAP> cudaError_t run_codes(const AttendParams& P, int num_sms, cudaStream_t stream)
{
    return P.d == 64 ? run_codes<T, 64, CAP>(P, num_sms, stream) : P.d == 128 ? run_codes<T, 128, CAP>(P, num_sms, stream)
                                                                             : run_codes<T, 256, CAP>(P, num_sms, stream);
}

}  // namespace

cudaError_t launch_attend_codes(const AttendParams& P, int dtype, int num_sms, cudaStream_t stream, int* launches)
{
    *launches = 0;
    if (P.T == 0) return cudaSuccess;
    *launches = 2;
    if (dtype == KVX_BF16) return P.cap > 0.0f ? launch_attend_tc_codes_capped(P, num_sms, stream) : launch_attend_tc_codes(P, num_sms, stream);
    return P.cap > 0.0f ? run_codes<float, true>(P, num_sms, stream) : run_codes<float, false>(P, num_sms, stream);
}

}  // namespace kvx
