// attend_bf16.cu -- the attention kernels over a cache of type bf16.

#include "attend_kernels.cuh"

namespace kvx {

cudaError_t launch_attend_bf16(const AttendParams& p, int num_sms, cudaStream_t s) { return attend<Bf16, false>(p, num_sms, s); }
cudaError_t prepare_attend_bf16() { return prepare<Bf16, false>(); }

}  // namespace kvx
