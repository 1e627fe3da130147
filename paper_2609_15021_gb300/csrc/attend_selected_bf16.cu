// attend_selected_bf16.cu -- the attention kernels over selected pages of a cache of type bf16.

#include "attend_kernels.cuh"

namespace kvx {

cudaError_t launch_attend_selected_bf16(const AttendParams& p, int num_sms, cudaStream_t s) { return attend<Bf16, true>(p, num_sms, s); }
cudaError_t prepare_attend_selected_bf16() { return prepare<Bf16, true>(); }

}  // namespace kvx
