// attend_selected_fp16.cu -- the attention kernels over selected pages of a cache of type fp16.

#include "attend_kernels.cuh"

namespace kvx {

cudaError_t launch_attend_selected_fp16(const AttendParams& p, int num_sms, cudaStream_t s) { return attend<Fp16, true>(p, num_sms, s); }
cudaError_t prepare_attend_selected_fp16() { return prepare<Fp16, true>(); }

}  // namespace kvx
