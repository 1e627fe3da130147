// attend_e4m3.cu -- the attention kernels over a cache of type e4m3.

#include "attend_kernels.cuh"

namespace kvx {

cudaError_t launch_attend_e4m3(const AttendParams& p, int num_sms, cudaStream_t s) { return attend<E4m3>(p, num_sms, s); }
cudaError_t prepare_attend_e4m3() { return prepare<E4m3>(); }

}  // namespace kvx
