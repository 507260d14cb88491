/* The attention's kernels for f16 queries over a cache in 8 bits (cfa_attend.cuh). */
#include "cfa_attend.cuh"

cudaError_t cfa_launch_attend_f16_f8(const cfa_attend_work *w, cudaStream_t stream)
{
    return cfa_attend_dev::launch_any<__half, true>(*w, stream);
}
