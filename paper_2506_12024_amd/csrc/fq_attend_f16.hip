// Attention over binary16.
#include "fq_attend_kernels.h"

hipError_t fq_launch_attend_f16(const FqAttendArgs &a, const FqAttendWork &w0, const FqAttendWork &w1, int rt0, int rt1, hipStream_t stream)
{
    const int dim = a.kv.dim;
    return dim == 64    ? launch<false, 64, true>(a, w0, w1, rt0, rt1, stream)
           : dim == 128 ? launch<false, 128, true>(a, w0, w1, rt0, rt1, stream)
           : dim <= 96  ? launch<false, 96, false>(a, w0, w1, rt0, rt1, stream)
                        : launch<false, 256, false>(a, w0, w1, rt0, rt1, stream);
}
