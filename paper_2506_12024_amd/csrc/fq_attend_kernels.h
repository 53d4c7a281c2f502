// The attention kernels of one 16-bit type: a launch holds one or two pieces of work, few or many rows to a key head each.  A
// prefix that a batch shares and the sequences' own keys are one launch, so that neither waits for the other's last workgroup
// (48 sequences behind 8197 keys: 31 + 19 us as two launches, 41 as one, 37 with the tiles as they are now).
#ifndef FQ_ATTEND_KERNELS_H
#define FQ_ATTEND_KERNELS_H

#include "fq_attend_few.h"
#include "fq_attend_many.h"

namespace {

// The workgroup's place in a piece's own grid.
__device__ __forceinline__ dim3 place_in(const FqAttendWork &w, uint32_t at)
{
    const uint32_t x = at % w.blocks_x, yz = at / w.blocks_x;
    return dim3(x, yz % w.parts, yz / w.parts);
}

// RT0, RT1: tiles of 16 rows of the two pieces, 0 for many rows.
template <bool BF16, int DP, bool FULL, int RT0, int RT1>
__global__ __launch_bounds__(FQ_ATTEND_THREADS, DP <= 128 ? 2 : 1) void attend_kernel(FqAttendArgs a, FqAttendWork w0, FqAttendWork w1)
{
    const bool first = blockIdx.x < w0.blocks;
    const FqAttendWork &w = first ? w0 : w1;
    const dim3 at = place_in(w, first ? blockIdx.x : blockIdx.x - w0.blocks);
    if constexpr (RT0 == 0 && RT1 != 0) {
        union Lds {
            many::Lds<DP> m;
            few::Lds<DP, RT1> f;
            __device__ Lds() {}
        };
        __shared__ Lds lds;
        if (first)
            many::attend<BF16, DP, FULL>(a, w, at, lds.m);
        else
            few::attend<BF16, DP, FULL, RT1>(a, w, at, lds.f);
    } else if constexpr (RT0 == 0) {
        __shared__ many::Lds<DP> lds;
        many::attend<BF16, DP, FULL>(a, w, at, lds);
    } else {
        __shared__ few::Lds<DP, RT1> lds;
        few::attend<BF16, DP, FULL, RT1>(a, w, at, lds);
    }
}

template <bool BF16, int DP, bool FULL>
hipError_t launch(const FqAttendArgs &a, const FqAttendWork &w0, const FqAttendWork &w1, int rt0, int rt1, hipStream_t stream)
{
    const uint32_t grid = w0.blocks + w1.blocks;
    if (rt1 == 0)
        attend_kernel<BF16, DP, FULL, 0, 0><<<grid, FQ_ATTEND_THREADS, 0, stream>>>(a, w0, w1);
    else if (rt1 == 1 && rt0 == 0)
        attend_kernel<BF16, DP, FULL, 0, 1><<<grid, FQ_ATTEND_THREADS, 0, stream>>>(a, w0, w1);
    else if (rt1 == 1)
        attend_kernel<BF16, DP, FULL, 1, 1><<<grid, FQ_ATTEND_THREADS, 0, stream>>>(a, w0, w1);
    else if constexpr (DP <= 128) {
        if (rt0 == 0)
            attend_kernel<BF16, DP, FULL, 0, 2><<<grid, FQ_ATTEND_THREADS, 0, stream>>>(a, w0, w1);
        else
            attend_kernel<BF16, DP, FULL, 2, 2><<<grid, FQ_ATTEND_THREADS, 0, stream>>>(a, w0, w1);
    }
    return hipGetLastError();
}

} // namespace

#endif
