// Low-rank adapters of many requests beside a projection that they share: out = y + scale (x A^T) B^T, row by row.
//
// A workgroup takes a row: its wavefronts form x A^T, a rank each in turn, then every thread an output.
#include <hip/hip_runtime.h>

#include "../../include/flexq.h"
#include "fq_kv.h"

namespace {

constexpr int THREADS = 256;

struct alignas(16) Eight {
    uint16_t v[8];
};

__global__ __launch_bounds__(THREADS) void adapters_kernel(FqAdaptersArgs a)
{
    __shared__ float low[FQ_MAX_ADAPTER_RANK];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool bf16 = a.set.bf16;
    for (int m = blockIdx.x; m < a.M; m += gridDim.x) {
        const int slot = a.adapter[m];
        const bool served = slot >= 0 && slot < a.set.slots;
        int rank = 0;
        if (served)
            rank = a.set.ranks ? min(max(a.set.ranks[slot], 0), a.set.rank) : a.set.rank;
        const uint16_t *y = a.y + m * a.y_stride;
        uint16_t *out = a.out + m * a.out_stride;
        if (rank == 0) {
            for (int n = tid; n < a.set.N; n += THREADS)
                out[n] = y[n];
            continue;
        }
        const uint16_t *x = a.x + m * a.x_stride;
        const uint16_t *am = a.set.a + slot * a.set.a_stride, *bm = a.set.b + slot * a.set.b_stride;
        for (int r = wave; r < rank; r += THREADS / 64) {
            float sum = 0.0f;
            for (int k = 8 * lane; k < a.set.K; k += 512) {
                const Eight p = *(const Eight *)(x + k), q = *(const Eight *)(am + (size_t)r * a.set.K + k);
                for (int i = 0; i < 8; i++)
                    sum += fq_to_float(p.v[i], bf16) * fq_to_float(q.v[i], bf16);
            }
            for (int off = 32; off >= 1; off >>= 1)
                sum += __shfl_xor(sum, off, 64);
            if (lane == 0)
                low[r] = sum;
        }
        __syncthreads();
        const float scale = a.set.scales ? a.set.scales[slot] : 1.0f;
        for (int n = tid; n < a.set.N; n += THREADS) {
            const uint16_t *b = bm + (size_t)n * a.set.rank;
            float sum = 0.0f;
            for (int r = 0; r < rank; r++)
                sum += low[r] * fq_to_float(b[r], bf16);
            out[n] = fq_from_float(fq_to_float(y[n], bf16) + scale * sum, bf16);
        }
        __syncthreads();
    }
}

} // namespace

size_t fq_adapters_bytes(const FqAdaptersView &, int) { return 256; }

hipError_t fq_launch_adapters(const FqAdaptersArgs &a, void *, hipStream_t stream)
{
    adapters_kernel<<<a.M < 65536 ? a.M : 65536, THREADS, 0, stream>>>(a);
    return hipGetLastError();
}
