// Log probabilities of given tokens, the entropy and the likeliest tokens of rows of logits.
//
// A workgroup takes a row: its largest logit, then the sums beside that one's weight of 1, then one alternative after the other.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/flexq.h"
#include "fq_internal.h"

namespace {

constexpr int THREADS = 256;

struct Best {
    float x;
    int i; // V: none
};

__device__ __forceinline__ Best better(Best a, Best b) { return b.x > a.x || (b.x == a.x && b.i < a.i) ? b : a; }

__device__ Best block_best(Best v, Best *s)
{
    for (int off = 32; off >= 1; off >>= 1)
        v = better(v, Best{__shfl_xor(v.x, off, 64), __shfl_xor(v.i, off, 64)});
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        s[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < THREADS / 64; w++)
        v = better(v, s[w]);
    return v;
}

__device__ double block_sum(double v, double *s)
{
    for (int off = 32; off >= 1; off >>= 1)
        v += __shfl_xor(v, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        s[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < THREADS / 64; w++)
        v += s[w];
    return v;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void logprobs_kernel(FqLogprobsArgs a)
{
    __shared__ Best s_best[THREADS / 64];
    __shared__ double s_sum[THREADS / 64];
    const int tid = threadIdx.x;
    for (long long r = blockIdx.x; r < a.R; r += gridDim.x) {
        const T *row = (const T *)a.logits + r * a.row_stride;
        auto at = [&](int i) {
            const float x = (float)row[i];
            return x == x ? x : -INFINITY;
        };
        Best top{-INFINITY, a.V};
        for (int i = tid; i < a.V; i += THREADS)
            top = better(top, Best{at(i), i});
        top = block_best(top, s_best);
        const bool none = top.x == -INFINITY, infinite = top.x == INFINITY;
        double rest = 0.0, turned = 0.0;
        for (int i = tid; i < a.V; i += THREADS) {
            const float x = at(i);
            if (i == top.i || none || (infinite && x < INFINITY))
                continue;
            const float t = infinite ? 0.0f : x - top.x, w = expf(t);
            rest += w;
            turned += w > 0.0f ? (double)w * t : 0.0;
        }
        rest = block_sum(rest, s_sum);
        turned = block_sum(turned, s_sum);
        const double log_sum = log1p(rest);
        auto logprob = [&](float x) {
            return none || x == -INFINITY || (infinite && x < INFINITY) ? -INFINITY
                   : infinite ? (float)-log_sum : (float)((double)x - (double)top.x - log_sum);
        };
        if (a.entropy && tid == 0)
            a.entropy[r] = (float)(log_sum - turned / (1.0 + rest));
        for (int j = tid; j < a.n_given; j += THREADS) {
            const int i = a.given[r * a.n_given + j];
            a.given_logprob[r * a.n_given + j] = i >= 0 && i < a.V ? logprob(at(i)) : -INFINITY;
        }
        Best last{INFINITY, -1};
        for (int j = 0; j < a.top_n; j++) {
            Best next{-INFINITY, a.V};
            for (int i = tid; i < a.V; i += THREADS) {
                const float x = at(i);
                if (x < last.x || (x == last.x && i > last.i))
                    next = better(next, Best{x, i});
            }
            last = block_best(next, s_best);
            if (tid == 0) {
                const bool found = last.x > -INFINITY && !(infinite && last.x < INFINITY);
                a.top_token[r * a.top_n + j] = found ? last.i : -1;
                a.top_logprob[r * a.top_n + j] = found ? logprob(last.x) : -INFINITY;
            }
        }
    }
}

} // namespace

size_t fq_logprobs_bytes(int, int) { return 256; }

hipError_t fq_launch_logprobs(const FqLogprobsArgs &a, bool half, void *, hipStream_t stream)
{
    const int grid = a.R < 65536 ? a.R : 65536;
    if (half)
        logprobs_kernel<_Float16><<<grid, THREADS, 0, stream>>>(a);
    else
        logprobs_kernel<float><<<grid, THREADS, 0, stream>>>(a);
    return hipGetLastError();
}
