// Drawing the next token from a row of logits: temperature, top-k, top-p, min-p and a given random number.
#include <hip/hip_runtime.h>

#include "fq_internal.h"

namespace {

constexpr int THREADS = 1024;
constexpr int WAVES = THREADS / 64;
typedef unsigned long long u64;

// Binary32 values as unsigned numbers in the same order; -0 is 0, a NaN is -inf.
__device__ __forceinline__ float clean(float f) { return f != f ? -INFINITY : f + 0.0f; }
__device__ __forceinline__ uint32_t ordered(float f)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k)
{
    return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// Where a logit stands: larger is earlier, of equal ones the smaller index.
__device__ __forceinline__ u64 standing(float f, int i) { return ((u64)ordered(f) << 32) | (0xffffffffu - (uint32_t)i); }

// floor(x * w) for x in [0, 1) with 24 bits of precision, and whether anything was cut off
__device__ __forceinline__ u64 share(float x, u64 w, bool &rest)
{
    const u64 f = (u64)((double)x * 18446744073709551616.0);
    rest = f * w != 0;
    return __umul64hi(f, w);
}

struct Weigh {
    float top;
    double inv_t; // 1 / temperature
    double unit;
    __device__ __forceinline__ u64 operator()(float l) const
    {
        if (l == -INFINITY)
            return 0;
        if (l == top)
            return (u64)unit;
        return (u64)rint(exp(((double)l - (double)top) * inv_t) * unit);
    }
};

__device__ __forceinline__ u64 wg_sum(u64 v, u64 *buf)
{
    for (int o = 32; o; o >>= 1)
        v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        buf[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 s = 0;
    for (int i = 0; i < WAVES; i++)
        s += buf[i];
    return s;
}

// Of the entries whose key is known to f(i, key, weight) (weight 0: not among them), taken from the largest key down:
// the key at which the running sum of weights reaches `target` (1 <= target <= the sum).  Eight bits at a time.
template <int BITS, class F>
__device__ u64 reach(const F &f, int V, u64 target, u64 *hist, u64 *word)
{
    u64 found = 0;
    for (int shift = BITS - 8; shift >= 0; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256)
            hist[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < V; i += THREADS) {
            u64 key, w;
            f(i, key, w);
            if (w && (shift == BITS - 8 || (key >> (shift + 8)) == (found >> (shift + 8))))
                atomicAdd(&hist[(key >> shift) & 255], w);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int d = 255;
            while (d > 0 && hist[d] < target)
                target -= hist[d--];
            word[0] = d;
            word[1] = target;
        }
        __syncthreads();
        found |= word[0] << shift;
        target = word[1];
    }
    return found;
}

template <class T>
__global__ __launch_bounds__(THREADS) void sample_row_kernel(FqSampleArgs a, double unit)
{
    __shared__ u64 hist[256], word[2], buf[WAVES];
    const int r = blockIdx.x, V = a.V, tid = threadIdx.x;
    const T *x = (const T *)a.logits + r * a.row_stride;
    u64 first = 0;
    for (int i = tid; i < V; i += THREADS) {
        const u64 s = standing(clean((float)x[i]), i);
        first = s > first ? s : first;
    }
    for (int o = 32; o; o >>= 1) {
        const u64 s = __shfl_xor(first, o);
        first = s > first ? s : first;
    }
    if ((tid & 63) == 0)
        buf[tid >> 6] = first;
    __syncthreads();
    for (int i = 0; i < WAVES; i++)
        first = buf[i] > first ? buf[i] : first;
    __syncthreads();
    const float top = unordered((uint32_t)(first >> 32));
    const int best = (int)(0xffffffffu - (uint32_t)first);
    const float temperature = a.temperature ? a.temperature[r] : 1.0f;
    if (top == -INFINITY || !(temperature > 0.0f)) {
        if (tid == 0) {
            a.token[r] = top == -INFINITY ? -1 : best;
            if (a.prob)
                a.prob[r] = top == -INFINITY ? 0.0f : 1.0f;
        }
        return;
    }
    const Weigh weigh{top, top == INFINITY ? (double)INFINITY : 1.0 / (double)temperature, unit};
    u64 cut = 0; // entries whose standing is below it are out
    const int k = a.top_k ? a.top_k[r] : 0;
    if (k > 0 && k < V)
        cut = reach<64>([&](int i, u64 &key, u64 &w) { key = standing(clean((float)x[i]), i); w = 1; }, V, k, hist, word);
    auto weight = [&](int i, u64 &key) {
        const float l = clean((float)x[i]);
        key = standing(l, i);
        return key >= cut ? weigh(l) : 0;
    };
    const float p = a.top_p ? a.top_p[r] : 1.0f;
    if (!(p >= 1.0f)) {
        u64 sum = 0, key;
        for (int i = tid; i < V; i += THREADS)
            sum += weight(i, key);
        sum = wg_sum(sum, buf);
        bool rest = false;
        u64 target = p > 0.0f ? share(p, sum, rest) : 0;
        target += rest || target == 0;
        const u64 at = reach<64>([&](int i, u64 &s, u64 &w) { w = weight(i, s); }, V, target, hist, word);
        cut = at > cut ? at : cut;
    }
    const float m = a.min_p ? a.min_p[r] : 0.0f;
    const double least = m > 0.0f ? (double)fminf(m, 1.0f) : 0.0;
    auto kept = [&](int i) -> u64 {
        const float l = clean((float)x[i]);
        if (standing(l, i) < cut || l == -INFINITY)
            return 0;
        if (least > 0.0 && l != top && !(exp(((double)l - (double)top) * weigh.inv_t) >= least))
            return 0;
        return weigh(l);
    };
    u64 sum = 0;
    for (int i = tid; i < V; i += THREADS)
        sum += kept(i);
    sum = wg_sum(sum, buf);
    const float u = a.u[r];
    bool rest;
    u64 target = u >= 1.0f ? sum - 1 : u > 0.0f ? share(u, sum, rest) : 0;
    const int token = (int)(0xffffffffu - (uint32_t)reach<32>(
        [&](int i, u64 &key, u64 &w) { key = 0xffffffffu - (uint32_t)i; w = kept(i); }, V, target + 1, hist, word));
    if (tid == 0) {
        a.token[r] = token;
        if (a.prob)
            a.prob[r] = (float)((double)kept(token) / (double)sum);
    }
}

} // namespace

size_t fq_sample_bytes(int, int) { return 256; }

hipError_t fq_launch_sample(const FqSampleArgs &a, bool half, void *, hipStream_t stream)
{
    const int log_v = a.V > 1 ? 32 - __builtin_clz((unsigned)a.V - 1) : 0;
    const double unit = (double)(1ULL << (62 - log_v));
    if (half)
        sample_row_kernel<_Float16><<<a.R, THREADS, 0, stream>>>(a, unit);
    else
        sample_row_kernel<float><<<a.R, THREADS, 0, stream>>>(a, unit);
    return hipGetLastError();
}
