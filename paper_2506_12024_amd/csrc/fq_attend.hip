// Attention of new tokens over a paged cache.
#include <hip/hip_runtime.h>

#include "fq_kv.h"

namespace {

constexpr int THREADS = 256;

__device__ __forceinline__ float wg_reduce(float v, bool largest, float *buf)
{
    for (int o = 32; o; o >>= 1) {
        const float w = __shfl_xor(v, o);
        v = largest ? fmaxf(v, w) : v + w;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        buf[threadIdx.x >> 6] = v;
    __syncthreads();
    return largest ? fmaxf(fmaxf(buf[0], buf[1]), fmaxf(buf[2], buf[3])) : buf[0] + buf[1] + buf[2] + buf[3];
}

// One workgroup to a new token and query head: 256 keys at a time, a thread to a key for the scores, a thread to a
// dimension for the values.
__global__ __launch_bounds__(THREADS) void attend_row_kernel(FqAttendArgs a)
{
    __shared__ float q[256], p[THREADS], buf[4];
    __shared__ long long at[THREADS];
    const int b = blockIdx.z, j = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
    const FqSeq seq = fq_seq(a.seqs, a.kv.page_shift, b);
    if (j >= seq.n)
        return;
    const int kh = h / (a.q_heads / a.kv.kv_heads), dim = a.kv.dim;
    const bool bf16 = a.kv.bf16;
    if (tid < dim)
        q[tid] = fq_to_float(a.q[(seq.q0 + j) * a.q_stride + h * dim + tid], bf16);
    const int seen = max(min(seq.len - seq.n + j + 1, a.max_kv), 0), all = a.seqs.prefix_len + seen;
    float m = -INFINITY, l = 0.f, acc = 0.f;
    for (int k0 = 0; k0 < all; k0 += THREADS) {
        __syncthreads();
        const int key = k0 + tid;
        float s = -INFINITY;
        long long from = -1;
        if (key < all) {
            const bool own = key >= a.seqs.prefix_len;
            const int place = own ? key - a.seqs.prefix_len : key;
            const int page = own ? a.seqs.table[(long long)b * a.seqs.table_width + (place >> a.kv.page_shift)]
                                 : a.seqs.prefix_table[place >> a.kv.page_shift];
            if (page >= 0 && page < a.kv.n_pages) {
                from = page * a.kv.page_stride + kh * a.kv.head_stride + (place & ((1 << a.kv.page_shift) - 1)) * a.kv.token_stride;
                s = 0.f;
                for (int d = 0; d < dim; d++)
                    s += q[d] * fq_to_float(a.kv.k[from + d], bf16);
                s *= a.scale;
            }
        }
        const float top = fmaxf(m, wg_reduce(s, true, buf));
        const float fall = top == -INFINITY ? 1.f : expf(m - top);
        p[tid] = from < 0 ? 0.f : expf(s - top);
        at[tid] = from;
        l = l * fall + wg_reduce(p[tid], false, buf);
        acc *= fall;
        m = top;
        if (tid < dim)
            for (int i = 0; i < THREADS; i++)
                if (at[i] >= 0)
                    acc += p[i] * fq_to_float(a.kv.v[at[i] + tid], bf16);
    }
    const long long row = seq.q0 + j;
    if (tid < dim)
        a.out[row * a.out_stride + h * dim + tid] = fq_from_float(l > 0.f || l != l ? acc / l : 0.f, bf16);
    if (tid == 0 && a.lse)
        a.lse[row * a.q_heads + h] = l == 0.f ? -INFINITY : m + logf(l);
}

} // namespace

size_t fq_attend_bytes(const FqAttendArgs &, int) { return 256; }

hipError_t fq_launch_attend(const FqAttendArgs &a, void *, hipStream_t stream)
{
    attend_row_kernel<<<dim3(a.max_q, a.q_heads, a.seqs.seqs), THREADS, 0, stream>>>(a);
    return hipGetLastError();
}
