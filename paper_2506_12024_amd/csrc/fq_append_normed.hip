// Norms of the heads of queries and keys, rotary positions and the append to a paged cache, one launch.
//
// A workgroup takes a token, a wavefront a head: its sum of squares, then its values in binary32 through LDS, where a pair's partner
// is found wherever it lies.
#include <hip/hip_runtime.h>

#include "../../include/flexq.h"
#include "fq_kv.h"

namespace {

constexpr int THREADS = 256;

__global__ __launch_bounds__(THREADS) void append_normed_kernel(FqAppendArgs a, FqNormArgs norm, int interleaved)
{
    __shared__ float cs[FQ_MAX_HEAD_DIM / 2], sn[FQ_MAX_HEAD_DIM / 2], head[THREADS / 64][FQ_MAX_HEAD_DIM];
    const int t = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const bool bf16 = a.kv.bf16;
    const int half = a.rot >> 1, dim = a.kv.dim, qk = a.q_heads + a.kv.kv_heads;
    int b = -1;
    for (int i = 0; i < a.seqs.seqs && a.seqs.q_start[i] <= t; i++)
        b = i;
    if (b < 0)
        return;
    const FqSeq seq = fq_seq(a.seqs, a.kv.page_shift, b);
    if (t < seq.q0 || t >= seq.q0 + seq.n)
        return; // nobody's row
    const int place = seq.len - seq.n + (t - seq.q0);
    int page = -1;
    if (place >= 0)
        page = a.seqs.table[(long long)b * a.seqs.table_width + (place >> a.kv.page_shift)];
    for (int i = tid; i < half; i += THREADS) {
        const int pos = a.positions ? a.positions[t] : a.seqs.prefix_len + place;
        double turns = (double)pos * (a.freqs[i] * 0.15915494309189533577);
        turns -= rint(turns);
        float s, c;
        sincospif(2.0f * (float)turns, &s, &c);
        cs[i] = c * a.amplitude;
        sn[i] = s * a.amplitude;
    }
    const bool stored = page >= 0 && page < a.kv.n_pages;
    const long long at = stored ? page * a.kv.page_stride + (place & ((1 << a.kv.page_shift) - 1)) * a.kv.token_stride : 0;
    __syncthreads();
    for (int h = wave; h < qk + a.kv.kv_heads; h += THREADS / 64) {
        const int kind = h < a.q_heads ? 0 : h < qk ? 1 : 2, own = h - (kind == 0 ? 0 : kind == 1 ? a.q_heads : qk);
        if (kind != 0 && !stored)
            continue;
        const uint16_t *row = (kind == 0 ? a.q + t * a.q_stride : kind == 1 ? a.k + t * a.k_stride : a.v + t * a.v_stride) + own * dim;
        uint16_t *to = kind == 0 ? a.q_out + t * a.q_out_stride + own * dim : (kind == 2 ? a.kv.v : a.kv.k) + at + own * a.kv.head_stride;
        if (kind == 2) {
            for (int d = lane; d < dim; d += 64)
                to[d] = row[d];
            continue;
        }
        // (bfloat16 squares may leave binary32: then the head is taken 2^-70 or 2^70 times as large)
        float f = 1.0f, mean;
        for (int again = 0; again < 2; again++) {
            float sum = 0.0f;
            for (int d = lane; d < dim; d += 64) {
                const float v = fq_to_float(row[d], bf16) * f;
                sum += v * v;
            }
            for (int off = 32; off >= 1; off >>= 1)
                sum += __shfl_xor(sum, off, 64);
            mean = sum / dim + norm.eps * f * f;
            if (again || (mean >= 0x1p-100f && mean < 0x1p100f))
                break;
            f = mean > 1.0f ? 0x1p-70f : 0x1p70f;
        }
        const float inv = 1.0f / sqrtf(mean);
        const uint16_t *w = (kind == 0 ? norm.q_weight : norm.k_weight) + own * norm.weight_stride;
        for (int d = lane; d < dim; d += 64)
            head[wave][d] = fq_to_float(row[d], bf16) * f * inv * (fq_to_float(w[d], bf16) + norm.offset);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        for (int d = lane; d < dim; d += 64) {
            float v = head[wave][d];
            if (d < a.rot) {
                const bool low = interleaved ? (d & 1) == 0 : d < half;
                const int pair = interleaved ? d >> 1 : low ? d : d - half;
                const float p = head[wave][interleaved ? d ^ 1 : low ? d + half : d - half];
                v = low ? v * cs[pair] - p * sn[pair] : v * cs[pair] + p * sn[pair];
            }
            to[d] = fq_from_float(v, bf16);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

} // namespace

hipError_t fq_launch_append_normed(const FqAppendArgs &a, const FqNormArgs &n, bool interleaved, hipStream_t stream)
{
    append_normed_kernel<<<a.seqs.tokens, THREADS, 0, stream>>>(a, n, interleaved);
    return hipGetLastError();
}
