// Rotary positions and the append of keys and values to a paged cache, one launch.
//
// A token's angles are the same for all its heads: a workgroup takes one token (or a share of its heads, where there
// are few tokens), computes cos and sin of every pair once into LDS, and streams the token's rows of q, k and v
// through registers, 8 values (16 bytes) to a thread and step.  The angle is a binary64 product taken in whole turns: position
// * freq / 2 pi minus its nearest integer, so a place of 10^6 keeps the accuracy of place 1 (in binary32 it would be off by
// 0.06 rad); the fraction then goes through a binary32 sincospi.  Bound by the traffic of q, k, v for prompts, by one launch
// for a token.
#include <hip/hip_runtime.h>

#include "fq_kv.h"

namespace {

constexpr int THREADS = 256;
constexpr int MAX_PAIRS = 128; // FQ_MAX_HEAD_DIM / 2

// The sequence that owns row t: the last b with q_start[b] <= t (empty sequences share a start with the next), or
// -1.  64 starts at a time, one load of latency for up to 64 sequences.
__device__ __forceinline__ int owner(const FqSeqsView &s, int t)
{
    const int lane = threadIdx.x & 63;
    int begun = 0;
    for (int b0 = 0; b0 < s.seqs; b0 += 64) {
        const bool in = b0 + lane < s.seqs && s.q_start[b0 + lane] <= t;
        const int n = __popcll(__ballot(in));
        begun += n;
        if (n < 64)
            break;
    }
    return begun - 1;
}

struct alignas(16) Eight {
    uint16_t v[8];
};

template <bool INTERLEAVED>
__global__ __launch_bounds__(THREADS) void append_kernel(FqAppendArgs a)
{
    __shared__ float cs[MAX_PAIRS], sn[MAX_PAIRS];
    const int t = blockIdx.x, tid = threadIdx.x;
    const bool bf16 = a.kv.bf16;
    const int b = owner(a.seqs, t);
    if (b < 0)
        return;
    const FqSeq seq = fq_seq(a.seqs, a.kv.page_shift, b);
    if (t < seq.q0 || t >= seq.q0 + seq.n)
        return; // nobody's row
    const int place = seq.len - seq.n + (t - seq.q0);
    const int half = a.rot >> 1;
    for (int i = tid; i < half; i += THREADS) {
        const int pos = a.positions ? a.positions[t] : a.seqs.prefix_len + place;
        double turns = (double)pos * (a.freqs[i] * 0.15915494309189533577);
        turns -= rint(turns);
        float s, c;
        sincospif(2.0f * (float)turns, &s, &c);
        cs[i] = c * a.amplitude;
        sn[i] = s * a.amplitude;
    }
    int page = -1;
    if (place >= 0)
        page = a.seqs.table[(long long)b * a.seqs.table_width + (place >> a.kv.page_shift)];
    const bool stored = page >= 0 && page < a.kv.n_pages;
    const long long at = stored ? page * a.kv.page_stride + (place & ((1 << a.kv.page_shift) - 1)) * a.kv.token_stride : 0;
    __syncthreads();
    const int per_head = a.kv.dim >> 3;
    const int q_units = a.q_heads * per_head, kv_units = a.kv.kv_heads * per_head;
    const int units = q_units + 2 * kv_units;
    for (int u = blockIdx.y * THREADS + tid; u < units; u += gridDim.y * THREADS) {
        const bool is_q = u < q_units, is_v = u >= q_units + kv_units;
        const int w = is_q ? u : u - q_units - (is_v ? kv_units : 0);
        const int head = w / per_head, d = (w - head * per_head) << 3;
        if (!is_q && !stored)
            continue;
        const uint16_t *row = (is_q ? a.q + t * a.q_stride : is_v ? a.v + t * a.v_stride : a.k + t * a.k_stride) + head * a.kv.dim;
        uint16_t *to = is_q ? a.q_out + t * a.q_out_stride + head * a.kv.dim + d
                            : (is_v ? a.kv.v : a.kv.k) + at + head * a.kv.head_stride + d;
        Eight x = *(const Eight *)(row + d);
        if (!is_v && d < a.rot) {
            if (INTERLEAVED) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    if (d + i < a.rot) {
                        const float c = cs[(d + i) >> 1], s = sn[(d + i) >> 1];
                        const float p = fq_to_float(x.v[i], bf16), q = fq_to_float(x.v[i + 1], bf16);
                        x.v[i] = fq_from_float(p * c - q * s, bf16);
                        x.v[i + 1] = fq_from_float(q * c + p * s, bf16);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const int e = d + i;
                    if (e < a.rot) {
                        const bool low = e < half;
                        const int pair = low ? e : e - half;
                        const float c = cs[pair], s = sn[pair];
                        const float p = fq_to_float(x.v[i], bf16), q = fq_to_float(row[low ? e + half : pair], bf16);
                        x.v[i] = fq_from_float(low ? p * c - q * s : p * c + q * s, bf16);
                    }
                }
            }
        }
        *(Eight *)to = x;
    }
}

} // namespace

hipError_t fq_launch_append(const FqAppendArgs &a, bool interleaved, hipStream_t stream)
{
    const int units = (a.q_heads + 2 * a.kv.kv_heads) * (a.kv.dim / 8);
    // a token's rows over as many workgroups as there are steps in them, where the tokens alone do not fill the chip
    const int steps = (units + THREADS - 1) / THREADS;
    const int room = (4 * fq_device_cus() + a.seqs.tokens - 1) / a.seqs.tokens;
    const dim3 grid(a.seqs.tokens, steps < room ? steps : room);
    if (interleaved)
        append_kernel<true><<<grid, THREADS, 0, stream>>>(a);
    else
        append_kernel<false><<<grid, THREADS, 0, stream>>>(a);
    return hipGetLastError();
}
