// Norms of the heads of queries and keys, rotary positions and the append to a paged cache, one launch.
//
//   y_d = x_d (w_d + offset) / sqrt(mean_i x_i^2 + eps),  then pairs turn as in fq_append.hip,  one rounding at the end
//
// A head lies in the registers of a group of lanes, two 16-byte pieces to a lane: those of a pair of pieces that turn together where a half rotation is
// whole pieces, else neighbours.  Its sum of squares is a sum over the group's lanes, and a head is read once.  Only where pairs lie anyhow
// (a half rotation that is no multiple of 8) the part of the normed head that turns goes through LDS.  A workgroup takes a token, or a share of
// its heads where there are few tokens; cos and sin of its angles, computed as fq_append.hip does, are in LDS.
//
// Bound by the traffic of q, k, v for prompts (2048 tokens of 64 / 8 heads of 128: 84 MB in 16.5 us, 5.1 TB/s, against 5.2 of a large copy; a wavefront to a
// head and its values one by one 65 us), by launch and marshalling for a token (3.3 us on the device, 8.4 a call from Python).  Heads of 80 leave three of
// eight lanes idle: 9 chunks, 32 heads, 20 of 80 turned, 45 MB in 12.5 us, 3.6 TB/s (with each turning value's partner read from LDS by the lane that has
// the value, instead of a pair to a lane, 17.2).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../include/flexq.h"
#include "fq_kv.h"

namespace {

constexpr int THREADS = 256;

struct alignas(16) Eight {
    uint16_t v[8];
};

// The sequence that owns row t: the last b with q_start[b] <= t, or -1 (64 starts at a time).
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

// The sum over a group of 4, 8 or 16 lanes, in all of them.
template <int GROUP>
__device__ __forceinline__ float group_sum(float x)
{
    auto step = [](float v, auto ctrl) {
        const int t = __builtin_bit_cast(int, v);
        return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(t, t, decltype(ctrl)::value, 0xf, 0xf, false));
    };
    x = step(x, std::integral_constant<int, 0xb1>()); // quad_perm 1, 0, 3, 2
    x = step(x, std::integral_constant<int, 0x4e>()); // quad_perm 2, 3, 0, 1
    if (GROUP >= 8)
        x = step(x, std::integral_constant<int, 0x141>()); // half a row mirrored
    if (GROUP >= 16)
        x = step(x, std::integral_constant<int, 0x140>()); // a row mirrored
    return x;
}

// What a group's lanes hand each other through LDS: a wavefront's operations there are in order, the compiler has to keep them so.
__device__ __forceinline__ void own_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

enum Layout { NEIGHBOURS, PIECES, ANYHOW };

// GROUP lanes to a head, a power of two, 2 GROUP pieces at least.
template <Layout LAYOUT, int GROUP, bool BF16>
__global__ __launch_bounds__(THREADS) void append_normed_kernel(FqAppendArgs a, FqNormArgs norm)
{
    __shared__ float cs[FQ_MAX_HEAD_DIM / 2], sn[FQ_MAX_HEAD_DIM / 2];
    __shared__ float normed[LAYOUT == ANYHOW ? THREADS * 16 : 1];
    const int t = blockIdx.x, tid = threadIdx.x;
    const int half = a.rot >> 1, dim = a.kv.dim, pieces = dim >> 3, qk = a.q_heads + a.kv.kv_heads, heads = qk + a.kv.kv_heads;
    const int i = tid & (GROUP - 1), c = LAYOUT == PIECES && i < half >> 3 ? i : 2 * i;
    const int c2 = LAYOUT == PIECES && i < half >> 3 ? i + (half >> 3) : 2 * i + 1; // (past the rotation pieces go on at rot / 8 = 2 half / 8)
    const bool has = c < pieces, has2 = c2 < pieces;
    struct Head {
        Eight x, y, w, w2;
        int kind, own; // 0, 1, 2: q, k, v
    };
    auto ask = [&](int h) {
        Head n;
        n.kind = h < a.q_heads ? 0 : h < qk ? 1 : 2;
        n.own = h - (n.kind == 0 ? 0 : n.kind == 1 ? a.q_heads : qk);
        const uint16_t *row = (n.kind == 0 ? a.q + t * a.q_stride : n.kind == 1 ? a.k + t * a.k_stride : a.v + t * a.v_stride) + n.own * dim;
        const uint16_t *w = (n.kind == 0 ? norm.q_weight : norm.k_weight) + n.own * norm.weight_stride;
        n.x = n.y = n.w = n.w2 = Eight{};
        if (has) {
            n.x = *(const Eight *)(row + 8 * c);
            if (n.kind != 2)
                n.w = *(const Eight *)(w + 8 * c);
        }
        if (has2) {
            n.y = *(const Eight *)(row + 8 * c2);
            if (n.kind != 2)
                n.w2 = *(const Eight *)(w + 8 * c2);
        }
        return n;
    };
    const int h0 = blockIdx.y * (THREADS / GROUP) + tid / GROUP, stride = gridDim.y * (THREADS / GROUP);
    Head now;
    if (h0 < heads)
        now = ask(h0);

    const int b = owner(a.seqs, t);
    if (b < 0)
        return;
    const FqSeq seq = fq_seq(a.seqs, a.kv.page_shift, b);
    if (t < seq.q0 || t >= seq.q0 + seq.n)
        return; // nobody's row
    const int place = seq.len - seq.n + (t - seq.q0);
    int page = -1;
    if (place >= 0)
        page = a.seqs.table[(long long)b * a.seqs.table_width + (place >> a.kv.page_shift)];
    for (int j = tid; j < half; j += THREADS) {
        const int pos = a.positions ? a.positions[t] : a.seqs.prefix_len + place;
        double turns = (double)pos * (a.freqs[j] * 0.15915494309189533577);
        turns -= rint(turns);
        float s, k;
        sincospif(2.0f * (float)turns, &s, &k);
        cs[j] = k * a.amplitude;
        sn[j] = s * a.amplitude;
    }
    const bool stored = page >= 0 && page < a.kv.n_pages;
    const long long at = stored ? page * a.kv.page_stride + (place & ((1 << a.kv.page_shift) - 1)) * a.kv.token_stride : 0;
    __syncthreads();

    // (a group's lanes take part in its sums together: heads past the last one are computed on and not written)
    const int rounds = (heads + stride - 1) / stride;
    for (int round = 0; round < rounds; round++) {
        const int h = h0 + round * stride;
        Head n = now;
        if (h + stride < heads)
            now = ask(h + stride);
        const bool live = h < heads && (n.kind == 0 || stored);
        if (live && n.kind != 2) {
            float x[8], y[8], sum = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                x[e] = fq_to_float(n.x.v[e], BF16);
                y[e] = fq_to_float(n.y.v[e], BF16);
            }
            // (bfloat16 squares may leave binary32: then the head is taken 2^-70 or 2^70 times as large)
            auto mean_of = [&](float f) {
                float own = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; e++)
                    own += (x[e] * f) * (x[e] * f) + (y[e] * f) * (y[e] * f);
                return group_sum<GROUP>(own) / dim + norm.eps * f * f;
            };
            float f = 1.0f;
            sum = mean_of(f);
            if (BF16 && !(sum >= 0x1p-100f && sum < 0x1p100f)) {
                f = sum > 1.0f ? 0x1p-70f : 0x1p70f;
                sum = mean_of(f);
            }
            const float inv = 1.0f / sqrtf(sum);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                x[e] = x[e] * f * inv * (fq_to_float(n.w.v[e], BF16) + norm.offset);
                y[e] = y[e] * f * inv * (fq_to_float(n.w2.v[e], BF16) + norm.offset);
            }
            if (LAYOUT == PIECES) {
                if (c < half >> 3) {
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const float k = cs[8 * c + e], s = sn[8 * c + e], p = x[e], q = y[e];
                        x[e] = p * k - q * s;
                        y[e] = q * k + p * s;
                    }
                }
            } else if (LAYOUT == NEIGHBOURS) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    if (8 * c + e < a.rot) {
                        const float k = cs[4 * c + e / 2], s = sn[4 * c + e / 2], p = x[e], q = x[e + 1];
                        x[e] = p * k - q * s;
                        x[e + 1] = q * k + p * s;
                    }
                    if (8 * c2 + e < a.rot) {
                        const float k = cs[4 * c2 + e / 2], s = sn[4 * c2 + e / 2], p = y[e], q = y[e + 1];
                        y[e] = p * k - q * s;
                        y[e + 1] = q * k + p * s;
                    }
                }
            } else { // the part that turns through LDS, its pairs over the group's lanes
                float *head = normed + tid / GROUP * (16 * GROUP);
                const bool mine = 16 * i < a.rot;
                if (mine) {
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        head[16 * i + e] = x[e];
                        head[16 * i + 8 + e] = y[e];
                    }
                }
                own_fence();
                for (int pair = i; pair < half; pair += GROUP) {
                    const float k = cs[pair], s = sn[pair], p = head[pair], q = head[pair + half];
                    head[pair] = p * k - q * s;
                    head[pair + half] = q * k + p * s;
                }
                own_fence();
                if (mine) {
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        x[e] = head[16 * i + e];
                        y[e] = head[16 * i + 8 + e];
                    }
                }
                own_fence();
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {
                n.x.v[e] = fq_from_float(x[e], BF16);
                n.y.v[e] = fq_from_float(y[e], BF16);
            }
        }
        if (live) {
            uint16_t *to = n.kind == 0 ? a.q_out + t * a.q_out_stride + n.own * dim
                                       : (n.kind == 2 ? a.kv.v : a.kv.k) + at + n.own * a.kv.head_stride;
            if (has)
                *(Eight *)(to + 8 * c) = n.x;
            if (has2)
                *(Eight *)(to + 8 * c2) = n.y;
        }
    }
}

template <Layout LAYOUT, bool BF16>
void launch(const FqAppendArgs &a, const FqNormArgs &n, hipStream_t stream)
{
    const int lanes = (a.kv.dim / 8 + 1) / 2, group = lanes <= 4 ? 4 : lanes <= 8 ? 8 : 16;
    const int heads = a.q_heads + 2 * a.kv.kv_heads;
    // a token's heads over as many workgroups as there are rounds in them, where the tokens alone do not fill the chip
    const int rounds = (heads * group + THREADS - 1) / THREADS;
    const int room = (4 * fq_device_cus() + a.seqs.tokens - 1) / a.seqs.tokens;
    const dim3 grid(a.seqs.tokens, rounds < room ? rounds : room);
    if (group == 4)
        append_normed_kernel<LAYOUT, 4, BF16><<<grid, THREADS, 0, stream>>>(a, n);
    else if (group == 8)
        append_normed_kernel<LAYOUT, 8, BF16><<<grid, THREADS, 0, stream>>>(a, n);
    else
        append_normed_kernel<LAYOUT, 16, BF16><<<grid, THREADS, 0, stream>>>(a, n);
}

template <bool BF16>
void launch(const FqAppendArgs &a, const FqNormArgs &n, bool interleaved, hipStream_t stream)
{
    if (interleaved)
        launch<NEIGHBOURS, BF16>(a, n, stream);
    else if (a.rot % 16 == 0)
        launch<PIECES, BF16>(a, n, stream);
    else
        launch<ANYHOW, BF16>(a, n, stream);
}

} // namespace

hipError_t fq_launch_append_normed(const FqAppendArgs &a, const FqNormArgs &n, bool interleaved, hipStream_t stream)
{
    if (a.kv.bf16)
        launch<true>(a, n, interleaved, stream);
    else
        launch<false>(a, n, interleaved, stream);
    return hipGetLastError();
}
