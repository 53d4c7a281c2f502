// Rotary positions and the append of keys and values to a paged cache, one launch.
//
// A token's angles are the same for all its heads: a workgroup takes one token (or a share of its heads, where there
// are few tokens), computes cos and sin of every pair once into LDS, and streams the token's rows of q, k and v
// through registers, 8 values (16 bytes) to a thread and step.  The angle is a binary64 product taken in whole turns: position
// * freq / 2 pi minus its nearest integer, so a place of 10^6 keeps the accuracy of place 1 (in binary32 it would be off by
// 0.06 rad); the fraction then goes through a binary32 sincospi.  Bound by the traffic of q, k, v for prompts (2048 tokens of
// the 70B shapes: 84 MB in 14.7 to 15.2 us, 5.5 to 5.7 TB/s, against 4.8 of a large copy), by one launch for a token (3.5 us on the device, 8.0 a
// call from Python).
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

// How a head's pairs lie in 16-byte pieces: two neighbours in one piece; piece against piece half a rotation on; or (a half
// that is no multiple of 8) anyhow, the partner fetched by itself.
enum Layout { NEIGHBOURS, PIECES, ANYHOW };

// A thread's unit is two pieces of a head, which a pair of pieces turns together: what is asked for before any of it is used.
// (One piece at a time, the partners value by value: 27 us for 2048 tokens of the 70B shapes where this takes 15.)  Where
// partners are fetched value by value a unit is one piece, and those that turn come first, so that other wavefronts do not pass
// through it.
template <Layout LAYOUT>
__global__ __launch_bounds__(THREADS) void append_kernel(FqAppendArgs a, int per_head, int turning)
{
    __shared__ float cs[MAX_PAIRS], sn[MAX_PAIRS];
    const int t = blockIdx.x, tid = threadIdx.x;
    const bool bf16 = a.kv.bf16;
    const int half = a.rot >> 1, pieces = a.kv.dim >> 3;
    // units: the first `turning` of every head of q and k, the others of these heads, v
    const int qk = a.q_heads + a.kv.kv_heads, first = qk * turning, copied = qk * (per_head - turning);
    const int units = first + copied + a.kv.kv_heads * per_head;

    struct Unit {
        Eight x, y;
        const uint16_t *row;
        int kind, head, c, c2; // 0, 1, 2: q, k, v; its two pieces (c2 < 0: one)
    };
    auto ask = [&](int u) {
        Unit n;
        int i;
        if (LAYOUT == ANYHOW && u < first) {
            n.head = u / turning;
            i = u - n.head * turning;
        } else if (u < first + copied) {
            const int w = u - first, each = per_head - turning;
            n.head = w / each;
            i = w - n.head * each + turning;
        } else {
            const int w = u - first - copied;
            n.head = w / per_head;
            i = w - n.head * per_head;
            n.head += qk;
        }
        n.kind = n.head < a.q_heads ? 0 : n.head < qk ? 1 : 2;
        n.head -= n.kind == 0 ? 0 : n.kind == 1 ? a.q_heads : qk;
        if (LAYOUT == PIECES && i < half >> 3) { // (v likewise: any two pieces do)
            n.c = i;
            n.c2 = i + (half >> 3);
        } else {
            n.c = LAYOUT == ANYHOW ? i : 2 * i; // (rot is a multiple of 16 where pieces pair up: past the rotation they go on at rot / 8 = 2 half / 8)
            n.c2 = LAYOUT != ANYHOW && n.c + 1 < pieces ? n.c + 1 : -1;
        }
        n.row = (n.kind == 0 ? a.q + t * a.q_stride : n.kind == 1 ? a.k + t * a.k_stride : a.v + t * a.v_stride) + n.head * a.kv.dim;
        n.x = *(const Eight *)(n.row + 8 * n.c);
        if (n.c2 >= 0)
            n.y = *(const Eight *)(n.row + 8 * n.c2);
        return n;
    };
    const int u0 = blockIdx.y * THREADS + tid, stride = gridDim.y * THREADS;
    Unit now;
    if (u0 < units)
        now = ask(u0);

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

    auto turn = [&](Eight &x, int d, const uint16_t *row) { // pairs that one piece does not hold with another
        if (LAYOUT == NEIGHBOURS) {
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
    };
    for (int u = u0; u < units; u += stride) {
        Unit n = now;
        if (u + stride < units)
            now = ask(u + stride);
        if (n.kind != 0 && !stored)
            continue;
        if (n.kind != 2) {
            if (LAYOUT == PIECES) {
                if (n.c < half >> 3) {
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        const float c = cs[8 * n.c + i], s = sn[8 * n.c + i];
                        const float p = fq_to_float(n.x.v[i], bf16), q = fq_to_float(n.y.v[i], bf16);
                        n.x.v[i] = fq_from_float(p * c - q * s, bf16);
                        n.y.v[i] = fq_from_float(q * c + p * s, bf16);
                    }
                }
            } else if (LAYOUT == NEIGHBOURS || u < first) {
                turn(n.x, 8 * n.c, n.row);
                if (n.c2 >= 0)
                    turn(n.y, 8 * n.c2, n.row);
            }
        }
        uint16_t *to = n.kind == 0 ? a.q_out + t * a.q_out_stride + n.head * a.kv.dim
                                   : (n.kind == 2 ? a.kv.v : a.kv.k) + at + n.head * a.kv.head_stride;
        *(Eight *)(to + 8 * n.c) = n.x;
        if (n.c2 >= 0)
            *(Eight *)(to + 8 * n.c2) = n.y;
    }
}

} // namespace

hipError_t fq_launch_append(const FqAppendArgs &a, bool interleaved, hipStream_t stream)
{
    const bool anyhow = !interleaved && a.rot % 16 != 0;
    const int per_head = anyhow ? a.kv.dim / 8 : (a.kv.dim / 8 + 1) / 2;
    const int units = (a.q_heads + 2 * a.kv.kv_heads) * per_head;
    // a token's rows over as many workgroups as there are steps in them, where the tokens alone do not fill the chip
    const int steps = (units + THREADS - 1) / THREADS;
    const int room = (4 * fq_device_cus() + a.seqs.tokens - 1) / a.seqs.tokens;
    const dim3 grid(a.seqs.tokens, steps < room ? steps : room);
    if (interleaved)
        append_kernel<NEIGHBOURS><<<grid, THREADS, 0, stream>>>(a, per_head, 0);
    else if (!anyhow)
        append_kernel<PIECES><<<grid, THREADS, 0, stream>>>(a, per_head, 0);
    else
        append_kernel<ANYHOW><<<grid, THREADS, 0, stream>>>(a, per_head, (a.rot + 7) / 8);
    return hipGetLastError();
}
