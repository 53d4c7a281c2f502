// Attention of many rows to a sequence and key head: prompts, chunks of them, and a prefix that a batch shares.
//
// Bound by the matrix cores and by the exponentials between the two products.  Four wavefronts take 32 rows each and share
// tiles of 64 keys in LDS, two of them in turn: while one is computed the next one's rows are in flight to registers, and go
// to the other tile before the one barrier of a step.
#ifndef FQ_ATTEND_MANY_H
#define FQ_ATTEND_MANY_H

#include "fq_attend.h"

namespace many {

constexpr int KEYS = 64;

// 16-byte pieces to a key in LDS, and where piece c of key r goes: 16 keys of one piece (the reads of K), 4 keys of four pieces
// in a row (the writes, and the transposed reads of V) fall on different bank groups.
template <int DP>
struct Place {
    static constexpr int PITCH = DP <= 64 ? 8 : DP <= 128 ? 16 : 32;
    static __device__ __forceinline__ int at(int r, int c)
    {
        const int s = PITCH == 8 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : ((r & 3) << 2) | ((r >> 2) & 3);
        return (r * PITCH + (c ^ s)) << 4;
    }
};

// LDS of a workgroup.
template <int DP>
struct Lds {
    static constexpr int TILE = KEYS * Place<DP>::PITCH * 16;
    alignas(16) char tiles[4 * TILE]; // K, V; K, V
    uint64_t missing[2][4];           // keys of a tile that are not there, by the wavefront that fetched them
};

// Workgroup `at` of the launch.  DP: dimensions computed; FULL: the head has all of them.
template <bool BF16, int DP, bool FULL>
__device__ __forceinline__ void attend(const FqAttendArgs &a, const FqAttendWork &w, dim3 at_block, Lds<DP> &shared)
{
    constexpr int NQ = DP / 16, ND = DP / 32, NC = DP / 32; // steps of the first product, tiles of dimensions, pieces to a thread
    constexpr int TILE = Lds<DP>::TILE;
    char *const lds = shared.tiles;
    auto &missing = shared.missing;

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int head = at_block.x % a.kv.kv_heads, b = at_block.z;
    // the last rows see most keys: they begin first
    const int row0 = (w.row_blocks - 1 - (int)(at_block.x / a.kv.kv_heads)) * FQ_MANY_ROWS;
    const int group = a.q_heads / a.kv.kv_heads, dim = FULL ? DP : a.kv.dim;
    const FqAttendRows rs = fq_attend_rows(a, w, b, group);
    if (row0 >= rs.rows)
        return;
    const int last = min(row0 + FQ_MANY_ROWS, rs.rows) - 1;
    const long long begin64 = w.key0 + (long long)at_block.y * w.chunk;
    const int most = rs.limit(last / group);
    if (begin64 >= most && w.part_o)
        return; // nobody reads this part
    const int begin = begin64 < most ? (int)begin64 : most;
    const int end = (int)(begin64 + w.chunk < most ? begin64 + w.chunk : most);

    const int r = row0 + wave * 32 + col;
    const bool real = r <= last;
    const int j = (real ? r : row0) / group, h = head * group + (real ? r : row0) % group;
    const int lim = min(rs.limit(j), end);
    // this wavefront's rows: all of them see the keys before `all_seen`, none those from `wave_end` on
    const int w_first = min(row0 + wave * 32, last), w_last = min(row0 + wave * 32 + 31, last);
    const int all_seen = rs.limit(w_first / group), wave_end = min(rs.limit(w_last / group), end);

    u32x4 q[NQ]; // dimensions 16 s + 8 half ..
    {
        const uint16_t *from = a.q + (rs.q0 + j) * a.q_stride + h * dim;
#pragma unroll
        for (int s = 0; s < NQ; s++) {
            const int d = 16 * s + 8 * half;
            q[s] = u32x4{0, 0, 0, 0};
            if (real && (FULL || d < dim))
                q[s] = fq_signed(*(const u32x4 *)(from + d), a.scale);
        }
    }
    float16_t o[ND];
#pragma unroll
    for (int d = 0; d < ND; d++)
#pragma unroll
        for (int i = 0; i < 16; i++)
            o[d][i] = 0.0f;
    float m = -INFINITY, l = 0.0f;
    const float c = fq_score_factor(a.scale);
    const int32_t *table = a.seqs.table + (rs.shared ? 0 : (long long)b * a.seqs.table_width);

    // fetching: thread -> key threadIdx.x / 4 of a tile, pieces threadIdx.x % 4 + 4 i of its rows of K and V
    const int my_key = threadIdx.x >> 2, my_piece = threadIdx.x & 3;
    u32x4 ks[NC], vs[NC];
    bool there = false;
    int page = -1;
    auto fetch = [&](int key) { // from the page found a step before
        there = page >= 0 && page < a.kv.n_pages;
        const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NC; i++)
            ks[i] = vs[i] = zero;
        if (there) {
            const long long at = fq_key_offset(a, page, key + my_key, head) + 8 * my_piece;
#pragma unroll
            for (int i = 0; i < NC; i++) {
                if (FULL || 32 * i + 8 * my_piece < dim) {
                    ks[i] = *(const u32x4 *)(a.kv.k + at + 32 * i);
                    vs[i] = *(const u32x4 *)(a.kv.v + at + 32 * i);
                }
            }
        }
    };
    auto put = [&](int buf) {
        char *kt = lds + buf * 2 * TILE, *vt = kt + TILE;
#pragma unroll
        for (int i = 0; i < NC; i++) {
            *(u32x4 *)(kt + Place<DP>::at(my_key, my_piece + 4 * i)) = ks[i];
            *(u32x4 *)(vt + Place<DP>::at(my_key, my_piece + 4 * i)) = vs[i];
        }
        const uint64_t gone = __ballot(!there); // lane 4 k + piece: key 16 wave + k
        if (lane == 0)
            missing[buf][wave] = gone;
    };

    if (begin < end) {
        page = fq_key_page(a, table, begin + my_key, end);
        fetch(begin);
        page = fq_key_page(a, table, min(begin + KEYS, end) + my_key, end);
        put(0);
    }
    int buf = 0;
    for (int key = begin; key < end; key += KEYS, buf ^= 1) {
        const bool more = key + KEYS < end;
        __syncthreads();
        if (more) {
            fetch(key + KEYS);
            page = fq_key_page(a, table, (key + 2 * KEYS < end ? key + 2 * KEYS : end) + my_key, end);
        }
        const char *kt = lds + buf * 2 * TILE, *vt = kt + TILE;
        if (key < wave_end) {
            float16_t sc[2];
#pragma unroll
            for (int t = 0; t < 2; t++) {
#pragma unroll
                for (int i = 0; i < 16; i++)
                    sc[t][i] = 0.0f;
#pragma unroll
                for (int s = 0; s < NQ; s++) {
                    const u32x4 k = *(const u32x4 *)(kt + Place<DP>::at(32 * t + col, 2 * s + half));
                    sc[t] = fq_mfma32<BF16>(k, q[s], sc[t]);
                }
            }
            const uint64_t gone0 = missing[buf][0], gone1 = missing[buf][1], gone2 = missing[buf][2], gone3 = missing[buf][3];
            const bool masked = (gone0 | gone1 | gone2 | gone3) != 0 || key + KEYS > all_seen;
            // register i of tile t holds key 32 t + 8 (i / 4) + 4 half + i % 4
            float top = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    if (masked) {
                        const int at = 32 * t + 8 * (i >> 2) + 4 * half + (i & 3);
                        const uint64_t gone = t == 0 ? (i < 8 ? gone0 : gone1) : (i < 8 ? gone2 : gone3);
                        if (((gone >> (4 * (at & 15))) & 1) || key + at >= lim)
                            sc[t][i] = -INFINITY;
                    }
                    top = fmaxf(top, sc[t][i]);
                }
            top = fq_over32<false>(top) * c;
            if (__any(top > m + FQ_ATTEND_SLACK)) {
                const float now = fmaxf(m, top);
                const float fall = __builtin_amdgcn_exp2f(m - fq_reference(now));
                m = now;
                l *= fall;
#pragma unroll
                for (int d = 0; d < ND; d++)
#pragma unroll
                    for (int i = 0; i < 16; i++)
                        o[d][i] *= fall;
            }
            const float ref = fq_reference(m);
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    sc[t][i] = __builtin_amdgcn_exp2f(fmaf(sc[t][i], c, -ref));
                    l += sc[t][i];
                }
#pragma unroll
            for (int s = 0; s < 4; s++) { // 16 keys: 16 s + 4 half + 0 .. 3 and 8 on
                u32x4 p;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    p[e] = fq_pack2<BF16>(sc[s >> 1][8 * (s & 1) + 2 * e], sc[s >> 1][8 * (s & 1) + 2 * e + 1]);
                const int t16 = lane & 15, key_at = 16 * s + 4 * half + (t16 >> 2);
#pragma unroll
                for (int d = 0; d < ND; d++) {
                    const int piece = 4 * d + 2 * ((lane >> 4) & 1) + ((t16 & 3) >> 1);
                    const u32x2 lo = fq_read_transposed(vt + Place<DP>::at(key_at, piece) + 8 * (t16 & 1));
                    const u32x2 hi = fq_read_transposed(vt + Place<DP>::at(key_at + 8, piece) + 8 * (t16 & 1));
                    o[d] = fq_mfma32<BF16>(u32x4{lo[0], lo[1], hi[0], hi[1]}, p, o[d]);
                }
            }
        }
        if (more)
            put(buf ^ 1);
    }

    l = fq_over32<true>(l);
    if (!real)
        return;
    const long long t = rs.q0 + j;
    // register i of tile d holds dimension 32 d + 8 (i / 4) + 4 half + i % 4
    if (w.part_o) {
        const long long at = (w.part0 + (long long)at_block.y) * a.seqs.tokens * a.q_heads + t * a.q_heads + h;
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int e = 32 * d + 8 * i + 4 * half;
                if (FULL || e < dim)
                    *(float4_t *)(w.part_o + at * dim + e) = float4_t{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
            }
        if (half == 0)
            w.part_ml[at] = float2{m, l};
    } else {
        const float inv = fq_inverse(l);
        uint16_t *to = a.out + t * a.out_stride + h * dim;
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int e = 32 * d + 8 * i + 4 * half;
                if (FULL || e < dim)
                    *(u32x2 *)(to + e) = u32x2{fq_pack2<BF16>(o[d][4 * i] * inv, o[d][4 * i + 1] * inv),
                                               fq_pack2<BF16>(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv)};
            }
        if (half == 0 && a.lse)
            a.lse[t * a.q_heads + h] = fq_lse(m, l);
    }
}

} // namespace many

#endif
