// Attention of many rows to a sequence and key head: prompts, chunks of them, and a prefix that a batch shares.
//
// Bound by the matrix cores and by the exponentials between the two products.  Four wavefronts take 32 rows each and share
// tiles of 64 keys in LDS, two of them in turn.  Rows come through registers, two tiles ahead: while one is computed, the next has
// had the time of a whole tile to arrive, is written to the other half of LDS at the end and the one barrier of a step follows.
// (One tile ahead a lone workgroup of a compute unit waited for memory.)
#ifndef FQ_ATTEND_MANY_H
#define FQ_ATTEND_MANY_H

#include <type_traits>

#include "fq_attend.h"

namespace many {

constexpr int KEYS = 64;

// Where 16-byte piece c of key r lies in a tile: blocks of 16 keys, in them pieces of four a key at a time (64 bytes) key by key, the
// four turned by the key's number.  16 keys of one piece (the reads of K), 4 keys of four pieces in a row (the writes, and the
// transposed reads of V) fall on different banks, and all but the lowest bits of a lane's address are constants.
template <int DP>
__device__ __forceinline__ constexpr int place(int r, int c)
{
    return (r >> 4) * (DP * 32) + (c >> 2) * 1024 + (r & 15) * 64 + (((c & 3) ^ ((r >> 2) & 3)) << 4);
}

// LDS of a workgroup.
template <int DP>
struct Lds {
    static constexpr int TILE = KEYS * DP * 2;
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
    constexpr int DEEP = DP <= 96 ? 2 : 1; // tiles ahead (the registers of a wider head hold one)
    u32x4 ks[DEEP][NC], vs[DEEP][NC];
    bool there[DEEP];
    int page = -1; // of the tile that is fetched next
    auto find = [&](int key) { page = fq_key_page(a, table, (key < end ? key : end) + my_key, end); };
    auto fetch = [&](auto P, int key) {
        const int p = DEEP == 2 ? P.value : 0;
        there[p] = page >= 0 && page < a.kv.n_pages;
        const u32x4 zero = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NC; i++)
            ks[p][i] = vs[p][i] = zero;
        if (there[p]) {
            const long long at = fq_key_offset(a, page, key + my_key, head) + 8 * my_piece;
#pragma unroll
            for (int i = 0; i < NC; i++) {
                if (FULL || 32 * i + 8 * my_piece < dim) {
                    ks[p][i] = *(const u32x4 *)(a.kv.k + at + 32 * i);
                    vs[p][i] = *(const u32x4 *)(a.kv.v + at + 32 * i);
                }
            }
        }
    };
    auto put = [&](auto P) {
        const int p = DEEP == 2 ? P.value : 0;
        char *kt = lds + P.value * 2 * TILE + place<DP>(my_key, my_piece), *vt = kt + TILE;
#pragma unroll
        for (int i = 0; i < NC; i++) {
            *(u32x4 *)(kt + 1024 * i) = ks[p][i];
            *(u32x4 *)(vt + 1024 * i) = vs[p][i];
        }
        const uint64_t gone = __ballot(!there[p]); // lane 4 k + piece: key 16 wave + k
        if (lane == 0)
            missing[P.value][wave] = gone;
    };
    // a lane's piece of K: key col, dimensions 8 half .. of 16 (even and odd steps); of V: key 4 half + t16 / 4 (and 8 on)
    const int t16 = lane & 15;
    const int k_at[2] = {place<DP>(col, half), place<DP>(col, 2 + half)};
    const int v_key = 4 * half + (t16 >> 2), v_piece = 2 * ((lane >> 4) & 1) + ((t16 & 3) >> 1);
    const int v_at[2] = {place<DP>(v_key, v_piece) + 8 * (t16 & 1), place<DP>(v_key + 8, v_piece) + 8 * (t16 & 1)};

    constexpr int RING = NQ < 8 ? NQ : 8; // pieces of K and V that are read ahead of the products
    auto step = [&](auto P, auto Q, int key) { // P, Q: the halves of LDS with this tile and for the next
        const int p = P.value;
        __syncthreads();
        if (key + DEEP * KEYS < end) {
            fetch(P, key + DEEP * KEYS);
            find(key + (DEEP + 1) * KEYS);
        }
        const char *kt = lds + p * 2 * TILE, *vt = kt + TILE;
        if (key < wave_end) {
            float16_t sc[2];
#pragma unroll
            for (int t = 0; t < 2; t++)
#pragma unroll
                for (int i = 0; i < 16; i++)
                    sc[t][i] = 0.0f;
            // The compiler reads a piece just before its product and waits for it; here eight are under way.
            auto piece_k = [&](int i) {
                const int t = i / NQ, s = i % NQ;
                return *(const u32x4 *)(kt + k_at[s & 1] + t * (DP * 64) + (s >> 1) * 1024);
            };
            auto piece_v = [&](int i) {
                const int s = i / ND, d = i % ND;
                const u32x2 lo = fq_read_transposed(vt + v_at[0] + s * (DP * 32) + d * 1024);
                const u32x2 hi = fq_read_transposed(vt + v_at[1] + s * (DP * 32) + d * 1024);
                return u32x4{lo[0], lo[1], hi[0], hi[1]};
            };
            u32x4 ring[RING];
#pragma unroll
            for (int i = 0; i < RING; i++)
                ring[i] = piece_k(i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 2 * NQ; i++) {
                sc[i / NQ] = fq_mfma32<BF16>(ring[i % RING], q[i % NQ], sc[i / NQ]);
                if (i + RING < 2 * NQ)
                    ring[i % RING] = piece_k(i + RING);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < RING; i++)
                ring[i] = piece_v(i);
            __builtin_amdgcn_sched_barrier(0);
            const uint64_t gone0 = missing[p][0], gone1 = missing[p][1], gone2 = missing[p][2], gone3 = missing[p][3];
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
            u32x4 pk[4]; // 16 keys each: 16 s + 4 half + 0 .. 3 and 8 on
#pragma unroll
            for (int s = 0; s < 4; s++)
#pragma unroll
                for (int e = 0; e < 4; e++)
                    pk[s][e] = fq_pack2<BF16>(sc[s >> 1][8 * (s & 1) + 2 * e], sc[s >> 1][8 * (s & 1) + 2 * e + 1]);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4 * ND; i++) {
                o[i % ND] = fq_mfma32<BF16>(ring[i % RING], pk[i / ND], o[i % ND]);
                if (i + RING < 4 * ND)
                    ring[i % RING] = piece_v(i + RING);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (key + KEYS < end)
            put(Q);
    };
    constexpr std::integral_constant<int, 0> EVEN;
    constexpr std::integral_constant<int, 1> ODD;
    if (begin < end) {
        find(begin);
        fetch(EVEN, begin);
        find(begin + KEYS);
        if constexpr (DEEP == 2) {
            fetch(ODD, begin + KEYS);
            find(begin + 2 * KEYS);
        }
        put(EVEN);
    }
    if constexpr (DEEP == 2) {
        for (int key = begin; key < end; key += 2 * KEYS) {
            step(EVEN, ODD, key);
            if (key + KEYS < end)
                step(ODD, EVEN, key + KEYS);
        }
    } else {
        struct Half {
            int value;
        } now{0};
        for (int key = begin; key < end; key += KEYS, now.value ^= 1)
            step(now, Half{now.value ^ 1}, key);
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
