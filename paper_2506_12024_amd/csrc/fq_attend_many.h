// Attention of many rows to a sequence and key head: prompts, chunks of them, and a prefix that a batch shares.
//
// Four wavefronts take 32 rows each and share tiles of 64 keys in LDS, two of them in turn; a tile's rows come through
// registers while the one before is computed.  A wavefront works in steps of 32 keys, three of them under way at once: the matrix cores sum V of the last one and score the next one while the
// vector units take the exponentials of this one.  Measured: 2048 new tokens behind 951 of the 70B shapes 178 us in fp16 and 171 in bf16
// (743 and 775 TFLOP/s), 8192 tokens 818 and 863 TFLOP/s, where a library product of 8192^3 reaches 1160 to 1220.  Neither unit is
// full: the matrix cores are busy 37 % of the cycles (the clock falls to 1.9 GHz under them), the vector units 48 %; two wavefronts to a SIMD
// have two barriers and a pass through registers to hide in every tile.  With exponentials and products one after the other 9 % longer.
// More pieces read ahead than four changed nothing.
#ifndef FQ_ATTEND_MANY_H
#define FQ_ATTEND_MANY_H

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
    int odd[4];                       // values that are not finite were taken out of what the wavefront fetched
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
    const int group = a.q_heads / a.kv.kv_heads, dim = FULL ? DP : a.kv.dim;
    const int head = at_block.x % a.kv.kv_heads;
    int b = at_block.z, block = w.row_blocks - 1 - (int)(at_block.x / a.kv.kv_heads); // the last rows see most keys: they begin first
    if (w.row_blocks == 0 && !fq_find_row_block(a, (int)(at_block.x / a.kv.kv_heads), group, FQ_MANY_ROWS, b, block))
        return;
    b = __builtin_amdgcn_readfirstlane(b);
    const int row0 = __builtin_amdgcn_readfirstlane(block) * FQ_MANY_ROWS;
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

    const int block_sees = rs.limit(row0 / group); // every row of the workgroup sees the keys before this one
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
    float m = -INFINITY, l = 0.0f, lost = 0.0f;
    const float c = fq_score_factor(a.scale);
    const int32_t *table = a.seqs.table + (rs.shared ? 0 : (long long)b * a.seqs.table_width);

    // fetching: thread -> key threadIdx.x / 4 of a tile, pieces threadIdx.x % 4 + 4 i of its rows of K and V
    const int my_key = threadIdx.x >> 2, my_piece = threadIdx.x & 3;
    u32x4 ks[NC], vs[NC];
    bool there = false;
    int page = -1; // of the tile that is fetched next
    auto find = [&](int key) { page = fq_key_page(a, table, (key < end ? key : end) + my_key, end); };
    auto fetch = [&](int key) {
        there = page >= 0 && page < a.kv.n_pages;
        // (a key that is not there is read from the pool's begin, and zeroed when it is put)
        const long long at = (there ? fq_key_offset(a, page, key + my_key, head) : 0) + 8 * my_piece;
#pragma unroll
        for (int i = 0; i < NC; i++) {
            const int d = FULL || 32 * i + 8 * my_piece < dim ? 32 * i : -8 * my_piece;
            ks[i] = *(const u32x4 *)(a.kv.k + at + d);
            vs[i] = *(const u32x4 *)(a.kv.v + at + d);
        }
    };
    uint32_t odd = 0;
    auto put = [&](int half_of_lds, int key) {
        const uint64_t gone = __ballot(!there); // lane 4 k + piece: key 16 wave + k
        if (gone) {
            if (!there)
#pragma unroll
                for (int i = 0; i < NC; i++)
                    ks[i] = vs[i] = u32x4{0, 0, 0, 0};
        }
        if (key + KEYS > block_sees) {
            if (key + my_key >= block_sees)
#pragma unroll
                for (int i = 0; i < NC; i++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const uint32_t out = fq_odd<BF16>(vs[i][e]);
                        vs[i][e] &= ~out;
                        odd |= out;
                    }
            const bool wave_odd = __any(odd != 0);
            if (lane == 0)
                shared.odd[wave] = wave_odd;
        }
        char *kt = lds + half_of_lds * 2 * TILE + place<DP>(my_key, my_piece), *vt = kt + TILE;
#pragma unroll
        for (int i = 0; i < NC; i++) {
            const u32x4 zero = {0, 0, 0, 0};
            const bool real = FULL || 32 * i + 8 * my_piece < dim;
            *(u32x4 *)(kt + 1024 * i) = real ? ks[i] : zero;
            *(u32x4 *)(vt + 1024 * i) = real ? vs[i] : zero;
        }
        if (lane == 0)
            missing[half_of_lds][wave] = gone;
    };
    // a lane's piece of K: key col, dimensions 8 half .. of 16 (even and odd steps); of V: key 4 half + t16 / 4 (and 8 on)
    const int t16 = lane & 15;
    const int k_at[2] = {place<DP>(col, half), place<DP>(col, 2 + half)};
    const int v_key = 4 * half + (t16 >> 2), v_piece = 2 * ((lane >> 4) & 1) + ((t16 & 3) >> 1);
    const int v_at[2] = {place<DP>(v_key, v_piece) + 8 * (t16 & 1), place<DP>(v_key + 8, v_piece) + 8 * (t16 & 1)};

    float16_t next; // scores of the step to come; register i holds key 8 (i / 4) + 4 half + i % 4 of its 32
    u32x4 pk[2];    // weights of the last step, 16 keys each
    pk[0] = pk[1] = u32x4{0, 0, 0, 0};
    // The products of a step: 2 ND with V of the last one, NQ with K of the next one.
    constexpr int PRODUCTS = 2 * ND + NQ, AHEAD = 4;
    auto piece = [&](int i, const char *vt, const char *kt) {
        if (i >= 2 * ND)
            return *(const u32x4 *)(kt + k_at[i & 1] + ((i - 2 * ND) >> 1) * 1024);
        const int at = i / ND * (DP * 32) + i % ND * 1024;
        const u32x2 lo = fq_read_transposed(vt + v_at[0] + at), hi = fq_read_transposed(vt + v_at[1] + at);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    };
    auto product = [&](int i, u32x4 x) {
        const float16_t zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        if (i >= 2 * ND)
            next = fq_mfma32<BF16>(x, q[i - 2 * ND], i == 2 * ND ? zero : next);
        else
            o[i % ND] = fq_mfma32<BF16>(x, pk[i / ND], o[i % ND]);
    };
    // One step: the keys from `key` on (half `t` of the tile in half `p` of LDS), whose scores are in `next`; V of the
    // step before at `v_last`, K of the step after at `k_next` (after the last step: any tile, nobody looks at the scores).
    // Between any two products stands a share of the exponentials (a fence each: left to itself the compiler puts all products
    // first), and four pieces are on their way from LDS.
    auto step = [&](int key, int p, int t, const char *v_last, const char *k_next) {
        float16_t x = next;
        const uint64_t gone0 = missing[p][2 * t], gone1 = missing[p][2 * t + 1];
        u32x4 ring[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; i++)
            ring[i] = piece(i, v_last, k_next);
        if ((gone0 | gone1) != 0 || key + 32 > all_seen) {
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int at = 8 * (i >> 2) + 4 * half + (i & 3);
                if ((((i < 8 ? gone0 : gone1) >> (4 * (at & 15))) & 1) || key + at >= lim)
                    x[i] = -INFINITY;
            }
        }
#pragma unroll
        for (int i = 0; i < 16; i++)
            x[i] = fq_score(x[i], c);
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 16; i++)
            top = fmaxf(top, x[i]);
        top = fq_over32<false>(top);
        const bool raise = __any(top - m > FQ_ATTEND_SLACK + FQ_ATTEND_BELOW<BF16>);
        const float now = raise ? fmaxf(m, top - FQ_ATTEND_BELOW<BF16>) : m, ref = fq_reference(now);
        const float fall = __builtin_amdgcn_exp2f(m - ref);
        l *= fall; // (1 where nothing is raised)
        lost *= fall;
        float sum = 0.0f;
        m = now;
        u32x4 weights[2];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < PRODUCTS; i++) {
            product(i, ring[i % AHEAD]);
            if (i + AHEAD < PRODUCTS)
                ring[i % AHEAD] = piece(i + AHEAD, v_last, k_next);
#pragma unroll
            for (int e = i * 16 / PRODUCTS; e < (i + 1) * 16 / PRODUCTS; e++) {
                x[e] = __builtin_amdgcn_exp2f(x[e] - ref);
                if (e > 0)
                    sum += x[e - 1]; // (one behind: the exponential takes a while)
                if (e > 1 && e % 2 == 0)
                    weights[(e - 2) >> 3][((e - 2) & 7) >> 1] = fq_pack2<BF16>(x[e - 2], x[e - 1]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        fq_add_weights(l, lost, sum + x[15]);
        weights[1][3] = fq_pack2<BF16>(x[14], x[15]);
        pk[0] = weights[0];
        pk[1] = weights[1];
        int rescale = raise;
        // (else the compiler moves the exponentials behind this branch)
        asm volatile("" : "+v"(rescale), "+v"(pk[0]), "+v"(pk[1]), "+v"(l));
        if (__builtin_amdgcn_readfirstlane(rescale)) {
#pragma unroll
            for (int d = 0; d < ND; d++)
#pragma unroll
                for (int i = 0; i < 16; i++)
                    o[d][i] *= fall;
        }
    };

    if (begin < end) {
        find(begin);
        fetch(begin);
        find(begin + KEYS);
        put(0, begin);
        if (begin + KEYS < end) {
            fetch(begin + KEYS);
            find(begin + 2 * KEYS);
        }
    }
    // the first step has none before it: its weights are 0, and so is what they meet, in the half of LDS that is not yet filled
    constexpr int HALF = DP * 64; // bytes of 32 keys
    char *const none = lds + 3 * TILE;
    for (int i = threadIdx.x * 16; i < HALF; i += FQ_ATTEND_THREADS * 16)
        *(u32x4 *)(none + i) = u32x4{0, 0, 0, 0};
    __syncthreads();
    if (begin < wave_end)
#pragma unroll
        for (int i = 2 * ND; i < PRODUCTS; i++)
            product(i, piece(i, lds, lds));
    const char *v_last = none;
    int p = 0;
    for (int key = begin; key < end; key += KEYS, p ^= 1) {
        const char *kt = lds + p * 2 * TILE, *vt = kt + TILE, *kn = lds + (p ^ 1) * 2 * TILE;
        const bool more = key + KEYS < end;
        if (key < wave_end)
            step(key, p, 0, v_last, kt + HALF);
        if (more) {
            __syncthreads(); // the other half of LDS is read no more
            put(p ^ 1, key + KEYS);
            if (key + 2 * KEYS < end) {
                fetch(key + 2 * KEYS);
                find(key + 3 * KEYS);
            }
            __syncthreads();
        }
        v_last = vt;
        if (key + 32 < wave_end) {
            step(key + 32, p, 1, vt, kn);
            v_last = vt + HALF;
        }
        if (key + KEYS >= wave_end && key < wave_end) // the last step's V
#pragma unroll
            for (int i = 0; i < 2 * ND; i++)
                product(i, piece(i, v_last, lds));
    }

    l = fq_over32<true>(l);
    if (!real)
        return;
    // register i of tile d holds dimension 32 d + 8 (i / 4) + 4 half + i % 4
    if (block_sees < end && (shared.odd[0] | shared.odd[1] | shared.odd[2] | shared.odd[3])) // (the last tile's put wrote them all)
        for (int at = max(block_sees, begin); at < lim; at++) {
            const int page_at = fq_key_page(a, table, at, lim);
            if (page_at < 0 || page_at >= a.kv.n_pages)
                continue;
            const uint16_t *from = a.kv.v + fq_key_offset(a, page_at, at, head);
#pragma unroll
            for (int d = 0; d < ND; d++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int e = 32 * d + 8 * i + 4 * half;
                    if (FULL || e < dim) {
                        const u32x2 y = *(const u32x2 *)(from + e);
#pragma unroll
                        for (int f = 0; f < 4; f++)
                            o[d][4 * i + f] += fq_odd_value<BF16>(y, f);
                    }
                }
        }
    const long long t = rs.q0 + j;
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
