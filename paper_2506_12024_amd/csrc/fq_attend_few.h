// Attention of up to 32 rows to a sequence and key head: the single tokens of a decode step, and a few more.
//
// Bound by reading the cache once.  A wavefront takes 32 keys at a time, its own ones: the rows of K go from memory straight
// into the registers of the first product's left operand (a lane holds 16 bytes of a key; any order of the head's
// dimensions serves if Q has the same), the rows of V pass through a piece of LDS that belongs to the wavefront alone and
// are read back transposed.  No barrier until the end, where the wavefronts' rows are added up; a lane asks for the next
// 32 keys as soon as the registers of the last are free, and for the page numbers a step before that.  Measured: 16 sequences of
// up to 4096 of the 7B shapes 102 us (5.0 TB/s), 32 of up to 16384 of the 70B shapes 251 us (5.3 TB/s); with the registers held to 168
// so that three workgroups fit a compute unit instead of two, 8 % longer.  One token behind 777 keys takes 7.1 us on the device,
// three trips to memory one after the other (lengths, page, keys), and 3.7 more to join its seven parts.
#ifndef FQ_ATTEND_FEW_H
#define FQ_ATTEND_FEW_H

#include "fq_attend.h"

namespace few {

constexpr int WAVES = FQ_ATTEND_THREADS / 64;
static_assert(WAVES == 4, "the flags of four are read");
constexpr int KEYS = 32; // to a wavefront and step

// 16-byte pieces to a row of V in LDS, and where piece c of row r goes: 16 rows of one piece fall on 16 different bank
// groups (the writes), and so do the pairs of pieces of any two neighbouring or next but one quarters of the rows (the transposed
// reads, whichever lanes LDS takes together).
template <int DP>
struct Place {
    static constexpr int PITCH = DP <= 64 ? 8 : DP <= 128 ? 16 : 32;
    static __device__ __forceinline__ int at(int r, int c)
    {
        const int s = PITCH == 8 ? (((r >> 1) & 1) << 1 | (((r >> 2) ^ (r >> 3)) & 1) << 2) | ((r >> 3) & 1)
                                 : ((r & 3) << 1 | (((r >> 2) ^ (r >> 3)) & 1) << 3) | ((r >> 3) & 1);
        return (r * PITCH + (c ^ s)) << 4;
    }
};

// The rows' sums at the end, 4 dimensions to a piece: 16 rows of one piece on different bank groups (8 where a row has 24).
template <int DP>
__device__ __forceinline__ int sum_place(int r, int piece)
{
    return (r * (DP / 4) + (piece ^ (r & (DP == 96 ? 7 : 15)))) << 4;
}

// LDS of a workgroup.
template <int DP, int RT>
struct Lds {
    static constexpr int WAVE = KEYS * Place<DP>::PITCH * 16; // a wavefront's V, its part of the rows at the end
    static_assert(WAVE >= 16 * DP * 4, "the rows are added up in the same piece");
    alignas(16) char v[WAVES * WAVE];
    float m[WAVES][RT * 16], l[WAVES][RT * 16];
    int odd[WAVES]; // values that are not finite were taken out of its keys
};

// Workgroup `at` of the launch.  DP: dimensions computed; FULL: the head has all of them; RT: tiles of 16 rows.
template <bool BF16, int DP, bool FULL, int RT>
__device__ __forceinline__ void attend(const FqAttendArgs &a, const FqAttendWork &w, dim3 at_block, Lds<DP, RT> &shared)
{
    constexpr int NS = DP / 32, ND = DP / 16;
    constexpr int WAVE_LDS = Lds<DP, RT>::WAVE;
    char *const lds = shared.v;
    auto &all_m = shared.m;
    auto &all_l = shared.l;

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
    const int head = at_block.x % a.kv.kv_heads, row0 = at_block.x / a.kv.kv_heads * (16 * RT), b = at_block.z;
    const int group = a.q_heads / a.kv.kv_heads, dim = FULL ? DP : a.kv.dim;
    const FqAttendRows rs = fq_attend_rows(a, w, b, group);
    if (row0 >= rs.rows)
        return;
    const int last = min(row0 + 16 * RT, rs.rows) - 1;
    const long long begin64 = w.key0 + (long long)at_block.y * w.chunk;
    const int most = rs.limit(last / group);
    if (begin64 >= most && w.part_o)
        return; // nobody reads this part
    const int begin = begin64 < most ? (int)begin64 : most;
    const int end = (int)(begin64 + w.chunk < most ? begin64 + w.chunk : most);
    const int all_seen = rs.limit(row0 / group); // every row sees the keys before this one

    // Q: row col of tile rt, dimensions 32 s + 8 quad ..
    u32x4 q[RT][NS];
    int lim[RT];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        const int r = row0 + rt * 16 + col;
        const bool real = r <= last;
        const int j = (real ? r : row0) / group, h = head * group + (real ? r : row0) % group;
        lim[rt] = min(rs.limit(j), end);
        const uint16_t *from = a.q + (rs.q0 + j) * a.q_stride + h * dim;
#pragma unroll
        for (int s = 0; s < NS; s++) {
            const int d = 32 * s + 8 * quad;
            q[rt][s] = u32x4{0, 0, 0, 0};
            if (real && (FULL || d < dim))
                q[rt][s] = fq_signed(*(const u32x4 *)(from + d), a.scale);
        }
    }

    float4_t o[RT][ND];
    float m[RT], l[RT], lost[RT];
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        m[rt] = -INFINITY;
        l[rt] = lost[rt] = 0.0f;
#pragma unroll
        for (int d = 0; d < ND; d++)
            o[rt][d] = float4_t{0, 0, 0, 0};
    }
    const float c = fq_score_factor(a.scale);
    const int32_t *table = a.seqs.table + (rs.shared ? 0 : (long long)b * a.seqs.table_width);
    char *mine = lds + wave * WAVE_LDS;

    const uint16_t *kp[2], *vp[2]; // the lane's two keys (col, col + 16)
    bool ok[2];
    u32x4 k[2][NS], v[2][NS];
    int page[2];
    auto pages = [&](int key) {
#pragma unroll
        for (int t = 0; t < 2; t++)
            page[t] = fq_key_page(a, table, key + 16 * t + col, end);
    };
    auto addresses = [&](int key) {
#pragma unroll
        for (int t = 0; t < 2; t++) {
            ok[t] = page[t] >= 0 && page[t] < a.kv.n_pages;
            const long long at = ok[t] ? fq_key_offset(a, page[t], key + 16 * t + col, head) : 0; // (any address of the pool)
            kp[t] = a.kv.k + at;
            vp[t] = a.kv.v + at;
        }
    };
    auto load = [&](const uint16_t *const (&p)[2], u32x4 (&x)[2][NS]) {
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
            for (int s = 0; s < NS; s++) {
                const int d = 32 * s + 8 * quad;
                x[t][s] = *(const u32x4 *)(p[t] + (FULL || d < dim ? d : 0));
            }
    };

    uint32_t odd = 0;
    constexpr int STEP = WAVES * KEYS;
    int key = begin + wave * KEYS;
    if (key < end) {
        pages(key);
        addresses(key);
        load(kp, k);
        load(vp, v);
        pages(key + STEP < end ? key + STEP : end);
    }
    for (; key < end; key += STEP) {
        const bool more = key + STEP < end;
        const uint64_t there0 = __ballot(ok[0]), there1 = __ballot(ok[1]);
        const uint32_t there = (uint32_t)(there0 & 0xffff) | ((uint32_t)(there1 & 0xffff) << 16);
        float4_t sc[RT][2];
#pragma unroll
        for (int t = 0; t < 2; t++) {
            if (!FULL) {
#pragma unroll
                for (int s = 0; s < NS; s++)
                    if (32 * s + 8 * quad >= dim)
                        k[t][s] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int rt = 0; rt < RT; rt++) {
                sc[rt][t] = float4_t{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < NS; s++)
                    sc[rt][t] = fq_mfma16<BF16>(k[t][s], q[rt][s], sc[rt][t]);
            }
        }
        // V of a key that is not there must be 0, whatever lies at its address: 0 times NaN is NaN
        if (there != 0xffffffffu) {
#pragma unroll
            for (int t = 0; t < 2; t++)
                if (!ok[t])
#pragma unroll
                    for (int s = 0; s < NS; s++)
                        v[t][s] = u32x4{0, 0, 0, 0};
        }
        if (key + KEYS > all_seen) {
#pragma unroll
            for (int t = 0; t < 2; t++)
                if (key + 16 * t + col >= all_seen)
#pragma unroll
                    for (int s = 0; s < NS; s++)
#pragma unroll
                        for (int e = 0; e < 4; e++) {
                            const uint32_t out = fq_odd<BF16>(v[t][s][e]);
                            v[t][s][e] &= ~out;
                            odd |= out;
                        }
        }
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
            for (int s = 0; s < NS; s++)
                *(u32x4 *)(mine + Place<DP>::at(16 * t + col, 4 * s + quad)) = v[t][s];
        if (more) {
            addresses(key + STEP);
            load(kp, k);
            load(vp, v);
            pages(key + 2 * STEP < end ? key + 2 * STEP : end);
        }
        const bool masked = there != 0xffffffffu || key + KEYS > all_seen;
        u32x4 p[RT];
#pragma unroll
        for (int rt = 0; rt < RT; rt++) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; i++)
                x[i] = fq_score(sc[rt][i >> 2][i & 3], c);
            if (masked) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const int at = 16 * (i >> 2) + 4 * quad + (i & 3);
                    if (!((there >> at) & 1) || key + at >= lim[rt])
                        x[i] = -INFINITY;
                }
            }
            float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
            top = fq_over32<false>(fq_over16<false>(top));
            if (__any(top - m[rt] > FQ_ATTEND_SLACK + FQ_ATTEND_BELOW<BF16>)) {
                const float now = fmaxf(m[rt], top - FQ_ATTEND_BELOW<BF16>);
                const float fall = __builtin_amdgcn_exp2f(m[rt] - fq_reference(now));
                m[rt] = now;
                l[rt] *= fall;
                lost[rt] *= fall;
#pragma unroll
                for (int d = 0; d < ND; d++)
                    o[rt][d] *= fall;
            }
            const float ref = fq_reference(m[rt]);
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                x[i] = __builtin_amdgcn_exp2f(x[i] - ref);
                sum += x[i];
            }
            fq_add_weights(l[rt], lost[rt], sum);
            p[rt] = u32x4{fq_pack2<BF16>(x[0], x[1]), fq_pack2<BF16>(x[2], x[3]), fq_pack2<BF16>(x[4], x[5]),
                          fq_pack2<BF16>(x[6], x[7])};
        }
        // the wavefront's own writes, read by other lanes of it: LDS serves a wavefront in order, the compiler is told so
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int d = 0; d < ND; d++) {
            const int r = 4 * quad + (col >> 2), piece = 2 * d + ((col & 3) >> 1), half = (col & 1) * 8;
            const u32x2 lo = fq_read_transposed(mine + Place<DP>::at(r, piece) + half);
            const u32x2 hi = fq_read_transposed(mine + Place<DP>::at(16 + r, piece) + half);
            const u32x4 vt = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
            for (int rt = 0; rt < RT; rt++)
                o[rt][d] = fq_mfma16<BF16>(vt, p[rt], o[rt][d]);
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }

#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        l[rt] = fq_over32<true>(fq_over16<true>(l[rt]));
        if (quad == 0) {
            all_m[wave][rt * 16 + col] = m[rt];
            all_l[wave][rt * 16 + col] = l[rt];
        }
    }
    const bool wave_odd = __any(odd != 0);
    if (lane == 0)
        shared.odd[wave] = wave_odd;
    const long long rows_all = (long long)a.seqs.tokens * a.q_heads;
#pragma unroll
    for (int rt = 0; rt < RT; rt++) {
        __syncthreads();
        const int r16 = rt * 16 + col;
        float top = all_m[0][r16];
#pragma unroll
        for (int i = 1; i < WAVES; i++)
            top = fmaxf(top, all_m[i][r16]);
        const float fall = __builtin_amdgcn_exp2f(m[rt] - fq_reference(top));
#pragma unroll
        for (int d = 0; d < ND; d++)
            *(float4_t *)(mine + sum_place<DP>(col, 4 * d + quad)) = o[rt][d] * fall;
        __syncthreads();
        // thread: row tid / (DP / 8), 8 dimensions of it
        for (int u = threadIdx.x; u < 16 * (DP / 8); u += WAVES * 64) {
            const int rr = u / (DP / 8), d = u % (DP / 8) * 8, r = row0 + rt * 16 + rr;
            if (r > last || d >= dim)
                continue;
            float sum[8];
            float best = all_m[0][rt * 16 + rr], total = 0.0f;
#pragma unroll
            for (int i = 1; i < WAVES; i++)
                best = fmaxf(best, all_m[i][rt * 16 + rr]);
#pragma unroll
            for (int e = 0; e < 8; e++)
                sum[e] = 0.0f;
#pragma unroll
            for (int i = 0; i < WAVES; i++) {
                total += all_l[i][rt * 16 + rr] * __builtin_amdgcn_exp2f(all_m[i][rt * 16 + rr] - fq_reference(best));
                const float4_t x = *(const float4_t *)(lds + i * WAVE_LDS + sum_place<DP>(rr, d >> 2));
                const float4_t y = *(const float4_t *)(lds + i * WAVE_LDS + sum_place<DP>(rr, (d >> 2) + 1));
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    sum[e] += x[e];
                    sum[4 + e] += y[e];
                }
            }
            if (all_seen < end && (shared.odd[0] | shared.odd[1] | shared.odd[2] | shared.odd[3])) {
                const int sees = min(rs.limit(r / group), end);
                for (int at = max(all_seen, begin); at < sees; at++) {
                    const int page_at = fq_key_page(a, table, at, sees);
                    if (page_at < 0 || page_at >= a.kv.n_pages)
                        continue;
                    const u32x4 y = *(const u32x4 *)(a.kv.v + fq_key_offset(a, page_at, at, head) + d);
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        sum[e] += fq_odd_value<BF16>(u32x2{y[e >> 2 << 1], y[(e >> 2 << 1) + 1]}, e & 3);
                }
            }
            const long long t = rs.q0 + r / group;
            const int h = head * group + r % group;
            if (w.part_o) {
                const long long at = (w.part0 + (long long)at_block.y) * rows_all + t * a.q_heads + h;
                *(float4_t *)(w.part_o + at * dim + d) = float4_t{sum[0], sum[1], sum[2], sum[3]};
                *(float4_t *)(w.part_o + at * dim + d + 4) = float4_t{sum[4], sum[5], sum[6], sum[7]};
                if (d == 0)
                    w.part_ml[at] = float2{best, total};
            } else {
                const float inv = fq_inverse(total);
                u32x4 y;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    y[e] = fq_pack2<BF16>(sum[2 * e] * inv, sum[2 * e + 1] * inv);
                *(u32x4 *)(a.out + t * a.out_stride + h * dim + d) = y;
                if (d == 0 && a.lse)
                    a.lse[t * a.q_heads + h] = fq_lse(best, total);
            }
        }
    }
}

} // namespace few

#endif
