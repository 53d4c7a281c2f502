// Attention of new tokens over a paged cache: which kernel takes which rows, how the keys are split, and the sum of the parts.
#include "fq_attend.h"

namespace {

// What one call launches.  The rows of a sequence and a key head share its keys; where they are few, the rows of the whole
// batch share the prefix besides, and the prefix is a piece of its own.
struct Plan {
    int n, parts;
    int most_parts; // for this many keys or any fewer
    FqAttendWork work[2];
    int row_tiles[2]; // 0: the kernel for many rows
};

constexpr int MAX_PARTS = 512; // of one launch

int div_up(long long a, long long b) { return (int)((a + b - 1) / b); }

int tiles_of(const FqAttendArgs &a, long long rows)
{
    const bool wide = a.kv.dim > 96 && a.kv.dim != 128; // (the registers of such a head hold one tile)
    return rows > (wide ? 16 : 32) ? 0 : rows > 16 ? 2 : 1;
}

FqAttendWork work(const FqAttendArgs &a, bool shared, int key0, long long keys, int seqs, int tokens, int row_tiles, int cus, int &most_parts)
{
    const long long rows = (long long)tokens * (a.q_heads / a.kv.kv_heads);
    const int step = row_tiles ? 128 : 64; // keys that a workgroup takes at once
    FqAttendWork w{};
    w.shared = shared;
    w.key0 = key0;
    w.row_blocks = div_up(rows, row_tiles ? 16 * row_tiles : FQ_MANY_ROWS);
    long long blocks = (long long)w.row_blocks * seqs;
    if (!row_tiles && seqs > 1) {
        // sequences of different lengths: no workgroups for rows that most of them do not have (a prompt of 2048 among 63
        // single tokens, eight rows to a token and key head: 1560 workgroups instead of 65536, 182 us instead of 318)
        const long long all = (long long)a.seqs.tokens * (a.q_heads / a.kv.kv_heads) / FQ_MANY_ROWS + seqs;
        if (all < blocks) {
            blocks = all;
            w.row_blocks = 0;
            seqs = 1;
        }
    }
    const long long groups = blocks * a.kv.kv_heads;
    const long long steps = div_up(keys > 0 ? keys : 1, step);
    // Steps to a part.  Few rows: one step each while that makes no more than three workgroups to a compute unit (by their registers three or
    // four of width 64 fit at once, two of 128, one of more); else four times as many of them (sequences differ in length), of as many steps that a part's sums (8 bytes to a row and dimension, written and read) are a
    // sixteenth of its keys and values at most.  Many rows write 64 KiB of sums a part: one workgroup to a compute unit (48
    // sequences behind a prefix of 8197: 66 us with a quarter as many, 48, 52 with half as many again, 54 with twice), of
    // four steps at least.
    const long long slots = (row_tiles ? 3LL : 1LL) * cus;
    long long take;
    if (row_tiles) {
        const long long in_block = rows < 16 * row_tiles ? rows : 16 * row_tiles, least = in_block > 8 ? in_block / 4 : 2;
        take = groups * steps <= slots ? 1 : div_up(groups * steps, 4 * slots);
        take = take < least && groups * steps > slots ? least : take;
    } else {
        const long long parts = groups < slots ? slots / groups : 1;
        take = div_up(steps, parts);
        take = take < 4 ? 4 : take;
    }
    if (div_up(steps, take) > MAX_PARTS)
        take = div_up(steps, MAX_PARTS);
    long long most = row_tiles ? 4 * slots / groups + 1 : slots / groups;
    most = most > steps ? steps : most < 1 ? 1 : most;
    most_parts += (int)(most > MAX_PARTS ? MAX_PARTS : most);
    w.chunk = (int)(take < steps ? take : steps) * step;
    w.parts = div_up(keys > 0 ? keys : 1, w.chunk);
    const long long in_all = groups * w.parts;
    w.blocks = in_all < FQ_ATTEND_BLOCKS ? (uint32_t)in_all : FQ_ATTEND_BLOCKS;
    w.blocks_x = (uint32_t)(blocks / seqs * a.kv.kv_heads);
    return w;
}

Plan plan(const FqAttendArgs &a, int cus)
{
    const long long group = a.q_heads / a.kv.kv_heads;
    const int P = a.seqs.prefix_len;
    Plan pl{};
    if (P > 0 && a.seqs.seqs > 1 && a.max_q * group < 64) {
        int &t0 = pl.row_tiles[0], &t1 = pl.row_tiles[1];
        t0 = tiles_of(a, a.seqs.tokens * group); // 0 where the batch has more rows than the kernel of few rows takes
        t1 = t0 ? t0 : tiles_of(a, a.max_q * group); // (a sequence has no more than the batch: the same tiles serve both)
        pl.work[0] = work(a, true, 0, P, 1, a.seqs.tokens, t0, cus, pl.most_parts);
        pl.work[1] = work(a, false, P, a.max_kv, a.seqs.seqs, a.max_q, t1, cus, pl.most_parts);
        pl.n = 2;
    } else {
        pl.row_tiles[0] = pl.row_tiles[1] = tiles_of(a, a.max_q * group);
        pl.work[0] = work(a, false, 0, (long long)P + a.max_kv, a.seqs.seqs, a.max_q, pl.row_tiles[0], cus, pl.most_parts);
        pl.n = 1;
    }
    for (int i = 0; i < pl.n; i++) {
        pl.work[i].part0 = pl.parts;
        pl.parts += pl.work[i].parts;
    }
    return pl;
}

size_t bytes(const FqAttendArgs &a, int parts)
{
    if (parts == 1)
        return 256;
    const size_t rows = (size_t)a.seqs.tokens * a.q_heads;
    return (rows * parts * (a.kv.dim * sizeof(float) + sizeof(float2)) + 255) & ~(size_t)255;
}

// The parts of a row, added up.  dim / 4 threads take 4 dimensions each of every `lanes`-th part, each with a reference of its own;
// then the lanes are added up through LDS in their order.  (One thread walking all parts waited for each load in turn: 196
// parts took 160 us of 186 for one token of the 70B shapes behind 100000.)
__global__ __launch_bounds__(256) void attend_join_kernel(FqAttendArgs a, FqAttendWork w0, FqAttendWork w1, int n, int lanes)
{
    __shared__ float4_t sums[256];
    __shared__ float2 stats[256];
    const int per = a.kv.dim >> 2, rows_wg = 256 / (per * lanes);
    const int unit = threadIdx.x / per, mine = unit / lanes, lane = unit - mine * lanes;
    const int d = (threadIdx.x - unit * per) << 2, b = blockIdx.z;
    const FqSeq s = fq_seq(a.seqs, a.kv.page_shift, b);
    const int rows = min(s.n, a.max_q) * a.q_heads;
    const int r = blockIdx.x * rows_wg + mine;
    if ((int)blockIdx.x * rows_wg >= rows)
        return;
    const bool real = mine < rows_wg && r < rows;
    const int j = real ? r / a.q_heads : 0, h = real ? r - j * a.q_heads : 0;
    const long long t = s.q0 + j, row = t * a.q_heads + h, rows_all = (long long)a.seqs.tokens * a.q_heads;
    float m = -INFINITY, l = 0.0f;
    float4_t o = {0, 0, 0, 0};
    if (real) {
        const int P = a.seqs.prefix_len, lim = P + min(max(s.len - s.n + j + 1, 0), a.max_kv);
        // parts that hold keys this row sees: the first `have0`, and `have1` from parts0 on
        const int parts0 = w0.parts, parts1 = w1.parts;
        const int have0 = w0.shared ? parts0 : min(parts0, lim > w0.key0 ? (lim - w0.key0 - 1) / w0.chunk + 1 : 0);
        const int have1 = n > 1 ? min(parts1, lim > w1.key0 ? (lim - w1.key0 - 1) / w1.chunk + 1 : 0) : 0;
        const int have = have0 + have1;
        constexpr int AHEAD = 4;
        for (int p0 = lane; p0 < have; p0 += AHEAD * lanes) {
            float2 ml[AHEAD];
            float4_t x[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; i++) {
                const int p = p0 + i * lanes;
                ml[i] = float2{-INFINITY, 0.0f};
                x[i] = float4_t{0, 0, 0, 0};
                if (p < have) {
                    const long long at = (p < have0 ? p : parts0 + p - have0) * rows_all + row;
                    ml[i] = w0.part_ml[at];
                    x[i] = *(const float4_t *)(w0.part_o + at * a.kv.dim + d);
                }
            }
            float top = m;
#pragma unroll
            for (int i = 0; i < AHEAD; i++)
                top = fmaxf(top, ml[i].x);
            const float ref = fq_reference(top), fall = __builtin_amdgcn_exp2f(m - ref);
            m = top;
            l *= fall;
            o *= fall;
#pragma unroll
            for (int i = 0; i < AHEAD; i++) {
                const float f = __builtin_amdgcn_exp2f(ml[i].x - ref);
                l += ml[i].y * f;
                o += x[i] * f;
            }
        }
    }
    sums[threadIdx.x] = o;
    stats[threadIdx.x] = float2{m, l};
    __syncthreads();
    if (!real || lane != 0)
        return;
    for (int i = 1; i < lanes; i++)
        m = fmaxf(m, stats[threadIdx.x + i * per].x);
    const float ref = fq_reference(m);
    l = 0.0f;
    o = float4_t{0, 0, 0, 0};
    for (int i = 0; i < lanes; i++) {
        const float2 ml = stats[threadIdx.x + i * per];
        const float f = __builtin_amdgcn_exp2f(ml.x - ref);
        l += ml.y * f;
        o += sums[threadIdx.x + i * per] * f;
    }
    const float inv = fq_inverse(l);
    u32x2 y;
    if (a.kv.bf16)
        y = u32x2{fq_pack2<true>(o[0] * inv, o[1] * inv), fq_pack2<true>(o[2] * inv, o[3] * inv)};
    else
        y = u32x2{fq_pack2<false>(o[0] * inv, o[1] * inv), fq_pack2<false>(o[2] * inv, o[3] * inv)};
    *(u32x2 *)(a.out + t * a.out_stride + h * a.kv.dim + d) = y;
    if (d == 0 && a.lse)
        a.lse[row] = fq_lse(m, l);
}

} // namespace

size_t fq_attend_bytes(const FqAttendArgs &a, bool for_fewer_keys, int cus)
{
    const Plan pl = plan(a, cus);
    return bytes(a, for_fewer_keys ? pl.most_parts : pl.parts);
}

hipError_t fq_launch_attend(const FqAttendArgs &a, void *workspace, hipStream_t stream)
{
    Plan pl = plan(a, fq_device_cus());
    if (pl.work[0].blocks + pl.work[1].blocks >= FQ_ATTEND_BLOCKS)
        return hipErrorInvalidConfiguration; // a launch has 2^32 threads at most
    const size_t rows = (size_t)a.seqs.tokens * a.q_heads;
    for (int i = 0; i < pl.n; i++)
        if (pl.parts > 1) {
            pl.work[i].part_o = (float *)workspace;
            pl.work[i].part_ml = (float2 *)((float *)workspace + rows * pl.parts * a.kv.dim);
        }
    const hipError_t e = (a.kv.bf16 ? fq_launch_attend_bf16 : fq_launch_attend_f16)(a, pl.work[0], pl.work[1], pl.row_tiles[0], pl.row_tiles[1],
                                                                                    stream);
    if (e != hipSuccess)
        return e;
    if (pl.parts == 1)
        return hipSuccess;
    const int per = a.kv.dim / 4;
    int lanes = 1; // of a row: as many as take four parts each at least, where a workgroup has them
    while (lanes * 4 < pl.parts && per * lanes * 2 <= 256)
        lanes *= 2;
    const dim3 grid(div_up((long long)a.max_q * a.q_heads, 256 / (per * lanes)), 1, a.seqs.seqs);
    attend_join_kernel<<<grid, 256, 0, stream>>>(a, pl.work[0], pl.work[1], pl.n, lanes);
    return hipGetLastError();
}
