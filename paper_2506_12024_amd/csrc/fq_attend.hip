// Attention of new tokens over a paged cache: which kernel takes which rows, how the keys are split, and the sum of the parts.
#include "fq_attend.h"

namespace {

// What one call launches.  The rows of a sequence and a key head share its keys; where they are few, the rows of the whole
// batch share the prefix besides, and the prefix is a launch of its own.
struct Piece {
    FqAttendWork work;
    int row_tiles; // 0: the kernel for many rows
    dim3 grid;
};
struct Plan {
    int n, parts;
    Piece piece[2];
};

int div_up(long long a, long long b) { return (int)((a + b - 1) / b); }

Piece piece(const FqAttendArgs &a, bool shared, int key0, long long keys, int seqs, int tokens, int cus)
{
    const long long rows = (long long)tokens * (a.q_heads / a.kv.kv_heads);
    Piece p{};
    const int few = a.kv.dim <= 96 || a.kv.dim == 128 ? 64 : 32; // (the registers of a wider head hold 32 rows)
    p.row_tiles = rows > few ? 0 : rows > 32 ? 4 : rows > 16 ? 2 : 1;
    const int step = p.row_tiles ? 128 : 64; // keys that a workgroup takes at once
    p.work.shared = shared;
    p.work.key0 = key0;
    p.work.row_blocks = div_up(rows, p.row_tiles ? 16 * p.row_tiles : FQ_MANY_ROWS);
    const long long groups = (long long)p.work.row_blocks * a.kv.kv_heads * seqs;
    // parts: enough workgroups to fill the chip several times over, of a few steps each at least
    const long long want = (p.row_tiles ? 12LL : 4LL) * cus;
    long long parts = div_up(want, groups);
    const long long most = div_up(keys, 4 * step);
    parts = parts < 1 ? 1 : parts > most ? (most < 1 ? 1 : most) : parts;
    if (parts > 256)
        parts = 256;
    p.work.chunk = div_up(div_up(keys > 0 ? keys : 1, parts), step) * step;
    const int chunks = div_up(keys > 0 ? keys : 1, p.work.chunk);
    p.grid = dim3((unsigned)(p.work.row_blocks * a.kv.kv_heads), chunks, seqs);
    return p;
}

Plan plan(const FqAttendArgs &a, int cus)
{
    const int group = a.q_heads / a.kv.kv_heads, P = a.seqs.prefix_len;
    Plan pl{};
    if (P > 0 && a.seqs.seqs > 1 && (long long)a.max_q * group < 64) {
        pl.piece[0] = piece(a, true, 0, P, 1, a.seqs.tokens, cus);
        pl.piece[1] = piece(a, false, P, a.max_kv, a.seqs.seqs, a.max_q, cus);
        pl.n = 2;
    } else {
        pl.piece[0] = piece(a, false, 0, (long long)P + a.max_kv, a.seqs.seqs, a.max_q, cus);
        pl.n = 1;
    }
    for (int i = 0; i < pl.n; i++) {
        pl.piece[i].work.part0 = pl.parts;
        pl.parts += pl.piece[i].grid.y;
    }
    return pl;
}

size_t bytes(const FqAttendArgs &a, const Plan &pl)
{
    if (pl.parts == 1)
        return 256;
    const size_t rows = (size_t)a.seqs.tokens * a.q_heads;
    return (rows * pl.parts * (a.kv.dim * sizeof(float) + sizeof(float2)) + 255) & ~(size_t)255;
}

// The parts of a row, added up in their order: a thread takes 4 dimensions of a row, 256 / (dim / 4) rows to a workgroup.
__global__ __launch_bounds__(256) void attend_join_kernel(FqAttendArgs a, FqAttendWork w0, FqAttendWork w1, int n, int parts0, int parts1)
{
    const int per = a.kv.dim >> 2, rows_wg = 256 / per;
    const int mine = threadIdx.x / per, d = (threadIdx.x - mine * per) << 2, b = blockIdx.z;
    const FqSeq s = fq_seq(a.seqs, a.kv.page_shift, b);
    const long long r = (long long)blockIdx.x * rows_wg + mine;
    if (mine >= rows_wg || r >= (long long)min(s.n, a.max_q) * a.q_heads)
        return;
    const int j = (int)(r / a.q_heads);
    const long long t = s.q0 + j, row = t * a.q_heads + r % a.q_heads, rows_all = (long long)a.seqs.tokens * a.q_heads;
    const int P = a.seqs.prefix_len, lim = P + min(max(s.len - s.n + j + 1, 0), a.max_kv);
    // parts that hold keys this row sees
    int have[2];
    have[0] = w0.shared ? parts0 : min(parts0, lim > w0.key0 ? (lim - w0.key0 - 1) / w0.chunk + 1 : 0);
    have[1] = n > 1 ? min(parts1, lim > w1.key0 ? (lim - w1.key0 - 1) / w1.chunk + 1 : 0) : 0;
    float m = -INFINITY;
    for (int i = 0; i < 2; i++)
        for (int p = 0; p < have[i]; p++)
            m = fmaxf(m, w0.part_ml[((i ? parts0 : 0) + p) * rows_all + row].x);
    const float ref = fq_reference(m);
    float l = 0.0f;
    float4_t o = {0, 0, 0, 0};
    for (int i = 0; i < 2; i++)
        for (int p = 0; p < have[i]; p++) {
            const long long at = ((i ? parts0 : 0) + p) * rows_all + row;
            const float2 ml = w0.part_ml[at];
            const float f = __builtin_amdgcn_exp2f(ml.x - ref);
            l += ml.y * f;
            o += *(const float4_t *)(w0.part_o + at * a.kv.dim + d) * f;
        }
    const float inv = fq_inverse(l);
    uint16_t *to = a.out + t * a.out_stride + r % a.q_heads * a.kv.dim + d;
    u32x2 y;
    if (a.kv.bf16)
        y = u32x2{fq_pack2<true>(o[0] * inv, o[1] * inv), fq_pack2<true>(o[2] * inv, o[3] * inv)};
    else
        y = u32x2{fq_pack2<false>(o[0] * inv, o[1] * inv), fq_pack2<false>(o[2] * inv, o[3] * inv)};
    *(u32x2 *)to = y;
    if (d == 0 && a.lse)
        a.lse[row] = fq_lse(m, l);
}

} // namespace

size_t fq_attend_bytes(const FqAttendArgs &a, int cus) { return bytes(a, plan(a, cus)); }

hipError_t fq_launch_attend(const FqAttendArgs &a, void *workspace, hipStream_t stream)
{
    Plan pl = plan(a, fq_device_cus());
    const size_t rows = (size_t)a.seqs.tokens * a.q_heads;
    for (int i = 0; i < pl.n; i++) {
        if (pl.parts > 1) {
            pl.piece[i].work.part_o = (float *)workspace;
            pl.piece[i].work.part_ml = (float2 *)((float *)workspace + rows * pl.parts * a.kv.dim);
        }
        const Piece &p = pl.piece[i];
        const hipError_t e = p.row_tiles ? fq_launch_attend_few(a, p.work, p.row_tiles, p.grid, stream)
                                         : fq_launch_attend_many(a, p.work, p.grid, stream);
        if (e != hipSuccess)
            return e;
    }
    if (pl.parts == 1)
        return hipSuccess;
    const int rows_wg = 256 / (a.kv.dim / 4);
    const dim3 grid(div_up((long long)a.max_q * a.q_heads, rows_wg), 1, a.seqs.seqs);
    attend_join_kernel<<<grid, 256, 0, stream>>>(a, pl.piece[0].work, pl.piece[1].work, pl.n, pl.piece[0].grid.y,
                                                 pl.n > 1 ? pl.piece[1].grid.y : 0);
    return hipGetLastError();
}
