// Low-rank adapters of many requests beside a projection that they share: out = y + scale (x A^T) B^T, row by row.
//
// Both products are on the matrix cores, in two launches: `low_kernel` forms u = x A^T, its K split over the wavefronts of a workgroup and over
// workgroups, whose parts (binary32) lie in the workspace; `out_kernel` adds them up, and B meets them as two 16-bit numbers each, u =
// hi + lo (binary16: 22 bits of it, a row scaled by a power of two so that its largest fills the range; bfloat16: 17), so that x A^T is
// nowhere rounded to 16 bits.  A tile is up to 16 or 64 rows of one slot, wherever in the call they stand: a row's sums do not
// depend on its place in a tile.  Up to SMALL_ROWS rows every workgroup finds its tile itself (the row it is numbered by leads a tile if
// the rows of its slot before it fill whole ones); for more a launch of one workgroup sorts the rows by slot first.
#include <hip/hip_runtime.h>

#include "../../include/flexq.h"
#include "fq_kv.h"

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int SMALL_ROWS = 256, SMALL_TILE = 16, TILE = 64;
constexpr int GROUP_THREADS = 1024;

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <bool BF16>
__device__ __forceinline__ float4_t mfma(u32x4 a, u32x4 b, float4_t c)
{
    if (BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8_t, a), __builtin_bit_cast(bf8_t, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
}

// The workspace: the parts of u, [part][row][rank]; for more than SMALL_ROWS rows the rows in the order of their slots and the tiles.
struct Tile {
    int slot, from, count, pad; // slot: -1 for rows without an adapter
};
struct Work {
    float *low;
    int *order;
    Tile *tiles;
    int parts, max_tiles;
};

int tiles_of(const FqAdaptersView &set, int M) // at most
{
    return M <= SMALL_ROWS ? M : M / TILE + (M < set.slots + 1 ? M : set.slots + 1);
}

// Parts of K: workgroups for the whole chip while rows are few, at least a step of 64 to each wavefront.
int parts_of(const FqAdaptersView &set, int M)
{
    const int tiles = M <= SMALL_ROWS ? M : (M + TILE - 1) / TILE;
    int parts = 512 / tiles;
    parts = parts > 16 ? 16 : M <= SMALL_ROWS && parts < 4 ? 4 : parts < 1 ? 1 : parts;
    const int most = (set.K + 64 * WAVES - 1) / (64 * WAVES);
    return parts < most ? parts : most;
}

// Rows times parts, from above and never less for more rows: what parts_of gives is at most this.
size_t low_rows(int M)
{
    const size_t m = M, few = M <= SMALL_ROWS ? (4 * m > 512 ? 4 * m : 512) : (m > 512 * TILE ? m : 512 * TILE);
    return 16 * m < few ? 16 * m : few;
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// A row's adapter, or -1.
__device__ __forceinline__ int slot_of(const FqAdaptersArgs &a, int m)
{
    const int s = a.adapter[m];
    return s >= 0 && s < a.set.slots ? s : -1;
}

__device__ __forceinline__ int rank_of(const FqAdaptersArgs &a, int slot)
{
    if (slot < 0)
        return 0;
    return a.set.ranks ? min(max(a.set.ranks[slot], 0), a.set.rank) : a.set.rank;
}

// The rows of this workgroup's tile into LDS; its slot through `slot`; the number of rows, 0 if there is no tile.
template <bool SMALL>
__device__ __forceinline__ int find_tile(const FqAdaptersArgs &a, const Work &w, int *rows, int &slot)
{
    const int tid = threadIdx.x, lane = tid & 63;
    if (!SMALL) {
        const Tile t = w.tiles[blockIdx.x];
        slot = t.slot;
        if (tid < t.count)
            rows[tid] = w.order[t.from + tid];
        __syncthreads();
        return t.count;
    }
    const int own = blockIdx.x;
    slot = slot_of(a, own);
    int found[SMALL_ROWS / 64];
#pragma unroll
    for (int c = 0; c < SMALL_ROWS / 64; c++)
        found[c] = 64 * c + lane < a.M ? slot_of(a, 64 * c + lane) : -2;
    int before = 0, seen = 0, count = 0;
    uint64_t mask[SMALL_ROWS / 64];
#pragma unroll
    for (int c = 0; c < SMALL_ROWS / 64; c++) {
        mask[c] = __ballot(found[c] == slot);
        const int upto = own - 64 * c;
        before += __popcll(upto <= 0 ? 0 : upto >= 64 ? mask[c] : mask[c] & ((1ull << upto) - 1));
    }
    if (before % SMALL_TILE != 0)
        return 0;
#pragma unroll
    for (int c = 0; c < SMALL_ROWS / 64; c++) {
        const int at = seen + __popcll(mask[c] & ((1ull << lane) - 1)) - before;
        if (tid < 64 && found[c] == slot && at >= 0 && at < SMALL_TILE)
            rows[at] = 64 * c + lane;
        seen += __popcll(mask[c]);
    }
    count = min(seen - before, SMALL_TILE);
    __syncthreads();
    return count;
}

// One workgroup: rows counted by slot, slots' first places and tiles, rows put in order.  (The order of a slot's rows among themselves
// does not show: a row's sums are the same anywhere in a tile.)
__global__ __launch_bounds__(GROUP_THREADS) void group_kernel(FqAdaptersArgs a, Work w)
{
    extern __shared__ int count[]; // slots + 1: the last for rows without one
    __shared__ int sums[2][GROUP_THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, keys = a.set.slots + 1;
    for (int i = tid; i < keys; i += GROUP_THREADS)
        count[i] = 0;
    __syncthreads();
    // the place of a row among its slot's, as far as they have come; a wavefront whose rows are all of one slot asks once
    auto take = [&](int key) {
        const uint64_t live = __ballot(true);
        const int first = __builtin_amdgcn_readfirstlane(key);
        if (__ballot(key == first) == live) {
            int from = 0;
            if (lane == __ffsll((unsigned long long)live) - 1)
                from = atomicAdd(&count[key], (int)__popcll(live));
            from = __builtin_amdgcn_readfirstlane(from);
            return from + (int)__popcll(live & ((1ull << lane) - 1));
        }
        return atomicAdd(&count[key], 1);
    };
    for (int m = tid; m < a.M; m += GROUP_THREADS) {
        const int s = slot_of(a, m);
        take(s < 0 ? keys - 1 : s);
    }
    __syncthreads();
    int rows = 0, tiles = 0; // of the slots before these
    for (int k0 = 0; k0 < keys; k0 += GROUP_THREADS) {
        const int k = k0 + tid, n = k < keys ? count[k] : 0, t = (n + TILE - 1) / TILE;
        int row = n, tile = t;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int r = __shfl_up(row, off, 64), q = __shfl_up(tile, off, 64);
            if (lane >= off) {
                row += r;
                tile += q;
            }
        }
        if (lane == 63) {
            sums[0][wave] = row;
            sums[1][wave] = tile;
        }
        __syncthreads();
        int all_rows = 0, all_tiles = 0;
        for (int v = 0; v < GROUP_THREADS / 64; v++) {
            if (v == wave) {
                row += all_rows;
                tile += all_tiles;
            }
            all_rows += sums[0][v];
            all_tiles += sums[1][v];
        }
        row += rows - n;
        tile += tiles - t;
        if (k < keys) {
            count[k] = row;
            for (int i = 0; i < t; i++)
                w.tiles[tile + i] = Tile{k == keys - 1 ? -1 : k, row + i * TILE, min(n - i * TILE, TILE), 0};
        }
        rows += all_rows;
        tiles += all_tiles;
        __syncthreads();
    }
    for (int i = tiles + tid; i < w.max_tiles; i += GROUP_THREADS)
        w.tiles[i] = Tile{-1, 0, 0, 0};
    for (int m = tid; m < a.M; m += GROUP_THREADS) {
        const int s = slot_of(a, m);
        w.order[take(s < 0 ? keys - 1 : s)] = m;
    }
}

// u = x A^T of a tile: TT * 16 rows, RT * 16 ranks from 16 RT blockIdx.z on, the part blockIdx.y of K.  A step is 64 of K, of which a lane has
// 16 that follow each other (32 bytes of its row of x and of A): 128 bytes of a row to four lanes.
template <int TT, int RT, bool BF16>
__global__ __launch_bounds__(THREADS) void low_kernel(FqAdaptersArgs a, Work w)
{
    constexpr bool SMALL = TT == 1;
    __shared__ int rows[16 * TT];
    __shared__ float4_t sums[WAVES / 2][TT * RT][64];
    int slot;
    const int count = find_tile<SMALL>(a, w, rows, slot);
    const int rank = rank_of(a, slot), r0 = 16 * RT * blockIdx.z;
    if (count == 0 || r0 >= rank)
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const uint16_t *xp[TT], *ap[RT];
#pragma unroll
    for (int t = 0; t < TT; t++)
        xp[t] = a.x + rows[16 * t + col < count ? 16 * t + col : 0] * a.x_stride + 16 * g;
#pragma unroll
    for (int r = 0; r < RT; r++)
        ap[r] = a.set.a + slot * a.set.a_stride + (size_t)min(r0 + 16 * r + col, rank - 1) * a.set.K + 16 * g;
    float4_t acc[TT][RT] = {};
    const int K = a.set.K, steps = (K + 63) / 64;
    const int stride = WAVES * gridDim.y;
    struct Step {
        u32x4 x[TT][2], a[RT][2];
    };
    auto ask = [&](Step &s, int step) {
        const int k = 64 * step;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const bool in = k + 16 * g + 8 * h < K;
#pragma unroll
            for (int t = 0; t < TT; t++)
                s.x[t][h] = in ? *(const u32x4 *)(xp[t] + k + 8 * h) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int r = 0; r < RT; r++)
                s.a[r][h] = in ? *(const u32x4 *)(ap[r] + k + 8 * h) : u32x4{0, 0, 0, 0};
        }
    };
    Step now, next;
    int step = wave + WAVES * blockIdx.y;
    if (step < steps)
        ask(now, step);
    for (; step < steps; step += stride) {
        if (step + stride < steps)
            ask(next, step + stride);
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int t = 0; t < TT; t++)
#pragma unroll
                for (int r = 0; r < RT; r++)
                    acc[t][r] = mfma<BF16>(now.a[r][h], now.x[t][h], acc[t][r]);
        now = next;
    }
    // the wavefronts' sums, in one order
    if (wave >= WAVES / 2) {
#pragma unroll
        for (int i = 0; i < TT * RT; i++)
            sums[wave - WAVES / 2][i][lane] = acc[i / RT][i % RT];
    }
    __syncthreads();
    if (wave < WAVES / 2) {
#pragma unroll
        for (int i = 0; i < TT * RT; i++)
            acc[i / RT][i % RT] += sums[wave][i][lane];
    }
    __syncthreads();
    if (wave == 1) {
#pragma unroll
        for (int i = 0; i < TT * RT; i++)
            sums[0][i][lane] = acc[i / RT][i % RT];
    }
    __syncthreads();
    if (wave == 0) {
#pragma unroll
        for (int t = 0; t < TT; t++) {
            if (16 * t + col >= count)
                continue;
            float *to = w.low + ((size_t)blockIdx.y * a.M + rows[16 * t + col]) * a.set.rank + r0 + 4 * g;
#pragma unroll
            for (int r = 0; r < RT; r++)
                if (r0 + 16 * r + 4 * g < a.set.rank)
                    *(float4_t *)(to + 16 * r) = acc[t][r] + sums[0][t * RT + r][lane];
        }
    }
}

// out = y + scale u B^T of a tile, blocks of 64 outputs to a wavefront.  u lies in LDS as the second operands' registers, 32 ranks
// to an instruction, hi and lo.  Row i of a first operand is output 16 (i / 4) + 4 j + i % 4 of the block in instruction j of four, so that a lane's results
// of the four are 16 outputs of its row that follow each other.
template <int TT, bool BF16, bool VEC>
__global__ __launch_bounds__(THREADS) void out_kernel(FqAdaptersArgs a, Work w)
{
    constexpr bool SMALL = TT == 1;
    __shared__ int rows[16 * TT];
    extern __shared__ u32x4 low[]; // [rank / 32][TT][2][64]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
    int slot;
    const int count = find_tile<SMALL>(a, w, rows, slot);
    if (count == 0)
        return;
    const int rank = rank_of(a, slot), N = a.set.N;
    const int first = blockIdx.y * WAVES + wave, stride = gridDim.y * WAVES, blocks = (N + 63) / 64;
    if (rank == 0) {
        if (a.out == a.y && a.out_stride == a.y_stride)
            return;
        for (int b = first; b < blocks; b += stride)
            if (64 * b + lane < N)
                for (int i = 0; i < count; i++)
                    a.out[rows[i] * a.out_stride + 64 * b + lane] = a.y[rows[i] * a.y_stride + 64 * b + lane];
        return;
    }
    const int chunks = (rank + 31) / 32;
    __shared__ float factor[16 * TT];
    // 16 threads to a row, 4 ranks to a thread and turn
    for (int row = tid >> 4; row < 16 * TT; row += THREADS / 16) {
        const int m = rows[row < count ? row : 0];
        const float *from = w.low + (size_t)m * a.set.rank;
        float4_t u[FQ_MAX_ADAPTER_RANK / 64];
        float most = 0.0f;
#pragma unroll
        for (int c = 0; c < FQ_MAX_ADAPTER_RANK / 64; c++) {
            const int r = 64 * c + 4 * (tid & 15);
            u[c] = float4_t{0, 0, 0, 0};
            if (64 * c < rank && r < rank) {
                for (int p = 0; p < w.parts; p++)
                    u[c] += *(const float4_t *)(from + (size_t)p * a.M * a.set.rank + r);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    u[c][i] = r + i < rank ? u[c][i] : 0.0f;
                    most = fmaxf(most, fabsf(u[c][i]) < INFINITY ? fabsf(u[c][i]) : 0.0f);
                }
            }
        }
#pragma unroll
        for (int off = 8; off >= 1; off >>= 1)
            most = fmaxf(most, __shfl_xor(most, off, 64));
        // binary16: the row's largest becomes 2^13 to 2^14 (a power of two changes no digit)
        const int e = BF16 || most == 0.0f ? 0 : min(max(14 - __builtin_amdgcn_frexp_expf(most), -126), 126);
        if ((tid & 15) == 0)
            factor[row] = ldexpf(a.set.scales ? a.set.scales[slot] : 1.0f, -e);
#pragma unroll
        for (int c = 0; c < FQ_MAX_ADAPTER_RANK / 64; c++) {
            const int r = 64 * c + 4 * (tid & 15);
            if (64 * c < rank && r < 32 * chunks) {
                uint16_t hi[4], lo[4];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float v = BF16 ? u[c][i] : ldexpf(u[c][i], e);
                    hi[i] = fq_from_float(v, BF16);
                    const float rest = v - fq_to_float(hi[i], BF16);
                    lo[i] = fabsf(rest) < INFINITY ? fq_from_float(rest, BF16) : 0; // (not where hi is infinite or NaN)
                }
                // operand: lane col + 16 (rank % 32 / 8), its 8 ranks
                uint2 *at = (uint2 *)&low[((r >> 5) * TT + (row >> 4)) * 128 + (row & 15) + 16 * ((r & 31) >> 3)];
                at[(r & 7) >> 2] = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
                at[128 + ((r & 7) >> 2)] = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
            }
        }
    }
    __syncthreads();
    const uint16_t *bp = a.set.b + slot * a.set.b_stride;
    for (int b = first; b < blocks; b += stride) {
        const int n0 = 64 * b;
        float4_t acc[TT][4] = {};
        for (int c = 0; c < chunks; c++) {
            const int r = 32 * c + 8 * g;
            u32x4 bv[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int n = n0 + 16 * (col >> 2) + 4 * j + (col & 3);
                bv[j] = n < N && r < rank ? *(const u32x4 *)(bp + (size_t)n * a.set.rank + r) : u32x4{0, 0, 0, 0};
            }
            if (rank & 7) { // (what lies behind a rank may be anything)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const uint32_t mask = (r + 2 * i < rank ? 0xffffu : 0u) | (r + 2 * i + 1 < rank ? 0xffff0000u : 0u);
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        bv[j][i] &= mask;
                }
            }
#pragma unroll
            for (int t = 0; t < TT; t++) {
                const u32x4 hi = low[(c * TT + t) * 128 + lane], lo = low[(c * TT + t) * 128 + 64 + lane];
#pragma unroll
                for (int j = 0; j < 4; j++)
                    acc[t][j] = mfma<BF16>(bv[j], lo, mfma<BF16>(bv[j], hi, acc[t][j]));
            }
        }
        const int n = n0 + 16 * g;
#pragma unroll
        for (int t = 0; t < TT; t++) {
            if (16 * t + col >= count)
                continue;
            const long long m = rows[16 * t + col];
            const uint16_t *y = a.y + m * a.y_stride + n;
            uint16_t *out = a.out + m * a.out_stride + n;
            const float f = factor[16 * t + col];
            if (VEC) {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    if (n + 8 * h >= N)
                        continue;
                    u32x4 v = *(const u32x4 *)(y + 8 * h);
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const float4_t s = acc[t][2 * h + i / 2];
                        const uint16_t p = fq_from_float(fq_to_float((uint16_t)v[i], BF16) + f * s[2 * (i & 1)], BF16);
                        const uint16_t q = fq_from_float(fq_to_float((uint16_t)(v[i] >> 16), BF16) + f * s[2 * (i & 1) + 1], BF16);
                        v[i] = p | (uint32_t)q << 16;
                    }
                    *(u32x4 *)(out + 8 * h) = v;
                }
            } else {
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (n + i < N)
                        out[i] = fq_from_float(fq_to_float(y[i], BF16) + f * acc[t][i >> 2][i & 3], BF16);
            }
        }
    }
}

template <int TT, bool BF16>
hipError_t launch(const FqAdaptersArgs &a, const Work &w, hipStream_t stream)
{
    const int ranks = a.set.rank, rt = ranks <= 16 ? 1 : ranks <= 32 ? 2 : 4;
    const dim3 low_grid(w.max_tiles, w.parts, (ranks + 16 * rt - 1) / (16 * rt));
    if (rt == 1)
        low_kernel<TT, 1, BF16><<<low_grid, THREADS, 0, stream>>>(a, w);
    else if (rt == 2)
        low_kernel<TT, 2, BF16><<<low_grid, THREADS, 0, stream>>>(a, w);
    else
        low_kernel<TT, 4, BF16><<<low_grid, THREADS, 0, stream>>>(a, w);
    if (hipError_t e = hipGetLastError())
        return e;
    const bool vec = a.set.N % 8 == 0 && a.y_stride % 8 == 0 && a.out_stride % 8 == 0 && ((uintptr_t)a.y & 15) == 0 && ((uintptr_t)a.out & 15) == 0;
    const int blocks = (a.set.N + 63) / 64, tiles = TT == 1 ? a.M : (a.M + TILE - 1) / TILE;
    // outputs over as many workgroups as fill the chip
    const int most = (blocks + WAVES - 1) / WAVES, room = (512 + tiles - 1) / tiles;
    const dim3 out_grid(w.max_tiles, most < room ? most : room);
    const size_t lds = (size_t)(ranks + 31) / 32 * TT * 2 * 64 * sizeof(u32x4);
    const void *func = vec ? (const void *)out_kernel<TT, BF16, true> : (const void *)out_kernel<TT, BF16, false>;
    if (hipError_t e = fq_raise_dynamic_lds(func, lds))
        return e;
    if (vec)
        out_kernel<TT, BF16, true><<<out_grid, THREADS, lds, stream>>>(a, w);
    else
        out_kernel<TT, BF16, false><<<out_grid, THREADS, lds, stream>>>(a, w);
    return hipGetLastError();
}

} // namespace

size_t fq_adapters_bytes(const FqAdaptersView &set, int M)
{
    const size_t low = up(low_rows(M) * set.rank * sizeof(float));
    return M <= SMALL_ROWS ? low + 256 : low + 256 + up((size_t)M * sizeof(int)) + up(tiles_of(set, M) * sizeof(Tile));
}

hipError_t fq_launch_adapters(const FqAdaptersArgs &a, void *workspace, hipStream_t stream)
{
    Work w{};
    char *at = (char *)workspace;
    w.low = (float *)at;
    at += up(low_rows(a.M) * a.set.rank * sizeof(float));
    w.order = (int *)at;
    w.tiles = (Tile *)(at + up((size_t)a.M * sizeof(int)));
    w.parts = parts_of(a.set, a.M);
    w.max_tiles = tiles_of(a.set, a.M);
    if (a.M <= SMALL_ROWS)
        return a.set.bf16 ? launch<1, true>(a, w, stream) : launch<1, false>(a, w, stream);
    const size_t lds = (a.set.slots + 1) * sizeof(int);
    if (hipError_t e = fq_raise_dynamic_lds((const void *)group_kernel, lds))
        return e;
    group_kernel<<<1, GROUP_THREADS, lds, stream>>>(a, w);
    if (hipError_t e = hipGetLastError())
        return e;
    return a.set.bf16 ? launch<4, true>(a, w, stream) : launch<4, false>(a, w, stream);
}
