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
constexpr int MIDDLE_ROWS = 4096, MIDDLE_SLOTS = 1023;
constexpr int GROUP_THREADS = 1024, MANY_THREADS = 512;
constexpr int CHUNK = 256, MAX_PARTS = 16; // of K
enum Find { ALONE, COUNTED, LISTED }; // how a workgroup finds its tile: of few rows; of MIDDLE_ROWS; in the workspace's list

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

// The workspace: the parts of u, [part][row][rank], and the tiles, whose rows are rows[TILE * tile] and on.
struct Tile {
    int slot, count, rank; // slot -1, rank 0: rows without an adapter
    float scale;
};
struct Work {
    float *low;
    int *rows;
    Tile *tiles;
    int parts, max_tiles;
};

int tiles_of(const FqAdaptersView &set, int M) // at most
{
    return M <= SMALL_ROWS ? M : M / TILE + (M < set.slots + 1 ? M : set.slots + 1);
}

// Parts of K: workgroups for the whole chip while rows are few, at least a chunk to each.
int parts_of(const FqAdaptersView &set, int M)
{
    const int tiles = M <= SMALL_ROWS ? M : (M + TILE - 1) / TILE, room = 256;
    int parts = room / tiles;
    parts = parts > MAX_PARTS ? MAX_PARTS : M <= SMALL_ROWS && parts < 4 ? 4 : parts < 1 ? 1 : parts;
    const int most = (set.K + CHUNK - 1) / CHUNK;
    return parts < most ? parts : most;
}

// Rows times parts, from above and never less for more rows: what parts_of gives is at most this.
size_t low_rows(int M)
{
    const size_t m = M, few = M <= SMALL_ROWS ? (4 * m > 256 ? 4 * m : 256) : (m > 256 * TILE ? m : 256 * TILE);
    return MAX_PARTS * m < few ? MAX_PARTS * m : few;
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
__device__ __forceinline__ int find_alone(const FqAdaptersArgs &a, int *rows, int &slot)
{
    const int tid = threadIdx.x, lane = tid & 63, own = blockIdx.x;
    int found[SMALL_ROWS / 64];
    uint64_t mask[SMALL_ROWS / 64];
    slot = slot_of(a, own);
#pragma unroll
    for (int c = 0; c < SMALL_ROWS / 64; c++)
        found[c] = 64 * c + lane < a.M ? slot_of(a, 64 * c + lane) : -2;
    int before = 0, seen = 0;
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
    __syncthreads();
    return min(seen - before, SMALL_TILE);
}

__device__ __forceinline__ Tile find_listed(const Work &w, int *rows)
{
    const Tile t = w.tiles[blockIdx.x];
    if (threadIdx.x < TILE)
        rows[threadIdx.x] = w.rows[TILE * blockIdx.x + threadIdx.x]; // (beyond the count: not used)
    __syncthreads();
    return t;
}

// What one of a tile's workgroups leaves for the second launch.
__device__ __forceinline__ void leave(const FqAdaptersArgs &a, const Work &w, const int *rows, Tile t)
{
    if (blockIdx.y != 0 || blockIdx.z != 0)
        return;
    if (threadIdx.x == 0) {
        t.scale = t.slot >= 0 && a.set.scales ? a.set.scales[t.slot] : 1.0f;
        w.tiles[blockIdx.x] = t;
    }
    if ((int)threadIdx.x < t.count)
        w.rows[TILE * blockIdx.x + threadIdx.x] = rows[threadIdx.x];
}

// Every workgroup of the first launch counts all rows by slot, finds the slot that its tile is of and takes the tile's rows in their order.
// (A launch of one workgroup that sorts them took 4.6 us for 701 rows, 5.9 for 2048.)
__device__ __forceinline__ int find_counted(const FqAdaptersArgs &a, int *rows, int &slot, int *count)
{
    constexpr int PER = MIDDLE_ROWS / THREADS;
    __shared__ int found[2], each[MIDDLE_ROWS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, keys = a.set.slots + 1;
    int key[PER]; // rows i * THREADS + tid
#pragma unroll
    for (int i = 0; i < PER; i++) {
        key[i] = -1;
        if (i * THREADS < a.M && i * THREADS + tid < a.M) {
            const int s = slot_of(a, i * THREADS + tid);
            key[i] = s < 0 ? keys - 1 : s;
        }
    }
    for (int i = tid; i < keys; i += THREADS)
        count[i] = 0;
    if (tid == 0)
        found[0] = -1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; i++) {
        if (i * THREADS >= a.M)
            break;
        const int first = __builtin_amdgcn_readfirstlane(key[i]);
        if (__ballot(key[i] == first) == ~0ull) { // (rows of one prompt)
            if (lane == 0 && first >= 0)
                atomicAdd(&count[first], 64);
        } else if (key[i] >= 0) {
            atomicAdd(&count[key[i]], 1);
        }
    }
    __syncthreads();
    if (wave == 0) { // the slot in whose tiles this one's number lies
        int begun = 0;
        for (int k0 = 0; k0 < keys; k0 += 64) {
            const int n = k0 + lane < keys ? (count[k0 + lane] + TILE - 1) / TILE : 0;
            int upto = n;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const int t = __shfl_up(upto, off, 64);
                upto += lane >= off ? t : 0;
            }
            const int from = begun + upto - n;
            if ((int)blockIdx.x >= from && (int)blockIdx.x < from + n) {
                found[0] = k0 + lane;
                found[1] = ((int)blockIdx.x - from) * TILE;
            }
            begun += __shfl(upto, 63, 64);
        }
    }
    __syncthreads();
    const int mine = found[0], skip = found[1];
    if (mine < 0)
        return 0;
    uint64_t mask[PER];
#pragma unroll
    for (int i = 0; i < PER; i++) {
        mask[i] = __ballot(key[i] == mine);
        if (lane == 0)
            each[i * WAVES + wave] = __popcll(mask[i]);
    }
    __syncthreads();
    const int total = min(count[mine] - skip, TILE);
    static_assert(MIDDLE_ROWS == 64 * 64, "a lane to 64 rows");
    int upto = each[lane];
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int t = __shfl_up(upto, off, 64);
        upto += lane >= off ? t : 0;
    }
    upto -= each[lane];
#pragma unroll
    for (int i = 0; i < PER; i++) {
        if (i * THREADS >= a.M)
            break;
        const int before = __shfl(upto, i * WAVES + wave, 64) - skip;
        const int at = before + (int)__popcll(mask[i] & ((1ull << lane) - 1));
        if (key[i] == mine && at >= 0 && at < TILE)
            rows[at] = i * THREADS + tid;
    }
    __syncthreads();
    slot = mine == keys - 1 ? -1 : mine;
    return total;
}

// One workgroup: rows counted by slot, slots' first places and tiles, rows put in order.  (The order of a slot's rows among themselves
// does not show: a row's sums are the same anywhere in a tile.)
__global__ __launch_bounds__(GROUP_THREADS) void group_kernel(FqAdaptersArgs a, Work w)
{
    extern __shared__ int count[]; // slots + 1: the last for rows without one
    __shared__ int sums[GROUP_THREADS / 64];
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
    int tiles = 0; // of the slots before these
    for (int k0 = 0; k0 < keys; k0 += GROUP_THREADS) {
        const int k = k0 + tid, n = k < keys ? count[k] : 0, t = (n + TILE - 1) / TILE;
        int tile = t;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int q = __shfl_up(tile, off, 64);
            tile += lane >= off ? q : 0;
        }
        if (lane == 63)
            sums[wave] = tile;
        __syncthreads();
        int all = 0;
        for (int v = 0; v < GROUP_THREADS / 64; v++) {
            tile += v < wave ? sums[v] : 0;
            all += sums[v];
        }
        tile += tiles - t;
        if (k < keys) {
            count[k] = tile * TILE;
            const int slot = k == keys - 1 ? -1 : k;
            const int rank = t ? rank_of(a, slot) : 0;
            const float scale = t && slot >= 0 && a.set.scales ? a.set.scales[slot] : 1.0f;
            for (int i = 0; i < t; i++)
                w.tiles[tile + i] = Tile{slot, min(n - i * TILE, TILE), rank, scale};
        }
        tiles += all;
        __syncthreads();
    }
    for (int i = tiles + tid; i < w.max_tiles; i += GROUP_THREADS)
        w.tiles[i] = Tile{-1, 0, 0, 1.0f};
    for (int m = tid; m < a.M; m += GROUP_THREADS) {
        const int s = slot_of(a, m);
        w.rows[take(s < 0 ? keys - 1 : s)] = m;
    }
}

// The sums that the wavefronts of a workgroup have of the same u, in one order; the first wavefront's become whole.
template <int TILES>
__device__ __forceinline__ void join_waves(float4_t (&acc)[TILES], float4_t (*sums)[TILES][64])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int half = WAVES / 2; half >= 1; half /= 2) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int i = 0; i < TILES; i++)
                sums[wave - half][i][lane] = acc[i];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int i = 0; i < TILES; i++)
                acc[i] += sums[wave][i][lane];
        }
        __syncthreads();
    }
}

// u = x A^T of a tile of few rows: RT * 16 ranks from 16 RT blockIdx.z on, the part blockIdx.y of K.  A step is 64 of K, of which a lane
// has 16 that follow each other (32 bytes of its row of x and of A): 128 bytes of a row to four lanes.
template <int RT, bool BF16>
__global__ __launch_bounds__(THREADS) void low_few_kernel(FqAdaptersArgs a, Work w)
{
    __shared__ int rows[SMALL_TILE];
    __shared__ float4_t sums[WAVES / 2][RT][64];
    int slot = -1;
    const int count = find_alone(a, rows, slot);
    const int rank = count ? rank_of(a, slot) : 0, r0 = 16 * RT * blockIdx.z;
    leave(a, w, rows, Tile{slot, count, rank, 1.0f});
    if (r0 >= rank)
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, g = lane >> 4;
    const uint16_t *xp = a.x + rows[col < count ? col : 0] * a.x_stride + 16 * g, *ap[RT];
#pragma unroll
    for (int r = 0; r < RT; r++)
        ap[r] = a.set.a + slot * a.set.a_stride + (size_t)min(r0 + 16 * r + col, rank - 1) * a.set.K + 16 * g;
    float4_t acc[RT] = {};
    const int K = a.set.K, steps = (K + 63) / 64;
    // a workgroup's part is one piece of K, its wavefronts' steps alternate
    const int part = (steps + gridDim.y - 1) / gridDim.y, end = min(steps, part * ((int)blockIdx.y + 1));
    struct Step {
        u32x4 x[2], a[RT][2];
    };
    auto ask = [&](Step &s, int step) {
        const int k = 64 * step;
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const bool in = k + 16 * g + 8 * h < K;
            s.x[h] = in ? *(const u32x4 *)(xp + k + 8 * h) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int r = 0; r < RT; r++)
                s.a[r][h] = in ? *(const u32x4 *)(ap[r] + k + 8 * h) : u32x4{0, 0, 0, 0};
        }
    };
    Step now, next;
    int step = part * blockIdx.y + wave;
    if (step < end)
        ask(now, step);
    for (; step < end; step += WAVES) {
        if (step + WAVES < end)
            ask(next, step + WAVES);
#pragma unroll
        for (int h = 0; h < 2; h++)
#pragma unroll
            for (int r = 0; r < RT; r++)
                acc[r] = mfma<BF16>(now.a[r][h], now.x[h], acc[r]);
        now = next;
    }
    join_waves(acc, sums);
    if (wave == 0 && col < count) {
        float *to = w.low + ((size_t)blockIdx.y * a.M + rows[col]) * a.set.rank + r0 + 4 * g;
#pragma unroll
        for (int r = 0; r < RT; r++)
            if (r0 + 16 * r + 4 * g < a.set.rank)
                *(float4_t *)(to + 16 * r) = acc[r];
    }
}

// The same for tiles of up to 64 rows.  Chunks of 256 of K go through LDS: 32 lanes ask for 512 bytes of a row (the operands' own order asks
// for 16 bytes of 16 rows at once, which the address unit takes a row at a time), a row's 16-byte piece p lies at place p ^ (row % 16), so that the
// 16 rows of an operand are read without conflicts.  A wavefront multiplies a quarter of the chunk while the next one is on its way.
template <int RT, bool BF16, Find FIND>
__global__ __launch_bounds__(THREADS) void low_many_kernel(FqAdaptersArgs a, Work w)
{
    constexpr int TT = TILE / 16, PIECES = CHUNK / 8, ROWS_A_TURN = THREADS / PIECES, X_TURNS = TILE / ROWS_A_TURN,
                  A_TURNS = 16 * RT / ROWS_A_TURN;
    __shared__ int rows[TILE];
    __shared__ u32x4 tile[(TILE + 16 * RT) * PIECES];
    static_assert(sizeof(tile) >= (MIDDLE_SLOTS + 1) * sizeof(int) && sizeof(tile) >= WAVES / 2 * TT * RT * 64 * sizeof(float4_t), "");
    static_assert(THREADS == WAVES * 64 && CHUNK == 64 * WAVES, "a wavefront to 64 of a chunk");
    Tile own;
    if (FIND == LISTED) {
        own = find_listed(w, rows);
    } else {
        own.slot = -1;
        own.count = find_counted(a, rows, own.slot, (int *)tile);
        own.rank = own.count ? rank_of(a, own.slot) : 0;
        leave(a, w, rows, own);
    }
    const int slot = own.slot, count = own.count, rank = own.rank, r0 = 16 * RT * blockIdx.z;
    if (r0 >= rank)
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
    const int K = a.set.K, chunks = (K + CHUNK - 1) / CHUNK;
    const int part = (chunks + gridDim.y - 1) / gridDim.y, from = part * blockIdx.y, end = min(chunks, from + part);
    const int piece = tid % PIECES, row0 = tid / PIECES;
    const uint16_t *xp[X_TURNS], *ap = a.set.a + slot * a.set.a_stride;
#pragma unroll
    for (int i = 0; i < X_TURNS; i++)
        xp[i] = a.x + rows[min(row0 + i * ROWS_A_TURN, count - 1)] * a.x_stride + 8 * piece;
    u32x4 xv[X_TURNS], av[A_TURNS];
    auto ask = [&](int c) {
        const int k = CHUNK * c + 8 * piece;
        const bool in = k < K;
#pragma unroll
        for (int i = 0; i < X_TURNS; i++)
            xv[i] = in && row0 + i * ROWS_A_TURN < count ? *(const u32x4 *)(xp[i] + CHUNK * c) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < A_TURNS; i++)
            av[i] = in ? *(const u32x4 *)(ap + (size_t)min(r0 + row0 + i * ROWS_A_TURN, rank - 1) * K + k) : u32x4{0, 0, 0, 0};
    };
    float4_t acc[TT * RT] = {};
    if (from < end)
        ask(from);
    __syncthreads(); // (the counts lay where the chunk goes)
    for (int c = from; c < end; c++) {
#pragma unroll
        for (int i = 0; i < X_TURNS; i++) {
            const int row = row0 + i * ROWS_A_TURN;
            tile[row * PIECES + (piece ^ (row & 15))] = xv[i];
        }
#pragma unroll
        for (int i = 0; i < A_TURNS; i++) {
            const int row = TILE + row0 + i * ROWS_A_TURN;
            tile[row * PIECES + (piece ^ (row & 15))] = av[i];
        }
        __syncthreads();
        if (c + 1 < end)
            ask(c + 1);
#pragma unroll
        for (int h = 0; h < 2; h++) {
            const int at = (8 * wave + 4 * h + g) ^ col;
            u32x4 xf[TT], af[RT];
#pragma unroll
            for (int t = 0; t < TT; t++)
                xf[t] = tile[(16 * t + col) * PIECES + at];
#pragma unroll
            for (int r = 0; r < RT; r++)
                af[r] = tile[(TILE + 16 * r + col) * PIECES + at];
#pragma unroll
            for (int t = 0; t < TT; t++)
#pragma unroll
                for (int r = 0; r < RT; r++)
                    acc[t * RT + r] = mfma<BF16>(af[r], xf[t], acc[t * RT + r]);
        }
        __syncthreads();
    }
    join_waves(acc, (float4_t(*)[TT * RT][64])tile);
    if (wave != 0)
        return;
#pragma unroll
    for (int t = 0; t < TT; t++) {
        if (16 * t + col >= count)
            continue;
        float *to = w.low + ((size_t)blockIdx.y * a.M + rows[16 * t + col]) * a.set.rank + r0 + 4 * g;
#pragma unroll
        for (int r = 0; r < RT; r++)
            if (r0 + 16 * r + 4 * g < a.set.rank)
                *(float4_t *)(to + 16 * r) = acc[t * RT + r];
    }
}

// out = y + scale u B^T of a tile, blocks of 64 outputs to a wavefront.  u lies in LDS as the second operands' registers, 32 ranks
// to an instruction, hi and lo.  Row i of a first operand is output 16 (i / 4) + 4 j + i % 4 of the block in instruction j of four, so that a lane's results
// of the four are 16 outputs of its row that follow each other.
template <int TT, bool BF16, bool VEC>
__global__ __launch_bounds__(TT == 1 ? THREADS : MANY_THREADS) void out_kernel(FqAdaptersArgs a, Work w)
{
    constexpr int THREADS = TT == 1 ? ::THREADS : MANY_THREADS, WAVES = THREADS / 64;
    __shared__ int rows[TILE];
    __shared__ float factor[16 * TT];
    extern __shared__ u32x4 low[]; // [rank / 32][TT][2][64]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
    const Tile own = find_listed(w, rows);
    const int slot = own.slot, count = own.count, rank = own.rank, N = a.set.N;
    if (count == 0)
        return;
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
    const uint16_t *bp = a.set.b + slot * a.set.b_stride;
    // What a block of 64 outputs needs from memory, asked for a block ahead: B of the first 64 ranks, and y.
    struct Block {
        u32x4 b[2][4], y[VEC ? TT : 1][2];
    };
    auto ask_b = [&](u32x4(&v)[4], int b, int c) {
        const int r = 32 * c + 8 * g;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int n = 64 * b + 16 * (col >> 2) + 4 * j + (col & 3);
            v[j] = n < N && r < rank ? *(const u32x4 *)(bp + (size_t)n * a.set.rank + r) : u32x4{0, 0, 0, 0};
        }
    };
    auto ask = [&](Block &k, int b) {
        ask_b(k.b[0], b, 0);
        if (chunks > 1)
            ask_b(k.b[1], b, 1);
        if (VEC) {
#pragma unroll
            for (int t = 0; t < TT; t++)
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    const int n = 64 * b + 16 * g + 8 * h;
                    k.y[t][h] = 16 * t + col < count && n < N ? *(const u32x4 *)(a.y + rows[16 * t + col] * a.y_stride + n) : u32x4{0, 0, 0, 0};
                }
        }
    };
    Block now, next;
    if (first < blocks)
        ask(now, first);

    // u: as many threads to a row as its ranks take four at a time, up to 16; everything that a turn adds is asked for together
    const int wide = rank <= 16 ? 4 : rank <= 32 ? 8 : 16, turn = THREADS / wide;
    const size_t apart = (size_t)a.M * a.set.rank;
    for (int row = tid / wide; row < 16 * TT; row += turn) {
        const float *from = w.low + (size_t)rows[row < count ? row : 0] * a.set.rank;
        float4_t u[FQ_MAX_ADAPTER_RANK / 64];
        float most = 0.0f;
#pragma unroll
        for (int c = 0; c < FQ_MAX_ADAPTER_RANK / 64; c++) {
            const int r = 64 * c + 4 * (tid & (wide - 1));
            u[c] = float4_t{0, 0, 0, 0};
            if (64 * c < rank && r < rank) {
                for (int p0 = 0; p0 < w.parts; p0 += 8) {
                    float4_t part[8];
#pragma unroll
                    for (int p = 0; p < 8; p++)
                        part[p] = *(const float4_t *)(from + (size_t)min(p0 + p, w.parts - 1) * apart + r);
#pragma unroll
                    for (int p = 0; p < 8; p++)
                        if (p0 + p < w.parts)
                            u[c] += part[p];
                }
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    u[c][i] = r + i < rank ? u[c][i] : 0.0f;
                    most = fmaxf(most, fabsf(u[c][i]) < INFINITY ? fabsf(u[c][i]) : 0.0f);
                }
            }
        }
        for (int off = wide / 2; off >= 1; off >>= 1)
            most = fmaxf(most, __shfl_xor(most, off, 64));
        // binary16: the row's largest becomes 2^13 to 2^14 (a power of two changes no digit)
        const int e = BF16 || most == 0.0f ? 0 : min(max(14 - __builtin_amdgcn_frexp_expf(most), -126), 126);
        if ((tid & (wide - 1)) == 0)
            factor[row] = ldexpf(own.scale, -e);
#pragma unroll
        for (int c = 0; c < FQ_MAX_ADAPTER_RANK / 64; c++) {
            const int r = 64 * c + 4 * (tid & (wide - 1));
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
                if (wide == 4 && rank <= 16) { // ranks 16 to 31 of the instruction
                    at[64 + ((r & 7) >> 2)] = make_uint2(0, 0);
                    at[128 + 64 + ((r & 7) >> 2)] = make_uint2(0, 0);
                }
            }
        }
    }
    __syncthreads();
    for (int b = first; b < blocks; b += stride) {
        if (b + stride < blocks)
            ask(next, b + stride);
        float4_t acc[TT][4] = {};
        auto multiply = [&](u32x4(&bv)[4], int c) {
            if (rank & 7) { // (what lies behind a rank may be anything)
                const int r = 32 * c + 8 * g;
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
        };
        multiply(now.b[0], 0);
        if (chunks > 1)
            multiply(now.b[1], 1);
        for (int c = 2; c < chunks; c++) {
            u32x4 bv[4];
            ask_b(bv, b, c);
            multiply(bv, c);
        }
        const int n = 64 * b + 16 * g;
#pragma unroll
        for (int t = 0; t < TT; t++) {
            if (16 * t + col >= count)
                continue;
            const long long m = rows[16 * t + col];
            uint16_t *out = a.out + m * a.out_stride + n;
            const float f = factor[16 * t + col];
            if (VEC) {
#pragma unroll
                for (int h = 0; h < 2; h++) {
                    if (n + 8 * h >= N)
                        continue;
                    u32x4 v = now.y[t][h];
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
                const uint16_t *y = a.y + m * a.y_stride + n;
#pragma unroll
                for (int i = 0; i < 16; i++)
                    if (n + i < N)
                        out[i] = fq_from_float(fq_to_float(y[i], BF16) + f * acc[t][i >> 2][i & 3], BF16);
            }
        }
        now = next;
    }
}

template <int RT, bool BF16, Find FIND>
void launch_low(const FqAdaptersArgs &a, const Work &w, hipStream_t stream)
{
    const dim3 grid(w.max_tiles, w.parts, (a.set.rank + 16 * RT - 1) / (16 * RT));
    if constexpr (FIND == ALONE)
        low_few_kernel<RT, BF16><<<grid, THREADS, 0, stream>>>(a, w);
    else
        low_many_kernel<RT, BF16, FIND><<<grid, THREADS, 0, stream>>>(a, w);
}

template <bool BF16, Find FIND>
hipError_t launch(const FqAdaptersArgs &a, const Work &w, hipStream_t stream)
{
    constexpr int TT = FIND == ALONE ? 1 : TILE / 16, threads = FIND == ALONE ? THREADS : MANY_THREADS;
    if (a.set.rank <= 16)
        launch_low<1, BF16, FIND>(a, w, stream);
    else if (a.set.rank <= 32)
        launch_low<2, BF16, FIND>(a, w, stream);
    else
        launch_low<4, BF16, FIND>(a, w, stream);
    if (hipError_t e = hipGetLastError())
        return e;
    const bool vec = a.set.N % 8 == 0 && a.y_stride % 8 == 0 && a.out_stride % 8 == 0 && ((uintptr_t)a.y & 15) == 0 && ((uintptr_t)a.out & 15) == 0;
    // outputs over as many workgroups as fill the chip
    const int blocks = (a.set.N + 63) / 64, tiles = TT == 1 ? a.M : (a.M + TILE - 1) / TILE;
    const int most = (blocks + threads / 64 - 1) / (threads / 64), room = ((TT == 1 ? 512 : 256) + tiles - 1) / tiles;
    const dim3 grid(w.max_tiles, most < room ? most : room);
    const size_t lds = (size_t)(a.set.rank + 31) / 32 * TT * 2 * 64 * sizeof(u32x4);
    const void *func = vec ? (const void *)out_kernel<TT, BF16, true> : (const void *)out_kernel<TT, BF16, false>;
    if (hipError_t e = fq_raise_dynamic_lds(func, lds))
        return e;
    if (vec)
        out_kernel<TT, BF16, true><<<grid, threads, lds, stream>>>(a, w);
    else
        out_kernel<TT, BF16, false><<<grid, threads, lds, stream>>>(a, w);
    return hipGetLastError();
}

} // namespace

size_t fq_adapters_bytes(const FqAdaptersView &set, int M)
{
    const size_t tiles = tiles_of(set, M);
    return up(low_rows(M) * set.rank * sizeof(float)) + up(tiles * TILE * sizeof(int)) + up(tiles * sizeof(Tile)) + 256;
}

hipError_t fq_launch_adapters(const FqAdaptersArgs &a, void *workspace, hipStream_t stream)
{
    Work w{};
    w.parts = parts_of(a.set, a.M);
    w.max_tiles = tiles_of(a.set, a.M);
    char *at = (char *)workspace;
    w.low = (float *)at;
    at += up(low_rows(a.M) * a.set.rank * sizeof(float));
    w.rows = (int *)at;
    at += up((size_t)w.max_tiles * TILE * sizeof(int));
    w.tiles = (Tile *)at;
    if (a.M <= SMALL_ROWS)
        return a.set.bf16 ? launch<true, ALONE>(a, w, stream) : launch<false, ALONE>(a, w, stream);
    if (a.M <= MIDDLE_ROWS && a.set.slots <= MIDDLE_SLOTS)
        return a.set.bf16 ? launch<true, COUNTED>(a, w, stream) : launch<false, COUNTED>(a, w, stream);
    const size_t lds = (a.set.slots + 1) * sizeof(int);
    if (hipError_t e = fq_raise_dynamic_lds((const void *)group_kernel, lds))
        return e;
    group_kernel<<<1, GROUP_THREADS, lds, stream>>>(a, w);
    if (hipError_t e = hipGetLastError())
        return e;
    return a.set.bf16 ? launch<true, LISTED>(a, w, stream) : launch<false, LISTED>(a, w, stream);
}
