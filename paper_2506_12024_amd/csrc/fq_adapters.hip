// Low-rank adapters of many requests beside a projection that they share: out = y + scale (x A^T) B^T, row by row.
//
// Both products are on the matrix cores.  u = x A^T is a binary32 sum, and meets B as two 16-bit numbers each, u = hi + lo (binary16: 22
// bits of it, a row scaled by a power of two so that its largest fills the range; bfloat16: 17), so that it is nowhere rounded to
// 16 bits.  A tile is up to 16 or 64 rows of one slot, wherever in the call they stand: a row's sums do not depend on its place in a
// tile.  Few rows are one launch (few_kernel), whose workgroups form u for themselves; many are two to four: low_kernel forms u in parts of K, which lie in
// the workspace; out_kernel adds them up, parts them into hi and lo and multiplies by B, or join_kernel does the first where each of its workgroups
// would have much to add; group_kernel sorts the rows ahead of them where the workgroups of low_kernel are too many to count them each.
//
// What bounds it: a token (4096 -> 4096, rank 16) 7.2 us a call from Python, of which the host takes 6.7 and the device as much: four trips to memory one
// after another, launch, the exchange through LDS; 32 rows of 24 slots (4096 -> 11008, rank 32) 11.3 us, A and B once 3.3, A read again by every workgroup
// of a tile.  701 rows, chunks and single tokens (11008 -> 4096, rank 16) 17.8 us, low_kernel 9.6 (3.5 until it knows its rows), out_kernel 9.1, everything once 6.0.
// A prompt of 2048 rows (8192 -> 8192, rank 64, bfloat16) 42 us, of which low_kernel has 19 (4.6 until it knows its rows, then x at 2/3 of the
// rate of a large copy), join_kernel 5, out_kernel 19 (67 MB of y and out, 3.5 TB/s); everything once at 5.2 TB/s would be 20.
//
// What the operands' registers hold (16 bytes of 16 rows to a quarter of a wavefront) is nowhere loaded from memory in that order: the address unit
// takes such a quarter a row at a time, 131 KB of A 3.4 us a workgroup as against 0.8 to 1.1 with 128 bytes of a row to eight lanes.
// It goes through LDS, 16-byte pieces placed so that both sides are free of conflicts.
#include <hip/hip_runtime.h>

#include <math.h>
#include <type_traits>

#include "../../include/flexq.h"
#include "fq_kv.h"

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int FEW_ROWS = 256, FEW_TILE = 16, TILE = 64;
constexpr int MIDDLE_ROWS = 4096, MIDDLE_SLOTS = 1023;
// With more workgroups of the first launch than these, one that sorts the rows goes ahead of it: each that counts the rows for itself, those without a tile, too, takes 3.5
// to 5 us for that, behind a list one read.  (4 slots named, us counted / sorted: 257 rows, 4096 -> 4096, rank 16, of a set of 32 13.4 / 14.4, of 300 27.0 / 18.8; 700 of 50
// 20.4 / 20.7, of 100 20.6 / 19.0, of 1000 74 / 27; 2048 of 100 22.9 / 24.8, of 300 30.2 / 26.9; 257 rows, 4096 -> 1024, rank 256, of 1000 141 / 39.  Over 2300 shapes this choice
// is 0.3 % from the better, 1500 0.7, 512 0.9.)
constexpr int COUNTING = 1024;
constexpr int GROUP_THREADS = 1024, OUT_THREADS = 512, MANY_THREADS = 256, JOIN_THREADS = 256, JOIN_ROWS = JOIN_THREADS / 16;
constexpr int CHUNK = 256, MAX_PARTS = 16; // of K
enum Find { COUNTED, LISTED }; // how a workgroup of low_kernel finds its tile: by itself, or in the workspace's list

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
    u32x4 *operands; // u as out_kernel's operands, tile_operands to a tile
    float *factor;   // [tile][TILE]
    int parts, max_tiles, tile_operands;
};

// Whether a call is one launch: every workgroup of a tile reads its slot's A whole, which is less than another launch and the parts while A is
// small, and the tiles of 16 rows suit many slots.  One launch / more (us on the device): 1 row, 4096 -> 4096, rank 16 7.1 / 8.4, rank 64 11.7 / 9.8; 32 rows of
// 24 slots, 4096 -> 11008, rank 32 10.7 / 17.5, of 2 11.9 / 9.7; 64 of 64, 4096 -> 4096, rank 32 10.9 / 22.6, of 4 10.6 / 9.6; 128 of 64, rank 16 11.7 / 20.7, of 4
// 12.6 / 10.0, of 4 with 2048 outputs 9.7 / 10.4; 64 of 4, 4096 -> 11008, rank 16 14.6 / 9.7.  An A above 2^17 pays where many slots may be in the call, whose tiles, empty
// or not, cost more launches most (all of a set's slots named, or one of them): with a tile's x up to 2^18 in rank 32, 5120 -> 5120, 16 rows of 16 slots 10.5 / 12.3,
// 10.3 / 11.5, 32 of 32 11.8 / 15.0, 11.6 / 15.8, of 8 12.0 / 12.1, 11.4 / 12.7, 64 of 64 13.9 / 26.3, of 32 13.2 / 16.5, 12.9 / 15.5, of 16 14.0 / 13.1, 12.9 / 14.7; beyond
// of nearly as many slots as rows: rank 16, 11008 -> 4096, 16 of 16 11.9 / 11.2, 11.5 / 10.2, 32 of 32 12.3 / 14.5, 12.0 / 14.6, 64 of 32 13.7 / 15.9, 13.7 / 13.4; rank 64,
// 4096 -> 4096, 24 of 24 14.2 / 14.7, 13.5 / 12.4, 32 of 32 15.0 / 16.9, 14.0 / 17.9, 64 of 64 24.3 / 32.7, 15.7 / 19.7; with more than 6144 outputs (out_tiles) later:
// rank 32, 8192 -> 8192, 32 of 32 15.3 / 20.4, 14.8 / 13.2, 48 of 64 19.6 / 31.4, 17.0 / 16.3, 64 of 64 21.3 / 39.5, 17.2 / 15.7, of 32 17.1 / 20.7, 17.2 / 14.1; rank 64,
// 4096 -> 11008, 32 of 32 26.9 / 29.9, 18.1 / 15.1, 64 of 64 37.9 / 52.6, 24.1 / 18.2.
bool few(const FqAdaptersView &set, int M)
{
    const long long rank = set.rank < 16 ? 16 : set.rank, a = rank * set.K, b = rank * set.N; // (the instructions take 16)
    if (set.rank > 64 || M > FEW_ROWS)
        return false;
    if (8 * (set.slots + 1) <= M) // many rows of a slot
        return a <= 1 << 17 && M * (a + b) <= 3 << 22;
    const int named = M < set.slots ? M : set.slots; // slots that the call may name
    if (M <= 64)
        return a <= 1 << 17 || (a + 16 * set.K <= 1 << 18 && named >= 16 && 2 * named >= M) ||
               (a <= 1 << 18 && named >= (set.N <= 6144 ? 28 : 40) && 5 * named >= 4 * M);
    return a + b <= 1 << 18 && set.N <= 8192;
}

// Workgroups to a row of that launch: outputs over as many as fill the chip if every row led a tile (32 rows of 20 slots, 4096 -> 11008, rank 32: 8 of them 11.6 us,
// 12 15.0, 4 14.0).  Up to 64 rows not one more than there are compute units: a unit that has two takes twice as long (40 rows of 40 slots, 4096 -> 4096, rank 16
// 7 11.5 us, 6 9.0; 48 of 48, 4096 -> 11008, rank 32 6 19.1, 5 15.9).
int few_shares(const FqAdaptersView &set, int M)
{
    const int blocks = (set.N + 63) / 64, most = (blocks + OUT_THREADS / 64 - 1) / (OUT_THREADS / 64);
    const int room = M <= 64 ? 256 / M : M <= 128 ? (256 + M - 1) / M : 2;
    return most < room ? most : room;
}

int tiles_of(const FqAdaptersView &set, int M) { return M / TILE + (M < set.slots + 1 ? M : set.slots + 1); } // at most

// Tiles to a row of the last launch's grid.  With a multiple of 8 all of a tile's workgroups are on one XCD, and find B and the parts in its L2; but XCDs have unequal
// shares of y and out, and one has all where a call names one slot; with an odd number they are on all XCDs.  (us with a multiple of 8 / odd: 701 rows of rank 16, N =
// 4096 17.5 / 18.9, 8192 20.6 / 19.5; 2048 rows, 1024 18.5 / 21.4, 6144 25.3 / 25.9, 8200 31.5 / 30.7, 11008 42 / 37; 24 rows of 24 slots of rank 128, 4096 -> 4096 23.6 / 27.0,
// 64 of one of 64 25.2 / 23.1; 32 rows of one of 64 slots of rank 64, 4096 -> 11008 32.3 / 14.6, of 32 27.9 / 28.1, 4096 -> 5120 19.6 / 13.5 and 18.9 / 19.2.)
int out_tiles(const FqAdaptersView &set, int M) { return set.N <= 6144 ? (tiles_of(set, M) + 7) / 8 * 8 : tiles_of(set, M) | 1; }

// As many as there may well be, between what rows fill and that: the adapters of the rows are not known here.  (Against what rows fill: 300 rows of 200 slots, 4096 ->
// 11008, rank 64 129 instead of 158 us, 1000 rows of 500 141 instead of 179.)
int tiles_likely(const FqAdaptersView &set, int M)
{
    const int least = (M + TILE - 1) / TILE + 1, mean = (int)(0.5f * sqrtf((float)least * tiles_of(set, M)));
    return least > mean ? least : mean;
}

// Parts of K: workgroups for the whole chip while rows are few, at least a chunk to each.
int parts_of(const FqAdaptersView &set, int M)
{
    int parts = 256 / ((M + TILE - 1) / TILE);
    parts = parts > MAX_PARTS ? MAX_PARTS : parts < 1 ? 1 : parts;
    const int most = (set.K + CHUNK - 1) / CHUNK;
    return parts < most ? parts : most;
}

// Rows times parts, from above and never less for more rows: what parts_of gives is at most this.
size_t low_rows(int M)
{
    const size_t m = M, most = m > 256 * TILE ? m : 256 * TILE;
    return MAX_PARTS * m < most ? MAX_PARTS * m : most;
}

int tile_operands(const FqAdaptersView &set) { return (set.rank + 31) / 32 * (TILE / 16) * 2 * 64; } // 16 bytes each

// Threads to a row where the last launch adds up the parts: four ranks to each.
__host__ __device__ inline int threads_a_row(const FqAdaptersView &set)
{
    return set.rank <= 8 ? 2 : set.rank <= 16 ? 4 : set.rank <= 32 ? 8 : set.rank <= 64 ? 16 : set.rank <= 128 ? 32 : 64;
}

// Ranks to a workgroup of low_kernel.
int low_ranks(const FqAdaptersView &set) { return set.rank <= 16 ? 16 : set.rank <= 32 ? 32 : 64; }

size_t up(size_t n) { return (n + 255) / 256 * 256; }

// What a wavefront hands to itself through LDS: its operations there are in order, the compiler has to keep them so.
__device__ __forceinline__ void own_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The sum over this lane and those before it.
__device__ __forceinline__ int sum_upto(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false); // within rows of 16: one, two, four, eight lanes down
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false); // the last lane of rows 0 and 2 to rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false); // lane 31 to rows 2 and 3
    return x;
}

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

// Ranks and scales of the first slots, a lane to each, asked for beside the rows' slots: one trip to memory fewer where a slot is among them.
struct Some {
    int rank;
    float scale;
    __device__ __forceinline__ explicit Some(const FqAdaptersArgs &a)
    {
        const int s = min((int)threadIdx.x & 63, a.set.slots - 1);
        rank = a.set.ranks ? a.set.ranks[s] : a.set.rank;
        scale = a.set.scales ? a.set.scales[s] : 1.0f;
    }
    // (slot is the same in all lanes)
    __device__ __forceinline__ void of(const FqAdaptersArgs &a, int slot, int &r, float &s) const
    {
        r = 0;
        s = 1.0f;
        if (slot >= 64) {
            r = rank_of(a, slot);
            s = a.set.scales ? a.set.scales[slot] : 1.0f;
        } else if (slot >= 0) {
            r = min(max(__builtin_amdgcn_readlane(rank, slot), 0), a.set.rank);
            s = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, scale), slot));
        }
    }
};

__device__ __forceinline__ Tile find_listed(const Work &w, int *rows)
{
    const Tile t = w.tiles[blockIdx.x];
    if (threadIdx.x < TILE)
        rows[threadIdx.x] = w.rows[TILE * blockIdx.x + threadIdx.x]; // (beyond the count: not used)
    __syncthreads();
    return t;
}

// What one of a tile's workgroups leaves for the second launch.
__device__ __forceinline__ void leave(const Work &w, const int *rows, const Tile &t)
{
    if (blockIdx.y != 0 || blockIdx.z != 0)
        return;
    if (threadIdx.x == 0)
        w.tiles[blockIdx.x] = t;
    if ((int)threadIdx.x < t.count)
        w.rows[TILE * blockIdx.x + threadIdx.x] = rows[threadIdx.x];
}

// Every workgroup of the first launch counts all rows by slot, finds the slot that its tile is of and takes the tile's rows in their order.
// (A launch of one workgroup that sorts them took 4.6 us for 701 rows, 5.9 for 2048.)
__device__ __forceinline__ int find_counted(const FqAdaptersArgs &a, int *rows, int &slot, int *count)
{
    constexpr int PER = MIDDLE_ROWS / THREADS;
    __shared__ int found[2], each[MIDDLE_ROWS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), keys = a.set.slots + 1;
    int key[PER]; // rows i * THREADS + tid
#pragma unroll
    for (int i = 0; i < PER; i++)
        key[i] = a.adapter[min(i * THREADS + tid, a.M - 1)]; // (all asked for together)
#pragma unroll
    for (int i = 0; i < PER; i++)
        key[i] = i * THREADS + tid >= a.M ? -1 : key[i] >= 0 && key[i] < a.set.slots ? key[i] : keys - 1;
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
            const int upto = sum_upto(n), from = begun + upto - n;
            if ((int)blockIdx.x >= from && (int)blockIdx.x < from + n) {
                found[0] = k0 + lane;
                found[1] = ((int)blockIdx.x - from) * TILE;
            }
            begun += __builtin_amdgcn_readlane(upto, 63);
            if (begun > (int)blockIdx.x)
                break;
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
    const int upto = sum_upto(each[lane]) - each[lane];
#pragma unroll
    for (int i = 0; i < PER; i++) {
        if (i * THREADS >= a.M)
            break;
        const int before = __builtin_amdgcn_readlane(upto, i * WAVES + wave) - skip;
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
        int tile = sum_upto(t);
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

// u = x A^T of a tile of up to 64 rows: 16 RT ranks from 16 RT blockIdx.z on, the part blockIdx.y of K, 256 at a time.  32 lanes ask for 512
// bytes of a row, two chunks ahead; a row's piece p lies at place p ^ (row % 16).  A wavefront has 16 of the rows.
template <int RT, bool BF16, Find FIND>
__global__ __launch_bounds__(THREADS, 1) void low_kernel(FqAdaptersArgs a, Work w)
{
    constexpr int PIECES = CHUNK / 8, ROWS_A_TURN = THREADS / PIECES, X_TURNS = TILE / ROWS_A_TURN, A_TURNS = 16 * RT / ROWS_A_TURN;
    __shared__ int rows[TILE];
    __shared__ u32x4 tile[(TILE + 16 * RT) * PIECES];
    static_assert(sizeof(tile) >= (MIDDLE_SLOTS + 1) * sizeof(int) && TILE == 16 * WAVES, "");
    Tile own;
    if (FIND == LISTED) {
        own = find_listed(w, rows);
    } else {
        const Some some(a);
        own.slot = -1;
        own.count = find_counted(a, rows, own.slot, (int *)tile);
        own.slot = __builtin_amdgcn_readfirstlane(own.slot);
        some.of(a, own.count ? own.slot : -1, own.rank, own.scale);
        leave(w, rows, own);
    }
    const int slot = own.slot, count = own.count, rank = own.rank, r0 = 16 * RT * blockIdx.z;
    if (r0 >= rank)
        return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
    const int K = a.set.K, chunks = (K + CHUNK - 1) / CHUNK;
    // (a part's chunks lie among the others': what is read at a time lies together)
    const int from = blockIdx.y, apart = gridDim.y;
    const int piece = tid % PIECES, row0 = tid / PIECES;
    const uint16_t *xp[X_TURNS], *ap = a.set.a + slot * a.set.a_stride;
#pragma unroll
    for (int i = 0; i < X_TURNS; i++)
        xp[i] = a.x + rows[min(row0 + i * ROWS_A_TURN, count - 1)] * a.x_stride;
    struct Step {
        u32x4 x[X_TURNS], a[A_TURNS];
    };
    // (rows beyond the last are the last again, and not used)
    auto ask = [&](Step &s, int c) {
        const int k = min(CHUNK * c + 8 * piece, K - 8);
#pragma unroll
        for (int i = 0; i < X_TURNS; i++)
            s.x[i] = *(const u32x4 *)(xp[i] + k);
#pragma unroll
        for (int i = 0; i < A_TURNS; i++)
            s.a[i] = *(const u32x4 *)(ap + (size_t)min(r0 + row0 + i * ROWS_A_TURN, rank - 1) * K + k);
    };
    float4_t acc[RT] = {};
    auto use = [&](Step &s, int c) {
        if (CHUNK * (c + 1) > K && CHUNK * c + 8 * piece >= K) { // behind the end of K
#pragma unroll
            for (int i = 0; i < X_TURNS; i++)
                s.x[i] = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < A_TURNS; i++)
                s.a[i] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < X_TURNS; i++) {
            const int row = row0 + i * ROWS_A_TURN;
            tile[row * PIECES + (piece ^ (row & 15))] = s.x[i];
        }
#pragma unroll
        for (int i = 0; i < A_TURNS; i++) {
            const int row = TILE + row0 + i * ROWS_A_TURN;
            tile[row * PIECES + (piece ^ (row & 15))] = s.a[i];
        }
        __syncthreads();
        if (c + 2 * apart < chunks)
            ask(s, c + 2 * apart);
        if (16 * wave < count) {
#pragma unroll
            for (int h = 0; h < PIECES / 4; h++) {
                const int at = (4 * h + g) ^ col;
                const u32x4 x = tile[(16 * wave + col) * PIECES + at];
#pragma unroll
                for (int r = 0; r < RT; r++)
                    acc[r] = mfma<BF16>(tile[(TILE + 16 * r + col) * PIECES + at], x, acc[r]);
            }
        }
        __syncthreads();
    };
    Step even, odd;
    ask(even, from); // (chunks >= parts)
    if (from + apart < chunks)
        ask(odd, from + apart);
    __syncthreads(); // (the counts lay where the chunk goes)
    for (int c = from; c < chunks; c += 2 * apart) {
        use(even, c);
        if (c + apart < chunks)
            use(odd, c + apart);
    }
    if (16 * wave + col < count) {
        float *to = w.low + ((size_t)blockIdx.y * a.M + rows[16 * wave + col]) * a.set.rank + r0 + 4 * g;
#pragma unroll
        for (int r = 0; r < RT; r++)
            if (r0 + 16 * r + 4 * g < a.set.rank)
                *(float4_t *)(to + 16 * r) = acc[r];
    }
}

// The last step: 64 outputs of 16 TT rows to a wavefront and turn, out = y + factor u B^T.  u lies in LDS as the first operands' registers, 32
// ranks to an instruction, hi and lo: [rank / 32][ALL][2][64].  Column c of instruction j of four is output 4 c + j, so that a lane's results of the four
// are four outputs that follow each other, 128 bytes of a row to sixteen lanes; where rows are not aligned to 8 bytes it is output 16 j + c, 32 bytes of a
// row to an access.  B comes 32 ranks of 64 outputs at a time, through 4 KB of LDS of the wavefront's own; that of the first 32 AHEAD ranks is asked for
// beside y.
template <int TT, int ALL, int AHEAD, bool BF16, bool VEC>
struct Out {
    const FqAdaptersArgs &a;
    const int *rows;
    const float *factor;
    const u32x4 *low;
    u32x4 *mine; // [256]
    const uint16_t *b;
    int count, rank, chunks;
    struct Turn {
        u32x4 b[AHEAD][4];
        uint2 y[VEC ? TT : 1][4];
        uint16_t one[VEC ? 1 : TT][4][4];
    };

    // (what lies outside is loaded from inside and not used: a condition around each load is a branch around each)
    __device__ __forceinline__ void ask_b(u32x4 (&v)[4], int block, int c) const
    {
        const int lane = threadIdx.x & 63, r = min(32 * c + 8 * (lane & 3), a.set.rank - 8);
#pragma unroll
        for (int i = 0; i < 4; i++)
            v[i] = *(const u32x4 *)(b + (size_t)min(64 * block + 16 * i + (lane >> 2), a.set.N - 1) * a.set.rank + r);
    }

    __device__ __forceinline__ void ask(Turn &k, int block) const
    {
        const int lane = threadIdx.x & 63;
        ask_b(k.b[0], block, 0);
        if (AHEAD > 1 && chunks > 1)
            ask_b(k.b[AHEAD - 1], block, 1);
#pragma unroll
        for (int t = 0; t < TT; t++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint16_t *y = a.y + rows[min(16 * t + 4 * (lane >> 4) + i, count - 1)] * a.y_stride;
                if (VEC)
                    k.y[VEC ? t : 0][i] = *(const uint2 *)(y + min(64 * block + 4 * (lane & 15), a.set.N - 4));
                else
#pragma unroll
                    for (int j = 0; j < 4; j++)
                        k.one[VEC ? 0 : t][i][j] = y[min(64 * block + 16 * j + (lane & 15), a.set.N - 1)];
            }
    }

    // Infinities of B meet hi alone, whose product has u's sign: lo may be 0 or of the other sign, and would make NaN of them.  (A u that is 2^-38 of its row's
    // largest or less has a hi of 0 in binary16.)  SOUGHT: B is looked at while it lies in LDS, which costs out_kernel nothing, few_kernel 0.1 to 0.3 us of 5 to 10;
    // IGNORED: its sums are looked at, and where they are not all numbers the rest is walked APART (few_kernel up to rank 32 0 to 0.1 us, of rank 64 0.1 to 2 of 30).
    enum Infinities { SOUGHT, IGNORED, APART };
    template <Infinities B>
    __device__ __forceinline__ void multiply(float4_t (&acc)[TT][4], u32x4 (&v)[4], int c) const
    {
        const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
        if (32 * c + 32 > rank) { // (what lies behind a rank may be anything)
            const int r = 32 * c + 8 * (lane & 3);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t mask = (r + 2 * i < rank ? 0xffffu : 0u) | (r + 2 * i + 1 < rank ? 0xffff0000u : 0u);
#pragma unroll
                for (int j = 0; j < 4; j++)
                    v[j][i] &= mask;
            }
        }
        // piece g of column col of instruction j: place 64 j + 16 g + (col ^ (j + 4 g))
#pragma unroll
        for (int i = 0; i < 4; i++) { // output 16 i + lane / 4
            const int j = VEC ? (lane >> 2) & 3 : i, p = lane & 3, c = VEC ? 4 * i + (lane >> 4) : lane >> 2;
            mine[64 * j + 16 * p + (c ^ (j + 4 * p))] = v[i];
        }
        const bool infinite = B == APART || (B == SOUGHT && __ballot(has_infinity(v)));
        own_fence();
        u32x4 bv[4];
#pragma unroll
        for (int j = 0; j < 4; j++)
            bv[j] = mine[64 * j + 16 * g + (col ^ (j + 4 * g))];
        own_fence();
        u32x4 lo[TT];
#pragma unroll
        for (int t = 0; t < TT; t++) {
            if (16 * t >= count)
                break;
            const u32x4 hi = low[(c * ALL + t) * 128 + lane];
            lo[t] = low[(c * ALL + t) * 128 + 64 + lane];
#pragma unroll
            for (int j = 0; j < 4; j++)
                acc[t][j] = mfma<BF16>(hi, bv[j], acc[t][j]);
            if (B == IGNORED)
#pragma unroll
                for (int j = 0; j < 4; j++)
                    acc[t][j] = mfma<BF16>(lo[t], bv[j], acc[t][j]);
        }
        if (B == IGNORED)
            return;
        if (__builtin_expect(infinite, B == APART))
            without_infinities(bv);
#pragma unroll
        for (int t = 0; t < TT; t++) {
            if (16 * t >= count)
                break;
#pragma unroll
            for (int j = 0; j < 4; j++)
                acc[t][j] = mfma<BF16>(lo[t], bv[j], acc[t][j]);
        }
    }

    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    static constexpr uint32_t ONES = BF16 ? 0x7f807f80u : 0x7c007c00u; // the exponents of infinities and NaNs

    static __device__ __forceinline__ bool has_infinity(const u32x4 (&v)[4]) // or a NaN
    {
        u16x2 most = {0, 0};
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t u = v[j][i] & 0x7fff7fffu;
                most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, u));
            }
        return max(most[0], most[1]) >= (ONES & 0xffffu);
    }

    static __device__ __forceinline__ void without_infinities(u32x4 (&v)[4])
    {
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int i = 0; i < 4; i++) { // times 0 where exponent and fraction are an infinity's, else 1
                const uint32_t u = v[j][i], apart = (u & 0x7fff7fffu) ^ ONES;
                const u16x2 kept = __builtin_bit_cast(u16x2, u) * __builtin_elementwise_min(__builtin_bit_cast(u16x2, apart), u16x2{1, 1});
                v[j][i] = __builtin_bit_cast(uint32_t, kept);
            }
    }

    __device__ __forceinline__ void finish(const Turn &k, const float4_t (&acc)[TT][4], int block) const
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int t = 0; t < TT; t++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int row = 16 * t + 4 * (lane >> 4) + i;
                if (row >= count)
                    continue;
                const float f = factor[row];
                uint16_t *out = a.out + rows[row] * a.out_stride;
                if (VEC) {
                    const int n = 64 * block + 4 * (lane & 15);
                    const uint2 y = k.y[VEC ? t : 0][i];
                    const uint16_t v0 = fq_from_float(fq_to_float((uint16_t)y.x, BF16) + f * acc[t][0][i], BF16);
                    const uint16_t v1 = fq_from_float(fq_to_float((uint16_t)(y.x >> 16), BF16) + f * acc[t][1][i], BF16);
                    const uint16_t v2 = fq_from_float(fq_to_float((uint16_t)y.y, BF16) + f * acc[t][2][i], BF16);
                    const uint16_t v3 = fq_from_float(fq_to_float((uint16_t)(y.y >> 16), BF16) + f * acc[t][3][i], BF16);
                    if (n < a.set.N)
                        *(uint2 *)(out + n) = make_uint2(v0 | (uint32_t)v1 << 16, v2 | (uint32_t)v3 << 16);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; j++) {
                        const int n = 64 * block + 16 * j + (lane & 15);
                        if (n < a.set.N)
                            out[n] = fq_from_float(fq_to_float(k.one[VEC ? 0 : t][i][j], BF16) + f * acc[t][j][i], BF16);
                    }
                }
            }
    }

    static __device__ __forceinline__ bool all_numbers(const float4_t (&acc)[TT][4])
    {
        float most[2] = {}; // (a maximum that is NaN where one of its operands is)
#pragma unroll
        for (int t = 0; t < TT; t++)
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < 4; i++)
                    most[j & 1] = __builtin_elementwise_maximum(most[j & 1], fabsf(acc[t][j][i]));
        return __builtin_elementwise_maximum(most[0], most[1]) < INFINITY;
    }

    // The blocks first, first + stride ...; k: what was asked for the first, if it was.  (A turn ahead in registers would cost half of the wavefronts, which hide
    // more.)  IGNORED: ends before a block whose sums are not all numbers, and returns it.
    template <Infinities B>
    __device__ __forceinline__ int walk(Turn &k, int first, int stride) const
    {
        const int blocks = (a.set.N + 63) / 64;
        int block = first;
        for (; block < blocks; block += stride) {
            if (B == APART || block != first)
                ask(k, block);
            float4_t acc[TT][4] = {};
            multiply<B>(acc, k.b[0], 0);
            if (AHEAD > 1 && chunks > 1)
                multiply<B>(acc, k.b[AHEAD - 1], 1);
            for (int c = AHEAD; c < chunks; c++) {
                u32x4 v[4];
                ask_b(v, block, c);
                multiply<B>(acc, v, c);
            }
            // vmcnt(0): y is here before the first store, behind which a wait for the rest of it would be one for the store (64 rows of 8 slots, 1024 -> 28672, rank
            // 16 25.6 to 22.9 us; the 2048 rows 43.8 to 43.3)
            __builtin_amdgcn_s_waitcnt(0x0f70);
            if (B == IGNORED && __ballot(!all_numbers(acc)))
                break;
            finish(k, acc, block);
        }
        return block;
    }

    __device__ __forceinline__ void run(Turn &k, int first, int stride) const
    {
        if (TT > 1 || AHEAD > 1) {
            walk<SOUGHT>(k, first, stride);
        } else {
            const int block = walk<IGNORED>(k, first, stride);
            if (64 * block < a.set.N)
                walk<APART>(k, block, stride);
        }
    }
};

// Rows without an adapter: copied, where out is not y.
__device__ __forceinline__ void copy_rows(const FqAdaptersArgs &a, const int *rows, int count, int first, int stride)
{
    if (a.out == a.y && a.out_stride == a.y_stride)
        return;
    for (int n = 64 * first + (threadIdx.x & 63); n < a.set.N; n += 64 * stride)
        for (int i = 0; i < count; i++)
            a.out[rows[i] * a.out_stride + n] = a.y[rows[i] * a.y_stride + n];
}

// Four ranks r .. r + 3 of row `row` of u as hi and lo into the operands.  `e`: the row's power of two.
template <int TT, bool BF16>
__device__ __forceinline__ void put_low(u32x4 *low, const float4_t u, int e, int row, int r)
{
    uint16_t hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float v = BF16 ? u[i] : ldexpf(u[i], e);
        hi[i] = fq_from_float(v, BF16);
        if (BF16 && (hi[i] & 0x7fff) == 0x7f80 && fabsf(v) < INFINITY)
            hi[i]--; // a number beyond bfloat16's largest: that one, and the rest in lo
        const float rest = v - fq_to_float(hi[i], BF16);
        lo[i] = fabsf(rest) < INFINITY ? fq_from_float(rest, BF16) : 0; // (not where hi is infinite or NaN)
    }
    // operand: lane row % 16 + 16 (rank % 32 / 8), its 8 ranks
    uint2 *at = (uint2 *)&low[((r >> 5) * TT + (row >> 4)) * 128 + (row & 15) + 16 * ((r & 31) >> 3)] + ((r & 7) >> 2);
    at[0] = make_uint2(hi[0] | (uint32_t)hi[1] << 16, hi[2] | (uint32_t)hi[3] << 16);
    at[128] = make_uint2(lo[0] | (uint32_t)lo[1] << 16, lo[2] | (uint32_t)lo[3] << 16);
}

// binary16: the row's largest finite number becomes 2^13 to 2^14 (a power of two changes no digit)
template <bool BF16>
__device__ __forceinline__ int power_of(float most)
{
    return BF16 || most == 0.0f ? 0 : min(max(14 - __builtin_amdgcn_frexp_expf(most), -126), 126);
}

// What a row's sums are multiplied by.  A finite scale stays inside binary32: an infinity would make NaN of a sum of 0 (other sums pass binary16 either way: they are
// 2^-48 at least).
template <bool BF16>
__device__ __forceinline__ float factor_of(float scale, int e)
{
    const float f = BF16 ? scale : ldexpf(scale, -e);
    return !BF16 && fabsf(scale) < INFINITY ? fminf(fmaxf(f, -0x1.fffffep127f), 0x1.fffffep127f) : f;
}

__device__ __forceinline__ float finite(const float4_t v)
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; i++)
        most = fmaxf(most, fabsf(v[i]) < INFINITY ? fabsf(v[i]) : 0.0f);
    return most;
}

// The parts of a tile's u as the operands of the last launch: the tile's piece of `low`, and the rows' factors.  (By every workgroup of the last launch it would
// be 131 KB each for 64 ranks in 8 parts: see joined_here.)  64 C ranks at most.
template <int C, bool BF16>
__global__ __launch_bounds__(JOIN_THREADS) void join_kernel(FqAdaptersArgs a, Work w)
{
    constexpr int ALL = TILE / 16;
    const int tid = threadIdx.x;
    const Tile own = w.tiles[blockIdx.x];
    const int count = own.count, rank = own.rank;
    if (JOIN_ROWS * (int)blockIdx.y >= count || rank == 0)
        return;
    // 16 threads to a row, four ranks to a thread and 64
    const int row = JOIN_ROWS * blockIdx.y + (tid >> 4), mine = 4 * (tid & 15), chunks = (rank + 31) / 32;
    const size_t apart = (size_t)a.M * a.set.rank;
    const float *from = w.low + (size_t)w.rows[TILE * blockIdx.x + min(row, count - 1)] * a.set.rank;
    float4_t u[C];
    float most = 0.0f;
#pragma unroll
    for (int c = 0; c < C; c++) {
        const int r = 64 * c + mine;
        u[c] = float4_t{0, 0, 0, 0};
        if (64 * c < rank && r < rank) {
            for (int p0 = 0; p0 < w.parts; p0 += 8) { // eight asked for together
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
            for (int i = 0; i < 4; i++)
                u[c][i] = r + i < rank ? u[c][i] : 0.0f;
            most = fmaxf(most, finite(u[c]));
        }
    }
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1)
        most = fmaxf(most, __shfl_xor(most, off, 64));
    const int e = power_of<BF16>(most);
    if (mine == 0)
        w.factor[TILE * blockIdx.x + row] = factor_of<BF16>(own.scale, e);
    u32x4 *low = w.operands + (size_t)blockIdx.x * w.tile_operands;
#pragma unroll
    for (int c = 0; c < C; c++)
        if (64 * c < rank && 64 * c + mine < 32 * chunks)
            put_low<ALL, BF16>(low, u[c], e, row, 64 * c + mine);
}

// The same by every workgroup of the last launch, into operands and factors of its own: PARTS parts at most of the rows of PASSES turns, all asked for
// together (turn by turn, 701 rows of rank 32, 4096 -> 4096, 20.7 us instead of 19.5).
template <int PARTS, int PASSES, bool BF16>
__device__ __forceinline__ void join_rows(const FqAdaptersArgs &a, const Work &w, const Tile &own, const int *rows, float *factor, u32x4 *low, int wide)
{
    const int step = MANY_THREADS / wide, own_row = threadIdx.x / wide, r = 4 * (threadIdx.x & (wide - 1)), last = own.rank - 1;
    const size_t apart = (size_t)a.M * a.set.rank;
    for (int row0 = own_row; row0 < min((own.count + 15) & ~15, TILE); row0 += step * PASSES) { // (a row's threads together)
        float4_t part[PASSES][PARTS];
#pragma unroll
        for (int k = 0; k < PASSES; k++) {
            const float *from = w.low + (size_t)rows[min(row0 + k * step, own.count - 1)] * a.set.rank + min(r, last & ~3);
#pragma unroll
            for (int p = 0; p < PARTS; p++)
                part[k][p] = *(const float4_t *)(from + (size_t)min(p, w.parts - 1) * apart);
        }
#pragma unroll
        for (int k = 0; k < PASSES; k++) {
            const int row = row0 + k * step;
            float4_t u = {0, 0, 0, 0};
#pragma unroll
            for (int p = 0; p < PARTS; p++)
                if (p < w.parts)
                    u += part[k][p];
#pragma unroll
            for (int i = 0; i < 4; i++)
                u[i] = r + i <= last ? u[i] : 0.0f;
            float most = finite(u);
            for (int off = wide / 2; off >= 1; off >>= 1)
                most = fmaxf(most, __shfl_xor(most, off, 64));
            const int e = power_of<BF16>(most);
            if (row < TILE) {
                if (r == 0)
                    factor[row] = factor_of<BF16>(own.scale, e);
                if (r < (own.rank + 31) / 32 * 32)
                    put_low<TILE / 16, BF16>(low, u, e, row, r);
            }
        }
    }
}

// out = y + scale u B^T of a tile.  A wavefront has half of the tile's rows: with all of them 238 registers leave one workgroup to a compute unit.
template <bool BF16, bool VEC, bool JOIN>
__global__ __launch_bounds__(MANY_THREADS, 3) void out_kernel(FqAdaptersArgs a, Work w)
{
    constexpr int ALL = TILE / 16, TT = ALL / 2, COLUMNS = MANY_THREADS / 128;
    __shared__ int rows[TILE];
    __shared__ float factor[TILE];
    __shared__ u32x4 b_of[MANY_THREADS / 64][256];
    extern __shared__ u32x4 low[]; // [rank / 32][ALL][2][64]
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row0 = 16 * TT * (wave & 1);
    if ((int)blockIdx.x >= w.max_tiles)
        return;
    if (!JOIN && tid < TILE)
        factor[tid] = w.factor[TILE * blockIdx.x + tid];
    if (JOIN && a.set.rank <= 16)
        for (int i = tid; i < ALL * 128; i += MANY_THREADS)
            low[i] = u32x4{0, 0, 0, 0};
    const Tile own = find_listed(w, rows);
    const int count = own.count, rank = own.rank;
    if (count == 0)
        return;
    const int first = blockIdx.y * COLUMNS + (wave >> 1), stride = gridDim.y * COLUMNS;
    if (rank == 0)
        return copy_rows(a, rows + row0, min(count - row0, 16 * TT), first, stride);
    const Out<TT, ALL, 1, BF16, VEC> o{a, rows + row0, factor + row0, low + TT * 128 * (wave & 1), b_of[wave],
                                       a.set.b + own.slot * a.set.b_stride, count - row0, rank, (rank + 31) / 32};
    typename Out<TT, ALL, 1, BF16, VEC>::Turn now;
    if (JOIN) {
        if (64 * first < a.set.N)
            o.ask(now, first);
        const int wide = threads_a_row(a.set);
        if (w.parts <= 4)
            join_rows<4, 4, BF16>(a, w, own, rows, factor, low, wide);
        else if (w.parts <= 8)
            join_rows<8, 2, BF16>(a, w, own, rows, factor, low, wide);
        else
            join_rows<MAX_PARTS, 1, BF16>(a, w, own, rows, factor, low, wide);
    } else {
        const u32x4 *from = w.operands + (size_t)blockIdx.x * w.tile_operands;
        for (int i = tid; i < o.chunks * ALL * 128; i += MANY_THREADS)
            low[i] = from[i];
        if (64 * first < a.set.N)
            o.ask(now, first);
    }
    __syncthreads();
    if (row0 < count)
        o.run(now, first, stride);
}

// Few rows, up to 64 GROUPS, one launch: the tile that row blockIdx.x leads (the rows of its slot before it fill whole tiles), the outputs that are blockIdx.y's.  A
// wavefront forms u over pieces of K of its own, 128 / RT at a time, two asked for ahead, through LDS of its own (a row's piece p at p ^ row, or p ^ row /
// 2 where a row is 64 bytes); the sums of the eight meet there.  LDS for two workgroups to a compute unit: rows that lead no tile have one, too.
template <int RT, int GROUPS, bool BF16, bool VEC>
__global__ __launch_bounds__(OUT_THREADS, 4) void few_kernel(FqAdaptersArgs a)
{
    constexpr int WAVES = OUT_THREADS / 64, PIECES = 16 / RT, LANES = 64 / PIECES, A_TURNS = 16 * RT / LANES, X_TURNS = 16 / LANES;
    constexpr int OWN = (16 + 16 * RT) * PIECES, CHUNKS = (RT + 1) / 2;
    __shared__ int rows[FEW_TILE];
    __shared__ float factor[FEW_TILE];
    __shared__ u32x4 low[CHUNKS * 128];
    __shared__ u32x4 lds[WAVES][OWN > 256 ? OWN : 256];
    static_assert(RT * 64 <= OWN, "the sums of a wavefront");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, g = lane >> 4;
    const Some some(a);
    const int lead = blockIdx.x;
    int found[GROUPS], slot = -1, before = 0, seen = 0;
    uint64_t same[GROUPS];
#pragma unroll
    for (int i = 0; i < GROUPS; i++)
        found[i] = a.adapter[min(64 * i + lane, a.M - 1)];
#pragma unroll
    for (int i = 0; i < GROUPS; i++) {
        found[i] = 64 * i + lane >= a.M ? -2 : found[i] >= 0 && found[i] < a.set.slots ? found[i] : -1;
        if (lead >> 6 == i)
            slot = __builtin_amdgcn_readlane(found[i], lead & 63);
    }
#pragma unroll
    for (int i = 0; i < GROUPS; i++) {
        same[i] = __ballot(found[i] == slot);
        const int upto = lead - 64 * i;
        before += __popcll(upto <= 0 ? 0 : upto >= 64 ? same[i] : same[i] & ((1ull << upto) - 1));
    }
    if (before % FEW_TILE != 0)
        return;
#pragma unroll
    for (int i = 0; i < GROUPS; i++) {
        const int at = seen + __popcll(same[i] & ((1ull << lane) - 1)) - before;
        if (wave == 0 && found[i] == slot && at >= 0 && at < FEW_TILE)
            rows[at] = 64 * i + lane;
        seen += __popcll(same[i]);
    }
    const int count = min(seen - before, FEW_TILE);
    int rank;
    float scale;
    some.of(a, slot, rank, scale);
    __syncthreads();
    const int first = blockIdx.y * WAVES + wave, stride = gridDim.y * WAVES;
    if (rank == 0)
        return copy_rows(a, rows, count, first, stride);
    const int K = a.set.K, piece = lane % PIECES, row0 = lane / PIECES;
    const uint16_t *ap = a.set.a + slot * a.set.a_stride, *xp[X_TURNS];
#pragma unroll
    for (int i = 0; i < X_TURNS; i++)
        xp[i] = a.x + rows[min(row0 + i * LANES, count - 1)] * a.x_stride;
    struct Step {
        u32x4 x[X_TURNS], a[A_TURNS];
    };
    // (rows beyond the last are the last again, and not used)
    auto ask = [&](Step &s, int k) {
        const int at = min(k + 8 * piece, K - 8);
#pragma unroll
        for (int i = 0; i < A_TURNS; i++)
            s.a[i] = *(const u32x4 *)(ap + (size_t)min(row0 + i * LANES, rank - 1) * K + at);
#pragma unroll
        for (int i = 0; i < X_TURNS; i++)
            s.x[i] = *(const u32x4 *)(xp[i] + at);
    };
    auto place = [&](int row, int p) -> u32x4 & {
        return lds[wave][row * PIECES + (p ^ ((PIECES >= 8 ? row : row >> 1) & (PIECES - 1)))];
    };
    float4_t acc[RT] = {};
    constexpr int STEP = 8 * PIECES, APART = STEP * WAVES;
    auto use = [&](Step &s, int k) {
        if (k + STEP > K && k + 8 * piece >= K) { // behind the end of K
#pragma unroll
            for (int i = 0; i < A_TURNS; i++)
                s.a[i] = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < X_TURNS; i++)
                s.x[i] = u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < A_TURNS; i++)
            place(16 + row0 + i * LANES, piece) = s.a[i];
#pragma unroll
        for (int i = 0; i < X_TURNS; i++)
            place(row0 + i * LANES, piece) = s.x[i];
        own_fence();
        if (k + 2 * APART < K)
            ask(s, k + 2 * APART);
#pragma unroll
        for (int h = 0; h < PIECES / 4; h++) {
            const u32x4 x = place(col, 4 * h + g);
#pragma unroll
            for (int r = 0; r < RT; r++)
                acc[r] = mfma<BF16>(place(16 + 16 * r + col, 4 * h + g), x, acc[r]);
        }
        own_fence();
    };
    Step even, odd;
    int k = STEP * wave;
    if (k < K)
        ask(even, k);
    if (k + APART < K)
        ask(odd, k + APART);
    for (; k < K; k += 2 * APART) {
        use(even, k);
        if (k + APART < K)
            use(odd, k + APART);
    }
    const Out<1, 1, CHUNKS, BF16, VEC> o{a, rows, factor, low, lds[wave], a.set.b + slot * a.set.b_stride, count, rank, (rank + 31) / 32};
    typename Out<1, 1, CHUNKS, BF16, VEC>::Turn now;
    if (64 * first < a.set.N)
        o.ask(now, first);
    // u[rank 16 r + 4 g + i][row col] of each wavefront
#pragma unroll
    for (int r = 0; r < RT; r++)
        ((float4_t *)lds[wave])[64 * r + lane] = acc[r];
    __syncthreads();
    // four ranks to a thread, the threads of whole instructions (32 ranks) to a row
    constexpr int WIDE = RT == 1 ? 8 : 4 * RT;
    const int row = tid / WIDE, r = 4 * (tid % WIDE);
    if (row < FEW_TILE) {
        float4_t u = {0, 0, 0, 0};
        if (r < rank) {
#pragma unroll
            for (int v = 0; v < WAVES; v++)
                u += ((const float4_t *)lds[v])[64 * (r >> 4) + row + 16 * ((r & 15) >> 2)];
#pragma unroll
            for (int i = 0; i < 4; i++)
                u[i] = r + i < rank ? u[i] : 0.0f;
        }
        float most = finite(u);
#pragma unroll
        for (int off = WIDE / 2; off >= 1; off >>= 1)
            most = fmaxf(most, __shfl_xor(most, off, 64));
        const int e = power_of<BF16>(most);
        if (r == 0)
            factor[row] = factor_of<BF16>(scale, e);
        put_low<1, BF16>(low, u, e, row, r);
    }
    __syncthreads();
    o.run(now, first, stride);
}

template <int GROUPS, bool BF16, bool VEC>
hipError_t launch_few(const FqAdaptersArgs &a, hipStream_t stream)
{
    const dim3 grid(a.M, few_shares(a.set, a.M));
    if (a.set.rank <= 16)
        few_kernel<1, GROUPS, BF16, VEC><<<grid, OUT_THREADS, 0, stream>>>(a);
    else if (a.set.rank <= 32)
        few_kernel<2, GROUPS, BF16, VEC><<<grid, OUT_THREADS, 0, stream>>>(a);
    else
        few_kernel<4, GROUPS, BF16, VEC><<<grid, OUT_THREADS, 0, stream>>>(a);
    return hipGetLastError();
}

template <int RT, bool BF16, Find FIND>
void launch_low(const FqAdaptersArgs &a, const Work &w, hipStream_t stream)
{
    const dim3 grid(w.max_tiles, w.parts, (a.set.rank + 16 * RT - 1) / (16 * RT)); // (16 RT = low_ranks)
    low_kernel<RT, BF16, FIND><<<grid, THREADS, 0, stream>>>(a, w);
}

// Whether the workgroups of the last launch add up the parts by themselves: a thread's loads, times the workgroups of a compute unit.  By themselves / in a launch
// (us on the device, those loads): 701 rows, 11008 -> 4096, rank 16 17.5 / 20.1 (24); 3 rows, 9344 -> 634, rank 32 11.1 / 14.1 (16); 2048, 4096 -> 4096, rank 32 24.4 / 25.2
// (33); 701, rank 32 16.6 / 17.9 (48); 64, 8192 -> 8192, rank 64 16.2 / 16.7 (64); 300, 4096 -> 4096, rank 64 17.8 / 17.2 (64); 2048, 8192 -> 8192, rank 64 51 / 48 (105);
// 200, 4096 -> 4096, rank 128 21.4 / 18.3 (128).
bool joined_here(const FqAdaptersArgs &a, const Work &w, int workgroups)
{
    const int rows = a.M < TILE ? a.M : TILE, step = MANY_THREADS / threads_a_row(a.set), parts = w.parts <= 4 ? 4 : w.parts <= 8 ? 8 : MAX_PARTS;
    return (long long)((rows + step - 1) / step) * parts * (workgroups > 256 ? workgroups : 256) <= 64 * 256;
}

template <bool BF16, bool VEC, bool JOIN>
hipError_t launch_out(const FqAdaptersArgs &a, const Work &w, dim3 grid, size_t lds, hipStream_t stream)
{
    if (lds > 16384)
        if (hipError_t e = fq_raise_dynamic_lds((const void *)out_kernel<BF16, VEC, JOIN>, lds))
            return e;
    out_kernel<BF16, VEC, JOIN><<<grid, MANY_THREADS, lds, stream>>>(a, w);
    return hipGetLastError();
}

template <bool BF16, bool VEC, Find FIND>
hipError_t launch_many(const FqAdaptersArgs &a, const Work &w, hipStream_t stream)
{
    const int ranks = low_ranks(a.set);
    if (ranks == 16)
        launch_low<1, BF16, FIND>(a, w, stream);
    else if (ranks == 32)
        launch_low<2, BF16, FIND>(a, w, stream);
    else
        launch_low<4, BF16, FIND>(a, w, stream);
    if (hipError_t e = hipGetLastError())
        return e;
    // outputs over as many workgroups as fill the chip, three to a compute unit
    const int blocks = (a.set.N + 63) / 64, tiles = tiles_likely(a.set, a.M), columns = MANY_THREADS / 128;
    const int most = (blocks + columns - 1) / columns, room = 768 / tiles > 1 ? 768 / tiles : 1;
    const int turns = (most + room - 1) / room;
    const dim3 grid(out_tiles(a.set, a.M), (most + turns - 1) / turns);
    const size_t lds = (size_t)w.tile_operands * sizeof(u32x4);
    if (joined_here(a, w, tiles * grid.y))
        return launch_out<BF16, VEC, true>(a, w, grid, lds, stream);
    const dim3 join_grid(w.max_tiles, TILE / JOIN_ROWS);
    if (a.set.rank <= 64)
        join_kernel<1, BF16><<<join_grid, JOIN_THREADS, 0, stream>>>(a, w);
    else
        join_kernel<FQ_MAX_ADAPTER_RANK / 64, BF16><<<join_grid, JOIN_THREADS, 0, stream>>>(a, w);
    if (hipError_t e = hipGetLastError())
        return e;
    return launch_out<BF16, VEC, false>(a, w, grid, lds, stream);
}

template <bool BF16, bool VEC>
hipError_t launch(const FqAdaptersArgs &a, void *workspace, hipStream_t stream)
{
    const FqAdaptersRoute route = fq_adapters_route(a.set, a.M);
    if (route.few)
        return a.M <= 64 ? launch_few<1, BF16, VEC>(a, stream) : launch_few<FEW_ROWS / 64, BF16, VEC>(a, stream);
    Work w{};
    w.parts = parts_of(a.set, a.M);
    w.max_tiles = tiles_of(a.set, a.M);
    char *at = (char *)workspace;
    w.low = (float *)at;
    at += up(low_rows(a.M) * a.set.rank * sizeof(float));
    w.rows = (int *)at;
    at += up((size_t)w.max_tiles * TILE * sizeof(int));
    w.tiles = (Tile *)at;
    at += up(w.max_tiles * sizeof(Tile));
    w.factor = (float *)at;
    at += up((size_t)w.max_tiles * TILE * sizeof(float));
    w.operands = (u32x4 *)at;
    w.tile_operands = tile_operands(a.set);
    if (!route.listed)
        return launch_many<BF16, VEC, COUNTED>(a, w, stream);
    const size_t lds = (a.set.slots + 1) * sizeof(int);
    if (lds > 32768)
        if (hipError_t e = fq_raise_dynamic_lds((const void *)group_kernel, lds))
            return e;
    group_kernel<<<1, GROUP_THREADS, lds, stream>>>(a, w);
    if (hipError_t e = hipGetLastError())
        return e;
    return launch_many<BF16, VEC, LISTED>(a, w, stream);
}

} // namespace

FqAdaptersRoute fq_adapters_route(const FqAdaptersView &set, int M)
{
    if (few(set, M))
        return {1, 0, M * few_shares(set, M), 0};
    const int groups = tiles_of(set, M) * parts_of(set, M) * ((set.rank + low_ranks(set) - 1) / low_ranks(set));
    return {0, M > MIDDLE_ROWS || set.slots > MIDDLE_SLOTS || groups > COUNTING, groups, out_tiles(set, M)};
}

size_t fq_adapters_bytes(const FqAdaptersView &set, int M)
{
    const size_t tiles = tiles_of(set, M);
    return up(low_rows(M) * set.rank * sizeof(float)) + up(tiles * TILE * sizeof(int)) + up(tiles * sizeof(Tile)) + up(tiles * TILE * sizeof(float)) +
           tiles * tile_operands(set) * sizeof(u32x4) + 256;
}

hipError_t fq_launch_adapters(const FqAdaptersArgs &a, void *workspace, hipStream_t stream)
{
    // four outputs of a row at a time
    const bool vec = a.set.N % 4 == 0 && a.y_stride % 4 == 0 && a.out_stride % 4 == 0 && ((uintptr_t)a.y & 7) == 0 && ((uintptr_t)a.out & 7) == 0;
    if (a.set.bf16)
        return vec ? launch<true, true>(a, workspace, stream) : launch<true, false>(a, workspace, stream);
    return vec ? launch<false, true>(a, workspace, stream) : launch<false, false>(a, workspace, stream);
}
