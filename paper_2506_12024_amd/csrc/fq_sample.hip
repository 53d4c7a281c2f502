// Drawing the next token from a row of logits: temperature, top-k, top-p, min-p and a given random number.
//
// Weights are whole numbers (exp in binary64, rounded to a unit under which V of them still fit 62 bits), so sums are exact in any
// order and atomics give the same bits every time.  One workgroup takes a row, each of its wavefronts four stretches of it, side by side:
//   1. the largest logit
//   2. top-k of at most 1024: the k-th largest of the 1024 threads' own largest is no larger than the k-th of all, so the few
//      entries from it on go to a list in LDS, which takes the row's place
//   3. a cut (the entry at which a running count or sum, from the largest logit down, reaches its target): a histogram over 2048
//      steps of 1/32 octave from the top, the step that holds the target, and the entries of that step in order (a step of more than
//      1024 entries -- flat rows, equal logits -- is parted by standing first, 11 bits at a time)
//   4. the draw: kept weights summed over the 64 stretches, the one that holds the target, its entries in order
// Bound by reading a long row two (top-k, temperature, min-p) or three times (top-p), all but the first from the caches, and by
// the exponentials of the entries that count; by the chain of steps for a short one.  Measured, 256 rows of 128256 (131 MB, 22 us to
// read once): top-k 50 47 us, temperature alone 58, top-p 0.95 92, all of them mixed 107 to 116 (by the settings drawn); one row of
// 32000 with top-k 50 15 us, with top-p 0.95 26.  Rows count from the 16-byte boundary before them, so that any row is read 16 bytes at a
// time: 256 of 128255 with top-p 0.95 96 us; it costs aligned rows 0.5 to 2 %.  1024 threads have 128 registers each: the fp16 instance
// keeps 4 of its vector and both 64 of their scalar registers elsewhere (scratch, spare lanes).
#include <hip/hip_runtime.h>

#include "fq_internal.h"

namespace {

constexpr int THREADS = 1024;
constexpr int WAVES = THREADS / 64;
constexpr int ROOTS = 128;   // steps of an octave
constexpr int BINS = 2048;   // groups of four steps from the top, 64 octaves; the last one holds what lies further down (weight 0)
constexpr int STRETCHES = 64;
constexpr int LIST = 8192;  // entries of the list of step 2
constexpr int FEW = 256;     // entries of a list that need no histogram
constexpr int CELL = 1024;  // entries of one step that are put in order there
constexpr int DEEPEST = -128 * ROOTS; // no entry lies as far down, in steps
typedef unsigned long long u64;

// Binary32 values as unsigned numbers in the same order, -0 as 0.  (NaNs are nowhere larger or equal and weigh nothing.)
__device__ __forceinline__ uint32_t ordered(float f)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, f + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t k)
{
    return __builtin_bit_cast(float, k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// Where a logit stands: larger is earlier, of equal ones the smaller index.
__device__ __forceinline__ u64 standing(float f, int i) { return ((u64)ordered(f) << 32) | (0xffffffffu - (uint32_t)i); }

// floor(x * w) for x in [0, 1) with 24 bits of precision, and whether anything was cut off
__device__ __forceinline__ u64 share(float x, u64 w, bool &rest)
{
    const u64 f = (u64)((double)x * 18446744073709551616.0);
    rest = f * w != 0;
    return __umul64hi(f, w);
}

// 2^(j / 128): the series of exp to the 13th power on an argument of at most ln 2 / 2 (what is left out is under 2^-57)
__device__ __forceinline__ double root_of_two(int j)
{
    const double x = (j > ROOTS / 2 ? j - ROOTS : j) * (0.69314718055994530942 / ROOTS);
    double p = 1.0;
    for (int i = 13; i >= 1; i--)
        p = fma(p * x, 1.0 / i, 1.0);
    return j > ROOTS / 2 ? 2.0 * p : p;
}

// How far down a logit lies: n + f steps of 1/128 octave, n whole, |f| <= 1/2.
struct Depth {
    double f;
    int n;
};

// The weight of a logit, 2^((n + f) / 128): table[n % 128] times a polynomial in f (the series to the fourth power, under 2^-49
// left out) times 2^(n / 128).  Binary64 instructions bound the passes over a row, so there are ten of them: the distance from the
// top is multiplied twice (once rounded to a whole number by a sum with 1.5 * 2^52, once less that number), the weight is rounded to a
// whole number by the sum with 2^52 that its last product ends in, nothing is converted between double and integer, and what is too far
// down is held up in binary32.  The coefficients stay in vector registers (pinned: as literals or in scalar ones they took nine
// moves to a weight).
struct Weigh {
    double top, scale; // the largest logit; 128 / (temperature * ln 2)
    float lowest;      // 64 octaves down and more (-inf and NaNs too) the weight rounds to 0
    bool careful;      // temperature or logits so large or small that the above does not hold in binary32, or an infinite top
    double least;      // min_p times the unit, 0 for none
    const double *table;
    double c1 = 0.69314718055994530942 / ROOTS, c2 = c1 * c1 / 2, c3 = c1 * c2 / 3, c4 = c1 * c3 / 4;
    __device__ __forceinline__ Weigh(float top_, double temperature, double least_, const double *table_)
        : top(top_), scale(ROOTS * 1.4426950408889634074 / temperature), least(least_), table(table_)
    {
        // one step of binary32 at the top is less than the 64 octaves, and they end above the lowest value
        const double reach = 64.0 * ROOTS / scale;
        careful = !(fabs(top) * 0x1p-23 < reach && reach > 1e-30 && fabs(top) + reach < 1e38);
        if (top_ == INFINITY)
            scale = INFINITY; // what is finite has no weight
        lowest = careful ? 0.0f : __double2float_rd(top - 64.0 * ROOTS / scale);
        asm volatile("" : "+v"(c1), "+v"(c2), "+v"(c3), "+v"(c4));
    }
    __device__ __forceinline__ Depth depth(float l) const
    {
        double x, s;
        if (careful) { // (the same for the whole row)
            x = l == (float)top ? 0.0 : fmax(((double)l - top) * scale, -64.0 * ROOTS);
            s = 1.0;
        } else {
            x = (double)fmaxf(l, lowest) - top;
            s = scale;
        }
        const double m = fma(x, s, 0x1.8p52);
        return Depth{fma(x, s, 0x1.8p52 - m), (int)(uint32_t)__builtin_bit_cast(u64, m)};
    }
    __device__ __forceinline__ double series(double f) const
    {
        double p = fma(f, c4, c3);
        p = fma(f, p, c2);
        p = fma(f, p, c1);
        return fma(f, p, 1.0);
    }
    __device__ __forceinline__ double power(int n) const // times the unit
    {
        return __builtin_bit_cast(double, __builtin_bit_cast(u64, table[n & (ROOTS - 1)]) + ((u64)(uint32_t)((n & ~(ROOTS - 1)) << 13) << 32));
    }
    static __device__ __forceinline__ u64 low_bits(double v) { return __builtin_bit_cast(u64, v) & ((1ULL << 52) - 1); }
    __device__ __forceinline__ u64 whole(const Depth &d) const // at most 2^51
    {
        return low_bits(fma(power(d.n), series(d.f), 0x1p52));
    }
    __device__ __forceinline__ u64 kept(const Depth &d) const // what min-p leaves of it: all of the same whole number, or nothing
    {
        const double v = power(d.n) * series(d.f);
        return v >= least ? whole(d) : 0;
    }
    static __device__ __forceinline__ int bin(const Depth &d) { return min(max(-d.n, 0) >> 2, BINS - 1); }
    // no entry of the first `bins` bins lies below this
    __device__ __forceinline__ float floor_of(int bins) const
    {
        return careful ? -INFINITY : __double2float_rd(top - (4.0 * bins + 1.0) / scale);
    }
};

// The last entry that is kept, in the order of standing.
struct Cut {
    float l;
    int i;
    __device__ __forceinline__ bool keeps(float x, int at) const { return x > l || (x == l && at <= i); }
};
__device__ __forceinline__ Cut cut_of(u64 standing)
{
    return Cut{unordered((uint32_t)(standing >> 32)), (int)(0xffffffffu - (uint32_t)standing)};
}
constexpr Cut FQ_NO_CUT = {-INFINITY, 0x7fffffff};

// What lane i of a wavefront holds plus what the lanes before it hold: within rows of 16 lanes, then the rows' sums.
template <int DPP, int ROWS>
__device__ __forceinline__ u64 add_from(u64 v)
{
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)v, DPP, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(v >> 32), DPP, ROWS, 0xf, false);
    return v + (((u64)hi << 32) | lo);
}
__device__ __forceinline__ u64 wave_running(u64 v)
{
    v = add_from<0x111, 0xf>(v); // row_shr 1, 2, 4, 8
    v = add_from<0x112, 0xf>(v);
    v = add_from<0x114, 0xf>(v);
    v = add_from<0x118, 0xf>(v);
    v = add_from<0x142, 0xa>(v); // lane 15 of a row to the next row: rows 1 and 3
    v = add_from<0x143, 0xc>(v); // lane 31 to rows 2 and 3
    return v;
}
__device__ __forceinline__ u64 wave_sum(u64 v)
{
    v = wave_running(v);
    return ((u64)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(v >> 32), 63) << 32) | (uint32_t)__builtin_amdgcn_readlane((uint32_t)v, 63);
}

struct Shared {
    u64 bins[BINS];
    u64 stretch[STRETCHES];
    double table[ROOTS];
    u64 cell_key[CELL], cell_w[CELL];
    float list_l[LIST];
    int list_i[LIST];
    u64 wave[WAVES];
    u64 word[2];
    int count;
};

// Running sum of one value a thread, in thread order (its own included), and the sum of all.
__device__ __forceinline__ u64 running(Shared &s, u64 v, u64 &all)
{
    const int lane = threadIdx.x & 63;
    v = wave_running(v);
    __syncthreads();
    if (lane == 63)
        s.wave[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 before = 0;
    all = 0;
#pragma unroll
    for (int i = 0; i < WAVES; i++) {
        const u64 w = s.wave[i];
        before += i < (int)(threadIdx.x >> 6) ? w : 0;
        all += w;
    }
    return before + v;
}

// The row.  each(f) calls f(logits, index of the first) for every VEC entries once, all 64 lanes of a wavefront together (-inf where
// there is no entry); stretches(f, g) besides g(stretch) after each of the wavefront's stretches of `length` entries (a multiple of
// 64 VEC).
template <class T, int VEC_>
struct Row {
    static constexpr int VEC = VEC_;
    static constexpr bool LIST = false;
    const T *x;      // the row
    int V, skip, length; // skip: entries before it on a 16-byte boundary, which `at` below counts from (rows begin anywhere)
    typedef T Vec __attribute__((ext_vector_type(VEC)));

    __device__ __forceinline__ void block(int at, int end, float (&l)[VEC]) const
    {
        if (at >= skip && at + VEC <= end) {
            const Vec v = *(const Vec *)(x + (at - skip));
#pragma unroll
            for (int e = 0; e < VEC; e++)
                l[e] = (float)v[e];
        } else {
#pragma unroll
            for (int e = 0; e < VEC; e++)
                l[e] = at + e >= skip && at + e < end ? (float)x[at + e - skip] : -INFINITY;
        }
    }
    // LIGHT passes ask for 64 bytes a thread at once; the others (exponentials) for the next 32 while the last are worked on.  A
    // wavefront's stretches lie side by side, and requests run across their ends.
    template <bool LIGHT, class F, class G>
    __device__ __forceinline__ void stretches(const F &f, const G &g) const
    {
        constexpr int AHEAD = (LIGHT ? 64 : 32) / (VEC * (int)sizeof(T)), STEP = AHEAD * 64 * VEC;
        const int lane = threadIdx.x & 63;
        int part = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * (STRETCHES / WAVES);
        const int begin = part * length, end = min(begin + STRETCHES / WAVES * length, V + skip);
        int part_end = begin + length;
        float l[AHEAD][VEC];
        auto ask = [&](int first, float (&to)[AHEAD][VEC]) {
#pragma unroll
            for (int b = 0; b < AHEAD; b++)
                if (first + b * 64 * VEC < end)
                    block(first + (b * 64 + lane) * VEC, end, to[b]);
        };
        if (!LIGHT)
            ask(begin, l);
        for (int first = begin; first < end; first += STEP) {
            float next[AHEAD][VEC];
            if (LIGHT)
                ask(first, l);
            else if (first + STEP < end)
                ask(first + STEP, next);
#pragma unroll
            for (int b = 0; b < AHEAD; b++) {
                const int at = first + b * 64 * VEC;
                if (at < end) {
                    f(l[b], at + lane * VEC - skip);
                    if (at + 64 * VEC >= (part_end < end ? part_end : end)) {
                        g(part++);
                        part_end += length;
                    }
                }
            }
            if (!LIGHT)
#pragma unroll
                for (int b = 0; b < AHEAD; b++)
#pragma unroll
                    for (int e = 0; e < VEC; e++)
                        l[b][e] = next[b][e];
        }
    }
    template <bool LIGHT, class F>
    __device__ __forceinline__ void each(const F &f) const
    {
        stretches<LIGHT>(f, [](int) {});
    }
    template <bool LIGHT, class F, class G>
    __device__ __forceinline__ void each(const F &f, const G &flush) const // flush() after every stretch
    {
        stretches<LIGHT>(f, [&](int) { flush(); });
    }
};

// The row, with what is to be done at the end of a stretch.
template <class R, class End>
struct RowOf {
    static constexpr int VEC = R::VEC;
    static constexpr bool LIST = false;
    const R &row;
    const End &end;
    template <bool LIGHT, class F>
    __device__ __forceinline__ void each(const F &f) const
    {
        row.template stretches<LIGHT>(f, end);
    }
    template <bool LIGHT, class F, class G>
    __device__ __forceinline__ void each(const F &f, const G &flush) const
    {
        row.template stretches<LIGHT>(f, [&](int part) {
            flush();
            end(part);
        });
    }
};

struct Listed {
    static constexpr int VEC = 1;
    static constexpr bool LIST = true;
    const Shared *s;
    int n;
    template <bool LIGHT, class F>
    __device__ __forceinline__ void each(const F &f) const
    {
        for (int at = threadIdx.x; at - (int)threadIdx.x < n; at += THREADS) {
            const float l[1] = {at < n ? s->list_l[at] : -INFINITY};
            f(l, at < n ? s->list_i[at] : 0);
        }
    }
};

// Among the weights added up in s.bins (bins[0] first): the one at which the running sum reaches `target`; false if it never does.
// word[0]: that one; word[1]: what is left of the target there.  N <= 2048 bins, two to a thread.
template <int N, class Target>
__device__ __forceinline__ bool find_bin(Shared &s, const Target &target_of)
{
    __syncthreads();
    const int i = 2 * threadIdx.x;
    const u64 x = i < N ? s.bins[i] : 0, y = i + 1 < N ? s.bins[i + 1] : 0;
    u64 all;
    const u64 to = running(s, x + y, all), from = to - x - y;
    const u64 target = target_of(all);
    if (target == 0 || target > all)
        return false;
    if (from < target && target <= to) {
        const bool first = target <= from + x;
        s.word[0] = first ? i : i + 1;
        s.word[1] = target - (first ? from : from + x);
    }
    __syncthreads();
    return true;
}

// Of the n entries of the cell, from the largest standing down: the one at which the running sum of weights reaches `target`
// (1 <= target <= the sum).  More than 256 of them: eight bits of the standing at a time.
__device__ __forceinline__ u64 reach_cell(Shared &s, int n, u64 target)
{
    if (n > 256) {
        u64 found = 0;
        for (int shift = 56; shift >= 0; shift -= 8) {
            __syncthreads();
            if (threadIdx.x < 256)
                s.bins[threadIdx.x] = 0;
            __syncthreads();
            if ((int)threadIdx.x < n) {
                const u64 key = s.cell_key[threadIdx.x];
                if (shift == 56 || (key >> (shift + 8)) == (found >> (shift + 8)))
                    atomicAdd(&s.bins[255 - ((key >> shift) & 255)], s.cell_w[threadIdx.x]);
            }
            find_bin<256>(s, [&](u64) { return target; });
            found |= (255 - s.word[0]) << shift;
            target = s.word[1];
        }
        __syncthreads();
        return found;
    }
    // four threads to an entry: what stands before it
    const int mine = threadIdx.x >> 2;
    if (mine < n) {
        const u64 key = s.cell_key[mine], w = s.cell_w[mine];
        u64 before = 0;
        for (int i = threadIdx.x & 3; i < n; i += 4)
            before += s.cell_key[i] > key ? s.cell_w[i] : 0;
        before += __shfl_xor(before, 1);
        before += __shfl_xor(before, 2);
        if (before < target && target <= before + w)
            s.word[0] = key;
    }
    __syncthreads();
    const u64 found = s.word[0];
    __syncthreads();
    return found;
}

// Entries with a weight go to the cell, counted once for a wavefront (all of whose lanes call this).
__device__ __forceinline__ void put_in_cell(Shared &s, u64 w, u64 key, u64 &lowest, u64 &highest)
{
    const u64 who = __ballot(w != 0);
    if (!who)
        return;
    int base = 0;
    if ((threadIdx.x & 63) == 0)
        base = atomicAdd(&s.count, __popcll(who));
    const int at = __builtin_amdgcn_readfirstlane(base) + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
    if (w) {
        lowest = key < lowest ? key : lowest;
        highest = key > highest ? key : highest;
        if (at < CELL) {
            s.cell_key[at] = key;
            s.cell_w[at] = w;
        }
    }
}

// The largest of all threads' values.
__device__ __forceinline__ u64 wg_most(Shared &s, u64 v)
{
    for (int o = 32; o; o >>= 1) {
        const u64 x = __shfl_xor(v, o);
        v = x > v ? x : v;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        s.wave[threadIdx.x >> 6] = v;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; i++)
        v = s.wave[i] > v ? s.wave[i] : v;
    return v;
}

// The entry at which the running sum of weights, from the largest logit down, reaches its target (a function of the whole sum):
// weight(l, i, depth) -> u64.  False where it never does, and `cut` stays; else it is that entry, and entries of the source were handed
// to above(l, i, depth) if they stand before it for sure (a lower step), the others of its step are in the cell, `n` of them (-1: above
// was not called for all of them).
template <class Source, class Weight, class Target, class Above>
__device__ __forceinline__ bool cut_at(Shared &s, const Source &src, const Weigh &weigh, const Weight &weight, const Target &target_of,
                                       const Above &above, Cut &cut, int &n)
{
    __syncthreads();
    s.bins[threadIdx.x] = s.bins[threadIdx.x + THREADS] = 0;
    if (threadIdx.x == 0)
        s.count = 0;
    __syncthreads();
    constexpr int VEC = Source::VEC;
    src.template each<false>([&](const float (&l)[VEC], int i) {
        Depth d[VEC];
        int nearest = BINS, farthest = 0;
#pragma unroll
        for (int e = 0; e < VEC; e++) {
            d[e] = weigh.depth(l[e]);
            nearest = min(nearest, Weigh::bin(d[e]));
            farthest = max(farthest, Weigh::bin(d[e]));
        }
        if (__all(nearest == BINS - 1))
            return;
        const int one = __builtin_amdgcn_readfirstlane(nearest);
        if (__all(nearest == one && farthest == one)) { // (a flat row: additions to one place would wait for each other)
            u64 sum = 0;
#pragma unroll
            for (int e = 0; e < VEC; e++)
                sum += weight(l[e], i + e, d[e]);
            sum = wave_sum(sum);
            if ((threadIdx.x & 63) == 0)
                atomicAdd(&s.bins[one], sum);
            return;
        }
        u64 w[VEC];
#pragma unroll
        for (int e = 0; e < VEC; e++)
            w[e] = weight(l[e], i + e, d[e]);
#pragma unroll
        for (int e = 0; e < VEC; e++)
            if (w[e])
                atomicAdd(&s.bins[Weigh::bin(d[e])], w[e]);
    });
    u64 target = 0;
    if (!find_bin<BINS>(s, [&](u64 all) { return target = target_of(all); }))
        return false;
    const int cell = (int)s.word[0];
    const u64 left = s.word[1];
    u64 lowest = ~0ULL, highest = 0; // the standings that went into the cell, this thread's
    auto sort_in = [&](float l, int i) {
        const Depth d = weigh.depth(l);
        const int b = Weigh::bin(d);
        if (b < cell)
            above(l, i, d);
        put_in_cell(s, b == cell ? weight(l, i, d) : 0, standing(l, i), lowest, highest);
    };
    const float floor = weigh.floor_of(cell + 1);
    if constexpr (VEC == 1 && Source::LIST) {
        src.template each<true>([&](const float (&l)[VEC], int i) { sort_in(l[0], i); });
    } else {
        // What lies above the floor is collected, 64 entries to a wavefront, before any exponential is taken: a nucleus is a small
        // part of a row, and a wavefront with one such entry costs as much as one with 64.  (The list's place is free here.)
        float *const near_l = s.list_l + (threadIdx.x >> 6) * 128;
        int *const near_i = s.list_i + (threadIdx.x >> 6) * 128;
        const int lane = threadIdx.x & 63;
        int held = 0; // (the same in all lanes)
        auto take = [&](int from, int most) {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            sort_in(lane < most ? near_l[from + lane] : -INFINITY, lane < most ? near_i[from + lane] : 0);
        };
        src.template each<true>([&](const float (&l)[VEC], int i) {
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                const u64 who = __ballot(l[e] >= floor);
                if (who) {
                    if (l[e] >= floor) {
                        const int at = held + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
                        near_l[at] = l[e];
                        near_i[at] = i + e;
                    }
                    held += __popcll(who);
                    if (held >= 64) {
                        held -= 64;
                        take(held, 64);
                    }
                }
            }
        }, [&] {
            if (held)
                take(0, held);
            held = 0;
        });
    }
    __syncthreads();
    n = s.count;
    if (n <= CELL) {
        cut = cut_of(reach_cell(s, n, left));
        return true;
    }
    // More entries than the cell holds (flat rows, equal logits): the same again over their standings alone, 11 bits closer each
    // time; equal logits part by index.  The light passes skip what is not between the two ends.
    u64 low = wg_most(s, ~lowest), high = wg_most(s, highest), rest = left;
    low = ~low;
    int held = n;
    while (held > CELL) {
        const u64 range = high - low;
        const int shift = range < BINS ? 0 : 64 - __clzll((long long)range) - 11;
        __syncthreads();
        s.bins[threadIdx.x] = s.bins[threadIdx.x + THREADS] = 0;
        __syncthreads();
        src.template each<true>([&](const float (&l)[VEC], int i) {
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                const u64 key = standing(l[e], i + e);
                const bool in = key >= low && key <= high;
                if (!__any(in))
                    continue;
                const u64 w = in ? weight(l[e], i + e, weigh.depth(l[e])) : 0;
                if (w)
                    atomicAdd(&s.bins[(high - key) >> shift], w);
            }
        });
        find_bin<BINS>(s, [&](u64) { return rest; });
        high -= s.word[0] << shift;
        rest = s.word[1];
        const u64 width = (1ULL << shift) - 1;
        low = high - low > width ? high - width : low;
        if (threadIdx.x == 0)
            s.count = 0;
        __syncthreads();
        src.template each<true>([&](const float (&l)[VEC], int i) {
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                const u64 key = standing(l[e], i + e);
                const bool in = key >= low && key <= high;
                if (!__any(in))
                    continue;
                put_in_cell(s, in ? weight(l[e], i + e, weigh.depth(l[e])) : 0, key, lowest, highest);
            }
        });
        __syncthreads();
        held = s.count;
    }
    cut = cut_of(reach_cell(s, held, rest));
    n = -1;
    return true;
}

// The draw takes the first entry whose running sum is above this.
__device__ __forceinline__ u64 target_of(float u, u64 all)
{
    bool rest;
    return u >= 1.0f ? all - 1 : u > 0.0f ? share(u, all, rest) : 0;
}

// The draw among the kept entries, whose sums over the stretches are there.
template <class T, int VEC>
__device__ __forceinline__ void draw(Shared &s, const Row<T, VEC> &row, const Weigh &weigh, const Cut &cut, float u, int32_t *token,
                                     float *prob)
{
    __syncthreads();
    u64 all;
    const u64 mine = threadIdx.x < STRETCHES ? s.stretch[threadIdx.x] : 0, to = running(s, mine, all);
    const u64 target = target_of(u, all);
    if (to - mine <= target && target < to) {
        s.word[0] = threadIdx.x;
        s.word[1] = target - (to - mine);
    }
    __syncthreads();
    u64 left = s.word[1];
    const int first = (int)s.word[0] * row.length - row.skip, end = min(first + row.length, row.V);
    for (int base = first; base < end; base += THREADS) {
        const int i = base + threadIdx.x;
        const float l = i >= 0 && i < end ? (float)row.x[i] : -INFINITY;
        const u64 w = cut.keeps(l, i) ? weigh.kept(weigh.depth(l)) : 0;
        u64 sum;
        const u64 to = running(s, w, sum);
        if (to - w <= left && left < to) {
            *token = i;
            if (prob)
                *prob = (float)((double)w / (double)all);
        }
        if (left < sum)
            return;
        left -= sum;
    }
}

// All of it for a list of at most FEW entries, four threads to each: its place among them and what stands before it, then
// the running sum by index.
template <class Nucleus>
__device__ __forceinline__ void draw_few(Shared &s, int n, const Weigh &weigh, int k, float p, const Nucleus &nucleus, float u, int32_t *token,
                                         float *prob)
{
    const int mine = threadIdx.x >> 2, part = threadIdx.x & 3;
    const bool real = mine < n;
    const float l = real ? s.list_l[mine] : -INFINITY;
    const int at = real ? s.list_i[mine] : 0;
    const Depth d = weigh.depth(l);
    const u64 key = standing(l, at), w = real ? weigh.whole(d) : 0;
    if (real && part == 0) {
        s.cell_key[mine] = key;
        s.cell_w[mine] = w;
    }
    __syncthreads();
    int ahead = 0;
    u64 before = 0;
    for (int i = part; i < n; i += 4) {
        const bool larger = s.cell_key[i] > key;
        ahead += larger;
        before += larger ? s.cell_w[i] : 0;
    }
    ahead += __shfl_xor(ahead, 1);
    ahead += __shfl_xor(ahead, 2);
    before += __shfl_xor(before, 1);
    before += __shfl_xor(before, 2);
    u64 all;
    running(s, ahead < k && part == 0 ? w : 0, all); // (its barriers part the reads above from the writes below)
    const u64 target = p >= 1.0f ? all : nucleus(all);
    const u64 kept = ahead < k && before < target && real ? weigh.kept(d) : 0;
    if (real && part == 0)
        s.cell_w[mine] = kept;
    running(s, part == 0 ? kept : 0, all);
    const u64 to = target_of(u, all);
    u64 sum = 0;
    for (int i = part; i < n; i += 4)
        sum += s.list_i[i] < at ? s.cell_w[i] : 0;
    sum += __shfl_xor(sum, 1);
    sum += __shfl_xor(sum, 2);
    if (part == 0 && sum <= to && to < sum + kept) {
        *token = at;
        if (prob)
            *prob = (float)((double)kept / (double)all);
    }
}

template <class T, int VEC>
__global__ __launch_bounds__(THREADS) void sample_kernel(FqSampleArgs a, double unit, int length)
{
    __shared__ Shared s;
    const int r = blockIdx.x, V = a.V, tid = threadIdx.x, lane = tid & 63;
    const float temperature = a.temperature ? a.temperature[r] : 1.0f, p = a.top_p ? a.top_p[r] : 1.0f;
    const float min_p = a.min_p ? a.min_p[r] : 0.0f, u = a.u[r];
    const int k = a.top_k ? a.top_k[r] : 0;
    const T *const x = (const T *)a.logits + r * a.row_stride;
    const Row<T, VEC> row{x, V, (int)((uintptr_t)x / sizeof(T) % VEC), length};
    if (tid < ROOTS)
        s.table[tid] = root_of_two(tid) * unit;
    if (tid < STRETCHES)
        s.stretch[tid] = 0;
    float mine = -INFINITY;
    int at = 0;
    row.template each<true>([&](const float (&l)[VEC], int i) {
#pragma unroll
        for (int e = 0; e < VEC; e++)
            if (l[e] > mine) {
                mine = l[e];
                at = i + e;
            }
    });
    const u64 best = wg_most(s, standing(mine, at));
    const float top = unordered((uint32_t)(best >> 32));
    if (top == -INFINITY || !(temperature > 0.0f)) {
        if (tid == 0) {
            a.token[r] = top == -INFINITY ? -1 : (int)(0xffffffffu - (uint32_t)best);
            if (a.prob)
                a.prob[r] = top == -INFINITY ? 0.0f : 1.0f;
        }
        return;
    }
    const Weigh weigh(top, (double)temperature, min_p > 0.0f ? (double)fminf(min_p, 1.0f) * unit : 0.0, s.table);
    auto nucleus = [&](u64 all) { // the sum that top-p asks for
        bool rest = false;
        u64 t = p > 0.0f ? share(p, all, rest) : 0;
        t += rest;
        return t ? t : 1;
    };
    Cut cut = FQ_NO_CUT;
    // (an entry of the last step has no weight, a top-k that reaches it keeps all that has)
    auto count = [](float, int, const Depth &d) -> u64 { return Weigh::bin(d) < BINS - 1; };
    auto weight = [&](float l, int i, const Depth &d) -> u64 { return cut.keeps(l, i) ? weigh.whole(d) : 0; };
    // no entry this far down passes min-p (a step to spare)
    const int least_n = min_p > 0.0f ? (int)(ROOTS * log2f(fminf(min_p, 1.0f))) - 2 : DEEPEST;
    auto nothing = [](float, int, const Depth &) {};
    int in_cell;
    if (k > 0 && k <= THREADS && k < V && top < INFINITY) {
        // a bound: the k-th largest of the threads' own largest, its last 16 bits let go
        const uint32_t key = ordered(mine);
        u64 left = k;
        uint32_t bound = 0;
        for (int b = 24; b >= 16; b -= 8) {
            __syncthreads();
            if (tid < 256)
                s.bins[tid] = 0;
            __syncthreads();
            if (b == 24 || key >> (b + 8) == bound >> (b + 8))
                atomicAdd(&s.bins[255 - ((key >> b) & 255)], 1ULL);
            find_bin<256>(s, [&](u64) { return left; });
            bound |= (255 - (uint32_t)s.word[0]) << b;
            left = s.word[1];
        }
        // (below the order of the finite values lie -inf and what the bits that were let go make of it)
        const float least_l = bound < 0x00800000u ? -3.402823466e38f : unordered(bound);
        if (tid == 0)
            s.count = 0;
        __syncthreads();
        row.template each<true>([&](const float (&l)[VEC], int i) {
            float largest = l[0];
#pragma unroll
            for (int e = 1; e < VEC; e++)
                largest = fmaxf(largest, l[e]);
            if (!__any(largest >= least_l))
                return;
#pragma unroll
            for (int e = 0; e < VEC; e++)
                if (l[e] >= least_l) {
                    const int to = atomicAdd(&s.count, 1);
                    if (to < LIST) {
                        s.list_l[to] = l[e];
                        s.list_i[to] = i + e;
                    }
                }
        });
        __syncthreads();
        const int n = s.count;
        if (n <= FEW) {
            draw_few(s, n, weigh, k, p, nucleus, u, a.token + r, a.prob ? a.prob + r : nullptr);
            return;
        }
        if (n <= LIST) {
            const Listed list{&s, n};
            cut_at(s, list, weigh, count, [&](u64) { return (u64)k; }, nothing, cut, in_cell);
            if (!(p >= 1.0f))
                cut_at(s, list, weigh, weight, nucleus, nothing, cut, in_cell);
            list.template each<true>([&](const float (&l)[1], int i) {
                const u64 w = cut.keeps(l[0], i) ? weigh.kept(weigh.depth(l[0])) : 0;
                if (w)
                    atomicAdd(&s.stretch[(i + row.skip) / length], w);
            });
            draw(s, row, weigh, cut, u, a.token + r, a.prob ? a.prob + r : nullptr);
            return;
        }
    }
    if (k > 0 && k < V)
        cut_at(s, row, weigh, count, [&](u64) { return (u64)k; }, nothing, cut, in_cell);
    u64 sum = 0;
    auto add_stretch = [&](int part) {
        sum = wave_sum(sum);
        if (lane == 0)
            s.stretch[part] = sum;
        sum = 0;
    };
    bool summed = false;
    if (!(p >= 1.0f)) {
        const RowOf<Row<T, VEC>, decltype(add_stretch)> adding{row, add_stretch};
        const Cut k_cut = cut;
        if (cut.l == -INFINITY)
            summed = cut_at(s, adding, weigh, [&](float, int, const Depth &d) { return weigh.whole(d); }, nucleus,
                            [&](float, int, const Depth &d) { sum += weigh.kept(d); }, cut, in_cell);
        else
            summed = cut_at(s, adding, weigh, weight, nucleus, [&](float l, int i, const Depth &d) {
                if (k_cut.keeps(l, i))
                    sum += weigh.kept(d);
            }, cut, in_cell);
        summed = summed && in_cell >= 0;
        if (summed && tid < in_cell) {
            const Cut c = cut_of(s.cell_key[tid]);
            const u64 w = cut.keeps(c.l, c.i) ? weigh.kept(weigh.depth(c.l)) : 0;
            if (w)
                atomicAdd(&s.stretch[(c.i + row.skip) / length], w);
        }
    }
    if (!summed && cut.l == -INFINITY && weigh.least == 0.0)
        row.template stretches<false>([&](const float (&l)[VEC], int) {
#pragma unroll
            for (int e = 0; e < VEC; e++)
                sum += weigh.whole(weigh.depth(l[e]));
        }, add_stretch);
    else if (!summed)
        row.template stretches<false>([&](const float (&l)[VEC], int i) {
            Depth d[VEC];
            int nearest = DEEPEST;
#pragma unroll
            for (int e = 0; e < VEC; e++) {
                d[e] = weigh.depth(l[e]);
                nearest = max(nearest, d[e].n);
            }
            if (__any(nearest >= least_n))
#pragma unroll
                for (int e = 0; e < VEC; e++)
                    sum += cut.keeps(l[e], i + e) ? weigh.kept(d[e]) : 0;
        }, add_stretch);
    draw(s, row, weigh, cut, u, a.token + r, a.prob ? a.prob + r : nullptr);
}

template <class T, int VEC>
void launch(const FqSampleArgs &a, double unit, hipStream_t stream)
{
    const int blocks = (a.V + VEC - 1 + STRETCHES * 64 * VEC - 1) / (STRETCHES * 64 * VEC); // (with what a row may skip)
    sample_kernel<T, VEC><<<a.R, THREADS, 0, stream>>>(a, unit, blocks * 64 * VEC);
}

} // namespace

hipError_t fq_launch_sample(const FqSampleArgs &a, bool half, hipStream_t stream)
{
    const int log_v = a.V > 1 ? 32 - __builtin_clz((unsigned)a.V - 1) : 0;
    const double unit = (double)(1ULL << (log_v > 11 ? 62 - log_v : 51));
    if (half)
        launch<_Float16, 8>(a, unit, stream);
    else
        launch<float, 4>(a, unit, stream);
    return hipGetLastError();
}
