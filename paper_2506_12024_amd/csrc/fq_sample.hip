// Drawing the next token from a row of logits: temperature, top-k, top-p, min-p and a given random number.
//
// Weights are whole numbers (exp in binary64, rounded to a unit under which V of them still fit 62 bits), so sums are exact in any
// order and atomics give the same bits every time.  One workgroup takes a row:
//   1. the largest logit (a row of up to 32768 entries stays in registers from here on, a longer one is read again)
//   2. top-k of at most 1024: the k-th largest of the 1024 threads' own largest is no larger than the k-th of all, so the few
//      entries from it on go to a list in LDS, which takes the row's place
//   3. a cut (the entry at which a running count or sum, from the largest logit down, reaches its target): a histogram over 2048
//      steps of 1/64 nat from the top, the step that holds the target, and the entries of that step in order
//   4. the draw: kept weights summed over segments of the vocabulary, the segment that holds the target, its entries in order
// Bound by reading a long row two (top-k, temperature, min-p) or three times (top-p), the second and third from the caches;
// by the chain of steps for a short one.
#include <hip/hip_runtime.h>

#include "fq_internal.h"

namespace {

constexpr int THREADS = 1024;
constexpr int WAVES = THREADS / 64;
constexpr int HELD = 32;    // entries of a row that a thread holds in registers
constexpr int BINS = 2048;  // steps of 1/64 nat; the last one holds everything from 32 nats on
constexpr int LIST = 8192;  // entries of the list of step 2
constexpr int CELL = 1024;  // entries of one step that are put in order there
constexpr int SEGMENTS = 1024;
typedef unsigned long long u64;

// Binary32 values as unsigned numbers in the same order; -0 is 0, a NaN is -inf.
__device__ __forceinline__ float clean(float f) { return f != f ? -INFINITY : f + 0.0f; }
__device__ __forceinline__ uint32_t ordered(float f)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, f);
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

// exp(y) for y <= 0: y = n ln 2 + f, the series of exp(f) to f^13 (|f| <= 0.347: what is left out is under 2^-57)
__device__ __forceinline__ double exp_down(double y)
{
    if (!(y > -750.0))
        return 0.0;
    const double n = rint(y * 1.4426950408889634074);
    // ln 2 as its first 32 bits, of which n times is exact, and the rest
    double f = fma(n, -0x1.62e42fee00000p-1, y);
    f = fma(n, -0x1.a39ef35793c76p-33, f);
    double p = 1.0 / 6227020800.0;
    p = fma(p, f, 1.0 / 479001600.0);
    p = fma(p, f, 1.0 / 39916800.0);
    p = fma(p, f, 1.0 / 3628800.0);
    p = fma(p, f, 1.0 / 362880.0);
    p = fma(p, f, 1.0 / 40320.0);
    p = fma(p, f, 1.0 / 5040.0);
    p = fma(p, f, 1.0 / 720.0);
    p = fma(p, f, 1.0 / 120.0);
    p = fma(p, f, 1.0 / 24.0);
    p = fma(p, f, 1.0 / 6.0);
    p = fma(p, f, 0.5);
    p = fma(p, f, 1.0);
    p = fma(p, f, 1.0);
    return ldexp(p, (int)n);
}

struct Weigh {
    float top;
    double inv_t; // 1 / temperature
    double unit;
    double least; // min_p, 0 for none
    __device__ __forceinline__ double power(float l) const // l > -inf
    {
        return l == top ? 1.0 : exp_down(((double)l - (double)top) * inv_t);
    }
    __device__ __forceinline__ u64 whole(double e) const
    {
        const double v = rint(e * unit);
        const uint32_t hi = (uint32_t)(v * 0x1p-32);
        return ((u64)hi << 32) | (uint32_t)fma((double)hi, -0x1p32, v);
    }
    __device__ __forceinline__ u64 operator()(float l) const { return l == -INFINITY ? 0 : whole(power(l)); }
    // the weight of an entry that is kept where its standing is not under the cut
    __device__ __forceinline__ u64 kept(float l, int i, u64 cut) const
    {
        if (l == -INFINITY || standing(l, i) < cut)
            return 0;
        const double e = power(l);
        return e >= least ? whole(e) : 0;
    }
    __device__ __forceinline__ int bin(float l) const
    {
        if (l == top)
            return 0;
        const double x = ((double)top - (double)l) * inv_t * 64.0;
        return x < BINS - 1 ? (int)x : BINS - 1;
    }
};

__device__ __forceinline__ u64 wave_sum(u64 v)
{
    for (int o = 32; o; o >>= 1)
        v += __shfl_xor(v, o);
    return v;
}

struct Shared {
    u64 bins[BINS];
    u64 segments[SEGMENTS];
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
    for (int o = 1; o < 64; o <<= 1) {
        const u64 w = __shfl_up(v, o);
        v += lane >= o ? w : 0;
    }
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

// The row: each(f) calls f(logit, index) for every entry once, all 64 lanes of a wavefront together (-inf where there is
// no entry), blocks(f, g) besides g(first index of the lane's block) after a block of VEC entries.
template <class T, int VEC, bool IN_REGISTERS>
struct Row {
    const T *x;
    int V;
    float held[IN_REGISTERS ? HELD : 1];
    typedef T Vec __attribute__((ext_vector_type(VEC)));

    __device__ __forceinline__ void block(int at, float (&l)[VEC]) const
    {
        if (at + VEC <= V) {
            if constexpr (VEC > 1) {
                const Vec v = *(const Vec *)(x + at);
#pragma unroll
                for (int e = 0; e < VEC; e++)
                    l[e] = clean((float)v[e]);
            } else {
                l[0] = clean((float)x[at]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < VEC; e++)
                l[e] = at + e < V ? clean((float)x[at + e]) : -INFINITY;
        }
    }
    __device__ __forceinline__ void fill()
    {
        if constexpr (IN_REGISTERS) {
#pragma unroll
            for (int b = 0; b < HELD / VEC; b++) {
                float l[VEC];
                block((b * THREADS + threadIdx.x) * VEC, l);
#pragma unroll
                for (int e = 0; e < VEC; e++)
                    held[b * VEC + e] = l[e];
            }
        }
    }
    template <class F, class G>
    __device__ __forceinline__ void blocks(const F &f, const G &g) const
    {
        if constexpr (IN_REGISTERS) {
#pragma unroll
            for (int b = 0; b < HELD / VEC; b++) {
                if (b * THREADS * VEC < V) {
                    const int at = (b * THREADS + threadIdx.x) * VEC;
#pragma unroll
                    for (int e = 0; e < VEC; e++)
                        f(held[b * VEC + e], at + e);
                    g(at);
                }
            }
        } else {
            constexpr int AHEAD = 64 / (VEC * (int)sizeof(T)); // 64 bytes a thread in flight
            for (int first = 0; first < V; first += AHEAD * THREADS * VEC) {
                float l[AHEAD][VEC];
#pragma unroll
                for (int b = 0; b < AHEAD; b++)
                    block(first + (b * THREADS + threadIdx.x) * VEC, l[b]);
#pragma unroll
                for (int b = 0; b < AHEAD; b++) {
                    const int at = first + (b * THREADS + threadIdx.x) * VEC;
#pragma unroll
                    for (int e = 0; e < VEC; e++)
                        f(l[b][e], at + e);
                    g(at);
                }
            }
        }
    }
    template <class F>
    __device__ __forceinline__ void each(const F &f) const
    {
        blocks(f, [](int) {});
    }
};

struct Listed {
    const Shared *s;
    int n;
    template <class F>
    __device__ __forceinline__ void each(const F &f) const
    {
        for (int at = threadIdx.x; at - (int)threadIdx.x < n; at += THREADS)
            f(at < n ? s->list_l[at] : -INFINITY, at < n ? s->list_i[at] : 0);
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

// Of entries f(visit) names by visit(key, weight) (weight 0: not among them), from the largest key down: the key at which the running
// sum of weights reaches `target` (1 <= target <= the sum).  Eight bits at a time: any number of entries and equal keys'
// prefixes, the way out where a histogram over values does not tell entries apart.
template <int BITS, class F>
__device__ __forceinline__ u64 reach(Shared &s, const F &f, u64 target)
{
    u64 found = 0;
    for (int shift = BITS - 8; shift >= 0; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256)
            s.bins[threadIdx.x] = 0;
        __syncthreads();
        f([&](u64 key, u64 w) {
            if (w && (shift == BITS - 8 || (key >> (shift + 8)) == (found >> (shift + 8))))
                atomicAdd(&s.bins[255 - ((key >> shift) & 255)], w);
        });
        find_bin<256>(s, [&](u64) { return target; });
        found |= (255 - s.word[0]) << shift;
        target = s.word[1];
    }
    __syncthreads();
    return found;
}

// The entries of the cell, n of them: the same.
__device__ __forceinline__ u64 reach_cell(Shared &s, int n, u64 target)
{
    if (n > 256)
        return reach<64>(s, [&](const auto &visit) {
            for (int i = threadIdx.x; i < n; i += THREADS)
                visit(s.cell_key[i], s.cell_w[i]);
        }, target);
    if ((int)threadIdx.x < n) {
        const u64 key = s.cell_key[threadIdx.x], w = s.cell_w[threadIdx.x];
        u64 before = 0;
        for (int i = 0; i < n; i++)
            before += s.cell_key[i] > key ? s.cell_w[i] : 0;
        if (before < target && target <= before + w)
            s.word[0] = key;
    }
    __syncthreads();
    const u64 found = s.word[0];
    __syncthreads();
    return found;
}

// The standing at which the running sum of weight(l, i), from the largest logit down, reaches its target (a function of the
// whole sum); 0 where it never does.
template <class Source, class Weight, class Target>
__device__ __forceinline__ u64 cut_at(Shared &s, const Source &src, const Weigh &weigh, const Weight &weight, const Target &target_of)
{
    __syncthreads();
    s.bins[threadIdx.x] = s.bins[threadIdx.x + THREADS] = 0;
    if (threadIdx.x == 0)
        s.count = 0;
    __syncthreads();
    u64 far = 0;
    src.each([&](float l, int i) {
        const u64 w = weight(l, i);
        const int b = w ? weigh.bin(l) : BINS - 1;
        const int one = __builtin_amdgcn_readfirstlane(b);
        if (__all(b == one)) { // (a flat row: 64 additions to one place would wait for each other)
            if (one == BINS - 1) {
                far += w;
            } else {
                const u64 sum = wave_sum(w);
                if ((threadIdx.x & 63) == 0)
                    atomicAdd(&s.bins[one], sum);
            }
        } else if (b == BINS - 1) {
            far += w;
        } else {
            atomicAdd(&s.bins[b], w);
        }
    });
    far = wave_sum(far);
    if ((threadIdx.x & 63) == 0)
        atomicAdd(&s.bins[BINS - 1], far);
    u64 target = 0;
    if (!find_bin<BINS>(s, [&](u64 all) { return target = target_of(all); }))
        return 0;
    const int cell = (int)s.word[0];
    const u64 left = s.word[1];
    src.each([&](float l, int i) {
        const u64 w = weight(l, i);
        if (w && weigh.bin(l) == cell) {
            const int at = atomicAdd(&s.count, 1);
            if (at < CELL) {
                s.cell_key[at] = standing(l, i);
                s.cell_w[at] = w;
            }
        }
    });
    __syncthreads();
    const int n = s.count;
    if (n > CELL)
        return reach<64>(s, [&](const auto &visit) {
            src.each([&](float l, int i) { visit(standing(l, i), weight(l, i)); });
        }, target);
    return reach_cell(s, n, left);
}

// The draw among the kept entries: segments holds their sums, 2^shift entries each.
template <class T, int VEC, bool R>
__device__ __forceinline__ void draw(Shared &s, const Row<T, VEC, R> &row, const Weigh &weigh, u64 cut, int shift, float u, int32_t *token,
                                     float *prob)
{
    __syncthreads();
    u64 all;
    const u64 mine = s.segments[threadIdx.x], to = running(s, mine, all);
    bool rest;
    const u64 target = u >= 1.0f ? all - 1 : u > 0.0f ? share(u, all, rest) : 0; // the first running sum above it
    if (to - mine <= target && target < to) {
        s.word[0] = threadIdx.x;
        s.word[1] = target - (to - mine);
    }
    __syncthreads();
    u64 left = s.word[1];
    const int first = (int)s.word[0] << shift;
    for (int base = 0; base < 1 << shift; base += THREADS) {
        const int i = first + base + threadIdx.x;
        const u64 w = base + (int)threadIdx.x < 1 << shift && i < row.V ? weigh.kept(clean((float)row.x[i]), i, cut) : 0;
        u64 sum;
        const u64 end = running(s, w, sum);
        if (end - w <= left && left < end) {
            *token = i;
            if (prob)
                *prob = (float)((double)w / (double)all);
        }
        if (left < sum)
            return;
        left -= sum;
    }
}

template <class T, int VEC, bool IN_REGISTERS>
__global__ __launch_bounds__(THREADS) void sample_kernel(FqSampleArgs a, double unit, int shift)
{
    __shared__ Shared s;
    const int r = blockIdx.x, V = a.V, tid = threadIdx.x, lane = tid & 63;
    const float temperature = a.temperature ? a.temperature[r] : 1.0f, p = a.top_p ? a.top_p[r] : 1.0f;
    const float min_p = a.min_p ? a.min_p[r] : 0.0f, u = a.u[r];
    const int k = a.top_k ? a.top_k[r] : 0;
    Row<T, VEC, IN_REGISTERS> row;
    row.x = (const T *)a.logits + r * a.row_stride;
    row.V = V;
    row.fill();
    float mine = -INFINITY;
    int at = 0;
    row.each([&](float l, int i) {
        if (l > mine) {
            mine = l;
            at = i;
        }
    });
    u64 best = standing(mine, at);
    for (int o = 32; o; o >>= 1) {
        const u64 x = __shfl_xor(best, o);
        best = x > best ? x : best;
    }
    if (lane == 0)
        s.wave[tid >> 6] = best;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; i++)
        best = s.wave[i] > best ? s.wave[i] : best;
    const float top = unordered((uint32_t)(best >> 32));
    if (top == -INFINITY || !(temperature > 0.0f)) {
        if (tid == 0) {
            a.token[r] = top == -INFINITY ? -1 : (int)(0xffffffffu - (uint32_t)best);
            if (a.prob)
                a.prob[r] = top == -INFINITY ? 0.0f : 1.0f;
        }
        return;
    }
    // (with +inf in the row 1 / temperature is too, so that what is finite has no weight)
    const Weigh weigh{top, top == INFINITY ? (double)INFINITY : 1.0 / (double)temperature, unit,
                      min_p > 0.0f ? (double)fminf(min_p, 1.0f) : 0.0};
    auto nucleus = [&](u64 all) { // the sum that top-p asks for
        bool rest = false;
        u64 t = p > 0.0f ? share(p, all, rest) : 0;
        t += rest;
        return t ? t : 1;
    };
    u64 cut = 0; // entries whose standing is below it are out
    __syncthreads();
    s.segments[tid] = 0;
    if (k > 0 && k <= THREADS && k < V) {
        // a bound: the k-th largest of the threads' own largest, its last 8 bits let go
        const uint32_t key = ordered(mine);
        u64 left = k;
        uint32_t bound = 0;
        for (int b = 24; b >= 8; b -= 8) {
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
        if (tid == 0)
            s.count = 0;
        __syncthreads();
        row.each([&](float l, int i) {
            const bool in = l > -INFINITY && ordered(l) >= bound;
            const u64 who = __ballot(in);
            if (who) {
                int base = 0;
                if (lane == 0)
                    base = atomicAdd(&s.count, __popcll(who));
                const int to = __builtin_amdgcn_readfirstlane(base) + __popcll(who & ((1ULL << lane) - 1));
                if (in && to < LIST) {
                    s.list_l[to] = l;
                    s.list_i[to] = i;
                }
            }
        });
        __syncthreads();
        const int n = s.count;
        if (n <= LIST) {
            const Listed list{&s, n};
            cut = cut_at(s, list, weigh, [&](float l, int) -> u64 { return l > -INFINITY; }, [&](u64) { return (u64)k; });
            if (!(p >= 1.0f)) {
                const u64 c = cut_at(s, list, weigh, [&](float l, int i) { return standing(l, i) >= cut ? weigh(l) : 0; }, nucleus);
                cut = c > cut ? c : cut;
            }
            list.each([&](float l, int i) {
                const u64 w = weigh.kept(l, i, cut);
                if (w)
                    atomicAdd(&s.segments[i >> shift], w);
            });
            draw(s, row, weigh, cut, shift, u, a.token + r, a.prob ? a.prob + r : nullptr);
            return;
        }
    }
    if (k > 0 && k < V)
        cut = cut_at(s, row, weigh, [&](float l, int) -> u64 { return l > -INFINITY; }, [&](u64) { return (u64)k; });
    if (!(p >= 1.0f)) {
        const u64 c = cut_at(s, row, weigh, [&](float l, int i) { return standing(l, i) >= cut ? weigh(l) : 0; }, nucleus);
        cut = c > cut ? c : cut;
    }
    __syncthreads();
    u64 sum = 0;
    row.blocks([&](float l, int i) { sum += weigh.kept(l, i, cut); },
               [&](int i) { // the wavefront's blocks lie in one segment
                   sum = wave_sum(sum);
                   if (lane == 0 && sum)
                       atomicAdd(&s.segments[i >> shift], sum);
                   sum = 0;
               });
    draw(s, row, weigh, cut, shift, u, a.token + r, a.prob ? a.prob + r : nullptr);
}

template <class T, int VEC>
void launch(const FqSampleArgs &a, double unit, int shift, hipStream_t stream)
{
    if (a.V <= HELD * THREADS)
        sample_kernel<T, VEC, true><<<a.R, THREADS, 0, stream>>>(a, unit, shift);
    else
        sample_kernel<T, VEC, false><<<a.R, THREADS, 0, stream>>>(a, unit, shift);
}

} // namespace

size_t fq_sample_bytes(int, int) { return 256; }

hipError_t fq_launch_sample(const FqSampleArgs &a, bool half, void *, hipStream_t stream)
{
    const int log_v = a.V > 1 ? 32 - __builtin_clz((unsigned)a.V - 1) : 0;
    const double unit = (double)(1ULL << (62 - log_v));
    const int shift = log_v - 10 > 9 ? log_v - 10 : 9; // entries of a segment: no more than 1024 of them, 64 blocks of 8 at least
    const int vec = half ? 8 : 4;
    const bool wide = ((uintptr_t)a.logits & 15) == 0 && (a.R == 1 || a.row_stride % vec == 0);
    if (half && wide)
        launch<_Float16, 8>(a, unit, shift, stream);
    else if (half)
        launch<_Float16, 1>(a, unit, shift, stream);
    else if (wide)
        launch<float, 4>(a, unit, shift, stream);
    else
        launch<float, 1>(a, unit, shift, stream);
    return hipGetLastError();
}
