// Log probabilities of given tokens, the entropy and the likeliest tokens of rows of logits, one pass over them.
//
// With m the largest logit, s = sum of e^(l - m) over all others and t = sum of e^(l - m) (l - m):
//   ln p_i = (l_i - m) - log1p(s),   H = log1p(s) - t / (1 + s)
// -- the largest one's own 1 stays out of the sums, so that a nearly certain token keeps its digits.  A workgroup takes a row (a piece of one, where few
// rows are long).  Its wavefronts stream it in 16-byte loads; each keeps a running maximum that all its lanes share, so that a raise is a branch which
// it takes a few times in a row, and whose new largest logit is taken out of the lane that has it.  On the way the largest logit of every block of 64 goes
// to LDS.  The n likeliest tokens lie in the n blocks whose largest come first in the order (larger logit, smaller index): any token of another
// block comes behind the largest of each of them.  So the blocks' maxima are cut at about the n-th by a histogram over the distance from the
// largest, the few blocks above are read again (from a cache), and the tokens there that reach the cut, some more than n, are ranked against each other.
// Equal logits by the thousand, or all the best in one place, cost more rounds of the histogram, not another result.
//
// What bounds it: many long rows memory (500 x 128256 in binary32 with 20 alternatives 52 us, 4.9 TB/s), in binary16 the vector units too (2048 x 32000
// without alternatives 31 us, 4.2 TB/s: eleven instructions to a logit, one of them an exponential at a quarter of the rate); short rows what comes
// after the stream (8000 x 1000 with alternatives 49 us: some ten steps one after another to a row of 4 KB);
// one row the same and what one compute unit draws from memory (1 x 32000 in binary32 9.6 us a call: 5.3 until all is there, 1 the sums, 2.7 the alternatives).
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/flexq.h"
#include "fq_internal.h"

namespace {

constexpr int BLOCK = 64, MAX_BLOCKS = 2048; // logits; a row of more takes blocks twice, four times ... as large
constexpr int BINS = 256, LIST = 256, MAX_CHOSEN = 128;
// Rows in pieces (a workgroup of 1024 threads to a whole row / pieces and a second launch, us, 20 alternatives): 1 x 32000 in binary32 10.1 / 11.5, 65536
// 14.2 / 11.8, 128256 21.9 / 13.2, 262144 37.6 / 14.6; 32 x 65536 in binary16 13.5 / 12.4, 128256 20.8 / 13.8; 64 x 65536 13.8 / 14.5, 128256 21.1 / 16.1.
constexpr int SPLIT_ROWS = 64, SPLIT_LOGITS = 60000, MAX_PIECES = 64;
constexpr uint32_t LOWEST = 0x007fffffu; // the key of -inf

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Larger for larger numbers, equal for -0 and 0; a NaN is as -inf (a signalling one only once it is quiet: a maximum with one that is not is a NaN).
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, fmaxf(__builtin_canonicalizef(x), -INFINITY) + 0.0f);
    return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __builtin_bit_cast(float, (k >> 31) ? k & 0x7fffffffu : ~k); }

template <typename T>
struct Row {
    static constexpr int PER = 16 / sizeof(T); // logits to a 16-byte load
    const T *at;  // the row
    const T *from; // the 16-byte boundary before it
    unsigned shift, V;

    __device__ __forceinline__ Row(const FqLogprobsArgs &a, long long r) : at((const T *)a.logits + r * a.row_stride), V(a.V)
    {
        shift = (unsigned)((uintptr_t)at & 15) / sizeof(T);
        from = at - shift;
    }
    __device__ __forceinline__ unsigned loads() const { return (shift + V + PER - 1) / PER; }
    __device__ __forceinline__ float operator[](unsigned i) const { return (float)at[i]; }
};

template <typename T>
__device__ __forceinline__ void widen(const u32x4 v, float (&x)[16 / sizeof(T)])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t u = v[i]; // (a bit cast of v[i] itself takes the vector's first element)
            x[i] = __builtin_bit_cast(float, u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            x[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(v[i / 2] >> 16 * (i & 1)));
    }
}

// Element e of a load becomes -inf.
template <typename T>
__device__ __forceinline__ void blank(u32x4 &v, int e)
{
    if constexpr (sizeof(T) == 4)
        v[e] = 0xff800000u;
    else
        v[e / 2] = e & 1 ? (v[e / 2] & 0xffffu) | 0xfc000000u : (v[e / 2] & 0xffff0000u) | 0xfc00u;
}

// The largest of a group of 8 or 16 lanes, in all of them.
template <int LANES>
__device__ __forceinline__ float group_max(float x)
{
    auto step = [](float v, auto ctrl) {
        const int t = __builtin_bit_cast(int, v);
        return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(t, t, decltype(ctrl)::value, 0xf, 0xf, false)));
    };
    x = step(x, std::integral_constant<int, 0xb1>());  // quad_perm 1, 0, 3, 2
    x = step(x, std::integral_constant<int, 0x4e>());  // quad_perm 2, 3, 0, 1
    x = step(x, std::integral_constant<int, 0x141>()); // half a row mirrored
    if (LANES == 16)
        x = step(x, std::integral_constant<int, 0x140>()); // a row mirrored
    return x;
}

__device__ __forceinline__ float lane_of(float x, int lane)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

// Sums over the lanes of a wavefront; of binary32 numbers those of sixteen lanes in binary32 (four roundings, as a thread's own sums have more), the four in binary64.
__device__ __forceinline__ double wave_sum(float x)
{
    auto step = [](float v, auto ctrl) {
        const int t = __builtin_bit_cast(int, v);
        return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(t, t, decltype(ctrl)::value, 0xf, 0xf, false));
    };
    x = step(x, std::integral_constant<int, 0xb1>());
    x = step(x, std::integral_constant<int, 0x4e>());
    x = step(x, std::integral_constant<int, 0x141>());
    x = step(x, std::integral_constant<int, 0x140>());
    return ((double)lane_of(x, 0) + (double)lane_of(x, 16)) + ((double)lane_of(x, 32) + (double)lane_of(x, 48));
}
__device__ __forceinline__ double lane_of(double x, int lane)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t low = __builtin_amdgcn_readlane((int)u, lane), high = __builtin_amdgcn_readlane((int)(u >> 32), lane);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
__device__ __forceinline__ double wave_sum(double x)
{
    auto step = [](double v, auto ctrl) {
        const uint64_t t = __builtin_bit_cast(uint64_t, v);
        const uint32_t low = __builtin_amdgcn_update_dpp((int)t, (int)t, decltype(ctrl)::value, 0xf, 0xf, false);
        const uint32_t high = __builtin_amdgcn_update_dpp((int)(t >> 32), (int)(t >> 32), decltype(ctrl)::value, 0xf, 0xf, false);
        return v + __builtin_bit_cast(double, (uint64_t)high << 32 | low);
    };
    x = step(x, std::integral_constant<int, 0xb1>());
    x = step(x, std::integral_constant<int, 0x4e>());
    x = step(x, std::integral_constant<int, 0x141>());
    x = step(x, std::integral_constant<int, 0x140>());
    return (lane_of(x, 0) + lane_of(x, 16)) + (lane_of(x, 32) + lane_of(x, 48));
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

// A part of a row: its largest logit, the sums beside that one's weight.
struct Part {
    float m;
    double s, t;
};

struct Work {
    uint32_t *keys; // [row][MAX_BLOCKS]
    Part *parts;    // [row][pieces]
    int pieces, shift; // shift: blocks of BLOCK << shift logits
    unsigned piece; // loads to a piece
};

// What a workgroup needs in LDS.
template <int THREADS>
struct Shared {
    static constexpr int BLOCKS = THREADS == 64 ? 64 : MAX_BLOCKS;
    uint32_t keys[BLOCKS];
    Part parts[THREADS / 64];
    Part all; // of the row
    double log_sum;
    uint64_t list[LIST];
    int chosen[MAX_CHOSEN];
    int bins[BINS];
    int found[5];
};

// The loads [begin, end) of a row through the workgroup: parts of the wavefronts and the blocks' maxima, from block `first` on, into `sh`.
template <typename T, int THREADS, int AHEAD>
__device__ __forceinline__ void stream(const Row<T> &row, unsigned begin, unsigned end, int block_shift, unsigned first, bool top, Shared<THREADS> &sh)
{
    constexpr int PER = Row<T>::PER, LANES = BLOCK / PER; // lanes of a block
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned whole = (row.shift + row.V) / PER; // the loads before are whole, but for the first
    float m = -INFINITY, s = 0.0f, t = 0.0f;
    auto turn = [&](unsigned base, auto edge) {
        constexpr bool EDGE = decltype(edge)::value;
        u32x4 v[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
            const unsigned g = base + 64 * j + lane;
            v[j] = __builtin_nontemporal_load((const u32x4 *)row.from + (EDGE ? min(g, end - 1) : g));
        }
        if (EDGE) { // loads behind the end count as -inf, of the first and the last one what does not belong to the row
#pragma unroll
            for (int j = 0; j < AHEAD; j++) {
                const unsigned g = base + 64 * j + lane;
#pragma unroll
                for (int i = 0; i < 4; i++)
                    v[j][i] = g >= end ? sizeof(T) == 4 ? 0xff800000u : 0xfc00fc00u : v[j][i];
                if ((g == 0 && row.shift) || (g >= whole && g < end)) {
#pragma unroll
                    for (int e = 0; e < PER; e++)
                        if (g * PER + e < row.shift || g * PER + e >= row.shift + row.V)
                            blank<T>(v[j], e);
                }
            }
        }
        float most[AHEAD], peak = -INFINITY;
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
            float x[PER];
            widen<T>(v[j], x);
            most[j] = -INFINITY;
#pragma unroll
            for (int e = 0; e < PER; e++)
                most[j] = fmaxf(most[j], sizeof(T) == 4 ? __builtin_canonicalizef(x[e]) : x[e]); // (a conversion has made it quiet)
            const float b = group_max<LANES>(most[j]);
            peak = fmaxf(peak, b);
            const unsigned g = base + 64 * j + lane;
            if (top && (lane & (LANES - 1)) == 0 && (!EDGE || g < end)) {
                const unsigned block = (g * PER / BLOCK >> block_shift) - first;
                if (block_shift == 0)
                    sh.keys[block] = key_of(b);
                else
                    atomicMax(&sh.keys[block], key_of(b));
            }
        }
        peak = group_max<16>(peak);
        peak = fmaxf(fmaxf(lane_of(peak, 0), lane_of(peak, 16)), fmaxf(lane_of(peak, 32), lane_of(peak, 48)));
        if (peak > m) {
            const float d = m - peak, c = __expf(d);
            t = c > 0.0f ? c * (t + d * s) : 0.0f;
            s *= c;
            if (lane == 0 && c > 0.0f) { // the old largest one's 1
                s += c;
                t += c * d;
            }
            m = peak;
            bool looking = true; // the new one's is left out: one lane's first
#pragma unroll
            for (int j = 0; j < AHEAD; j++) {
                const uint64_t has = __ballot(most[j] == peak);
                if (looking && has) {
                    looking = false;
                    if (lane == __ffsll((unsigned long long)has) - 1) {
                        float x[PER];
                        widen<T>(v[j], x);
                        bool mine = true;
#pragma unroll
                        for (int e = 0; e < PER; e++)
                            if (mine && x[e] == peak) {
                                mine = false;
                                blank<T>(v[j], e);
                            }
                    }
                }
            }
        }
#pragma unroll
        for (int j = 0; j < AHEAD; j++) {
            float x[PER], w[PER], turned = 0.0f;
            widen<T>(v[j], x);
#pragma unroll
            for (int e = 0; e < PER; e++) {
                const float d = fmaxf(x[e] - m, -200.0f); // (-inf, NaN and what is not there: no weight)
                w[e] = __expf(d);
                turned += w[e] * d;
            }
#pragma unroll
            for (int e = PER / 2; e >= 1; e /= 2)
#pragma unroll
                for (int i = 0; i < e; i++)
                    w[i] += w[i + e];
            s += w[0];
            t += turned;
        }
    };
    constexpr unsigned STEP = 64 * AHEAD, STRIDE = STEP * (THREADS / 64);
    for (unsigned base = begin + wave * STEP; base < end; base += STRIDE) {
        if ((base == 0 && row.shift) || base + STEP > whole || base + STEP > end)
            turn(base, std::true_type());
        else
            turn(base, std::false_type());
    }
    const double all_s = wave_sum(s), all_t = wave_sum(t);
    if (lane == 0)
        sh.parts[wave] = Part{m, all_s, all_t};
}

// The blocks of a row.
template <typename T>
__device__ __forceinline__ int blocks_of(const Row<T> &row, int block_shift)
{
    static_assert(BLOCK == 64, "");
    return (int)((row.shift + row.V + (1u << (6 + block_shift)) - 1) >> (6 + block_shift));
}

// Whether the second wavefront takes the logarithm while the first is alone at work on the cut (32 x 128256 in binary16 14.2 to 13.7 us; the sums there, too, won
// nothing).
template <int THREADS, typename T>
__device__ __forceinline__ bool later(const FqLogprobsArgs &a, const Row<T> &row, int block_shift)
{
    return THREADS > 64 && a.top_n > 0 && blocks_of(row, block_shift) > a.top_n;
}

// The parts' sums as one, by the first wavefront: a lane to a part, up to 64.
template <int THREADS>
__device__ __forceinline__ void join(int n, const Part *parts, bool log_later, Shared<THREADS> &sh)
{
    const int lane = threadIdx.x;
    if (lane < 64) {
        const Part p = lane < n ? parts[lane] : Part{-INFINITY, 0.0, 0.0};
        float m = group_max<16>(p.m);
        m = fmaxf(fmaxf(lane_of(m, 0), lane_of(m, 16)), fmaxf(lane_of(m, 32), lane_of(m, 48)));
        const int first = __ffsll((unsigned long long)__ballot(p.m == m)) - 1; // whose 1 stays out
        double s = 0.0, t = 0.0;
        if (p.m > -INFINITY && m < INFINITY) {
            const double d = (double)p.m - (double)m, c = exp(d);
            if (c > 0.0) {
                s = c * (p.s + (lane == first ? 0.0 : 1.0));
                t = c * (p.t + (lane == first ? 0.0 : d * (p.s + 1.0)));
            }
        }
        if (n > 1) {
            s = wave_sum(s);
            t = wave_sum(t);
        }
        if (lane == 0) {
            sh.all = Part{m, s, t};
            if (!log_later)
                sh.log_sum = log1p(s);
        }
    }
    __syncthreads();
}

// The cut of items (logit, index) at about the n-th of the order (larger logit, smaller index): at least n of them, or all, lie at or above it, at most
// `cap` unless that is n.  In eighths of the distance from the row's largest logit m, the last for everything 31.9 and more below; within one of those by the
// bits of the logit; among equal ones by index.
struct Cut {
    float m;
    int below; // kept: fewer eighths, or as many and
    uint32_t key, turned; // a larger key, or this one with ~index >= turned
    static __device__ __forceinline__ int eighths(float m, float x) { return (int)fminf((m - x) * 8.0f, BINS - 1.0f); }
    __device__ __forceinline__ bool keeps(uint32_t k, uint32_t index) const
    {
        const int e = eighths(m, of_key(k));
        return e < below || (e == below && (k > key || (k == key && ~index >= turned)));
    }
};

// each(f) calls f(key, index) for a thread's items; keys from `low` on count.  meanwhile(): once, by a thread of the second wavefront.
template <int THREADS, typename Each, typename Meanwhile>
__device__ __forceinline__ Cut find_cut(int n, int cap, float m, uint32_t low, uint32_t last_index, Shared<THREADS> &sh, const Each &each,
                                        const Meanwhile &meanwhile)
{
    const int tid = threadIdx.x, lane = tid & 63;
    enum { EIGHTHS, KEYS, INDICES } by = EIGHTHS;
    Cut cut{m, 0, 0, 0};
    uint32_t high = BINS - 1; // of the fields that are counted, from `from` on
    uint32_t from = 0;
    int above = 0;
    for (;;) {
        const int bits = 32 - __clz((int)(high - from)), shift = high == from || bits < 8 ? 0 : bits - 8;
        for (int i = tid; i < BINS; i += THREADS)
            sh.bins[i] = 0;
        __syncthreads();
        each([&](uint32_t key, uint32_t index) {
            const int e = Cut::eighths(m, of_key(key));
            const uint32_t field = by == EIGHTHS ? BINS - 1 - e : by == KEYS ? key : ~index;
            if (key >= low && (by == EIGHTHS || e == cut.below) && (by != INDICES || key == cut.key) && field >= from && field <= high)
                atomicAdd(&sh.bins[(field - from) >> shift], 1);
        });
        __syncthreads();
        if (by == EIGHTHS && tid == 64)
            meanwhile();
        if (tid < 64) { // the highest bin from which on there are enough
            int own[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                own[i] = sh.bins[4 * (63 - lane) + 3 - i]; // from the top
                sum += own[i];
            }
            const int upto = sum_upto(sum);
            int before = above + upto - sum;
            const bool here = before < n && above + upto >= n;
            int bin = 0, count = above + upto, under = before;
            bool open = true;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (open && before + own[i] >= n) {
                    open = false;
                    bin = 4 * (63 - lane) + 3 - i;
                    under = before;
                    count = before + own[i];
                }
                before += own[i];
            }
            const uint64_t one = __ballot(here);
            if (one ? here : lane == 63) { // (fewer than n in all: everything)
                sh.found[0] = one ? bin : 0;
                sh.found[1] = count;
                sh.found[2] = under;
            }
        }
        __syncthreads();
        const int bin = sh.found[0], count = sh.found[1];
        const uint32_t edge = from + ((uint32_t)bin << shift);
        if (by == EIGHTHS)
            cut.below = BINS - 1 - (int)edge;
        else if (by == KEYS)
            cut.key = edge;
        else
            cut.turned = edge;
        if (count <= cap || count <= n || (by == INDICES && shift == 0))
            return cut;
        above = sh.found[2];
        if (by == EIGHTHS) { // the keys of these eighths, from well below to well above
            by = KEYS;
            const float top = m - 0.125f * cut.below;
            from = cut.below == BINS - 1 ? low : key_of(top - 0.25f - 0x1p-10f * fabsf(top));
            from = from > low ? from : low;
            high = key_of(m);
        } else if (shift > 0) {
            from = edge;
            if (high - edge > (1u << shift) - 1)
                high = edge + ((1u << shift) - 1);
        } else { // all equal
            by = INDICES;
            from = ~last_index;
            high = ~0u;
        }
        __syncthreads();
    }
}

// Everything that comes after a row's logits were streamed.  given: the thread's first given token.
template <typename T, int THREADS>
__device__ __forceinline__ void finish(const FqLogprobsArgs &a, long long r, const Row<T> &row, int given, int block_shift, Shared<THREADS> &sh)
{
    const int tid = threadIdx.x;
    float given_logit = -INFINITY; // (asked for ahead of the next lines)
    if (given >= 0 && given < a.V)
        given_logit = row[given];
    Part all = sh.all;
    const bool none = all.m == -INFINITY, infinite = all.m == INFINITY;
    if (infinite) { // weights of 1 for these alone
        int count = 0;
        for (unsigned i = tid; i < row.V; i += THREADS)
            count += row[i] == INFINITY;
        if (tid == 0)
            sh.found[3] = 0;
        __syncthreads();
        if (count)
            atomicAdd(&sh.found[3], count);
        __syncthreads();
        all.s = sh.found[3] - 1.0;
        all.t = 0.0;
        __syncthreads();
    }
    const double log_infinite = infinite ? log1p(all.s) : 0.0;
    auto logprob = [&](float x) {
        if (none || !(x > -INFINITY) || (infinite && x < INFINITY))
            return -INFINITY;
        return infinite ? (float)-log_infinite : (float)((double)x - (double)all.m - sh.log_sum);
    };
    auto log_now = [&]() { sh.log_sum = log1p(sh.all.s); };
    const int n = a.top_n;
    if (n > 0 && !none) {
        const uint32_t low = infinite ? key_of(INFINITY) : LOWEST + 1; // of what counts
        const int size_shift = 6 + block_shift;
        const int blocks = blocks_of(row, block_shift);
        uint32_t floor = low; // n tokens at least, or all that count, have such a key
        Cut cut{all.m, BINS, 0, 0}; // everything
        bool every = blocks <= n;
        if (tid == 0)
            sh.found[3] = sh.found[4] = 0;
        if (every) {
            for (int i = tid; i < blocks; i += THREADS)
                sh.chosen[i] = i;
            if (tid == 0)
                sh.found[3] = blocks;
        } else if (blocks <= 64) { // ranked against each other by one wavefront
            if (THREADS > 64 && tid == 64)
                log_now();
            if (tid < 64) {
                const uint32_t k = tid < blocks ? sh.keys[tid] : 0;
                int rank = 0;
                for (int j = 0; j < blocks; j++) {
                    const uint32_t o = __builtin_amdgcn_readlane(k, j);
                    rank += o > k || (o == k && j < tid);
                }
                if (tid < blocks && rank < n) {
                    sh.chosen[rank] = tid;
                    if (rank == n - 1) {
                        sh.found[0] = (int)k;
                        sh.found[3] = n;
                    }
                }
            }
            __syncthreads();
            floor = (uint32_t)sh.found[0] > low ? (uint32_t)sh.found[0] : low;
        } else {
            const int cap = n > 32 ? MAX_CHOSEN : MAX_CHOSEN / 2;
            cut = find_cut<THREADS>(n, cap, all.m, low, (uint32_t)blocks - 1, sh, [&](const auto &f) {
                for (int i = tid; i < blocks; i += THREADS)
                    f(sh.keys[i], (uint32_t)i);
            }, log_now);
            __syncthreads();
            for (int i = tid; i < blocks; i += THREADS) {
                const uint32_t k = sh.keys[i];
                if (k >= low && cut.keeps(k, i)) {
                    const int at = atomicAdd(&sh.found[3], 1);
                    if (at < MAX_CHOSEN) // (always)
                        sh.chosen[at] = i;
                }
            }
            cut.turned = 0; // (the tokens that are wanted reach the cut by their logits alone)
        }
        __syncthreads();
        const int tokens = min(sh.found[3], MAX_CHOSEN) << size_shift;
        auto each = [&](const auto &f) {
            for (int i = tid; i < tokens; i += THREADS) {
                const unsigned at = ((unsigned)sh.chosen[i >> size_shift] << size_shift) + (i & ((1 << size_shift) - 1));
                if (at >= row.shift && at < row.shift + row.V) {
                    const uint32_t key = key_of((float)row.from[at]);
                    if (key >= floor)
                        f(key, at - row.shift);
                }
            }
        };
        auto collect = [&](uint32_t key, uint32_t index) {
            if (cut.keeps(key, index)) {
                const int at = atomicAdd(&sh.found[4], 1);
                if (at < LIST)
                    sh.list[at] = (uint64_t)key << 32 | (uint32_t)~index;
            }
        };
        const bool many = every && tokens > LIST;
        if (!many)
            each(collect);
        __syncthreads();
        if (many || sh.found[4] > LIST) { // more than that reach the blocks' cut: one among the tokens
            __syncthreads();
            cut = find_cut<THREADS>(n, LIST, all.m, floor, row.V - 1, sh, each, [] {});
            __syncthreads();
            if (tid == 0)
                sh.found[4] = 0;
            __syncthreads();
            each(collect);
            __syncthreads();
        }
        const int listed = min(sh.found[4], LIST);
        for (int i = tid; i < listed; i += THREADS) {
            const uint64_t own = sh.list[i];
            int rank = 0;
            for (int j = 0; j < listed; j++)
                rank += sh.list[j] > own;
            if (rank < n) {
                a.top_token[r * n + rank] = (int32_t)~(uint32_t)own;
                a.top_logprob[r * n + rank] = logprob(of_key((uint32_t)(own >> 32)));
            }
        }
        for (int i = listed + tid; i < n; i += THREADS) {
            a.top_token[r * n + i] = -1;
            a.top_logprob[r * n + i] = -INFINITY;
        }
    } else {
        for (int i = tid; i < n; i += THREADS) {
            a.top_token[r * n + i] = -1;
            a.top_logprob[r * n + i] = -INFINITY;
        }
    }
    if (a.entropy && tid == 0)
        a.entropy[r] = none ? 0.0f : (float)((infinite ? log_infinite : sh.log_sum) - all.t / (1.0 + all.s));
    for (int j = tid; j < a.n_given; j += THREADS) {
        if (j != tid) {
            given = a.given[r * a.n_given + j];
            given_logit = given >= 0 && given < a.V ? row[given] : -INFINITY;
        }
        a.given_logprob[r * a.n_given + j] = logprob(given_logit);
    }
}

__device__ __forceinline__ int first_given(const FqLogprobsArgs &a, long long r)
{
    return (int)threadIdx.x < a.n_given ? a.given[r * a.n_given + threadIdx.x] : -1;
}

template <typename T, int THREADS, int AHEAD>
__global__ __launch_bounds__(THREADS, THREADS == 1024 ? 4 : 6) void row_kernel(FqLogprobsArgs a, int block_shift)
{
    __shared__ Shared<THREADS> sh;
    const long long r = blockIdx.x;
    const Row<T> row(a, r);
    const int given = first_given(a, r);
    if (block_shift) {
        for (int i = threadIdx.x; i < sh.BLOCKS; i += THREADS)
            sh.keys[i] = 0;
        __syncthreads();
    }
    stream<T, THREADS, AHEAD>(row, 0, row.loads(), block_shift, 0, a.top_n > 0, sh);
    __syncthreads();
    join(THREADS / 64, sh.parts, later<THREADS>(a, row, block_shift), sh);
    finish<T, THREADS>(a, r, row, given, block_shift, sh);
}

// Few long rows: a workgroup takes a piece, a second launch joins them.
template <typename T, int THREADS, int AHEAD>
__global__ __launch_bounds__(THREADS) void piece_kernel(FqLogprobsArgs a, Work w)
{
    __shared__ Shared<THREADS> sh;
    const int r = blockIdx.x / w.pieces, p = blockIdx.x % w.pieces;
    const Row<T> row(a, r);
    const unsigned begin = p * w.piece, loads = row.loads(), end = min(loads, begin + w.piece);
    constexpr int PER = Row<T>::PER;
    const unsigned first = begin * PER / BLOCK >> w.shift;
    if (w.shift) {
        for (int i = threadIdx.x; i < MAX_BLOCKS; i += THREADS)
            sh.keys[i] = 0;
        __syncthreads();
    }
    if (begin < end)
        stream<T, THREADS, AHEAD>(row, begin, end, w.shift, first, a.top_n > 0, sh);
    else if ((threadIdx.x & 63) == 0)
        sh.parts[threadIdx.x >> 6] = Part{-INFINITY, 0.0, 0.0};
    __syncthreads();
    if (begin < end) {
        const unsigned blocks = (((end * PER + BLOCK - 1) / BLOCK + (1u << w.shift) - 1) >> w.shift) - first;
        for (unsigned i = threadIdx.x; i < blocks; i += THREADS)
            w.keys[(size_t)r * MAX_BLOCKS + first + i] = sh.keys[i];
    }
    join(THREADS / 64, sh.parts, true, sh);
    if (threadIdx.x == 0)
        w.parts[r * MAX_PIECES + p] = sh.all;
}

template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void join_kernel(FqLogprobsArgs a, Work w)
{
    __shared__ Shared<THREADS> sh;
    __shared__ Part parts[MAX_PIECES];
    const int r = blockIdx.x;
    const Row<T> row(a, r);
    const int given = first_given(a, r);
    const int blocks = (int)(((row.shift + row.V + BLOCK - 1) / BLOCK + (1u << w.shift) - 1) >> w.shift);
    for (int i = threadIdx.x; i < blocks; i += THREADS)
        sh.keys[i] = w.keys[(size_t)r * MAX_BLOCKS + i];
    if ((int)threadIdx.x < w.pieces)
        parts[threadIdx.x] = w.parts[r * MAX_PIECES + threadIdx.x];
    __syncthreads();
    join(w.pieces, parts, later<THREADS>(a, row, w.shift), sh);
    finish<T, THREADS>(a, r, row, given, w.shift, sh);
}

template <typename T>
hipError_t launch(const FqLogprobsArgs &a, void *workspace, hipStream_t stream)
{
    constexpr int PER = Row<T>::PER;
    int shift = 0;
    while (((long long)a.V + PER + BLOCK - 1) / BLOCK > (long long)MAX_BLOCKS << shift)
        shift++;
    const long long loads = ((long long)a.V + PER - 1) / PER + 1;
    const int cus = fq_device_cus(), grid = a.R;
    constexpr int AHEAD = 32 / PER, T2 = 512, UNIT = T2 * AHEAD;
    if (a.R <= SPLIT_ROWS && a.V >= SPLIT_LOGITS) {
        Work w{};
        const long long units = (loads + UNIT - 1) / UNIT;
        long long pieces = 2 * cus / a.R;
        pieces = pieces > MAX_PIECES ? MAX_PIECES : pieces < 1 ? 1 : pieces;
        const long long each = (units + pieces - 1) / pieces;
        w.pieces = (int)((units + each - 1) / each);
        w.piece = (unsigned)(each * UNIT);
        w.shift = shift;
        w.parts = (Part *)workspace;
        w.keys = (uint32_t *)((char *)workspace + sizeof(Part) * SPLIT_ROWS * MAX_PIECES);
        piece_kernel<T, T2, AHEAD><<<a.R * w.pieces, T2, 0, stream>>>(a, w);
        if (hipError_t e = hipGetLastError())
            return e;
        join_kernel<T, T2><<<a.R, T2, 0, stream>>>(a, w);
        return hipGetLastError();
    }
    if (loads <= 256)
        row_kernel<T, 64, 4><<<grid, 64, 0, stream>>>(a, shift);
    else if (a.R < cus && loads > 4096)
        row_kernel<T, 1024, AHEAD><<<grid, 1024, 0, stream>>>(a, shift);
    else if (loads <= 2048)
        row_kernel<T, 256, 4><<<grid, 256, 0, stream>>>(a, shift);
    else
        row_kernel<T, 512, AHEAD><<<grid, 512, 0, stream>>>(a, shift);
    return hipGetLastError();
}

} // namespace

size_t fq_logprobs_bytes(int, int) { return sizeof(Part) * SPLIT_ROWS * MAX_PIECES + sizeof(uint32_t) * SPLIT_ROWS * MAX_BLOCKS; }

hipError_t fq_launch_logprobs(const FqLogprobsArgs &a, bool half, void *workspace, hipStream_t stream)
{
    constexpr int ROWS = 1 << 20; // to a launch
    for (long long r = 0; r < a.R; r += ROWS) {
        FqLogprobsArgs some = a;
        some.R = a.R - r < ROWS ? (int)(a.R - r) : ROWS;
        some.logits = (const char *)a.logits + r * a.row_stride * (half ? 2 : 4);
        some.given = a.n_given ? a.given + r * a.n_given : nullptr;
        some.given_logprob = a.n_given ? a.given_logprob + r * a.n_given : nullptr;
        some.top_token = a.top_n ? a.top_token + r * a.top_n : nullptr;
        some.top_logprob = a.top_n ? a.top_logprob + r * a.top_n : nullptr;
        some.entropy = a.entropy ? a.entropy + r : nullptr;
        if (hipError_t e = half ? launch<_Float16>(some, workspace, stream) : launch<float>(some, workspace, stream))
            return e;
    }
    return hipSuccess;
}
