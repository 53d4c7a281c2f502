// What the attention kernels share: which rows and keys a workgroup takes, how a key's row is found, the matrix
// instructions of both types, and the end of a row of the softmax.
//
// A sequence's keys are numbered through prefix and cache: key 0 .. prefix_len - 1, then its places.  Rows are (new token,
// query head of one key head), token by token.  Both kernels compute the scores transposed, S^T = K Q^T: a lane then holds
// scores of ONE row, over keys that run through its registers, so the statistics of a row are a lane's own but for one or two
// exchanges, and exp(S^T) is already the right-hand operand of O^T = V^T P^T.  The contraction over keys may run in any order,
// so the keys a lane holds after the first product are the keys it takes V's elements of (read transposed from LDS), and P never
// moves between lanes.
#ifndef FQ_ATTEND_H
#define FQ_ATTEND_H

#include <hip/hip_runtime.h>

#include "fq_kv.h"
#include "fq_mfma.h"

// One piece of work: the rows it takes and how their keys are split.
struct FqAttendWork {
    int shared;     // 1: all tokens' rows over the prefix; 0: a sequence's rows over its keys from key0 on
    int key0;
    int chunk;      // keys of one part
    int part0;      // its parts are part0 .. part0 + parts - 1
    int row_blocks; // of a sequence (shared: of all tokens); 0: the sequences' row blocks follow each other, as many as each has
    uint32_t blocks_x, parts, blocks; // its grid: key heads times row blocks, parts, sequences; workgroups in all
    float *part_o;  // [part][token][q_head][dim] not yet divided, or null: one part, the result goes out
    float2 *part_ml; // [part][token][q_head]: reference of the row's weights (a score times log2 e), their sum
};

constexpr float FQ_LOG2E = 1.4426950408889634f, FQ_LN2 = 0.6931471805599453f;
// A row's weights are 2^(score - its reference), rounded to the 16-bit type where they meet V.  binary16 ends under 2^16 and has fewer
// bits below 2^-14, so there the reference is set 2^7 below the row's largest score, and the row is rescaled when a score passes that
// one by more than 2^8 (most tiles rescale nothing): weights lie under 2^15, the largest at 2^7 or above, a key that has 2^-21 of it
// keeps all its bits and one of 2^-32 still counts.  (With the reference at the largest score those were 2^-14 and 2^-25: 32768 keys
// of 2^-27.5 beside one of 1 were lost, of 2^-24.3 a quarter too heavy.)  bfloat16 has binary32's range.
template <bool BF16>
constexpr float FQ_ATTEND_BELOW = BF16 ? 0.0f : 7.0f;
constexpr float FQ_ATTEND_SLACK = 8.0f;

// The rows of one workgroup's sequence and what they see.
struct FqAttendRows {
    int q0, rows;   // first token, rows
    int own, n;     // own keys before the first new token (may be negative)
    int P, max_kv;
    bool shared;
    __device__ __forceinline__ int limit(int j) const // keys 0 .. limit - 1 are seen by token j
    {
        return shared ? P : P + min(max(own + j + 1, 0), max_kv);
    }
};

__device__ __forceinline__ FqAttendRows fq_attend_rows(const FqAttendArgs &a, const FqAttendWork &w, int b, int group)
{
    FqAttendRows r;
    r.P = a.seqs.prefix_len;
    r.max_kv = a.max_kv;
    r.shared = w.shared != 0;
    if (r.shared) {
        r.q0 = 0;
        r.n = a.seqs.tokens;
        r.own = 0;
        r.rows = r.n * group;
    } else {
        const FqSeq s = fq_seq(a.seqs, a.kv.page_shift, b);
        r.q0 = s.q0;
        r.n = s.n;
        r.own = s.len - s.n;
        r.rows = min(s.n, a.max_q) * group;
    }
    return r;
}

// Row block `at` of those that the sequences have, one after the other: its sequence and its number there, the last one first (its
// rows see most keys); false past the end.  64 sequences at a time, every lane of the wavefront together.
__device__ __forceinline__ bool fq_find_row_block(const FqAttendArgs &a, int at, int group, int rows_per_block, int &b, int &block)
{
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < a.seqs.seqs; b0 += 64) {
        int mine = 0;
        if (b0 + lane < a.seqs.seqs)
            mine = (min(fq_seq(a.seqs, a.kv.page_shift, b0 + lane).n, a.max_q) * group + rows_per_block - 1) / rows_per_block;
        int to = mine;
        for (int o = 1; o < 64; o <<= 1) {
            const int x = __shfl_up(to, o);
            to += lane >= o ? x : 0;
        }
        const uint64_t after = __ballot(to > at);
        if (after) {
            const int who = __builtin_ctzll(after);
            b = b0 + who;
            block = __shfl(to, who) - 1 - at;
            return true;
        }
        at -= __shfl(to, 63);
    }
    return false;
}

// The page of a key, -1 for one that is not there (past `end`, or a hole).
__device__ __forceinline__ int fq_key_page(const FqAttendArgs &a, const int32_t *table, int key, int end)
{
    if (key >= end)
        return -1;
    const int P = a.seqs.prefix_len;
    return key < P ? a.seqs.prefix_table[key >> a.kv.page_shift] : table[(key - P) >> a.kv.page_shift];
}

// Where the row of a key's values begins, for a page that is there.
__device__ __forceinline__ long long fq_key_offset(const FqAttendArgs &a, int page, int key, int head)
{
    const int P = a.seqs.prefix_len;
    const int place = key < P ? key : key - P;
    return page * a.kv.page_stride + head * a.kv.head_stride + (place & ((1 << a.kv.page_shift) - 1)) * a.kv.token_stride;
}

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short4_t __attribute__((ext_vector_type(4)));

template <bool BF16>
__device__ __forceinline__ float4_t fq_mfma16(u32x4 x, u32x4 y, float4_t c)
{
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, x), __builtin_bit_cast(half8_t, y), c, 0, 0, 0);
}

template <bool BF16>
__device__ __forceinline__ float16_t fq_mfma32(u32x4 x, u32x4 y, float16_t c)
{
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, x), __builtin_bit_cast(half8_t, y), c, 0, 0, 0);
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Two values to the 16-bit type, each rounded to nearest even.
template <bool BF16>
__device__ __forceinline__ uint32_t fq_pack2(float x, float y)
{
    if constexpr (BF16)
        return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)x, (__bf16)y});
    else
        return __builtin_bit_cast(uint32_t, half2_t{(_Float16)x, (_Float16)y});
}

// The factor of the scores in powers of two.  It is never negative -- Q's signs are turned instead (exact), so that the largest
// product is the largest score -- nor 0, so that a masked -inf stays one: at least the smallest binary32 value, which leaves of any score
// that is finite (under 2^128) 2^-21 at most.
__device__ __forceinline__ float fq_score_factor(float scale) { return fmaxf(fabsf(scale) * FQ_LOG2E, 0x1p-149f); }
__device__ __forceinline__ u32x4 fq_signed(u32x4 q, float scale) { return scale < 0.0f ? q ^ 0x80008000u : q; }

// Four consecutive rows (keys) of a 16-column block of LDS, column by column: of 16 lanes, lane t names 8 bytes (row t / 4, columns
// 4 (t % 4) ..) and gets column t of the four rows.
__device__ __forceinline__ u32x2 fq_read_transposed(const char *at)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((FQ_LDS short4_t *)at));
}

// The larger of (the sum of) a value and that of the lane 32 on; of the lanes 16 on.
template <bool SUM>
__device__ __forceinline__ float fq_over32(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    const float x = __builtin_bit_cast(float, (uint32_t)r[0]), y = __builtin_bit_cast(float, (uint32_t)r[1]);
    return SUM ? x + y : fmaxf(x, y);
}
template <bool SUM>
__device__ __forceinline__ float fq_over16(float v)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float x = __builtin_bit_cast(float, (uint32_t)r[0]), y = __builtin_bit_cast(float, (uint32_t)r[1]);
    return SUM ? x + y : fmaxf(x, y);
}

// A score in powers of two, rounded by itself: references are such values, so that a row's largest score lies an exact distance from
// its reference.  In one rounding with the difference (fma) it is off by what x c loses: from 2^27 on by more than binary16
// has powers of two, and the row's weights overflow or vanish.  (Taken ahead of the products it costs prompts 0.5 %: 179.8 to 180.9 us for
// 2048 tokens behind 951 of the 70B shapes, 67.7 to 68.0 with heads of 64; between the products 183 and 70.6.)
__device__ __forceinline__ float fq_score(float x, float c)
{
#pragma clang fp contract(off)
    return x * c;
}

// exp2(x - m) for a row whose reference may still be -inf (nothing seen yet: 0)
__device__ __forceinline__ float fq_reference(float m) { return m == -INFINITY ? 0.0f : m; }

// Adds a step's sum of weights to a row's, with what rounding has taken from it: thousands of small sums beside one large weight lose the
// same part each time, or all of themselves (16 equal weights of 2^-24.3 at a time to a sum of 1).
__device__ __forceinline__ void fq_add_weights(float &l, float &lost, float sum)
{
#pragma clang fp contract(off)
    const float add = sum - lost, to = l + add;
    lost = (to - l) - add;
    l = to;
}

// lse in natural logarithms of a row with reference m (times log2 e) and sum l, whose power of two joins the reference: both parts would
// else be large and cancel where the lse is near 0.
__device__ __forceinline__ float fq_lse(float m, float l)
{
    int power = 0;
    const float part = frexpf(l, &power);
    return l == 0.0f ? -INFINITY : (fq_reference(m) + (float)power) * FQ_LN2 + logf(part);
}
__device__ __forceinline__ float fq_inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

// The products sum p v over all keys of a tile, and 0 times an infinity is NaN: a row must not meet a V that it does not see and that is
// not finite.  Keys past the end and holes are zeroed as they arrive.  So are the values that are not finite of those keys that some rows of
// a workgroup see and others do not (a chunk's own new tokens); the rows that see them get them back at the end, added to their sums:
// an infinity stays one whatever its weight, two of them or a NaN give NaN.
// All bits of those of two values that are not finite: an exponent of ones carries into the sign's place when one is added.
template <bool BF16>
__device__ __forceinline__ uint32_t fq_odd(uint32_t two)
{
    constexpr uint32_t EXPONENTS = BF16 ? 0x7f807f80 : 0x7c007c00, ONES = BF16 ? 0x00800080 : 0x04000400;
    const uint32_t signs = ((two & EXPONENTS) + ONES) & 0x80008000u;
    return signs | (signs - (signs >> 15));
}
// Value i of four if it is not finite, else 0.
template <bool BF16>
__device__ __forceinline__ float fq_odd_value(u32x2 four, int i)
{
    const uint32_t two = four[i >> 1] & fq_odd<BF16>(four[i >> 1]);
    return fq_to_float((uint16_t)(two >> (16 * (i & 1))), BF16);
}

// rt0, rt1: tiles of 16 rows of a workgroup of each piece, 0 for the kernel of many rows.  A launch of one piece has no workgroups in
// the second and names rt1 = rt0; of two pieces for few rows rt0 = rt1.
hipError_t fq_launch_attend_f16(const FqAttendArgs &a, const FqAttendWork &w0, const FqAttendWork &w1, int rt0, int rt1, hipStream_t stream);
hipError_t fq_launch_attend_bf16(const FqAttendArgs &a, const FqAttendWork &w0, const FqAttendWork &w1, int rt0, int rt1, hipStream_t stream);
constexpr int FQ_ATTEND_THREADS = 256;
constexpr uint32_t FQ_ATTEND_BLOCKS = 1u << 24; // fewer workgroups than this to a launch
constexpr int FQ_MANY_ROWS = 128; // rows of a workgroup of many rows

#endif
