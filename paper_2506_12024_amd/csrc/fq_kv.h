// What the kernels over a paged cache share: the tables of a batch as one token or one tile of keys sees them, and the
// two 16-bit types.
#ifndef FQ_KV_H
#define FQ_KV_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fq_internal.h"

// New tokens of sequence b, held inside the call's rows, and its places in the cache.
struct FqSeq {
    int q0, n, len;
};

__device__ __forceinline__ FqSeq fq_seq(const FqSeqsView &s, int page_shift, int b)
{
    FqSeq r;
    r.q0 = min(max(s.q_start[b], 0), s.tokens);
    r.n = min(max(s.q_start[b + 1], r.q0), s.tokens) - r.q0;
    r.len = min(max(s.kv_len[b], 0), s.table_width << page_shift);
    return r;
}

__device__ __forceinline__ float fq_to_float(uint16_t v, bool bf16)
{
    return bf16 ? __builtin_bit_cast(float, (uint32_t)v << 16) : (float)__builtin_bit_cast(_Float16, v);
}

// One rounding, to nearest even (NaNs stay NaNs).
__device__ __forceinline__ uint16_t fq_from_float(float f, bool bf16)
{
    if (!bf16)
        return __builtin_bit_cast(uint16_t, (_Float16)f);
    return __builtin_bit_cast(uint16_t, (__bf16)f);
}

#endif
