// Batches of sequences, paged caches and encoder states as kernels see them: where a row belongs, where a token lies, the
// 4-bit numbers.  Everything that comes from device memory (row starts, lengths, page numbers) is clamped here.
#pragma once
#include <atomic>
#include "nfd_common.cuh"
#include "nfd_paged_plan.h"

#define NFD_MAX_TOKENS (1 << 30)
#define NFD_PAGED_DEVICES 64

struct BatchD {
    const int *row_start, *kv_len, *table;
    int n_seqs, n_rows, max_rows, table_len;
    // first row and number of rows of sequence s (of which the first max_rows are computed)
    __device__ __forceinline__ int2 rows(int s) const {
        if (!row_start) return make_int2(s * max_rows, max_rows);
        const RowSpan r = rows_between(__ldg(row_start + s), __ldg(row_start + s + 1), n_rows);
        return make_int2(r.first, r.n);
    }
    // the sequence of a row, for a whole warp: as many as end at or before it
    __device__ __forceinline__ int seq_of(int row) const {
        if (!row_start) return row / max_rows;
        int s = 0;
        for (int s0 = 0; s0 < n_seqs; s0 += 32) {
            const int i = s0 + (threadIdx.x & 31);
            s += __popc(__ballot_sync(0xffffffffu, i < n_seqs && __ldg(row_start + i + 1) <= row));
        }
        return s;
    }
    __device__ __forceinline__ int tokens(int s) const { return min(max(__ldg(kv_len + s), 0), NFD_MAX_TOKENS); }
};

// What a token's place in a paged cache needs.
struct PagesD {
    void *k, *v;
    uint16_t *k_scale, *v_scale;
    int n_pages, heads, page_tokens;
    // Place of token p of sequence s: (page * heads) * page_tokens + offset, in rows; head h is h * page_tokens further on.
    // -1: there is none.
    __device__ __forceinline__ long long place(const BatchD &B, int s, int p) const {
        const int pg = p / page_tokens, page = __ldg(B.table + (size_t)s * B.table_len + pg % B.table_len);
        if ((unsigned)page >= (unsigned)n_pages) return -1;
        return (long long)page * heads * page_tokens + (p - pg * page_tokens);
    }
    // tokens below this one have been overwritten by the ring
    __device__ __forceinline__ int oldest(const BatchD &B, int tokens) const {
        const long long o = (long long)tokens - (long long)B.table_len * page_tokens;
        return o > 0 ? (int)o : 0;
    }
};

// ---- 4-bit numbers ------------------------------------------------------------------------------------------
// x / step to the nearest whole number, ties to even, in the low bits of the result's significand (less KV4_MAGIC's bits).  The quotient is
// corrected by its exact remainder, which makes it the rounded quotient; step having 4 significant bits, a quotient that is not half way
// between whole numbers is not rounded to one that is (it is off by more than half an ulp), so that rounding once more loses nothing.
#define KV4_MAGIC 12582912.0f                              // 1.5 x 2^23: an ulp is 1
__device__ __forceinline__ float kv4_quotient(float x, float step, float inv) {
    const float q = x * inv;
    return fmaf(fmaf(-q, step, x), inv, q) + KV4_MAGIC;
}
// bits of code i of a word of eight
__device__ __forceinline__ constexpr int kv4_shift(int i) { return 4 * (i >> 1) + 16 * (i & 1); }
// pair i of a word of codes as bf16 numbers: z2 = two bf16 numbers 128 + z, step2 = the step twice
__device__ __forceinline__ uint32_t kv4_pair(uint32_t codes, int i, uint32_t z2, uint32_t step2) {
    const uint32_t t = (codes >> (4 * i) & 0x000F000Fu) | 0x43004300u;
    __nv_bfloat162 a = *reinterpret_cast<const __nv_bfloat162 *>(&t);
    a = __hmul2(__hsub2(a, *reinterpret_cast<const __nv_bfloat162 *>(&z2)), *reinterpret_cast<const __nv_bfloat162 *>(&step2));
    return *reinterpret_cast<const uint32_t *>(&a);
}
__device__ __forceinline__ uint32_t kv4_z2(uint32_t w0, uint32_t w1) { return (w0 & 15u) | (w1 & 15u) << 16 | 0x43004300u; }
__device__ __forceinline__ uint32_t kv4_step2(uint32_t w0, uint32_t w1) { return (w0 & 0xFFF0u) | (w1 & 0xFFF0u) << 16; }

// The same for the operands of products, scaled by 2^-32 (KV4_UP undoes it in fp32): a code in the low bits of a bf16 is the subnormal number
// n 2^-133, and one fma with step 2^101 and -z step 2^-32 makes (n - z) step 2^-32 of it: two instructions and a
// shift for two numbers, where kv4_pair takes three.  Exactly for steps from 2^-98 on, whose numbers are whole multiples of 2^-101; the quantiser's smaller
// ones (2^-100 and 2^-99) lose half of 2^-101 in z step and half in the fma.  Steps of 2^27 and more (numbers beyond 10^8) count as not finite here.
#define KV4_UP 4294967296.0f
__device__ __forceinline__ bool kv4_not_finite(uint32_t word) { return (word & 0x7F80u) >= 0x4D00u; }
struct Kv4Scale {
    uint32_t step2, zero2;
    // check: the words may be of steps that are not finite
    __device__ __forceinline__ Kv4Scale(uint32_t w0, uint32_t w1, bool check) {
        auto up = [check](uint32_t w) { return check && kv4_not_finite(w) ? 0x7FC0u : (w & 0xFFF0u) + (101u << 7); };
        step2 = up(w0) | up(w1) << 16;
        const uint32_t z = (w0 & 15u) | (w1 & 15u) << 16;
        const __nv_bfloat162 p = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&z), *reinterpret_cast<const __nv_bfloat162 *>(&step2));
        zero2 = *reinterpret_cast<const uint32_t *>(&p) ^ 0x80008000u;
    }
    __device__ __forceinline__ uint32_t pair(uint32_t codes, int i) const {
        const uint32_t t = codes >> (4 * i) & 0x000F000Fu;
        const __nv_bfloat162 a = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&t), *reinterpret_cast<const __nv_bfloat162 *>(&step2),
                                         *reinterpret_cast<const __nv_bfloat162 *>(&zero2));
        return *reinterpret_cast<const uint32_t *>(&a);
    }
};

// ---- which keys a row sees ----------------------------------------------------------------------------------
struct KeyRange {
    int lo, hi;
};
// Block-wise causal: row i of n of a sequence of `len` tokens.
struct CausalMask {
    int frame_tokens, window;
    __device__ __forceinline__ KeyRange range(int len, int oldest, int n, int i) const {
        const int p = len - n + i;
        if (p < 0) return {0, 0};
        const int f = p / frame_tokens;
        const int lo = max(max(f - window, 0) * frame_tokens, oldest);
        return {lo, max(lo, min((f + 1) * frame_tokens, len))};
    }
};
