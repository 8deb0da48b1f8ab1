// Arithmetic of the calls on the caller's own memory on numbers alone, for the host and the kernels (and for a plain C++ compiler).
#pragma once
#include <string.h>
#include "nfd_attn_plan.h"

// Rows start .. end - 1 of a buffer of n_rows, whatever device memory says: both ends are clamped into 0 .. n_rows before anything is formed of
// them, so that first and first + n lie in 0 .. n_rows and no difference leaves an int.
struct RowSpan {
    int first, n;
};
NFD_HD int clamp_row(int row, int n_rows) { return row < 0 ? 0 : row > n_rows ? n_rows : row; }
NFD_HD RowSpan rows_between(int start, int end, int n_rows) {
    const int a = clamp_row(start, n_rows), b = clamp_row(end, n_rows);
    return {a, b > a ? b - a : 0};
}

// Keys that `rows` (one at least) tokens of a sequence, one behind the other, see under the block-wise causal mask, all together: those of the frames that the rows
// lie in (of as many as they can touch) and of `window` before, of `held` that there are.
NFD_HD long long keys_seen(long long held, int frame_tokens, int window, int rows) {
    const long long frames = (rows + (long long)frame_tokens - 2) / frame_tokens + 1, span = (window + frames) * frame_tokens;
    return held < span ? held : span;
}
// The same of a prompt's first `rows` rows, whose tokens begin at 0, in a buffer of n_rows: none sees further than the end of its frame, whatever other prompts there are.
NFD_HD long long prompt_keys_seen(int n_rows, int frame_tokens, int window, int rows) {
    const long long end = ((long long)rows + frame_tokens - 1) / frame_tokens * frame_tokens;
    return keys_seen(n_rows < end ? n_rows : end, frame_tokens, window, rows);
}
// Parts of so many keys that a run of `keys` touches, wherever in a part it begins.
NFD_HD int parts_touched(long long keys, int part) { return keys < 2 ? (int)keys : (int)((keys - 2) / part) + 2; }

// Probabilities of states are formed 2^-bits of their size: with a reference m of a row that may be short of its largest score, n of them of up to
// 2^growth have a sum of 1 at most then, so that O, a sum of values times them, is no larger than the largest value and leaves fp32 for no
// finite one; the quotient of O and the sum does not know of it.  (What it costs is at the other end: small values
// lose bits in O, which ends at 2^-149 whatever the scale.)
NFD_HD int sum_bits(int growth, int n) {
    if (n <= 1) return growth;
#ifdef __CUDA_ARCH__
    return growth + 32 - __clz(n - 1);
#else
    return growth + 32 - __builtin_clz((unsigned int)n - 1);
#endif
}

// ---- one wave of CTAs for rows that go through shared memory -------------------------------------------------
#define NORM_STAGES 6                    // rows of a CTA that are ahead, at most
#define NORM_MOST 196608                 // shared memory of a CTA for them
#define SM_SHARED 233472                 // of an SM; each CTA takes 1 KB beside its own, and whole units of 128 bytes
struct NormPlan {
    int ctas, stages;                    // CTAs that an SM holds at once; rows ahead of each
};
// regs: of a thread, in steps of 8; row_bytes: of a row in shared memory (0: rows do not go through it), of which two fit into NORM_MOST; own: a CTA's other shared memory.
NFD_HD NormPlan norm_plan(int regs, int threads, int row_bytes, int own) {
    NormPlan p = {65536 / (regs * threads), 0};
    p.ctas = p.ctas < 1 ? 1 : p.ctas > 2048 / threads ? 2048 / threads : p.ctas;
    if (!row_bytes) return p;
    // as many rows ahead as leave the CTAs that the registers allow, two at least
    const int fixed = own + 1024 + 128, share = SM_SHARED / p.ctas - fixed;
    p.stages = (share < NORM_MOST ? share : NORM_MOST) / row_bytes;
    p.stages = p.stages > NORM_STAGES ? NORM_STAGES : p.stages < 2 ? 2 : p.stages;
    const int fit = SM_SHARED / (p.stages * row_bytes + fixed);
    if (fit < p.ctas) p.ctas = fit;
    return p;
}

// ---- the step of 4-bit numbers ------------------------------------------------------------------------------
NFD_HD uint32_t bits_of(float x) {
#ifdef __CUDA_ARCH__
    return __float_as_uint(x);
#else
    uint32_t b;
    memcpy(&b, &x, 4);
    return b;
#endif
}
NFD_HD float float_of(uint32_t b) {
#ifdef __CUDA_ARCH__
    return __uint_as_float(b);
#else
    float x;
    memcpy(&x, &b, 4);
    return x;
#endif
}
// The smallest fp32 number that is at least hi - lo (lo <= 0 <= hi): the rounded difference, and the next number where what the rounding took away
// (exactly the second sum, the larger number standing first in it) is above 0.  An fp32 number is at least hi - lo exactly where it is at least this one.
NFD_HD float kv4_range(float lo, float hi) {
    const float big = hi > -lo ? hi : -lo, small = hi > -lo ? -lo : hi, r = big + small;
    return small - (r - big) > 0.f ? float_of(bits_of(r) + 1) : r;
}
// Step (upper 12 bits of the word) of a group with that range: the smallest number of 4 significant bits, at least 2^-100, 15 of which cover it.
// The fp32 product is within an ulp or two of range / 15; 15 step is exact with 4 significant bits (or infinite), so that one comparison on either
// side settles which of two neighbours it is.
NFD_HD float kv4_step(float range) {
    const float least = 7.8886090522101181e-31f, t = range * (1.0f / 15.0f);
    uint32_t b = (bits_of(t > least ? t : least) + 0xFFFFFu) & 0xFFF00000u;
    if (15.0f * float_of(b) < range) b += 0x100000u;
    const uint32_t down = b - 0x100000u;
    if (float_of(down) >= least && 15.0f * float_of(down) >= range) b = down;
    return float_of(b);
}
