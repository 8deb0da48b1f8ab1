// The rows of an attention call, and what they attend to: 4-bit pages, pages of whole numbers, the rows of a prompt, or encoder states.
#pragma once
#include <mutex>
#include "nfd_append.cuh"

// The rows of a call.
struct AttnRows {
    const void *q;
    void *out;
    long long q_stride;
    int heads, share;                    // heads, heads per head of the keys
    // row r of a unit (rows x heads that share a head of keys) as row and which of the heads; (without a division where there is none to share)
    __device__ __forceinline__ int2 split(int r) const {
        if (share == 1) return make_int2(r, 0);
        const int i = r / share;
        return make_int2(i, r - i * share);
    }
};

// Keys and values in 4-bit pages.
template <int DH> struct Kv4Keys {
    PagesD P;
    CausalMask mask;
    // tokens of sequence s (a load: asked for early); what row i of n of a sequence of that many sees
    __device__ __forceinline__ int length(const BatchD &B, int s) const { return B.tokens(s); }
    __device__ __forceinline__ KeyRange range(const BatchD &B, int len, int n, int i) const { return mask.range(len, P.oldest(B, len), n, i); }
};
// States of an encoder.
template <typename TS, int DH> struct StateKeys {
    const TS *k, *v;
    const unsigned char *mask;
    long long seq_stride, key_stride, head_stride;
    int n_keys;
    __device__ __forceinline__ const TS *first_k() const { return k; }
    __device__ __forceinline__ const TS *first_v() const { return v; }
    __device__ __forceinline__ int length(const BatchD &B, int s) const { return B.kv_len ? min(B.tokens(s), n_keys) : n_keys; }
    __device__ __forceinline__ KeyRange range(const BatchD &, int len, int, int) const { return {0, len}; }
};

// Pages of TS and the rows of packed sequences, both under the block-wise causal mask.  A reader walks keys p, p + step, ... with a cursor, which
// tells a key's row (-1: there is none): of the pages, (page, head, offset), or of the row buffers.
template <typename TS, int DH> struct PageKeys {
    static constexpr bool TMA = false, HOLES = true;                     // a key within the range may not be there
    PagesD P;
    CausalMask mask;
    __device__ __forceinline__ int length(const BatchD &B, int s) const { return B.tokens(s); }
    __device__ __forceinline__ KeyRange range(const BatchD &B, int len, int n, int i) const { return mask.range(len, P.oldest(B, len), n, i); }
    struct Cursor {
        const int *table;
        int pg, off, dq, dr;                                // entry of the table, offset in the page; how far they move (additions instead of two divisions a step)
    };
    __device__ __forceinline__ Cursor cursor(const BatchD &B, int s, int first_row, int p, int step) const {
        const int T = P.page_tokens, L = B.table_len;
        return {B.table + (size_t)s * L, p / T % L, p % T, step / T % L, step % T};
    }
    __device__ __forceinline__ long long next(Cursor &c, const BatchD &B, int h, bool there) const {
        const int T = P.page_tokens, L = B.table_len;
        long long row = -1;
        if (there) {
            const int page = __ldg(c.table + c.pg);
            if ((unsigned)page < (unsigned)P.n_pages) row = ((long long)page * P.heads + h) * T + c.off;
        }
        c.off += c.dr, c.pg += c.dq;
        if (c.off >= T) c.off -= T, ++c.pg;
        if (c.pg >= L) c.pg -= L;
        return row;
    }
    __device__ __forceinline__ const TS *first_k() const { return (const TS *)P.k; }         // (where nothing is read from)
    __device__ __forceinline__ const TS *first_v() const { return (const TS *)P.v; }
    __device__ __forceinline__ const TS *k_row(long long row, int) const { return (const TS *)P.k + row * DH; }
    __device__ __forceinline__ const TS *v_row(long long row, int) const { return (const TS *)P.v + row * DH; }
};
template <typename TS, int DH> struct PackedKeys {
    static constexpr bool TMA = false, HOLES = false;
    const TS *k, *v;
    long long k_stride, v_stride;
    CausalMask mask;
    __device__ __forceinline__ int length(const BatchD &B, int s) const { return B.rows(s).y; }
    __device__ __forceinline__ KeyRange range(const BatchD &, int len, int n, int i) const { return mask.range(len, 0, n, i); }
    struct Cursor {
        int row, step;
    };
    __device__ __forceinline__ Cursor cursor(const BatchD &, int, int first_row, int p, int step) const { return {first_row + p, step}; }
    __device__ __forceinline__ long long next(Cursor &c, const BatchD &, int, bool there) const {
        const int row = c.row;
        c.row += c.step;
        return there ? row : -1;
    }
    __device__ __forceinline__ const TS *first_k() const { return k; }
    __device__ __forceinline__ const TS *first_v() const { return v; }
    __device__ __forceinline__ const TS *k_row(long long row, int h) const { return k + row * k_stride + h * DH; }
    __device__ __forceinline__ const TS *v_row(long long row, int h) const { return v + row * v_stride + h * DH; }
};
// Is one of a pair of bf16 numbers not finite?  Which bits of it are those of finite ones.
__device__ __forceinline__ uint32_t finite_bits(uint32_t w) {
    return ((w & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((w & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
}

// What a kernel's first call on a device finds out, once for all threads: nobody reads it before it is complete.
struct OncePerDevice {
    std::atomic<bool> done[NFD_PAGED_DEVICES];
    std::mutex mutex;
    // f() returns false where it failed: the next call tries again
    template <typename F> bool run(int dev, F &&f) {
        if (done[dev]) return true;
        std::lock_guard<std::mutex> lock(mutex);
        if (!done[dev]) {
            if (!f()) {
                cudaGetLastError();                         // (the call's code tells)
                return false;
            }
            done[dev] = true;
        }
        return true;
    }
};
// Clusters of `ctas` CTAs that the device holds at once.
template <typename Kernel> static int clusters_that_fit(Kernel kern, int ctas, int threads, int smem) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas), cfg.blockDim = dim3(threads), cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension, at.val.clusterDim.x = ctas, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at, cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kern, &cfg) == cudaSuccess) return n;
    cudaGetLastError();
    return 0;
}
