// The rows of an attention call, and what they attend to: 4-bit pages or encoder states.
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
    __device__ __forceinline__ int length(const BatchD &B, int s) const { return B.kv_len ? min(B.tokens(s), n_keys) : n_keys; }
    __device__ __forceinline__ KeyRange range(const BatchD &, int len, int, int) const { return {0, len}; }
};


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
