// The rows of an attention call, and what they attend to: 4-bit pages or encoder states.
#pragma once
#include "nfd_append.cuh"

// The rows of a call.
struct AttnRows {
    const void *q;
    void *out;
    long long q_stride;
    int heads, share;                    // heads, heads per head of the keys
};

// Keys and values in 4-bit pages.
template <int DH> struct Kv4Keys {
    PagesD P;
    CausalMask mask;
    __device__ __forceinline__ KeyRange range(const BatchD &B, int s, int n, int i) const {
        const int len = B.tokens(s);
        return mask.range(len, P.oldest(B, len), n, i);
    }
};
// States of an encoder.
template <typename TS, int DH> struct StateKeys {
    const TS *k, *v;
    const unsigned char *mask;
    long long seq_stride, key_stride, head_stride;
    int n_keys;
    __device__ __forceinline__ KeyRange range(const BatchD &B, int s, int n, int i) const {
        return {0, B.kv_len ? min(B.tokens(s), n_keys) : n_keys};
    }
};

