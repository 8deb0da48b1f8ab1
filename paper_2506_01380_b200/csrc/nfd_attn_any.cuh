// Attention of a batch's rows to 4-bit pages or encoder states, one warp per (row, head): the plainest form.
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
    // dims d .. d+n-1 of key p; false: not seen
    template <int n> __device__ __forceinline__ bool get(const BatchD &B, int s, int h, int p, int d, float *k, float *v) const {
        const long long place = P.place(B, s, p);
        if (place < 0) return false;
        const size_t at = (size_t)(place + (long long)h * P.page_tokens);
        float x[8];
        kv4_unpack(reinterpret_cast<const uint32_t *>(P.k)[at * (DH / 8) + d / 8], P.k_scale[at * (DH / 32) + d / 32], x);
        for (int e = 0; e < n; ++e) k[e] = x[d % 8 + e];
        kv4_unpack(reinterpret_cast<const uint32_t *>(P.v)[at * (DH / 8) + d / 8], P.v_scale[at * (DH / 32) + d / 32], x);
        for (int e = 0; e < n; ++e) v[e] = x[d % 8 + e];
        return true;
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
    template <int n> __device__ __forceinline__ bool get(const BatchD &B, int s, int h, int p, int d, float *ko, float *vo) const {
        if (mask && !mask[(size_t)s * n_keys + p]) return false;
        const long long at = s * seq_stride + p * key_stride + h * head_stride + d;
        for (int e = 0; e < n; ++e) ko[e] = to_f<TS>(k[at + e]), vo[e] = to_f<TS>(v[at + e]);
        return true;
    }
};

template <typename TS, int DH, typename Keys>
__global__ void __launch_bounds__(256) k_attn_any(const BatchD B, const AttnRows A, const Keys K) {
    constexpr int N = DH / 32;
    const int lane = threadIdx.x & 31, w = blockIdx.x * 8 + (threadIdx.x >> 5), s = blockIdx.y;
    const int i = w / A.heads, h = w - i * A.heads;
    const int2 sr = B.rows(s);
    if (i >= min(sr.y, B.max_rows)) return;
    const KeyRange kr = K.range(B, s, sr.y, i);
    const TS *q = (const TS *)A.q + (long long)(sr.x + i) * A.q_stride + h * DH + lane * N;
    const float scale = rsqrtf((float)DH);
    float qv[N], o[N] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < N; ++e) qv[e] = to_f<TS>(q[e]) * scale;
    for (int p = kr.lo; p < kr.hi; ++p) {
        float k[N], v[N];
        if (!K.template get<N>(B, s, h / A.share, p, lane * N, k, v)) continue;
        float x = 0.f;
        for (int e = 0; e < N; ++e) x = fmaf(qv[e], k[e], x);
        x = warp_sum(x);
        if (x == -INFINITY) continue;
        const float mn = fmaxf(m, x), a = expf(m - mn), b = expf(x - mn);
        l = l * a + b;
        for (int e = 0; e < N; ++e) o[e] = o[e] * a + b * v[e];
        m = mn;
    }
    TS *out = (TS *)A.out + ((long long)(sr.x + i) * A.heads + h) * DH + lane * N;
    for (int e = 0; e < N; ++e) out[e] = from_f<TS>(l == 0.f ? 0.f : o[e] / l);
}

template <typename TS, int DH, typename Keys>
static int launch_attn_any(const BatchD &B, const AttnRows &A, const Keys &K, cudaStream_t st) {
    const dim3 grid((unsigned)(((long long)B.max_rows * A.heads + 7) / 8), B.n_seqs);
    k_attn_any<TS, DH, Keys><<<grid, 256, 0, st>>>(B, A, K);
    return cudaGetLastError() == cudaSuccess ? NFD_OK : NFD_E_CUDA;
}
