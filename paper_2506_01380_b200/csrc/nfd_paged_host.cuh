// The host's side of the calls on the caller's own memory: checks of arguments, the current device.
#pragma once
#include <math.h>
#include <stdio.h>
#include <string.h>

#include "nfd_append.cuh"

#define CK(call)                                                                                   \
    do {                                                                                           \
        cudaError_t e_ = (call);                                                                   \
        if (e_ != cudaSuccess) {                                                                   \
            fprintf(stderr, "libnfd: %s failed: %s (%s:%d)\n", #call, cudaGetErrorString(e_),      \
                    __FILE__, __LINE__);                                                           \
            return NFD_E_CUDA;                                                                     \
        }                                                                                          \
    } while (0)

#define RET(expr)                    \
    do {                             \
        int r_ = (expr);             \
        if (r_ != NFD_OK) return r_; \
    } while (0)

namespace {

bool aligned(const void *p, int bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
size_t type_size(int dtype) { return dtype == NFD_DTYPE_FP32 ? 4 : 2; }

template <typename F> int by_head_dim(int dh, F &&f) {
    switch (dh) {
        case 32: return f(std::integral_constant<int, 32>());
        case 64: return f(std::integral_constant<int, 64>());
        default: return f(std::integral_constant<int, 128>());
    }
}

int check_batch(const nfd_batch *b, bool paged, BatchD &B) {
    if (!b) return NFD_E_NULLPTR;
    if (paged && (!b->kv_len || !b->table)) return NFD_E_NULLPTR;
    if (!aligned(b->row_start, 4) || !aligned(b->kv_len, 4) || !aligned(b->table, 4)) return NFD_E_ALIGN;
    if (b->n_seqs < 1 || b->n_seqs > 65535 || b->n_rows < 0 || b->n_rows > NFD_MAX_TOKENS) return NFD_E_RANGE;
    if (b->max_rows < 0 || b->max_rows > b->n_rows) return NFD_E_RANGE;
    if (!b->row_start && (long long)b->n_seqs * b->max_rows != b->n_rows) return NFD_E_RANGE;
    if (paged && (b->table_len < 1 || b->table_len > NFD_MAX_TOKENS)) return NFD_E_RANGE;
    B = {b->row_start, b->kv_len, b->table, b->n_seqs, b->n_rows, b->max_rows, b->table_len};
    return NFD_OK;
}

int check_pages(const nfd_pages *p, PagesD &P) {
    if (!p || !p->k || !p->v) return NFD_E_NULLPTR;
    if (p->dtype != NFD_DTYPE_FP32 && p->dtype != NFD_DTYPE_BF16 && p->dtype != NFD_DTYPE_KV4) return NFD_E_BADCFG;
    if (p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) return NFD_E_BADCFG;
    if (p->dtype == NFD_DTYPE_KV4 && (!p->k_scale || !p->v_scale)) return NFD_E_NULLPTR;
    if (!aligned(p->k, 16) || !aligned(p->v, 16)) return NFD_E_ALIGN;
    if (p->dtype == NFD_DTYPE_KV4 && (!aligned(p->k_scale, 16) || !aligned(p->v_scale, 16))) return NFD_E_ALIGN;
    if (p->n_pages < 1 || p->n_heads < 1 || p->n_heads > 1024 || p->page_tokens < 1 || p->page_tokens > (1 << 20)) return NFD_E_RANGE;
    P = {p->k, p->v, (uint16_t *)p->k_scale, (uint16_t *)p->v_scale, p->n_pages, p->n_heads, p->page_tokens};
    return NFD_OK;
}

// rows of `heads` heads, `stride` elements apart, read in 16-byte words; where there are no rows they may be nowhere
int check_rows(const BatchD &B, const void *p, long long stride, int heads, int head_dim, int dtype) {
    if (!p && B.n_rows) return NFD_E_NULLPTR;
    if (!aligned(p, 16) || (stride * (long long)type_size(dtype)) % 16) return NFD_E_ALIGN;
    if (stride < (long long)heads * head_dim || stride > (1LL << 40)) return NFD_E_RANGE;
    return NFD_OK;
}

// heads that share heads of keys; rows x heads that share one are numbered within a sequence, 32 and more to a CTA of a grid's last dimension
int check_heads(int n_heads, int kv_heads, const BatchD &B) {
    if (n_heads < 1 || n_heads > 1024 || kv_heads < 1 || n_heads % kv_heads) return NFD_E_RANGE;
    if ((long long)B.max_rows * (n_heads / kv_heads) > 65535LL * 32) return NFD_E_RANGE;
    return NFD_OK;
}

// the current device and its SMs
int this_device(int &dev, int &n_sm) {
    static std::atomic<int> n_sms[NFD_PAGED_DEVICES];      // (the same value whichever thread stores it)
    CK(cudaGetDevice(&dev));
    if (dev < 0 || dev >= NFD_PAGED_DEVICES) return NFD_E_RANGE;
    n_sm = n_sms[dev];
    if (!n_sm) {
        CK(cudaDeviceGetAttribute(&n_sm, cudaDevAttrMultiProcessorCount, dev));
        n_sms[dev] = n_sm;
    }
    return NFD_OK;
}

// rows of a CTA: several where every SM has a few CTAs all the same
int append_rows(int n_rows, int n_sm) {
    int rows = 1;
    while (rows < APPEND_MAX_ROWS && n_rows >= 4 * rows * n_sm) rows *= 2;
    return rows;
}

}  // namespace
