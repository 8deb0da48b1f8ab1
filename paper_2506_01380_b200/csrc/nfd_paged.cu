// Entry points for callers that bring their own memory: appending to paged caches, attention over 4-bit pages, cross
// attention.  No context, no working memory; see include/nfd.h.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include "nfd_append.cuh"
#include "nfd_attn_f32.cuh"
#include "nfd_attn_tile.cuh"

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

extern "C" {

int nfd_kv_append(const nfd_pages *pages, const nfd_batch *batch, const nfd_rope *rope, int dtype, const void *k,
                  long long k_stride, const void *v, long long v_stride, int n_q_heads, const void *q,
                  long long q_stride, void *q_out, void *cuda_stream) {
    BatchD B;
    PagesD P;
    RET(check_pages(pages, P));
    RET(check_batch(batch, true, B));
    if (dtype != NFD_DTYPE_FP32 && dtype != NFD_DTYPE_BF16) return NFD_E_BADCFG;
    if (pages->dtype != dtype && pages->dtype != NFD_DTYPE_KV4) return NFD_E_BADCFG;
    const int dh = pages->head_dim;
    RET(check_rows(B, k, k_stride, P.heads, dh, dtype));
    RET(check_rows(B, v, v_stride, P.heads, dh, dtype));
    if (n_q_heads < 0 || n_q_heads > 1024) return NFD_E_RANGE;
    if (n_q_heads) {
        RET(check_rows(B, q, q_stride, n_q_heads, dh, dtype));
        if (!q_out && B.n_rows) return NFD_E_NULLPTR;
        if (!aligned(q_out, 16)) return NFD_E_ALIGN;
    }
    RopeD R;
    memset(&R, 0, sizeof(R));
    if (rope) {
        const int d[3] = {rope->rope_t, rope->rope_h, rope->rope_w};
        if (d[0] < 0 || d[1] < 0 || d[2] < 0 || d[0] % 2 || d[1] % 2 || d[2] % 2 || (long long)d[0] + d[1] + d[2] != dh) return NFD_E_BADCFG;
        if (!(rope->theta > 0.f) || !isfinite(rope->theta)) return NFD_E_BADCFG;
        if (rope->frame_tokens < 1 || rope->grid_w < 1 || rope->frame_tokens % rope->grid_w) return NFD_E_BADCFG;
        R.on = 1, R.frame_tokens = rope->frame_tokens, R.grid_w = rope->grid_w;
        R.half_t = d[0] / 2, R.half_th = (d[0] + d[1]) / 2;
        // (the powers of the last rotation of this thread: they took longer than the rest of the call)
        static thread_local struct {
            int d[3];
            float theta;
            double freq[64];
        } last = {};
        if (memcmp(last.d, d, sizeof(d)) || last.theta != rope->theta) {
            for (int a = 0, pair = 0; a < 3; ++a)
                for (int i = 0; i < d[a] / 2; ++i) last.freq[pair++] = pow((double)rope->theta, -2.0 * i / d[a]);
            memcpy(last.d, d, sizeof(d)), last.theta = rope->theta;
        }
        memcpy(R.freq, last.freq, dh / 2 * sizeof(double));
    }
    if (B.n_rows == 0 || B.max_rows == 0) return NFD_OK;
    int dev = 0, n_sm = 0;
    RET(this_device(dev, n_sm));
    const AppendIO io = {q, k, v, q_stride, k_stride, v_stride, q_out, n_q_heads};
    const int rows = append_rows(B.n_rows, n_sm);
    const unsigned grid = (unsigned)((B.n_rows + rows - 1) / rows);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    by_head_dim(dh, [&](auto d) {
        constexpr int DH = decltype(d)::value;
        const bool kv4 = pages->dtype == NFD_DTYPE_KV4;
        if (dtype == NFD_DTYPE_BF16) {
            if (kv4) k_kv_append<bf16, true, DH><<<grid, APPEND_THREADS, 0, st>>>(R, io, B, P, rows);
            else k_kv_append<bf16, false, DH><<<grid, APPEND_THREADS, 0, st>>>(R, io, B, P, rows);
        } else {
            if (kv4) k_kv_append<float, true, DH><<<grid, APPEND_THREADS, 0, st>>>(R, io, B, P, rows);
            else k_kv_append<float, false, DH><<<grid, APPEND_THREADS, 0, st>>>(R, io, B, P, rows);
        }
        return 0;
    });
    CK(cudaGetLastError());
    return NFD_OK;
}

int nfd_pages_read(const nfd_pages *pages, const nfd_batch *batch, int dtype, void *k_out, void *v_out, void *cuda_stream) {
    BatchD B;
    PagesD P;
    RET(check_pages(pages, P));
    RET(check_batch(batch, true, B));
    if (dtype != NFD_DTYPE_FP32 && dtype != NFD_DTYPE_BF16) return NFD_E_BADCFG;
    if (pages->dtype != dtype && pages->dtype != NFD_DTYPE_KV4) return NFD_E_BADCFG;
    if (!aligned(k_out, 16) || !aligned(v_out, 16)) return NFD_E_ALIGN;
    if (B.n_rows == 0 || B.max_rows == 0 || (!k_out && !v_out)) return NFD_OK;
    int dev = 0, n_sm = 0;
    RET(this_device(dev, n_sm));
    const int rows = append_rows(B.n_rows, n_sm);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    by_head_dim(pages->head_dim, [&](auto d) {
        constexpr int DH = decltype(d)::value;
        const unsigned grid = (unsigned)((B.n_rows + rows - 1) / rows);
        if (pages->dtype == NFD_DTYPE_KV4) {
            if (dtype == NFD_DTYPE_BF16) k_pages_read<bf16, bf16, true, DH><<<grid, APPEND_THREADS, 0, st>>>(B, P, (bf16 *)k_out, (bf16 *)v_out, rows);
            else k_pages_read<bf16, float, true, DH><<<grid, APPEND_THREADS, 0, st>>>(B, P, (float *)k_out, (float *)v_out, rows);
        } else if (dtype == NFD_DTYPE_BF16) {
            k_pages_read<bf16, bf16, false, DH><<<grid, APPEND_THREADS, 0, st>>>(B, P, (bf16 *)k_out, (bf16 *)v_out, rows);
        } else {
            k_pages_read<float, float, false, DH><<<grid, APPEND_THREADS, 0, st>>>(B, P, (float *)k_out, (float *)v_out, rows);
        }
        return 0;
    });
    CK(cudaGetLastError());
    return NFD_OK;
}

int nfd_attention_kv4(const nfd_pages *pages, const nfd_batch *batch, int n_heads, const void *q, long long q_stride,
                      int frame_tokens, int window, void *out, void *cuda_stream) {
    BatchD B;
    PagesD P;
    RET(check_pages(pages, P));
    RET(check_batch(batch, true, B));
    if (pages->dtype != NFD_DTYPE_KV4) return NFD_E_BADCFG;
    RET(check_heads(n_heads, P.heads, B));
    RET(check_rows(B, q, q_stride, n_heads, pages->head_dim, NFD_DTYPE_BF16));
    if (!out && B.n_rows) return NFD_E_NULLPTR;
    if (!aligned(out, 16)) return NFD_E_ALIGN;
    if (frame_tokens < 1 || frame_tokens > (1 << 20) || window < 0) return NFD_E_RANGE;
    if (B.n_rows == 0 || B.max_rows == 0) return NFD_OK;
    const AttnRows A = {q, out, q_stride, n_heads, n_heads / P.heads};
    int dev = 0, n_sm = 0;
    RET(this_device(dev, n_sm));
    // the most keys that a unit's rows can see: what the tables hold, what the window leaves
    const long long held = (long long)B.table_len * P.page_tokens, seen = ((long long)window + 1) * frame_tokens + B.max_rows;
    const long long keys = held < seen ? held : seen;
    return by_head_dim(pages->head_dim, [&](auto d) -> int {
        constexpr int DH = decltype(d)::value;
        if ((long long)B.max_rows * A.share > few_most(DH))
            return launch_attn_tile<TileKv4<DH>, DH>(B, A, TileKv4<DH>{{P, {frame_tokens, window}}}, P.heads, keys, dev, n_sm, (cudaStream_t)cuda_stream);
        FewKv4<DH> src;
        src.K = {P, {frame_tokens, window}};
        return launch_attn_few<FewKv4<DH>, DH>(B, A, src, P.heads, keys, dev, n_sm, (cudaStream_t)cuda_stream);
    });
}

int nfd_cross_attention(const nfd_states *states, const nfd_batch *batch, int n_heads, const void *q, long long q_stride,
                        void *out, void *cuda_stream) {
    if (!states || (states->n_keys && (!states->k || !states->v))) return NFD_E_NULLPTR;
    BatchD B;
    RET(check_batch(batch, false, B));
    const int dtype = states->dtype, dh = states->head_dim;
    if (dtype != NFD_DTYPE_FP32 && dtype != NFD_DTYPE_BF16) return NFD_E_BADCFG;
    if (dh != 32 && dh != 64 && dh != 128) return NFD_E_BADCFG;
    if (states->n_keys < 0 || states->n_keys > NFD_MAX_TOKENS) return NFD_E_RANGE;
    RET(check_heads(n_heads, states->n_heads, B));
    const long long unit = 16 / (long long)type_size(dtype), most = 1LL << 40;
    const long long st[3] = {states->seq_stride, states->key_stride, states->head_stride};
    for (long long s : st)
        if (s < 0 || s > most) return NFD_E_RANGE;
    for (long long s : st)
        if (s % unit) return NFD_E_ALIGN;
    if (!aligned(states->k, 16) || !aligned(states->v, 16)) return NFD_E_ALIGN;
    RET(check_rows(B, q, q_stride, n_heads, dh, dtype));
    if (!out && B.n_rows) return NFD_E_NULLPTR;
    if (!aligned(out, 16)) return NFD_E_ALIGN;
    if (B.n_rows == 0 || B.max_rows == 0) return NFD_OK;
    const AttnRows A = {q, out, q_stride, n_heads, n_heads / states->n_heads};
    int dev = 0, n_sm = 0;
    RET(this_device(dev, n_sm));
    return by_head_dim(dh, [&](auto d) -> int {
        constexpr int DH = decltype(d)::value;
        auto go = [&](auto *t) -> int {
            using TS = std::remove_pointer_t<decltype(t)>;
            const StateKeys<TS, DH> K = {(const TS *)states->k, (const TS *)states->v, states->mask, st[0], st[1], st[2], states->n_keys};
            if constexpr (std::is_same_v<TS, bf16>) {
                if ((long long)B.max_rows * A.share > few_most(DH))
                    return launch_attn_tile<TileStates<DH>, DH>(B, A, TileStates<DH>{K}, states->n_heads, states->n_keys, dev, n_sm, (cudaStream_t)cuda_stream);
                FewStates<DH> src;
                src.K = K, src.bits = (float)sum_bits(8, K.n_keys);    // (probabilities grow to 2^8 before m follows)
                return launch_attn_few<FewStates<DH>, DH>(B, A, src, states->n_heads, states->n_keys, dev, n_sm, (cudaStream_t)cuda_stream);
            } else {
                return launch_attn_f32<DH>(B, A, K, states->n_heads, dev, n_sm, (cudaStream_t)cuda_stream);
            }
        };
        return dtype == NFD_DTYPE_BF16 ? go((bf16 *)nullptr) : go((float *)nullptr);
    });
}

}  // extern "C"
