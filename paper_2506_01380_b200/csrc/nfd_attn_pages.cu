// Entry points for callers that bring their own memory: attention over pages of whole numbers and over packed prompts.  No context, no
// working memory; see include/nfd.h.
#include "nfd_paged_host.cuh"
#include "nfd_attn_f32.cuh"
#include "nfd_attn_block.cuh"

namespace {

// Attention of a batch's rows to keys under the block-wise causal mask, of the rows' type: by what their number and type ask for.  keys: the most that
// the rows of a sequence can see, all together.
template <template <typename, int> class Keys, typename Make>
int launch_rows(const BatchD &B, const AttnRows &A, int dtype, int head_dim, int kv_heads, long long keys, Make &&make, cudaStream_t st) {
    int dev = 0, n_sm = 0;
    RET(this_device(dev, n_sm));
    return by_head_dim(head_dim, [&](auto d) -> int {
        constexpr int DH = decltype(d)::value;
        if (dtype == NFD_DTYPE_FP32) {
            using K = Keys<float, DH>;
            return launch_attn_f32<DH>(B, A, F32Rows<K, DH>(make.template operator()<K>(), keys), kv_heads, dev, n_sm, st);
        }
        using K = Keys<bf16, DH>;
        if ((long long)B.max_rows * A.share > few_most(DH)) return attn_block<DH>(B, A, make.template operator()<K>(), kv_heads, keys, dev, n_sm, st);
        FewRows<K, DH> src;
        src.K = make.template operator()<K>(), src.bits = (float)sum_bits(8, (int)keys);       // (probabilities grow to 2^8 before m follows)
        return launch_attn_few<FewRows<K, DH>, DH>(B, A, src, kv_heads, keys, dev, n_sm, st);
    });
}
struct MakePageKeys {
    const PagesD &P;
    CausalMask mask;
    template <typename K> K operator()() const { return K{P, mask}; }
};
struct MakePackedKeys {
    const void *k, *v;
    long long k_stride, v_stride;
    CausalMask mask;
    template <typename K> K operator()() const {
        using TS = std::remove_const_t<std::remove_pointer_t<decltype(K::k)>>;
        return K{(const TS *)k, (const TS *)v, k_stride, v_stride, mask};
    }
};

int check_mask(int frame_tokens, int window) { return frame_tokens < 1 || frame_tokens > (1 << 20) || window < 0 ? NFD_E_RANGE : NFD_OK; }

}  // namespace

extern "C" {

int nfd_attention_pages(const nfd_pages *pages, const nfd_batch *batch, int n_heads, const void *q, long long q_stride,
                        int frame_tokens, int window, void *out, void *cuda_stream) {
    BatchD B;
    PagesD P;
    RET(check_pages(pages, P));
    RET(check_batch(batch, true, B));
    if (pages->dtype != NFD_DTYPE_FP32 && pages->dtype != NFD_DTYPE_BF16) return NFD_E_BADCFG;
    RET(check_heads(n_heads, P.heads, B));
    RET(check_rows(B, q, q_stride, n_heads, pages->head_dim, pages->dtype));
    if (!out && B.n_rows) return NFD_E_NULLPTR;
    if (!aligned(out, 16)) return NFD_E_ALIGN;
    RET(check_mask(frame_tokens, window));
    if (B.n_rows == 0 || B.max_rows == 0) return NFD_OK;
    const AttnRows A = {q, out, q_stride, n_heads, n_heads / P.heads};
    const long long held = (long long)B.table_len * P.page_tokens, most = held < NFD_MAX_TOKENS ? held : NFD_MAX_TOKENS;
    return launch_rows<PageKeys>(B, A, pages->dtype, pages->head_dim, P.heads, keys_seen(most, frame_tokens, window, B.max_rows),
                                 MakePageKeys{P, {frame_tokens, window}}, (cudaStream_t)cuda_stream);
}

int nfd_attention_packed(const nfd_batch *batch, int dtype, int n_heads, int kv_heads, int head_dim, const void *q, long long q_stride,
                         const void *k, long long k_stride, const void *v, long long v_stride, int frame_tokens, int window, void *out,
                         void *cuda_stream) {
    if (!batch) return NFD_E_NULLPTR;
    nfd_batch prompts = *batch;
    prompts.kv_len = prompts.table = NULL;                 // (not looked at, aligned or not)
    BatchD B;
    RET(check_batch(&prompts, false, B));
    if (dtype != NFD_DTYPE_FP32 && dtype != NFD_DTYPE_BF16) return NFD_E_BADCFG;
    if (head_dim != 32 && head_dim != 64 && head_dim != 128) return NFD_E_BADCFG;
    RET(check_heads(n_heads, kv_heads, B));
    RET(check_rows(B, q, q_stride, n_heads, head_dim, dtype));
    RET(check_rows(B, k, k_stride, kv_heads, head_dim, dtype));
    RET(check_rows(B, v, v_stride, kv_heads, head_dim, dtype));
    if (!out && B.n_rows) return NFD_E_NULLPTR;
    if (!aligned(out, 16)) return NFD_E_ALIGN;
    RET(check_mask(frame_tokens, window));
    if (B.n_rows == 0 || B.max_rows == 0) return NFD_OK;
    const AttnRows A = {q, out, q_stride, n_heads, n_heads / kv_heads};
    // (a sequence may have more rows than are computed, and these may see them: the rest of a frame)
    return launch_rows<PackedKeys>(B, A, dtype, head_dim, kv_heads, prompt_keys_seen(B.n_rows, frame_tokens, window, B.max_rows),
                                   MakePackedKeys{k, v, k_stride, v_stride, {frame_tokens, window}}, (cudaStream_t)cuda_stream);
}

}  // extern "C"
