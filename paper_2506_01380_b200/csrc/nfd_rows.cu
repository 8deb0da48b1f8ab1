// Entry points for callers that bring their own memory: rotation of rows, norms around a block.  No context, no working memory; see
// include/nfd.h.
#include "nfd_paged_host.cuh"
#include "nfd_rows.cuh"

namespace {

// parameters of a norm
int check_norm(const nfd_norm *n, NormD &N) {
    memset(&N, 0, sizeof(N));
    if (!n) return NFD_OK;
    if (n->kind != NFD_NORM_LAYER && n->kind != NFD_NORM_RMS) return NFD_E_BADCFG;
    if (n->dtype != NFD_DTYPE_FP32 && n->dtype != NFD_DTYPE_BF16) return NFD_E_BADCFG;
    if (!(n->eps >= 0.f) || !isfinite(n->eps)) return NFD_E_BADCFG;
    if (!aligned(n->weight, 16) || !aligned(n->bias, 16)) return NFD_E_ALIGN;
    N = {1, n->kind == NFD_NORM_LAYER, n->dtype == NFD_DTYPE_BF16, n->eps, n->weight, n->bias};
    return NFD_OK;
}
// n_rows rows of `width` numbers
int check_plain_rows(const void *p, long long stride, int width, int dtype) {
    if (!aligned(p, 16) || (stride * (long long)type_size(dtype)) % 16) return NFD_E_ALIGN;
    return stride < width || stride > (1LL << 40) ? NFD_E_RANGE : NFD_OK;
}

}  // namespace

extern "C" {

int nfd_rotate(const nfd_rope *rope, int flags, int dtype, int head_dim, int n_rows, const int *positions, int n_heads, const void *x,
               long long x_stride, void *x_out, long long x_out_stride, int n_heads2, const void *x2, long long x2_stride, void *x2_out,
               long long x2_out_stride, void *cuda_stream) {
    if (!rope) return NFD_E_NULLPTR;
    if (flags & ~(NFD_ROTATE_HALVES | NFD_ROTATE_BACK)) return NFD_E_BADCFG;
    if (dtype != NFD_DTYPE_FP32 && dtype != NFD_DTYPE_BF16) return NFD_E_BADCFG;
    if (head_dim < 16 || head_dim > ROTATE_MAX_DIM || head_dim % 16) return NFD_E_BADCFG;
    const int d[3] = {rope->rope_t, rope->rope_h, rope->rope_w};
    if (d[0] < 0 || d[1] < 0 || d[2] < 0 || d[0] % 2 || d[1] % 2 || d[2] % 2 || (long long)d[0] + d[1] + d[2] != head_dim) return NFD_E_BADCFG;
    if (!(rope->theta > 0.f) || !isfinite(rope->theta)) return NFD_E_BADCFG;
    if (n_rows < 0 || n_rows > NFD_MAX_TOKENS || n_heads < 0 || n_heads > 1024 || n_heads2 < 0 || n_heads2 > 1024) return NFD_E_RANGE;
    if (!aligned(positions, 4)) return NFD_E_ALIGN;
    RotateIO io = {{x, x2}, {x_out, x2_out}, {x_stride, x2_stride}, {x_out_stride, x2_out_stride}, {n_heads, n_heads2}, positions, n_rows};
    for (int i = 0; i < 2; ++i) {
        if (!io.heads[i]) continue;
        if (n_rows && (!io.in[i] || !io.out[i])) return NFD_E_NULLPTR;
        RET(check_plain_rows(io.in[i], io.in_stride[i], io.heads[i] * head_dim, dtype));
        RET(check_plain_rows(io.out[i], io.out_stride[i], io.heads[i] * head_dim, dtype));
        if (io.in[i] == io.out[i] && io.in_stride[i] != io.out_stride[i]) return NFD_E_BADCFG;
    }
    if (n_rows == 0 || n_heads + n_heads2 == 0) return NFD_OK;
    if (!positions) return NFD_E_NULLPTR;
    RotateD R;
    memset(&R, 0, sizeof(R));
    R.half_t = d[0] / 2, R.half_th = (d[0] + d[1]) / 2, R.dim = head_dim;
    // (theta^(-2 i / n) as a product of two powers, of i's multiple of eight and of the rest: two roundings more, and a quarter of the time)
    const double turn = 6.283185307179586476925286766559;
    for (int a = 0, pair = 0; a < 3; ++a) {
        double low[8];
        for (int i = 0; i < d[a] / 2; ++i) {
            if (i < 8) low[i] = pow((double)rope->theta, -2.0 * i / d[a]);
            if (i % 8 == 0) R.freq[pair + i] = (i ? pow((double)rope->theta, -2.0 * i / d[a]) : 1.0) / turn;
            else R.freq[pair + i] = R.freq[pair + i - i % 8] * low[i % 8];
        }
        pair += d[a] / 2;
    }
    int dev = 0, n_sm = 0;
    RET(this_device(dev, n_sm));
    const int rows = append_rows(n_rows, n_sm);
    const unsigned grid = (unsigned)((n_rows + rows - 1) / rows);
    const float sign = flags & NFD_ROTATE_BACK ? -1.0f : 1.0f;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == NFD_DTYPE_BF16) {
        if (flags & NFD_ROTATE_HALVES) k_rotate<bf16, true><<<grid, ROTATE_THREADS, 0, st>>>(R, io, rows, sign);
        else k_rotate<bf16, false><<<grid, ROTATE_THREADS, 0, st>>>(R, io, rows, sign);
    } else {
        if (flags & NFD_ROTATE_HALVES) k_rotate<float, true><<<grid, ROTATE_THREADS, 0, st>>>(R, io, rows, sign);
        else k_rotate<float, false><<<grid, ROTATE_THREADS, 0, st>>>(R, io, rows, sign);
    }
    CK(cudaGetLastError());
    return NFD_OK;
}

int nfd_gate_norm(int n_rows, int width, int x_dtype, const void *x, long long x_stride, int dtype, const void *y, long long y_stride,
                  void *x_out, long long x_out_stride, void *h, long long h_stride, const nfd_norm *post, const nfd_norm *pre,
                  const nfd_modulation *mod, float res_scale, void *cuda_stream) {
    if (x_dtype != NFD_DTYPE_FP32 && x_dtype != NFD_DTYPE_BF16) return NFD_E_BADCFG;
    if (dtype != NFD_DTYPE_FP32 && dtype != NFD_DTYPE_BF16) return NFD_E_BADCFG;
    if (n_rows < 0 || n_rows > NFD_MAX_TOKENS || width < 8 || width > NFD_MAX_WIDTH || width % 8) return NFD_E_RANGE;
    GateNormD N;
    memset(&N, 0, sizeof(N));
    RET(check_norm(y ? post : NULL, N.post));
    RET(check_norm(h ? pre : NULL, N.pre));
    if (h && !pre) return NFD_E_NULLPTR;
    N.n_rows = n_rows, N.width = width, N.res_scale = res_scale, N.n_mods = 1, N.rows_per_mod = NFD_MAX_TOKENS;
    if (mod) {
        if (mod->dtype != NFD_DTYPE_FP32 && mod->dtype != NFD_DTYPE_BF16) return NFD_E_BADCFG;
        if (mod->n_mods < 1 || (!mod->index && mod->rows_per_mod < 1)) return NFD_E_RANGE;
        // (a gate goes with y, scale and shift with h: without those they are not looked at)
        N.gate = y ? mod->gate : NULL, N.scale = h ? mod->scale : NULL, N.shift = h ? mod->shift : NULL;
        for (const void *p : {N.gate, N.scale, N.shift})
            if (p) RET(check_plain_rows(p, mod->stride, width, mod->dtype));
        if (!aligned(mod->index, 4)) return NFD_E_ALIGN;
        N.mod_stride = mod->stride, N.mod_bf = mod->dtype == NFD_DTYPE_BF16;
        N.index = mod->index, N.n_mods = mod->n_mods;
        if (!mod->index) N.rows_per_mod = mod->rows_per_mod;
    }
    if (n_rows == 0 || (!y && !h)) return NFD_OK;
    if (!x || (y && !x_out)) return NFD_E_NULLPTR;
    RET(check_plain_rows(x, x_stride, width, x_dtype));
    if (y) RET(check_plain_rows(y, y_stride, width, dtype));
    if (y) RET(check_plain_rows(x_out, x_out_stride, width, x_dtype));
    if (h) RET(check_plain_rows(h, h_stride, width, dtype));
    if ((y && x == x_out && x_stride != x_out_stride) || (y && y == h && y_stride != h_stride)) return NFD_E_BADCFG;
    N.x = x, N.x_stride = x_stride, N.y = y, N.y_stride = y_stride, N.x_out = x_out, N.x_out_stride = x_out_stride, N.h = h, N.h_stride = h_stride;
    int dev = 0, n_sm = 0;
    RET(this_device(dev, n_sm));
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (x_dtype == NFD_DTYPE_FP32)
        return dtype == NFD_DTYPE_FP32 ? launch_gate_norm<float, float>(N, dev, n_sm, st) : launch_gate_norm<float, bf16>(N, dev, n_sm, st);
    return dtype == NFD_DTYPE_FP32 ? launch_gate_norm<bf16, float>(N, dev, n_sm, st) : launch_gate_norm<bf16, bf16>(N, dev, n_sm, st);
}

}  // extern "C"
