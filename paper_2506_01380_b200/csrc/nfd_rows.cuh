// Rows on their way from one projection of a block to the next: rotary embedding with a position on several axes, and the norms around a block with
// its gate and residual scale.  Both read and write every number once; what bounds them is memory, or for few rows the launch and a chain of loads.
#pragma once
#include "nfd_append.cuh"

// ---- rotation -----------------------------------------------------------------------------------------------
#define ROTATE_THREADS 256
#define ROTATE_MAX_ROWS 8
#define ROTATE_MAX_DIM 256

struct RotateD {
    int half_t, half_th, dim;            // pairs that turn with the first axis; with the first or the second; numbers of a head
    double freq[ROTATE_MAX_DIM / 2];     // of each pair, in turns
};
struct RotateIO {
    const void *in[2];
    void *out[2];
    long long in_stride[2], out_stride[2];
    int heads[2];
    const int *pos;
    int n_rows;
};
// A CTA takes `rows` rows: sine and cosine of their pairs once for all heads (the angle, in turns, is formed and reduced in 64 bits, so that far
// positions keep their fraction; sine and cosine of what is left are fp32), then eight pairs to a thread: 16 numbers in a row, or eight of either half of a head.
template <typename TS, bool HALVES>
__global__ void __launch_bounds__(ROTATE_THREADS) k_rotate(const __grid_constant__ RotateD R, const RotateIO io, int rows, float sign) {
    constexpr int U = 4;                                       // rows in flight
    __shared__ float2 s_cs[ROTATE_MAX_ROWS * (ROTATE_MAX_DIM / 2)];
    const int tid = threadIdx.x, r0 = blockIdx.x * rows, nr = min(rows, io.n_rows - r0), pairs = R.dim / 2, per_head = R.dim / 16;
    const int n0 = io.heads[0] * per_head, n = n0 + io.heads[1] * per_head;
    for (int i = tid; i < nr * pairs; i += ROTATE_THREADS) {
        const int r = i / pairs, pair = i - r * pairs, axis = pair < R.half_t ? 0 : pair < R.half_th ? 1 : 2;
        const double turns = (double)__ldg(io.pos + 3LL * (r0 + r) + axis) * R.freq[pair];
        float sn, cs;
        sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
        s_cs[i] = make_float2(cs, sign * sn);
    }
    __syncthreads();
    for (int j = tid; j < n; j += ROTATE_THREADS) {
        const int w = j >= n0, jj = w ? j - n0 : j, h = jj / per_head, d = jj - h * per_head;
        const int first = h * R.dim + (HALVES ? 8 * d : 16 * d), second = first + (HALVES ? pairs : 8);
        const TS *in = (const TS *)io.in[w] + r0 * io.in_stride[w];
        TS *out = (TS *)io.out[w] + r0 * io.out_stride[w];
        for (int rb = 0; rb < nr; rb += U) {
            float a[U][8], b[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (rb + u < nr) load8<TS>(in + (rb + u) * io.in_stride[w] + first, a[u]), load8<TS>(in + (rb + u) * io.in_stride[w] + second, b[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (rb + u >= nr) break;
                const float4 *cs = reinterpret_cast<const float4 *>(s_cs + (rb + u) * pairs + 8 * d);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float4 c = cs[e];
                    auto turn = [](float &x, float &y, float co, float si) {
                        const float t = x * co - y * si;
                        y = y * co + x * si, x = t;
                    };
                    if (HALVES) {
                        turn(a[u][2 * e], b[u][2 * e], c.x, c.y), turn(a[u][2 * e + 1], b[u][2 * e + 1], c.z, c.w);
                    } else {
                        float *x = e < 2 ? a[u] + 4 * e : b[u] + 4 * (e - 2);
                        turn(x[0], x[1], c.x, c.y), turn(x[2], x[3], c.z, c.w);
                    }
                }
                store8<TS>(out + (rb + u) * io.out_stride[w] + first, a[u]), store8<TS>(out + (rb + u) * io.out_stride[w] + second, b[u]);
            }
        }
    }
}

// ---- norms around a block -----------------------------------------------------------------------------------
struct NormD {
    int on, layer, bf;                   // layer: LayerNorm, otherwise RMSNorm; bf: weight and bias are bf16, otherwise fp32
    float eps;
    const void *weight, *bias;
};
struct GateNormD {
    const void *x, *y, *gate, *scale, *shift;
    void *x_out, *h;
    long long x_stride, y_stride, x_out_stride, h_stride, mod_stride;
    const int *index;
    int n_rows, width, n_mods, rows_per_mod, mod_bf;
    float res_scale;
    NormD post, pre;
};
// eight parameters
__device__ __forceinline__ void load8_par(const void *p, int bf, long long at, float *x) {
    if (bf) load8<bf16>((const bf16 *)p + at, x);
    else load8<float>((const float *)p + at, x);
}
// Sum over the threads of a row (T of them: a warp, or a CTA).
template <int T> __device__ __forceinline__ float row_sum(float x, float *shared, int &turn) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    if constexpr (T > 32) {
        float *s = shared + (turn ^= 1) * (T / 32);            // (who writes one half again has been through the barrier of the other)
        if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
        __syncthreads();
        x = s[threadIdx.x & (T / 32 - 1)];
#pragma unroll
        for (int d = T / 64; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    }
    return x;
}
// t = post(y), x' = x + res_scale gate t, h = pre(x') (1 + scale) + shift, statistics in fp32 over numbers that stay in registers: the mean first, then
// the squares of what is left.  T threads to a row, V pieces of eight numbers to a thread.
template <typename TX, typename TY, int T, int V>
__global__ void __launch_bounds__(T == 32 ? 256 : T) k_gate_norm(const __grid_constant__ GateNormD N) {
    constexpr int RPC = T == 32 ? 8 : 1;                       // rows of a CTA
    __shared__ float shared[2 * (T / 32)];
    const int t = threadIdx.x % T, row = blockIdx.x * RPC + threadIdx.x / T, pieces = N.width / 8;
    if (row >= N.n_rows) return;                               // (whole warps; a CTA of T > 32 has one row)
    int turn = 0;
    float x[V][8], y[V][8];
    const TX *px = (const TX *)N.x + row * N.x_stride;
    const TY *py = (const TY *)N.y + row * N.y_stride;
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = y[i][e] = 0.f;
        if (i * T + t < pieces) {
            load8<TX>(px + (i * T + t) * 8, x[i]);
            if (N.y) load8<TY>(py + (i * T + t) * 8, y[i]);
        }
    }
    const int m = min(max(N.index ? __ldg(N.index + row) : row / N.rows_per_mod, 0), N.n_mods - 1);
    const long long mod = m * N.mod_stride;
    const float per = 1.0f / (float)N.width;
    // numbers to what they are off the mean, and the factor that makes their mean square 1
    auto stats = [&](float (&v)[V][8], const NormD &n) -> float {
        if (n.layer) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += v[i][e];
            const float mean = row_sum<T>(sum, shared, turn) * per;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i * T + t < pieces)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[i][e] -= mean;
        }
        float sq = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(v[i][e], v[i][e], sq);
        return rsqrtf(row_sum<T>(sq, shared, turn) * per + n.eps);
    };
    auto affine = [&](float *v, const NormD &n, int at, float f) {
        float w[8];
        if (n.weight) load8_par(n.weight, n.bf, at, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= n.weight ? f * w[e] : f;
        if (n.bias) {
            load8_par(n.bias, n.bf, at, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += w[e];
        }
    };
    if (N.y) {
        float f = 1.f;
        if (N.post.on) f = stats(y, N.post);
        TX *po = (TX *)N.x_out + row * N.x_out_stride;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int at = (i * T + t) * 8;
            if (i * T + t >= pieces) continue;
            if (N.post.on) affine(y[i], N.post, at, f);
            float g[8];
            if (N.gate) load8_par(N.gate, N.mod_bf, mod + at, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = fmaf(N.gate ? N.res_scale * g[e] : N.res_scale, y[i][e], x[i][e]);
            store8<TX>(po + at, x[i]);
        }
    }
    if (!N.h) return;
    const float f = stats(x, N.pre);
    TY *ph = (TY *)N.h + row * N.h_stride;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int at = (i * T + t) * 8;
        if (i * T + t >= pieces) continue;
        affine(x[i], N.pre, at, f);
        float w[8];
        if (N.scale) {
            load8_par(N.scale, N.mod_bf, mod + at, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = fmaf(x[i][e], w[e], x[i][e]);
        }
        if (N.shift) {
            load8_par(N.shift, N.mod_bf, mod + at, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] += w[e];
        }
        store8<TY>(ph + at, x[i]);
    }
}
template <typename TX, typename TY, int T, int V> static int launch_gate_norm_as(const GateNormD &N, cudaStream_t st) {
    constexpr int RPC = T == 32 ? 8 : 1;
    k_gate_norm<TX, TY, T, V><<<(unsigned)((N.n_rows + RPC - 1) / RPC), T == 32 ? 256 : T, 0, st>>>(N);
    return cudaGetLastError() == cudaSuccess ? NFD_OK : NFD_E_CUDA;
}
template <typename TX, typename TY> static int launch_gate_norm(const GateNormD &N, int n_sm, cudaStream_t st) {
    const int pieces = N.width / 8;
    if (pieces <= 128 && (pieces <= 32 || N.n_rows >= 16 * n_sm)) {
        if (pieces <= 32) return launch_gate_norm_as<TX, TY, 32, 1>(N, st);
        if (pieces <= 64) return launch_gate_norm_as<TX, TY, 32, 2>(N, st);
        return launch_gate_norm_as<TX, TY, 32, 4>(N, st);
    }
    if (pieces <= 128) return launch_gate_norm_as<TX, TY, 128, 1>(N, st);
    if (pieces <= 256) return launch_gate_norm_as<TX, TY, 128, 2>(N, st);
    if (pieces <= 512) return launch_gate_norm_as<TX, TY, 128, 4>(N, st);
    if (pieces <= 1024) return launch_gate_norm_as<TX, TY, 512, 2>(N, st);
    return launch_gate_norm_as<TX, TY, 512, 4>(N, st);
}
