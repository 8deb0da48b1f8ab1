// Rows into a paged cache, rotated and, where the pages hold 4 bits, quantised on the way; and back out of it.
//
// Bound by memory: every number of the new rows is read once and written once.  A CTA takes `rows` rows (one where that
// leaves SMs idle otherwise) with all their heads, so that the angles of a row (64-bit arithmetic, head_dim / 2 sines and
// cosines) are formed once for all of its heads, and each thread eight numbers of a head at a time: 16 bytes of bf16, four
// pairs of the rotation, a word of 4-bit codes; four neighbouring lanes hold a group of 32.  The first loads are issued
// before the row's sequence, its place and the angles are looked up.
#pragma once
#include "nfd_paged.cuh"

#define APPEND_THREADS 256
#define APPEND_MAX_ROWS 4

struct RopeD {
    int on, frame_tokens, grid_w;
    int half_t, half_th;                 // pairs that turn with the frame; with the frame or the row
    double freq[64];                     // of each pair
};
// Rows and their strides, in elements.
struct AppendIO {
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    void *q_out;
    int q_heads;
};

template <typename TS> __device__ __forceinline__ void load8(const TS *p, float *x);
template <> __device__ __forceinline__ void load8<float>(const float *p, float *x) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
template <> __device__ __forceinline__ void load8<bf16>(const bf16 *p, float *x) {
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
}
template <typename TS> __device__ __forceinline__ void store8(TS *p, const float *x);
template <> __device__ __forceinline__ void store8<float>(float *p, const float *x) {
    *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
template <> __device__ __forceinline__ void store8<bf16>(bf16 *p, const float *x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// The eight numbers of this lane to 4 bits, with the group's other three lanes: codes, and the group's word.
__device__ __forceinline__ uint32_t kv4_pack(const float *x, uint32_t &word) {
    float lo = 0.f, hi = 0.f;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) lo = fminf(lo, x[i]), hi = fmaxf(hi, x[i]), bad |= x[i] != x[i];
    if (bad) hi = INFINITY;
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    if (!(hi - lo < INFINITY)) {
        word = 0x7FC0u;
        return 0;
    }
    const float step = kv4_step(lo, hi), inv = __frcp_rn(step), z = kv4_round(-lo, step, inv);
    word = (__float_as_uint(step) >> 16) | (uint32_t)(int)z;
    uint32_t codes = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        codes |= (uint32_t)(int)fminf(fmaxf(kv4_round(x[i], step, inv) + z, 0.f), 15.f) << kv4_shift(i);
    return codes;
}

// TS: the rows' type; KV4: pages of 4 bits, otherwise of TS.
template <typename TS, bool KV4, int DH>
__global__ void __launch_bounds__(APPEND_THREADS) k_kv_append(const __grid_constant__ RopeD rope, const AppendIO io, const BatchD B,
                                                              const PagesD P, int rows) {
    constexpr int CPH = DH / 8;                                // chunks of eight numbers of a head
    constexpr int U = KV4 ? 2 : 4;                             // chunks of a thread in flight
    __shared__ float2 s_cs[APPEND_MAX_ROWS][DH / 2];
    __shared__ long long s_place[APPEND_MAX_ROWS];             // -1: none
    __shared__ int s_pos[APPEND_MAX_ROWS];                     // -1: dropped
    const int tid = threadIdx.x, warp = tid >> 5;
    const int r0 = blockIdx.x * rows, nr = min(rows, B.n_rows - r0);
    const int qc = io.q_heads * CPH, kc = P.heads * CPH, per_row = qc + 2 * kc, total = nr * per_row;
    float x[U][8];
    auto load = [&](int c, float *v) {
        const int r = c / per_row, j = c - r * per_row;
        const TS *p = j < qc ? (const TS *)io.q + (r0 + r) * io.q_stride + j * 8
                    : j < qc + kc ? (const TS *)io.k + (r0 + r) * io.k_stride + (j - qc) * 8
                                  : (const TS *)io.v + (r0 + r) * io.v_stride + (j - qc - kc) * 8;
        load8<TS>(p, v);
    };
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u * APPEND_THREADS + tid < total) load(u * APPEND_THREADS + tid, x[u]);
    if (warp < nr) {
        const int row = r0 + warp, s = B.seq_of(row);
        int pos = -1;
        long long place = -1;
        if (s < B.n_seqs) {
            const int2 sr = B.rows(s);
            const int i = row - sr.x, len = B.tokens(s), p = len - sr.y + i;
            if (i >= 0 && i < min(sr.y, B.max_rows) && p >= 0) {
                pos = p;
                if (p >= P.oldest(B, len)) place = P.place(B, s, p);
            }
        }
        if ((tid & 31) == 0) s_pos[warp] = pos, s_place[warp] = place;
    }
    __syncthreads();
    if (rope.on) {
        for (int i = tid; i < nr * (DH / 2); i += APPEND_THREADS) {
            const int r = i / (DH / 2), pair = i - r * (DH / 2), pos = max(s_pos[r], 0);
            const int f = pos / rope.frame_tokens, in = pos - f * rope.frame_tokens, gr = in / rope.grid_w;
            const int at = pair < rope.half_t ? f : pair < rope.half_th ? gr : in - gr * rope.grid_w;
            double sn, cs;
            sincos((double)at * rope.freq[pair], &sn, &cs);
            s_cs[r][pair] = make_float2((float)cs, (float)sn);
        }
        __syncthreads();
    }
    for (int c0 = 0; c0 < total; c0 += U * APPEND_THREADS) {
        if (c0) {
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c0 + u * APPEND_THREADS + tid < total) load(c0 + u * APPEND_THREADS + tid, x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * APPEND_THREADS + tid;
            if (c0 + u * APPEND_THREADS >= total) break;       // (the same for all threads)
            const bool here = c < total;                       // (a multiple of four: the lanes of a group agree)
            const int r = here ? c / per_row : 0, j = here ? c - r * per_row : 0;
            const bool is_q = j < qc, is_k = !is_q && j < qc + kc;
            if (rope.on && (is_q || is_k)) {
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float2 cs = s_cs[r][(j % CPH) * 4 + e / 2];
                    const float a = x[u][e], b = x[u][e + 1];
                    // (every rounding spelled out: a number next to a border of the 4-bit codes falls on the same side in
                    // every instance of the kernel)
                    x[u][e] = __fsub_rn(__fmul_rn(a, cs.x), __fmul_rn(b, cs.y));
                    x[u][e + 1] = __fadd_rn(__fmul_rn(b, cs.x), __fmul_rn(a, cs.y));
                }
            }
            uint32_t word = 0, codes = 0;
            if (KV4) codes = kv4_pack(x[u], word);
            if (!here || s_pos[r] < 0) continue;
            if (is_q) {
                store8<TS>((TS *)io.q_out + ((long long)(r0 + r) * qc + j) * 8, x[u]);
                continue;
            }
            if (s_place[r] < 0) continue;
            const int jj = is_k ? j - qc : j - qc - kc, h = jj / CPH, d = jj - h * CPH;
            const size_t at = (size_t)(s_place[r] + (long long)h * P.page_tokens);
            if (KV4) {
                reinterpret_cast<uint32_t *>(is_k ? P.k : P.v)[at * CPH + d] = codes;
                if (!(d & 3)) (is_k ? P.k_scale : P.v_scale)[at * (DH / 32) + d / 4] = (uint16_t)word;
            } else {
                store8<TS>((TS *)(is_k ? P.k : P.v) + at * DH + d * 8, x[u]);
            }
        }
    }
}

// TP: type of the pages (KV4: 4 bits), TO: of the result.
template <typename TP, typename TO, bool KV4, int DH>
__global__ void __launch_bounds__(256) k_pages_read(const BatchD B, const PagesD P, TO *k_out, TO *v_out) {
    constexpr int CPH = DH / 8;
    const int row = blockIdx.x, s = B.seq_of(row);
    if (s >= B.n_seqs) return;
    const int2 sr = B.rows(s);
    const int i = row - sr.x, len = B.tokens(s), p = len - sr.y + i;
    if (i < 0 || i >= min(sr.y, B.max_rows) || p < P.oldest(B, len)) return;
    const long long place = P.place(B, s, p);
    if (place < 0) return;
    const int per = P.heads * CPH;
    for (int c = threadIdx.x; c < 2 * per; c += blockDim.x) {
        const bool is_k = c < per;
        TO *out = is_k ? k_out : v_out;
        if (!out) continue;
        const int j = is_k ? c : c - per, h = j / CPH, d = j - h * CPH;
        const size_t at = (size_t)(place + (long long)h * P.page_tokens);
        float x[8];
        if (KV4)
            kv4_unpack(reinterpret_cast<const uint32_t *>(is_k ? P.k : P.v)[at * CPH + d],
                       (is_k ? P.k_scale : P.v_scale)[at * (DH / 32) + d / 4], x);
        else
            load8<TP>((const TP *)(is_k ? P.k : P.v) + at * DH + d * 8, x);
        store8<TO>(out + ((size_t)row * per + j) * 8, x);
    }
}
