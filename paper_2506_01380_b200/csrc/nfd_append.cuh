// Rows into a paged cache, rotated and, where the pages hold 4 bits, quantised on the way; and back out of it.
//
// Every number of the new rows is read once and written once; what bounds it is latency, not a rate (figures below).  A CTA takes `rows` rows (one
// where that leaves SMs idle otherwise) with all their heads, so that the angles of a row (64-bit arithmetic, head_dim / 2 sines and
// cosines) are formed once for all of its heads.  A thread has a place in the rows, eight numbers of a head (16 bytes of bf16, four
// pairs of the rotation, a word of 4-bit codes; four neighbouring lanes hold a group of 32), and takes it in one row after the other: what
// depends on the place is worked out once.  The first loads are issued before the rows' sequences, places and angles are looked up.
// Measured, 16 heads x 64 with q: 336 rows into bf16 pages 4.3 us, eight single rows 3.7 (a launch that does nothing takes 2.5).  10752 rows, in and back
// out: fp32 pages 51 us (5.1 TB/s) and 33 (5.3), bf16 36 (3.7) and 24 (3.7), bf16 rows in 4-bit pages 40 (2.5) and 14 (4.0), fp32 rows in them 45 (4.2)
// and 29 (3.5).  Under the profiler both kernels of 4-bit pages issue in 62 % of the clocks and their warps wait for loads and for shared memory as long; the
// append has 40 % of an SM's warps, 64 registers a thread (with bf16 rows it spills 8 bytes of them).
#pragma once
#include "nfd_paged.cuh"

#define APPEND_THREADS 256
#define APPEND_MAX_ROWS 8

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
__device__ __forceinline__ uint32_t kv4_pack(const float *x, uint32_t &word, uint32_t group) {
    float lo = 0.f, hi = 0.f, zero = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) lo = fminf(lo, x[i]), hi = fmaxf(hi, x[i]), zero = fmaf(x[i], 0.f, zero);
    if (zero != 0.f) hi = INFINITY;                            // NaN: one of them is not finite
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(group, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(group, hi, o));
    }
    const float range = kv4_range(lo, hi);
    if (!(range < INFINITY)) {
        word = 0x7FC0u;
        return 0;
    }
    const float step = kv4_step(range), inv = __frcp_rn(step);
    const int z = __float_as_int(kv4_quotient(-lo, step, inv)) - __float_as_int(KV4_MAGIC), up = z - __float_as_int(KV4_MAGIC);
    word = (__float_as_uint(step) >> 16) | (uint32_t)z;
    uint32_t codes = 0;
    // (no code is below 0: x >= lo, and rounding is symmetric; the largest may be 16, where lo and hi are both rounded away from 0)
#pragma unroll
    for (int i = 0; i < 8; ++i) codes += (uint32_t)min(__float_as_int(kv4_quotient(x[i], step, inv)) + up, 15) << kv4_shift(i);
    return codes;
}

// The rows of a CTA, a warp to each: token (-1: none, or one that is dropped) and place in the pages (-1: none).
__device__ __forceinline__ void rows_look_up(const BatchD &B, const PagesD &P, int r0, int nr, int *pos, long long *place) {
    for (int r = threadIdx.x >> 5; r < nr; r += APPEND_THREADS / 32) {
        const int s = B.seq_of(r0 + r);
        int p = -1;
        long long at = -1;
        if (s < B.n_seqs) {
            const int2 sr = B.rows(s);
            const int i = r0 + r - sr.x, len = B.tokens(s);
            if (i >= 0 && i < min(sr.y, B.max_rows)) p = max(len - sr.y + i, -1);
            if (p >= 0 && p >= P.oldest(B, len)) at = P.place(B, s, p);
        }
        if ((threadIdx.x & 31) == 0) pos[r] = p, place[r] = at;
    }
}

// TS: the rows' type; KV4: pages of 4 bits, otherwise of TS.
template <typename TS, bool KV4, int DH>
__global__ void __launch_bounds__(APPEND_THREADS, KV4 ? 4 : 1) k_kv_append(const __grid_constant__ RopeD rope, const AppendIO io, const BatchD B,
                                                              const PagesD P, int rows) {
    constexpr int CPH = DH / 8, U = 4;                         // chunks of eight numbers of a head; rows in flight
    __shared__ float2 s_cs[APPEND_MAX_ROWS][DH / 2];
    __shared__ long long s_place[APPEND_MAX_ROWS];
    __shared__ int s_pos[APPEND_MAX_ROWS];
    const int tid = threadIdx.x, r0 = blockIdx.x * rows, nr = min(rows, B.n_rows - r0);
    const int qc = io.q_heads * CPH, kc = P.heads * CPH, per_row = qc + 2 * kc;
    // a thread's place: chunk j of q, k and v side by side, and its numbers in row r0
    struct Place {
        const TS *src;
        long long stride;
        bool is_q, is_k;
    };
    auto at = [&](int j) -> Place {
        Place p;
        p.is_q = j < qc, p.is_k = !p.is_q && j < qc + kc;
        p.stride = p.is_q ? io.q_stride : p.is_k ? io.k_stride : io.v_stride;
        p.src = (p.is_q ? (const TS *)io.q + j * 8 : p.is_k ? (const TS *)io.k + (j - qc) * 8 : (const TS *)io.v + (j - qc - kc) * 8) + r0 * p.stride;
        return p;
    };
    float x[U][8];
    auto load = [&](const Place &p, int r) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r + u < nr) load8<TS>(p.src + (r + u) * p.stride, x[u]);
    };
    int j = tid;
    Place pl = at(j);
    if (j < per_row) load(pl, 0);
    rows_look_up(B, P, r0, nr, s_pos, s_place);
    __syncthreads();
    if (rope.on) {
        for (int i = tid; i < nr * (DH / 2); i += APPEND_THREADS) {
            const int r = i / (DH / 2), pair = i - r * (DH / 2), pos = max(s_pos[r], 0);
            const int f = pos / rope.frame_tokens, in = pos - f * rope.frame_tokens, gr = in / rope.grid_w;
            const int a = pair < rope.half_t ? f : pair < rope.half_th ? gr : in - gr * rope.grid_w;
            double sn, cs;
            sincos((double)a * rope.freq[pair], &sn, &cs);
            s_cs[r][pair] = make_float2((float)cs, (float)sn);
        }
        __syncthreads();
    }
    for (; j < per_row; j += APPEND_THREADS) {                 // (a multiple of four: the lanes of a group agree)
        if (j != tid) pl = at(j), load(pl, 0);
        const bool turn = rope.on && (pl.is_q || pl.is_k);
        const int jj = pl.is_q ? j : pl.is_k ? j - qc : j - qc - kc, h = jj / CPH, d = jj - h * CPH;
        const long long head = (long long)h * P.page_tokens;
        const uint32_t group = 0xFu << (tid & 28);             // the lanes that hold this group of 32
        for (int rb = 0; rb < nr; rb += U) {
            if (rb) load(pl, rb);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int r = rb + u;
                if (r >= nr) break;                            // (the same for all threads)
                if (s_pos[r] < 0) continue;                    // (and this)
                if (turn) {
#pragma unroll
                    for (int e = 0; e < 8; e += 4) {
                        const float4 cs = *reinterpret_cast<const float4 *>(&s_cs[r][d * 4 + e / 2]);
                        const float a0 = x[u][e], a1 = x[u][e + 1], b0 = x[u][e + 2], b1 = x[u][e + 3];
                        // (every rounding spelled out: a number next to a border of the 4-bit codes falls on the same side in
                        // every instance of the kernel)
                        x[u][e] = __fsub_rn(__fmul_rn(a0, cs.x), __fmul_rn(a1, cs.y));
                        x[u][e + 1] = __fadd_rn(__fmul_rn(a1, cs.x), __fmul_rn(a0, cs.y));
                        x[u][e + 2] = __fsub_rn(__fmul_rn(b0, cs.z), __fmul_rn(b1, cs.w));
                        x[u][e + 3] = __fadd_rn(__fmul_rn(b1, cs.z), __fmul_rn(b0, cs.w));
                    }
                }
                if (pl.is_q) {
                    store8<TS>((TS *)io.q_out + ((long long)(r0 + r) * qc + j) * 8, x[u]);
                    continue;
                }
                if (s_place[r] < 0) continue;
                const size_t to = (size_t)(s_place[r] + head);
                if (KV4) {
                    uint32_t word;
                    const uint32_t codes = kv4_pack(x[u], word, group);
                    reinterpret_cast<uint32_t *>(pl.is_k ? P.k : P.v)[to * CPH + d] = codes;
                    if (!(d & 3)) (pl.is_k ? P.k_scale : P.v_scale)[to * (DH / 32) + d / 4] = (uint16_t)word;
                } else {
                    store8<TS>((TS *)(pl.is_k ? P.k : P.v) + to * DH + d * 8, x[u]);
                }
            }
        }
    }
}

// TP: type of the pages (KV4: 4 bits), TO: of the result.  Rows and threads as above.
template <typename TP, typename TO, bool KV4, int DH>
__global__ void __launch_bounds__(APPEND_THREADS) k_pages_read(const BatchD B, const PagesD P, TO *k_out, TO *v_out, int rows) {
    constexpr int CPH = DH / 8, U = 4;
    __shared__ long long s_place[APPEND_MAX_ROWS];
    __shared__ int s_pos[APPEND_MAX_ROWS];
    const int r0 = blockIdx.x * rows, nr = min(rows, B.n_rows - r0), per = P.heads * CPH;
    rows_look_up(B, P, r0, nr, s_pos, s_place);
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * per; c += APPEND_THREADS) {
        const bool is_k = c < per;
        TO *out = is_k ? k_out : v_out;
        if (!out) continue;
        const int j = is_k ? c : c - per, h = j / CPH, d = j - h * CPH;
        const long long head = (long long)h * P.page_tokens;
        const void *src = is_k ? P.k : P.v;
        const uint16_t *words = is_k ? P.k_scale : P.v_scale;
        out += (size_t)r0 * per * 8 + j * 8;
        for (int rb = 0; rb < nr; rb += U) {
            uint32_t codes[U], word[U];
            float x[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (rb + u >= nr || s_place[rb + u] < 0) continue;
                const size_t at = (size_t)(s_place[rb + u] + head);
                if (KV4) codes[u] = reinterpret_cast<const uint32_t *>(src)[at * CPH + d], word[u] = words[at * (DH / 32) + d / 4];
                else load8<TP>((const TP *)src + at * DH + d * 8, x[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (rb + u >= nr || s_place[rb + u] < 0) continue;
                TO *to = out + (size_t)(rb + u) * per * 8;
                if constexpr (KV4) {
                    uint32_t b[4];                             // bf16 numbers, exactly
#pragma unroll
                    for (int i = 0; i < 4; ++i) b[i] = kv4_pair(codes[u], i, kv4_z2(word[u], word[u]), kv4_step2(word[u], word[u]));
                    if constexpr (sizeof(TO) == 2) {
                        *reinterpret_cast<uint4 *>(to) = make_uint4(b[0], b[1], b[2], b[3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[u][2 * i] = __uint_as_float(b[i] << 16), x[u][2 * i + 1] = __uint_as_float(b[i] & 0xffff0000u);
                        store8<TO>(to, x[u]);
                    }
                } else {
                    store8<TO>(to, x[u]);
                }
            }
        }
    }
}
