// Attention of a batch's rows to fp32 keys, on the fp32 pipes: an encoder's states, pages, the rows of packed prompts.
//
// k_attn_f32: a CTA takes 32 or 64 rows (rows x heads that share a head of keys) of a sequence and walks its keys in tiles of 64, the next tile's copies in
// flight: S = Q K^T with 4 rows x 4 keys to a thread, an online softmax per row over the 16 lanes that hold it, P through shared memory
// (a row's 16 lanes write and read it, no barrier), O += P V with 4 rows x DH / 16 dims to a thread.  All operands are read as 16-byte words
// along their rows, rows are padded by one word so that no two lanes of a quarter warp meet in a bank.  Keys that are not seen are copied as zeros and take a score of -inf.
// Probabilities are scaled down by a power of two (sum_bits), which no result shows but those whose sums would have left fp32.
// Few units with many keys are split over the CTAs of a cluster and merged through distributed shared memory.
// For many rows at 46 % of the FMA pipes' rate (eight 16-byte words from shared memory for 64 FMAs either way; what else holds it has not been taken
// apart), for few bound by the chain of a tile (copy, S, softmax, P V), and so k_attn_f32_few takes them.  Measured: four sequences of 1344
// rows, 16 heads x 64, against 1000 states 667 us (33 TFLOP/s of 72); three of 77 rows, 6 heads x 32, against up to 220, 7.0 us.
#pragma once
#include "nfd_attn_few.cuh"

#define F32_KEYS 64

// Keys, and the power of two by which probabilities are scaled: exact, one bit for the roundings of the sums.
template <int DH> struct F32States : StateKeys<float, DH> {
    static constexpr bool RANGES = false;                               // all rows see the same keys
    int most;                                                           // keys of a row
    float scale;
    explicit F32States(const StateKeys<float, DH> &k) : StateKeys<float, DH>(k), most(k.n_keys), scale(ldexpf(1.0f, -sum_bits(1, k.n_keys))) {}
};
// Pages, or the rows of packed prompts: under a mask, and what a row does not see may be anything, so that in tiles that not all rows see a product
// with a value is left out where the row does not see it.
template <typename Keys, int DH> struct F32Rows : Keys {
    static constexpr bool RANGES = true;
    int most;
    float scale;
    F32Rows(const Keys &k, long long keys) : Keys(k), most((int)keys), scale(ldexpf(1.0f, -sum_bits(1, (int)keys))) {}
};

template <int DH, int ROWS> struct F32Cfg {
    static constexpr int THREADS = 4 * ROWS;
    static constexpr int LD = DH + 4, LP = F32_KEYS + 4;                // floats of a padded row
    static constexpr int AT_K = ROWS * LD, AT_V = AT_K + 2 * F32_KEYS * LD, AT_P = AT_V + 2 * F32_KEYS * LD,
                         AT_M = AT_P + ROWS * LP, FLOATS = AT_M + 2 * F32_KEYS;
    static constexpr int SMEM = FLOATS * 4;
    static_assert(ROWS * (DH + 2) <= AT_K + F32_KEYS * LD, "a CTA's state lies over Q and K");
};

template <typename Src, int DH, int ROWS>
__global__ void __launch_bounds__(4 * ROWS) k_attn_f32(const BatchD B, const AttnRows A, const Src K, int split) {
    using C = F32Cfg<DH, ROWS>;
    constexpr int LD = C::LD, LP = C::LP, ND = DH / 16, W = DH / 4;
    extern __shared__ __align__(16) float f32_smem[];
    float *sQ = f32_smem, *sP = f32_smem + C::AT_P;
    uint32_t *sM = reinterpret_cast<uint32_t *>(f32_smem + C::AT_M);    // keys that are there, of two tiles
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int rank = blockIdx.x % split, h = blockIdx.x / split, s = blockIdx.y, r0 = blockIdx.z * ROWS;
    const int2 sr = B.rows(s);
    const int rows = min(sr.y, B.max_rows) * A.share;
    if (r0 >= rows) return;                                             // (the whole cluster)
    const int nr = min(ROWS, rows - r0);
    // keys lo .. hi - 1; of which those below edge_lo and from edge_hi on are not seen by all rows
    int lo = 0, hi = 0, edge_lo = 0, edge_hi = INT_MAX;
    const int len = K.length(B, s);
    KeyRange kr[4];                                                     // what rows 4 ty + i see
    if constexpr (Src::RANGES) {
        const KeyRange first = K.range(B, len, sr.y, A.split(r0).x), last = K.range(B, len, sr.y, A.split(r0 + nr - 1).x);
        lo = first.lo, hi = last.hi, edge_lo = last.lo, edge_hi = first.hi;
#pragma unroll
        for (int i = 0; i < 4; ++i) kr[i] = K.range(B, len, sr.y, A.split(r0 + min(4 * ty + i, nr - 1)).x);
    } else {
        hi = len;
    }
    const int tiles = max(0, (hi - lo + F32_KEYS - 1) / F32_KEYS), per = (tiles + split - 1) / split;
    const int t0 = min(tiles, rank * per), t1 = min(tiles, t0 + per);
    // G threads to a key, a share of its row each
    constexpr int G = C::THREADS / F32_KEYS, PART = DH / G;
    const int key = tid / G, part = tid % G;
    long long seq = 0;                                                  // of states: where the sequence's begin, and what the mask says
    const unsigned char *mask = nullptr;
    if constexpr (!Src::RANGES) {
        seq = s * K.seq_stride + h * K.head_stride;
        mask = K.mask ? K.mask + (size_t)s * K.n_keys : nullptr;
    }
    auto cursor = [&]() {
        if constexpr (Src::RANGES) return K.cursor(B, s, sr.x, lo + t0 * F32_KEYS + key, F32_KEYS);
        else return 0;
    }();
    auto fill = [&](int t) {                                            // (t0, t0 + 1, ...)
        const int b = t & 1, p = lo + t * F32_KEYS + key;
        bool here = p < hi;
        const float *k = K.first_k(), *v = K.first_v();
        if constexpr (Src::RANGES) {
            const long long row = K.next(cursor, B, h, here);
            here = row >= 0;
            k = K.k_row(here ? row : 0, h) + part * PART, v = K.v_row(here ? row : 0, h) + part * PART;
        } else {
            here = here && (!mask || mask[p]);
            const long long at = here ? seq + p * K.key_stride + part * PART : 0;
            k += at, v += at;
        }
        const uint32_t dk = smem_u32(f32_smem + C::AT_K + (b * F32_KEYS + key) * LD + part * PART);
        const uint32_t dv = smem_u32(f32_smem + C::AT_V + (b * F32_KEYS + key) * LD + part * PART);
#pragma unroll
        for (int i = 0; i < PART / 4; ++i) {
            cp_async16(dk + 16 * i, k + (here ? 4 * i : 0), here ? 16 : 0);
            cp_async16(dv + 16 * i, v + (here ? 4 * i : 0), here ? 16 : 0);
        }
        cp_async_commit();
        if (part == 0) sM[64 * b + key] = here;
    };
    for (int i = tid; i < ROWS * W; i += C::THREADS) {
        const int r = i / W, w = i % W;
        const int2 at = A.split(r0 + min(r, nr - 1));
        cp_async16(smem_u32(sQ + r * LD + 4 * w), (const float *)A.q + (long long)(sr.x + at.x) * A.q_stride + (h * A.share + at.y) * DH + 4 * w, 16);
    }
    cp_async_commit();
    if (t0 < t1) fill(t0);
    const float cs = 1.4426950408889634f * (1.0f / sqrtf((float)DH));
    float o[4][ND], m[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY, l[i] = 0.f;
#pragma unroll
        for (int e = 0; e < ND; ++e) o[i][e] = 0.f;
    }
    for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) {
            fill(t + 1);
            cp_async_wait<1>();
        } else {
            cp_async_wait<0>();
        }
        __syncthreads();
        const float *kt = f32_smem + C::AT_K + (t & 1) * F32_KEYS * LD, *vt = f32_smem + C::AT_V + (t & 1) * F32_KEYS * LD;
        // S: rows 4 ty + i, keys tx + 16 j
        float2 xx[4][4];                                                // sums over even and odd dims
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) xx[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int w = 0; w < W; ++w) {
            float4 q[4], k[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const float4 *>(sQ + (4 * ty + i) * LD + 4 * w);
#pragma unroll
            for (int j = 0; j < 4; ++j) k[j] = *reinterpret_cast<const float4 *>(kt + (tx + 16 * j) * LD + 4 * w);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    xx[i][j] = ffma2(make_float2(q[i].x, q[i].y), make_float2(k[j].x, k[j].y),
                                     ffma2(make_float2(q[i].z, q[i].w), make_float2(k[j].z, k[j].w), xx[i][j]));
        }
        float x[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i][j] = xx[i][j].x + xx[i][j].y;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (!sM[64 * (t & 1) + tx + 16 * j])
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i][j] = -INFINITY;
        const int p0 = lo + t * F32_KEYS;
        const bool edge = Src::RANGES && (p0 < edge_lo || p0 + F32_KEYS > edge_hi);
        if constexpr (Src::RANGES) {
            if (edge)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int p = p0 + tx + 16 * j;
                        if (p < kr[i].lo || p >= kr[i].hi) x[i][j] = -INFINITY;
                    }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mn = fmaxf(fmaxf(x[i][0], x[i][1]), fmaxf(x[i][2], x[i][3]));
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, d));
            mn = fmaxf(mn, m[i]);
            const float f = mn == m[i] ? 1.0f : exp2f((m[i] - mn) * cs), mc = mn == -INFINITY ? 0.f : mn;
            m[i] = mn, l[i] *= f;
#pragma unroll
            for (int e = 0; e < ND; ++e) o[i][e] *= f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = exp2f((x[i][j] - mc) * cs) * K.scale;
                l[i] += p, sP[(4 * ty + i) * LP + tx + 16 * j] = p;
            }
        }
        __syncwarp();
        // O: rows 4 ty + i, dims: words of up to four, tx-th of every 16 of them
        auto sum = [&](auto masked) {
#pragma unroll 4
            for (int k = 0; k < F32_KEYS; k += 4) {
                float4 p[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = *reinterpret_cast<const float4 *>(sP + (4 * ty + i) * LP + k);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    float v[ND];
                    if constexpr (DH == 32) {
                        const float2 a = *reinterpret_cast<const float2 *>(vt + (k + u) * LD + 2 * tx);
                        v[0] = a.x, v[1] = a.y;
                    } else {
#pragma unroll
                        for (int e = 0; e < ND; e += 4) {
                            const float4 a = *reinterpret_cast<const float4 *>(vt + (k + u) * LD + 16 * e + 4 * tx);
                            v[e] = a.x, v[e + 1] = a.y, v[e + 2] = a.z, v[e + 3] = a.w;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if constexpr (decltype(masked)::value) {
                            if (p0 + k + u < kr[i].lo || p0 + k + u >= kr[i].hi) continue;
                        }
                        const float pu = u == 0 ? p[i].x : u == 1 ? p[i].y : u == 2 ? p[i].z : p[i].w;
#pragma unroll
                        for (int e = 0; e < ND; e += 2) {
                            const float2 y = ffma2(make_float2(pu, pu), make_float2(v[e], v[e + 1]), make_float2(o[i][e], o[i][e + 1]));
                            o[i][e] = y.x, o[i][e + 1] = y.y;
                        }
                    }
                }
            }
        };
        if (Src::RANGES && edge) sum(std::integral_constant<bool, Src::RANGES>());
        else sum(std::false_type());
        __syncthreads();                                                // the tile may be overwritten
    }
    cp_async_wait<0>();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
    auto dim = [&](int e) { return DH == 32 ? 2 * tx + e : 16 * (e & ~3) + 4 * tx + (e & 3); };
    auto place = [&](int r) {
        const int2 at = A.split(r0 + r);
        return (float *)A.out + ((long long)(sr.x + at.x) * A.heads + h * A.share + at.y) * DH;
    };
    if (split == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * ty + i;
            if (r >= nr) continue;
            const float inv = l[i] == 0.f ? 0.f : 1.0f / l[i];
            float *out = place(r);
            if constexpr (DH == 32) {
                *reinterpret_cast<float2 *>(out + dim(0)) = make_float2(o[i][0] * inv, o[i][1] * inv);
            } else {
#pragma unroll
                for (int e = 0; e < ND; e += 4)
                    *reinterpret_cast<float4 *>(out + dim(e)) = make_float4(o[i][e] * inv, o[i][e + 1] * inv, o[i][e + 2] * inv, o[i][e + 3] * inv);
            }
        }
        return;
    }
    __syncthreads();
    float *S = f32_smem;                                                // [rows][DH], then m and l of the rows
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 4 * ty + i;
        if (tx == 0) S[ROWS * DH + 2 * r] = m[i] * cs, S[ROWS * DH + 2 * r + 1] = l[i];
#pragma unroll
        for (int e = 0; e < ND; ++e) S[r * DH + dim(e)] = o[i][e];
    }
    cluster_sync_all();
    const uint32_t Ss = smem_u32(S);
    for (int i = rank + split * tid; i < nr * W; i += split * C::THREADS) {
        const int r = i / W, d = i % W * 4;
        float mx = -INFINITY, sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < split; ++k) mx = fmaxf(mx, ld_cluster_f2(cluster_map(Ss + (ROWS * DH + 2 * r) * 4, k)).x);
        for (int k = 0; k < split; ++k) {
            const float2 ml = ld_cluster_f2(cluster_map(Ss + (ROWS * DH + 2 * r) * 4, k));
            const float4 x = ld_cluster_f4(cluster_map(Ss + (r * DH + d) * 4, k));
            const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - mx);
            sum = fmaf(ml.y, f, sum);
            v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
        }
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        *reinterpret_cast<float4 *>(place(r) + d) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    }
    cluster_sync_all();                                                 // nobody leaves while its state is read
}

template <typename Src, int DH, int ROWS>
static int launch_attn_f32_rows(const BatchD &B, const AttnRows &A, const Src &K, int kv_heads, int dev, int n_sm, cudaStream_t st) {
    using C = F32Cfg<DH, ROWS>;
    auto kern = k_attn_f32<Src, DH, ROWS>;
    static OncePerDevice once;
    if (!once.run(dev, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) == cudaSuccess; })) return NFD_E_CUDA;
    const long long tiles = ((long long)B.max_rows * A.share + ROWS - 1) / ROWS, units = kv_heads * tiles * B.n_seqs;
    const int blocks = (K.most + F32_KEYS - 1) / F32_KEYS;
    int split = 1;
    while (split < 8 && units * split * 2 <= 2 * n_sm && blocks > split) split *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kv_heads * split, B.n_seqs, (unsigned)tiles), cfg.blockDim = dim3(C::THREADS), cfg.dynamicSmemBytes = C::SMEM, cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension, at.val.clusterDim.x = split, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at, cfg.numAttrs = split > 1;
    if (cudaLaunchKernelEx(&cfg, kern, B, A, K, split) != cudaSuccess) {
        cudaGetLastError();
        return NFD_E_CUDA;
    }
    return NFD_OK;
}
// A few rows (8 of a unit to a cluster) to fp32 states: bound by the stream of K and V.  Each warp of a cluster's CTAs takes chunks of 1024 / DH keys in turn,
// with a cp.async ring of its own (8 KB a chunk, two chunks ahead: 128 KB of an SM on their way), an online softmax of its own and no barrier until
// the end.  S: a lane has a key's share of 32 dims; O: a lane has four dims and eight keys.  Rows of 16-byte words are swizzled by the key, so
// that neither way of reading meets in a bank.  Measured, four sequences of one row, 16 heads x 64, against 2000 states each: 14.6 us (66 MB: 4.5 TB/s), with the
// kernel above, whose tile of 32 rows one row has to itself, 50.
template <int DH, int R> struct F32Few {
    static constexpr int KC = 1024 / DH, PR = DH / 4, LPK = 32 / KC, NST = 3;
    static constexpr int QS = LPK * 36;                                 // floats of a query: 32 of each share, and 4 that nobody reads
    static constexpr int STAGE = 2 * KC * DH * 4;
    static constexpr int STATE = R * (DH + 2) * 4;
    static constexpr int AT_Q = FEW_WARPS * NST * STAGE, AT_P = AT_Q + R * QS * 4, AT_T = AT_P + FEW_WARPS * R * KC * 4, SMEM = AT_T + STATE;
    static_assert(STATE <= NST * STAGE && AT_T % 16 == 0 && SMEM <= 232448 - 1024, "shared memory of a CTA");
};
// (The rings leave one CTA to an SM, and so it may have all registers: not told so, the compiler took 128 and spilled, and eight rows took 25.6 us for 21.5.)
template <typename Src, int DH, int R>
__global__ void __launch_bounds__(32 * FEW_WARPS, 1) k_attn_f32_few(const BatchD B, const AttnRows A, const Src K, int split) {
    using C = F32Few<DH, R>;
    constexpr int KC = C::KC, PR = C::PR, NST = C::NST, STEP = 32 / PR;
    extern __shared__ __align__(16) uint8_t f32_few_smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % split, h = blockIdx.x / split, s = blockIdx.y;
    const int2 sr = B.rows(s);
    const int r0 = blockIdx.z * R, nr = min(min(sr.y, B.max_rows) * A.share - r0, R);
    if (nr <= 0) return;                                                // (the whole cluster)
    const int len = K.length(B, s);
    int lo = 0, hi = len, edge_lo = 0, edge_hi = INT_MAX;               // (as in the kernel above)
    KeyRange kr[R];
    if constexpr (Src::RANGES) {
#pragma unroll
        for (int r = 0; r < R; ++r) kr[r] = K.range(B, len, sr.y, A.split(r0 + min(r, nr - 1)).x);
        lo = kr[0].lo, hi = kr[R - 1].hi, edge_lo = kr[R - 1].lo, edge_hi = kr[0].hi;
    }
    float *ring = reinterpret_cast<float *>(f32_few_smem + warp * NST * C::STAGE), *sQ = reinterpret_cast<float *>(f32_few_smem + C::AT_Q);
    float *sP = reinterpret_cast<float *>(f32_few_smem + C::AT_P) + warp * R * KC;
    // copies: word `lane % PR` of keys lane / PR, + STEP, ...
    const int word = lane % PR, key0 = lane / PR, step = split * FEW_WARPS * KC;
    int next = lo + (rank * FEW_WARPS + warp) * KC, base = next;
    uint32_t raw = 0, bits[2] = {0, 0};                                 // key `lane` of the chunk that is filled next; which keys of the next two chunks are there
    long long place = -1;                                               // its row
    long long from = 0;                                                 // of states: where the sequence's begin, and what the mask says
    const unsigned char *mask = nullptr;
    if constexpr (!Src::RANGES) {
        from = s * K.seq_stride + h * K.head_stride + word * 4;
        mask = K.mask ? K.mask + (size_t)s * K.n_keys : nullptr;
    }
    auto cursor = [&]() {
        if constexpr (Src::RANGES) return K.cursor(B, s, sr.x, next + lane, step);
        else return 0;
    }();
    auto look = [&]() {
        const int p = next + lane;
        raw = p < hi && lane < KC;
        if constexpr (Src::RANGES) {
            place = K.next(cursor, B, h, raw);
            raw = place >= 0;
        } else {
            if (mask && raw) raw = mask[p];
        }
    };
    auto fill = [&](int st) -> uint32_t {
        const uint32_t there = __ballot_sync(0xffffffffu, raw != 0), dst = smem_u32(ring) + st * C::STAGE;
        long long at = 0;
        if constexpr (!Src::RANGES) at = from + (long long)(next + key0) * K.key_stride;
#pragma unroll
        for (int i = 0; i < KC / STEP; ++i) {
            const int key = key0 + i * STEP;
            const bool here = there >> key & 1;
            const uint32_t d = dst + (key * PR + (word ^ (key & 7))) * 16;
            const float *k = K.first_k(), *v = K.first_v();
            if constexpr (Src::RANGES) {
                const long long row = __shfl_sync(0xffffffffu, place, key);
                if (here) k = K.k_row(row, h) + word * 4, v = K.v_row(row, h) + word * 4;
            } else {
                if (here) k += at, v += at;
                at += STEP * K.key_stride;
            }
            cp_async16(d, k, here ? 16 : 0);
            cp_async16(d + KC * DH * 4, v, here ? 16 : 0);
        }
        next += step;
        look();
        return there;
    };
    look();
#pragma unroll
    for (int i = 0; i < NST - 1; ++i) {
        if (next < hi) bits[i] = fill(i);
        cp_async_commit();
    }
    for (int i = threadIdx.x; i < R * PR; i += 32 * FEW_WARPS) {
        const int r = i / PR, w = i % PR;
        const int2 at = A.split(r0 + min(r, nr - 1));
        *reinterpret_cast<float4 *>(sQ + r * C::QS + (w >> 3) * 36 + (w & 7) * 4) =
            *reinterpret_cast<const float4 *>((const float *)A.q + (long long)(sr.x + at.x) * A.q_stride + (h * A.share + at.y) * DH + 4 * w);
    }
    const float cs = 1.4426950408889634f * (1.0f / sqrtf((float)DH));
    const int key = lane % KC, part = lane / KC, g = lane / PR;
    float o[R][4], m[R], l[R];
#pragma unroll
    for (int r = 0; r < R; ++r) m[r] = -INFINITY, l[r] = o[r][0] = o[r][1] = o[r][2] = o[r][3] = 0.f;
    __syncthreads();
    int st = 0;
    for (; base < hi; base += step) {
        const uint32_t there = bits[0];
        const float *kt = ring + st * (C::STAGE / 4), *vt = kt + KC * DH;
        bits[0] = bits[1];
        if (next < hi) bits[1] = fill(st == 0 ? NST - 1 : st - 1);
        if (++st == NST) st = 0;
        cp_async_commit();
        cp_async_wait<NST - 1>();
        __syncwarp();
        float2 xx[R];
#pragma unroll
        for (int r = 0; r < R; ++r) xx[r] = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            const float4 k = *reinterpret_cast<const float4 *>(kt + (key * PR + ((part * 8 + w) ^ (key & 7))) * 4);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float4 q = *reinterpret_cast<const float4 *>(sQ + r * C::QS + part * 36 + 4 * w);
                xx[r] = ffma2(make_float2(q.x, q.y), make_float2(k.x, k.y), ffma2(make_float2(q.z, q.w), make_float2(k.z, k.w), xx[r]));
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float x = xx[r].x + xx[r].y;
#pragma unroll
            for (int d = KC; d < 32; d <<= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
            if (!(there >> key & 1)) x = -INFINITY;
            if (Src::RANGES && (base + key < kr[r].lo || base + key >= kr[r].hi)) x = -INFINITY;
            float mn = x;
#pragma unroll
            for (int d = 1; d < KC; d <<= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, d));
            mn = fmaxf(mn, m[r]);
            const float f = mn == m[r] ? 1.0f : exp2f((m[r] - mn) * cs), p = exp2f((x - (mn == -INFINITY ? 0.f : mn)) * cs) * K.scale;
            m[r] = mn, l[r] = fmaf(l[r], f, p);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[r][e] *= f;
            if (part == 0) sP[r * KC + key] = p;
        }
        __syncwarp();
        const bool edge = Src::RANGES && (base < edge_lo || base + KC > edge_hi);
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            float4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const float4 *>(vt + ((g * 8 + i + u) * PR + (word ^ (i + u))) * 4);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float4 p4 = *reinterpret_cast<const float4 *>(sP + r * KC + g * 8 + i);
                const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (Src::RANGES && edge && (base + g * 8 + i + u < kr[r].lo || base + g * 8 + i + u >= kr[r].hi)) continue;
                    const float2 a = ffma2(make_float2(p[u], p[u]), make_float2(v[u].x, v[u].y), make_float2(o[r][0], o[r][1]));
                    const float2 b = ffma2(make_float2(p[u], p[u]), make_float2(v[u].z, v[u].w), make_float2(o[r][2], o[r][3]));
                    o[r][0] = a.x, o[r][1] = a.y, o[r][2] = b.x, o[r][3] = b.y;
                }
            }
        }
        __syncwarp();                                                   // the stage and sP may be written again
    }
    cp_async_wait<0>();
    __syncwarp();
    // this warp's state into its (drained) ring: O by rows, then m and l of the rows
    float *S = ring;
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int d = 1; d < KC; d <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
#pragma unroll
        for (int d = PR; d < 32; d <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[r][e] += __shfl_xor_sync(0xffffffffu, o[r][e], d);
        if (g == 0) *reinterpret_cast<float4 *>(S + r * DH + word * 4) = make_float4(o[r][0], o[r][1], o[r][2], o[r][3]);
        if (lane == 0) S[R * DH + 2 * r] = m[r] * cs, S[R * DH + 2 * r + 1] = l[r];
    }
    __syncthreads();
    float *T = reinterpret_cast<float *>(f32_few_smem + C::AT_T);
    auto write = [&](int r, int d, float4 v, float sum) {
        const int2 at = A.split(r0 + r);
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        float *out = (float *)A.out + ((long long)(sr.x + at.x) * A.heads + h * A.share + at.y) * DH + d;
        *reinterpret_cast<float4 *>(out) = make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv);
    };
    auto join = [](float4 &v, float &sum, float4 x, float2 ml, float mx) {
        const float f = ml.x == -INFINITY ? 0.f : exp2f(ml.x - mx);
        sum = fmaf(ml.y, f, sum);
        v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
    };
    for (int i = threadIdx.x; i < nr * PR; i += 32 * FEW_WARPS) {
        const int r = i / PR, d = i % PR * 4;
        float mx = -INFINITY, sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        auto state = [&](int w) { return reinterpret_cast<const float *>(f32_few_smem + w * NST * C::STAGE); };
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) mx = fmaxf(mx, state(w)[R * DH + 2 * r]);
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w)
            join(v, sum, *reinterpret_cast<const float4 *>(state(w) + r * DH + d), *reinterpret_cast<const float2 *>(state(w) + R * DH + 2 * r), mx);
        if (split == 1) {
            write(r, d, v, sum);
        } else {
            *reinterpret_cast<float4 *>(T + r * DH + d) = v;
            if (d == 0) T[R * DH + 2 * r] = mx, T[R * DH + 2 * r + 1] = sum;
        }
    }
    if (split == 1) return;
    cluster_sync_all();
    const uint32_t Ts = smem_u32(T);
    for (int i = rank + split * threadIdx.x; i < nr * PR; i += split * 32 * FEW_WARPS) {
        const int r = i / PR, d = i % PR * 4;
        float mx = -INFINITY, sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < split; ++k) mx = fmaxf(mx, ld_cluster_f2(cluster_map(Ts + (R * DH + 2 * r) * 4, k)).x);
        for (int k = 0; k < split; ++k)
            join(v, sum, ld_cluster_f4(cluster_map(Ts + (r * DH + d) * 4, k)), ld_cluster_f2(cluster_map(Ts + (R * DH + 2 * r) * 4, k)), mx);
        write(r, d, v, sum);
    }
    cluster_sync_all();                                                 // nobody leaves while its state is read
}
template <typename Src, int DH, int R>
static int launch_attn_f32_few(const BatchD &B, const AttnRows &A, const Src &K, int kv_heads, int dev, cudaStream_t st) {
    using C = F32Few<DH, R>;
    auto kern = k_attn_f32_few<Src, DH, R>;
    static OncePerDevice once;
    static int fit[NFD_PAGED_DEVICES][5];
    if (!once.run(dev, [&] {
            if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) != cudaSuccess ||
                cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
                return false;
            for (int i = 1; i < 5; ++i) fit[dev][i] = clusters_that_fit(kern, 1 << i, 32 * FEW_WARPS, C::SMEM);
            return true;
        }))
        return NFD_E_CUDA;
    const int tiles = (int)(((long long)B.max_rows * A.share + R - 1) / R);
    const int split = few_split((long long)kv_heads * B.n_seqs * tiles, K.most, C::KC, fit[dev]);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kv_heads * split, B.n_seqs, tiles), cfg.blockDim = dim3(32 * FEW_WARPS), cfg.dynamicSmemBytes = C::SMEM, cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension, at.val.clusterDim.x = split, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at, cfg.numAttrs = split > 1;
    if (cudaLaunchKernelEx(&cfg, kern, B, A, K, split) != cudaSuccess) {
        cudaGetLastError();
        return NFD_E_CUDA;
    }
    return NFD_OK;
}
// Rows of a unit that the kernel for few takes, eight at a time, each eight reading the keys.  us there and in tiles of 32 rows: four sequences, 16 heads x
// 64, 2000 states, 8 and 16 rows 21.6, 32.7 and 51.0, 50.8 (24, when that kernel still spilled, 79.7 and 50.7); 64 sequences, 512 states, 81.7,
// 154 and 242, 242; head dimension 128, 32 sequences, 8 heads, 600 states, 16 and 32 rows 80, 139 and 183, 183.
constexpr int f32_few_most(int dh) { return dh == 128 ? 32 : 16; }
// 64 rows where that leaves no SM idle: twice the warps for the same tiles of keys
template <int DH, typename Src>
static int launch_attn_f32(const BatchD &B, const AttnRows &A, const Src &K, int kv_heads, int dev, int n_sm, cudaStream_t st) {
    const long long rows = (long long)B.max_rows * A.share;
    if (rows <= 1) return launch_attn_f32_few<Src, DH, 1>(B, A, K, kv_heads, dev, st);
    if (rows <= 4) return launch_attn_f32_few<Src, DH, 4>(B, A, K, kv_heads, dev, st);
    if (rows <= f32_few_most(DH)) return launch_attn_f32_few<Src, DH, 8>(B, A, K, kv_heads, dev, st);
    if ((((long long)B.max_rows * A.share + 63) / 64) * kv_heads * B.n_seqs >= n_sm) return launch_attn_f32_rows<Src, DH, 64>(B, A, K, kv_heads, dev, n_sm, st);
    return launch_attn_f32_rows<Src, DH, 32>(B, A, K, kv_heads, dev, n_sm, st);
}
