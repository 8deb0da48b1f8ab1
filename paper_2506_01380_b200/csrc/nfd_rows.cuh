// Rows on their way from one projection of a block to the next: rotary embedding with a position on several axes, and the norms around a block with
// its gate and residual scale.  Both read and write every number once; what bounds them is memory, or for few rows the launch and a chain of loads.
#pragma once
#include "nfd_attn_rows.cuh"
#include "nfd_sm100.cuh"

// eight numbers as they are in memory
template <typename TS> struct Raw8;
template <> struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float *p) { a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4); }
    __device__ __forceinline__ void get(float *x) const { x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w; }
};
template <> struct Raw8<bf16> {
    uint4 a;
    __device__ __forceinline__ void load(const bf16 *p) { a = *reinterpret_cast<const uint4 *>(p); }
    __device__ __forceinline__ void get(float *x) const {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
};

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
// positions keep their fraction; sine and cosine of what is left are fp32), then eight pairs to a thread: 16 numbers in a row, or eight of either half of a
// head.  A thread keeps its place in the rows and has the next of them on its way, the first before the angles are known.  (With four in flight and eight rows to
// unpack there were 142 registers, a CTA to an SM, and 21504 rows of 32 heads x 64 took 121 us.)
template <typename TS, bool HALVES>
__global__ void __launch_bounds__(ROTATE_THREADS, 5) k_rotate(const __grid_constant__ RotateD R, const RotateIO io, int rows, float sign) {
    __shared__ __align__(16) float2 s_cs[ROTATE_MAX_ROWS * (ROTATE_MAX_DIM / 2)];
    const int tid = threadIdx.x, r0 = blockIdx.x * rows, nr = min(rows, io.n_rows - r0), pairs = R.dim / 2, per_head = R.dim / 16;
    const int n0 = io.heads[0] * per_head, n = n0 + io.heads[1] * per_head;
    // a thread's place (of n to a row), and the rows that it takes: row, row + by, ...
    const int by = n < ROTATE_THREADS ? ROTATE_THREADS / n : 1, row = n < ROTATE_THREADS ? tid / n : 0;
    int j = n < ROTATE_THREADS ? tid - row * n : tid;
    struct Place {
        const TS *in;
        TS *out;
        long long in_stride, out_stride;
        int second, pair;                                      // the other eight numbers, the first pair
    };
    auto at = [&](int j) -> Place {
        const int w = j >= n0, jj = w ? j - n0 : j, h = jj / per_head, d = jj - h * per_head, first = h * R.dim + (HALVES ? 8 * d : 16 * d);
        return {(const TS *)io.in[w] + r0 * io.in_stride[w] + first, (TS *)io.out[w] + r0 * io.out_stride[w] + first, io.in_stride[w], io.out_stride[w],
                HALVES ? pairs : 8, 8 * d};
    };
    Raw8<TS> ra, rb;                                           // the next row's numbers
    auto load = [&](const Place &p, int r) { ra.load(p.in + r * p.in_stride), rb.load(p.in + r * p.in_stride + p.second); };
    const bool mine = row < by && row < nr && j < n;
    Place p = at(mine ? j : 0);
    if (mine) load(p, row);
    for (int i = tid; i < nr * pairs; i += ROTATE_THREADS) {
        const int r = i / pairs, pair = i - r * pairs, axis = pair < R.half_t ? 0 : pair < R.half_th ? 1 : 2;
        const double turns = (double)__ldg(io.pos + 3LL * (r0 + r) + axis) * R.freq[pair];
        float sn, cs;
        sincospif(2.0f * (float)(turns - rint(turns)), &sn, &cs);
        s_cs[i] = make_float2(cs, sign * sn);
    }
    __syncthreads();
    if (!mine) return;
    for (; j < n; j += ROTATE_THREADS) {
        if (j >= ROTATE_THREADS) p = at(j), load(p, row);
        for (int r = row; r < nr; r += by) {
            float a[8], b[8];
            ra.get(a), rb.get(b);
            if (r + by < nr) load(p, r + by);
            const float4 *cs = reinterpret_cast<const float4 *>(s_cs + r * pairs + p.pair);
            auto turn = [](float &x, float &y, float co, float si) {
                const float t = x * co - y * si;
                y = y * co + x * si, x = t;
            };
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float4 c = cs[e];
                if (HALVES) {
                    turn(a[2 * e], b[2 * e], c.x, c.y), turn(a[2 * e + 1], b[2 * e + 1], c.z, c.w);
                } else {
                    float *x = e < 2 ? a + 4 * e : b + 4 * (e - 2);
                    turn(x[0], x[1], c.x, c.y), turn(x[2], x[3], c.z, c.w);
                }
            }
            store8<TS>(p.out + r * p.out_stride, a), store8<TS>(p.out + r * p.out_stride + p.second, b);
        }
        if (n < ROTATE_THREADS) break;
    }
}

// ---- norms around a block -----------------------------------------------------------------------------------
#define NORM_FEW 8                       // rows to an SM up to which a CTA reads its own as it comes to it
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
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ bool bulk_wait(uint32_t bar, uint32_t parity) {
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = global_timer_ns();
    uint32_t spins = 0;
    while (!mbar_try_wait(bar, parity))
        if ((++spins & 0x3ff) == 0 && global_timer_ns() - t0 > NFD_WAIT_LIMIT_NS) return false;
    return true;
}
__device__ __forceinline__ void bulk_store(void *dst, uint32_t src, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(src), "r"(bytes) : "memory");
}
// eight parameters
__device__ __forceinline__ void load8_par(const void *p, int bf, long long at, float *x) {
    if (bf) load8<bf16>((const bf16 *)p + at, x);
    else load8<float>((const float *)p + at, x);
}
// Sum over the threads of a row: a warp, or a CTA of up to 16.
template <bool WARP> __device__ __forceinline__ float row_sum(float x, float *shared, int &turn) {
#pragma unroll
    for (int d = 16; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
    if constexpr (!WARP) {
        float *s = shared + (turn ^= 16);                      // (who writes one half again has been through the barrier of the other)
        const int lane = threadIdx.x & 31;
        if (lane == 0) s[threadIdx.x >> 5] = x;
        __syncthreads();
        x = lane < (int)blockDim.x / 32 ? s[lane] : 0.f;
#pragma unroll
        for (int d = 8; d; d >>= 1) x += __shfl_xor_sync(0xffffffffu, x, d);
        x = __shfl_sync(0xffffffffu, x, 0);
    }
    return x;
}
// What a row's numbers are multiplied by and what is added, of a piece of eight: x' = x + y f ym + ya, h = x' f hm + ha.
struct NormFactors {
    float ym[8], ya[8], hm[8], ha[8];
    __device__ __forceinline__ void load_y(const GateNormD &N, int m, int at) {
        const long long mod = m * N.mod_stride + at;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) ym[e] = N.res_scale, ya[e] = 0.f;
        if (N.gate) {
            load8_par(N.gate, N.mod_bf, mod, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) ym[e] *= w[e];
        }
        if (N.post.bias) {
            load8_par(N.post.bias, N.post.bf, at, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) ya[e] = ym[e] * w[e];
        }
        if (N.post.weight) {
            load8_par(N.post.weight, N.post.bf, at, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) ym[e] *= w[e];
        }
    }
    __device__ __forceinline__ void load_h(const GateNormD &N, int m, int at) {
        const long long mod = m * N.mod_stride + at;
        float w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) hm[e] = 1.f, ha[e] = 0.f;
        if (N.scale) {
            load8_par(N.scale, N.mod_bf, mod, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) hm[e] += w[e];
        }
        if (N.shift) load8_par(N.shift, N.mod_bf, mod, ha);
        if (N.pre.bias) {
            load8_par(N.pre.bias, N.pre.bf, at, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) ha[e] = fmaf(w[e], hm[e], ha[e]);
        }
        if (N.pre.weight) {
            load8_par(N.pre.weight, N.pre.bf, at, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) hm[e] *= w[e];
        }
    }
};
// t = post(y), x' = x + res_scale gate t, h = pre(x') (1 + scale) + shift, statistics in fp32 over numbers that stay in registers: the mean first, then
// the squares of what is left.  A warp (WARP: up to 256 numbers a row) or a CTA takes `rows` rows one after the other, V pieces of eight numbers to a thread.
// Weights, gate, scale and shift become one factor and one summand for either norm, kept from row to row as long as the modulation is the same (V = 1; wider
// rows form them anew).  Where a CTA has several rows, bulk copies bring `stages` of them ahead into shared memory: with the next row in registers the bytes on
// their way were too few (21504 rows of 1536, two norms: 119 us, 90 us with the copies, 82 us with the results going out the same way; 4.8 TB/s).
// 21504 rows in bulk are bound by memory, a few hundred by the launch and one chain of loads (336 rows: 8.9 us from Python).
enum { NORM_WARP, NORM_CTA, NORM_RING };
template <typename TX, typename TY, int HOW, int V>
__global__ void __launch_bounds__(HOW == NORM_WARP ? 128 : 512, HOW == NORM_RING && V == 1 ? 2 : 1) k_gate_norm(const __grid_constant__ GateNormD N, int rows, int stages) {
    constexpr bool WARP = HOW == NORM_WARP, ring = HOW == NORM_RING;
    extern __shared__ __align__(16) uint8_t norm_smem[];       // [stages] rows of x and y
    __shared__ float shared[32];
    __shared__ __align__(8) uint64_t s_full[NORM_STAGES];
    const int t = WARP ? threadIdx.x & 31 : threadIdx.x, T = WARP ? 32 : blockDim.x, pieces = N.width / 8;
    const long long first = (long long)(WARP ? blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x) * rows;
    if (first >= N.n_rows) return;                             // (whole warps, or the whole CTA)
    const int end = (int)min(first + rows, (long long)N.n_rows);
    const uint32_t bytes_x = N.width * sizeof(TX), bytes_y = N.width * sizeof(TY), bytes = bytes_x + bytes_y, bar = smem_u32(s_full), to = smem_u32(norm_smem);
    uint32_t laps = 0;                                         // copies into the stages so far, odd or even
    auto bring = [&](int row, int st) {                        // (one thread)
        laps ^= 1u << st;
        const uint32_t dst = to + st * bytes;
        mbar_expect_tx(bar + 8 * st, N.y ? bytes : bytes_x);
        bulk_load(dst, (const TX *)N.x + row * N.x_stride, bytes_x, bar + 8 * st);
        if (N.y) bulk_load(dst + bytes_x, (const TY *)N.y + row * N.y_stride, bytes_y, bar + 8 * st);
    };
    if (ring) {
        if (threadIdx.x == 0) {
            for (int i = 0; i < stages; ++i) mbar_init(bar + 8 * i, 1);
            fence_mbar_init();
            for (int i = 0; i < stages && first + i < end; ++i) bring((int)first + i, i);
        }
        __syncthreads();
    }
    int turn = 0, st = 0, m = -1;
    uint32_t par = 0;
    bool ok = true;
    const float per = 1.0f / (float)N.width;
    Raw8<TX> rx[V];
    Raw8<TY> ry[V];
    auto fetch = [&](const TX *px, const TY *py) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i * T + t < pieces) {
                rx[i].load(px + (i * T + t) * 8);
                if (N.y) ry[i].load(py + (i * T + t) * 8);
            }
    };
    auto fetch_row = [&](int row) { fetch((const TX *)N.x + row * N.x_stride, (const TY *)N.y + row * N.y_stride); };
    // (clamped when it is used, a row later: a warp stops at the first instruction that asks for a load's result)
    auto mod_of = [&](int row) { return N.index ? __ldg(N.index + row) : row / N.rows_per_mod; };
    int next_m = mod_of((int)first);
    if (WARP) fetch_row((int)first);
    NormFactors kept;
    // numbers to what they are off the mean, and the factor that makes their mean square 1
    auto stats = [&](float (&v)[V][8], const NormD &n) -> float {
        if (n.layer) {
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e & 3] += v[i][e];
            const float mean = row_sum<WARP>((sum[0] + sum[1]) + (sum[2] + sum[3]), shared, turn) * per;
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i * T + t < pieces)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[i][e] -= mean;
        }
        float sq[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) sq[e & 3] = fmaf(v[i][e], v[i][e], sq[e & 3]);
        return rsqrtf(row_sum<WARP>((sq[0] + sq[1]) + (sq[2] + sq[3]), shared, turn) * per + n.eps);
    };
#pragma unroll 1
    for (int row = (int)first; row < end; ++row) {
        if (ring) {
            ok = ok && bulk_wait(bar + 8 * st, par);
            const uint8_t *at = norm_smem + st * bytes;
            fetch(reinterpret_cast<const TX *>(at), reinterpret_cast<const TY *>(at + bytes_x));
        } else if (!WARP) {
            fetch_row(row);
        }
        float x[V][8], y[V][8];
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[i][e] = y[i][e] = 0.f;
            if (i * T + t < pieces) {
                rx[i].get(x[i]);
                if (N.y) ry[i].get(y[i]);
            }
        }
        if (!ok) x[0][0] = NAN;                                // (a copy that did not come: the row is NaN)
        const int now = min(max(next_m, 0), N.n_mods - 1);
        if (V == 1 && now != m && t < pieces) {
            if (N.y) kept.load_y(N, now, t * 8);
            if (N.h) kept.load_h(N, now, t * 8);
        }
        m = now;
        if (row + 1 < end) {
            next_m = mod_of(row + 1);
            if (WARP) fetch_row(row + 1);
        }
        if (N.y) {
            const float f = N.post.on ? stats(y, N.post) : 1.f;
            TX *po = ring ? reinterpret_cast<TX *>(norm_smem + st * bytes) : (TX *)N.x_out + row * N.x_out_stride;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (i * T + t >= pieces) continue;
                if (V > 1) kept.load_y(N, m, (i * T + t) * 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] = fmaf(y[i][e] * f, kept.ym[e], x[i][e] + kept.ya[e]);
                store8<TX>(po + (i * T + t) * 8, x[i]);
            }
        }
        if (N.h) {
            const float f = stats(x, N.pre);
            TY *ph = ring ? reinterpret_cast<TY *>(norm_smem + st * bytes + bytes_x) : (TY *)N.h + row * N.h_stride;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (i * T + t >= pieces) continue;
                if (V > 1) kept.load_h(N, m, (i * T + t) * 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[i][e] = fmaf(x[i][e] * f, kept.hm[e], kept.ha[e]);
                store8<TY>(ph + (i * T + t) * 8, x[i]);
            }
        }
        if (ring) {
            // The results lie where the row lay (a thread writes what it alone has read), and go out from there; a stage is filled again a row later, when
            // its results have been read.
            fence_proxy_async_smem();
            __syncthreads();
            if (threadIdx.x == 0) {
                const uint32_t from = to + st * bytes;
                if (N.y) bulk_store((TX *)N.x_out + row * N.x_out_stride, from, bytes_x);
                if (N.h) bulk_store((TY *)N.h + row * N.h_stride, from + bytes_x, bytes_y);
                bulk_commit();
                const int last = st ? st - 1 : stages - 1, again = row - 1 + stages;
                if (row > (int)first && ok && again < end) {
                    bulk_wait_read<1>();
                    bring(again, last);
                }
            }
            if (++st == stages) st = 0, par ^= 1;
        }
    }
    if (ring && threadIdx.x == 0) {                            // (nobody leaves with copies in flight)
        if (!ok)
            for (int i = 0; i < stages && first + i < end; ++i) bulk_wait(bar + 8 * i, laps >> i & 1 ^ 1);
        bulk_wait_all();
    }
}
// One wave of CTAs, the rows shared out evenly: a CTA for each row where the device holds them all at once.
template <typename TX, typename TY, int HOW, int V> static int launch_gate_norm_as(const GateNormD &N, int threads, int bytes, int dev, int n_sm, cudaStream_t st) {
    auto kern = k_gate_norm<TX, TY, HOW, V>;
    static OncePerDevice once;
    static int regs[NFD_PAGED_DEVICES], own[NFD_PAGED_DEVICES];
    if (!once.run(dev, [&] {
            cudaFuncAttributes at;
            if (cudaFuncGetAttributes(&at, kern) != cudaSuccess || cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, NORM_MOST) != cudaSuccess) return false;
            regs[dev] = (at.numRegs + 7) / 8 * 8;
            own[dev] = (int)at.sharedSizeBytes;
            return true;
        }))
        return NFD_E_CUDA;
    // (two rows fit into shared memory: the caller's rule)
    const auto [ctas, stages] = norm_plan(regs[dev], threads, HOW == NORM_RING ? bytes : 0, own[dev]);
    const long long per = HOW == NORM_WARP ? threads / 32 : 1, held = (long long)ctas * n_sm * per, rows = (N.n_rows + held - 1) / held;
    kern<<<(unsigned)((N.n_rows + rows * per - 1) / (rows * per)), threads, stages * bytes, st>>>(N, (int)rows, stages);
    return cudaGetLastError() == cudaSuccess ? NFD_OK : NFD_E_CUDA;
}
template <typename TX, typename TY> static int launch_gate_norm(const GateNormD &N, int dev, int n_sm, cudaStream_t st) {
    const int pieces = N.width / 8, v = pieces <= 512 ? 1 : pieces <= 1024 ? 2 : 4, threads = ((pieces + v - 1) / v + 31) / 32 * 32;
    const int bytes = N.width * (int)(sizeof(TX) + sizeof(TY));
    if (pieces <= 32) return launch_gate_norm_as<TX, TY, NORM_WARP, 1>(N, 128, bytes, dev, n_sm, st);
    auto go = [&](auto pieces_of_a_thread) -> int {
        constexpr int V = decltype(pieces_of_a_thread)::value;
        // (two of the widest fp32 rows do not fit into shared memory)
        if (N.n_rows >= NORM_FEW * n_sm && 2 * bytes <= NORM_MOST) return launch_gate_norm_as<TX, TY, NORM_RING, V>(N, threads, bytes, dev, n_sm, st);
        return launch_gate_norm_as<TX, TY, NORM_CTA, V>(N, threads, bytes, dev, n_sm, st);
    };
    return v == 1 ? go(std::integral_constant<int, 1>()) : v == 2 ? go(std::integral_constant<int, 2>()) : go(std::integral_constant<int, 4>());
}
