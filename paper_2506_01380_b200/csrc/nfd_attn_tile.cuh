// Attention of many rows on tcgen05 / TMEM, on 4-bit pages or bf16 states.
//
// The rows of a sequence that share a head of keys (rows x heads that share it) are cut into tiles of 128.  A CTA takes one
// tile, whose key blocks its softmax groups take in turn, or a tile for every group, which share every
// key block (a third or half of the copies and, for 4-bit pages, of the conversions).  Either way the work is a list of jobs
// (block, group), and the groups know nothing of one another until the end: each has its S accumulators, O, m and l of
// its own.  Per job
//     S = Q K^T     UMMA 128 x KB x DH, operands in shared memory, accumulator in tensor memory
//     P = exp2(S c - m)   one thread per row: S by columns to registers, exponentials, P as bf16 over the S it came from
//     O += P V      UMMA 128 x head_dim x KB, P from tensor memory, V as it lies (MN-major)
// m is the largest of the first 16 scores of the group's first block, and no other maximum is taken: a probability is exact to the
// same number of bits whatever its size.  Where a block's sum of a row passes 2^60 (states: 2^50) after all (or is NaN), or a row has no m yet, the
// warp takes the block again, S being untouched so far: maxima first, and where one has risen by more than 8 (a factor of 256) it becomes m and
// the row's O is rescaled in tensor memory by its thread.  What P grows to, O does: 4-bit values are scaled to less than 1, and O stays in fp32; states
// may be as large as bf16 goes, so that their P are scaled down by as much as all blocks together can grow (sum_bits), in the exponent.
//
// Warps 0 .. PW-1 fill the rings of K and V blocks: bf16 states with cp.async, several blocks in flight; 4-bit pages through
// registers, two blocks ahead, the codes becoming bf16 numbers on the way.  Warp PW issues the products, the last 4 NG are the
// softmax groups.  Which keys of a block are there is told beside K, a bit each, in a ring of its own: the softmax does not wait for V.
//
// A unit (sequence, head of keys, tile) with many keys and few others beside it is split over the CTAs of a cluster, which
// merge through distributed shared memory.  Every wait on a barrier in memory is bounded; after one that ran out the rows are NaN.  (The cluster's own
// barrier has no bound and needs none: every CTA comes to it, its other waits being bounded, or has left as a whole cluster.)
//
// P is one bf16 number.  (k_attn_tc carries it as two and doubles its second product for that, 9 to 16 % of its time; here the error of a result is 2.3e-3,
// 2-norm, normal data, for 1.66e-3 of one that is only rounded at the end.  4-bit numbers are themselves off by some 8 % of their group's deviation.)
//
// Nothing is saturated: with 4-bit pages and head dimension 64 an SM that has a CTA gives the special-function unit 62 % of its clocks and issues in 54 %
// of them (a fifth of the exponentials by a polynomial on the FMA pipe made 202 us 207), with head dimension 128 it issues in 44 % and the tensor pipe
// has 30 %.  What is left is the chain S - P - P V of few warps: three to a scheduler, two with head dimension 128.  (512 threads
// have 128 registers each; head dimensions 32 and 64 spill 16 to 24 bytes of them.)
// Measured, 16 heads x 64: 336 rows behind 5712 tokens in 4-bit pages 28.7 us (274 TFLOP/s: 96 CTAs, 12 blocks of three tiles each, the merge), eight
// streams of 336 rows behind 11088 202 us (604 TFLOP/s; 128 CTAs on 148 SMs); 16 heads on 4 x 128, eight batches of 1344 rows against up to 2048 states
// 126.5 us (620 TFLOP/s).
#pragma once
#include "nfd_attn_few.cuh"

#define TILE_THREADS 512
#define TILE_SPLIT 8                // most CTAs of a cluster
#define TILE_GROWTH_KV4 60          // bits that a block's sum may grow by before m follows it
#define TILE_GROWTH 50              // of states, whose probabilities start as many bits lower.  8 x 1344 rows against up to 2048 states, 16 heads on 4 x 128,
                                    // scores with a deviation of 10 nats, us: 24 bits 156, 40 135, 50 128, 60 127; with a deviation of 1 all 126 to 127

// (no status word: there is no context whose latch could be read)
__device__ __forceinline__ bool tile_wait(uint32_t bar, uint32_t parity) {
    if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long t0 = global_timer_ns();
    uint32_t spins = 0;
    while (!mbar_try_wait(bar, parity))
        if ((++spins & 0x3ff) == 0 && global_timer_ns() - t0 > NFD_WAIT_LIMIT_NS) return false;
    return true;
}
// two of them, their first looks overlapped
__device__ __forceinline__ bool tile_wait2(uint32_t a, uint32_t pa, uint32_t b, uint32_t pb) {
    const bool da = mbar_try_wait(a, pa), db = mbar_try_wait(b, pb);
    return (da || tile_wait(a, pa)) && (db || tile_wait(b, pb));
}
// Has the phase completed?  (try_wait may sleep for a while before it says no.)
__device__ __forceinline__ bool tile_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// registers that a tensor-memory load has filled are not touched before this point (which comes after its wait)
__device__ __forceinline__ void loaded32(float *x) {
    asm volatile("" : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]),
                      "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]));
    asm volatile("" : "+f"(x[16]), "+f"(x[17]), "+f"(x[18]), "+f"(x[19]), "+f"(x[20]), "+f"(x[21]), "+f"(x[22]), "+f"(x[23]),
                      "+f"(x[24]), "+f"(x[25]), "+f"(x[26]), "+f"(x[27]), "+f"(x[28]), "+f"(x[29]), "+f"(x[30]), "+f"(x[31]));
}
__device__ __forceinline__ void loaded8(float *x) {
    asm volatile("" : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]));
}
__device__ __forceinline__ void loaded16(float *x) {
    asm volatile("" : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]),
                      "+f"(x[8]), "+f"(x[9]), "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]));
}

template <int DH> struct TileCfg {
    static constexpr int SUB = DH == 128 ? 2 : 1;          // 64-dim parts of a row
    static constexpr int NG = DH == 128 ? 2 : 3;           // softmax groups
    static constexpr int KB = DH == 128 ? 64 : 80;         // keys of a block
    static constexpr int NB = 4;                           // S accumulators: job j has number j % NB
    static constexpr int PW = DH == 128 ? 4 : 3;           // producer warps
    static constexpr int SM0 = 16 - 4 * NG;                // first softmax warp
    static constexpr int NST = DH == 128 ? 5 : 6;          // blocks in the ring of K, and in that of V
    static constexpr int NM = 16;                          // and of their masks: K runs up to NST + NB blocks ahead of the softmax
    static constexpr int Q_BYTES = SUB * 128 * 128;        // a tile's queries
    static constexpr int BLK = SUB * KB * 128;             // a block of K or V
    static constexpr int AT_Q = 0, AT_K = NG * Q_BYTES, AT_V = AT_K + NST * BLK, AT_MASK = AT_V + NST * BLK,
                         AT_BAR = AT_MASK + NM * 32, SMEM = AT_BAR + 448 + 1024;
    static constexpr int TM_O = NB * KB;                   // S number i, and over it P, at i KB; O of group g at TM_O + g 64 SUB
    static constexpr uint32_t M1 = 0xffffffffu, M2 = KB >= 96 ? 0xffffffffu : KB > 64 ? (1u << (KB - 64)) - 1 : 0;      // bits of keys 32 .., 64 ..
    // a group's state, over queries and rings: O as [DH / 4][128] float4, then [128] (m, l)
    static constexpr int STATE = 128 * DH * 4 + 128 * 8;
    static_assert(TM_O + NG * 64 * SUB <= 512 && NG * STATE + 128 * 8 <= AT_MASK && SMEM <= 232448, "tensor and shared memory");
    static_assert(SMEM > 232448 / 2, "a CTA has an SM, and its tensor memory, to itself: nobody in a cluster waits for what another cluster holds");
    static_assert(NST + NB <= NM, "masks");
    static_assert(NST <= 6 && NB == 4 && NM == 16, "TileBars");
    static_assert(PW * 32 >= KB * SUB && KB >= 64 && KB <= 96 && KB % 16 == 0, "a thread for 64 dims of a key; three words of bits");
    static_assert(PW < SM0, "warps");
};

struct TileBars {
    uint32_t b;
    // per stage (up to 6)
    __device__ __forceinline__ uint32_t k_full(int s) const { return b + 8 * s; }
    __device__ __forceinline__ uint32_t k_empty(int s) const { return b + 48 + 8 * s; }
    __device__ __forceinline__ uint32_t v_full(int s) const { return b + 96 + 8 * s; }
    __device__ __forceinline__ uint32_t v_empty(int s) const { return b + 144 + 8 * s; }
    // per accumulator (up to 4)
    __device__ __forceinline__ uint32_t s_full(int i) const { return b + 192 + 8 * i; }
    __device__ __forceinline__ uint32_t p_full(int i) const { return b + 224 + 8 * i; }
    // of a group's even and odd jobs: a warp may be done with a job before the product of the one before it is
    __device__ __forceinline__ uint32_t pv_done(int g, int n) const { return b + 256 + 16 * g + 8 * (n & 1); }
    __device__ __forceinline__ uint32_t q_full() const { return b + 304; }
    // per mask (16)
    __device__ __forceinline__ uint32_t m_full(int s) const { return b + 312 + 8 * s; }
    static constexpr int BYTES = 440;
    __device__ __forceinline__ void init(int producers, int q_warps) const {
        for (int s = 0; s < 6; ++s) {
            mbar_init(k_full(s), producers), mbar_init(v_full(s), producers);      // a producer warp each
            mbar_init(k_empty(s), 1), mbar_init(v_empty(s), 1);
        }
        for (int i = 0; i < 4; ++i) mbar_init(s_full(i), 1), mbar_init(p_full(i), 4);      // a softmax warp each
        for (int g = 0; g < 3; ++g) mbar_init(pv_done(g, 0), 1), mbar_init(pv_done(g, 1), 1);
        for (int s = 0; s < 16; ++s) mbar_init(m_full(s), producers);
        mbar_init(q_full(), q_warps);                                              // the softmax warps
        fence_mbar_init();
    }
};
// at most n groups of this thread's copies are in flight
__device__ __forceinline__ void cp_async_wait_upto(int n) {
    switch (n) {
        case 0: cp_async_wait<0>(); break;
        case 1: cp_async_wait<1>(); break;
        case 2: cp_async_wait<2>(); break;
        case 3: cp_async_wait<3>(); break;
        case 4: cp_async_wait<4>(); break;
        default: cp_async_wait<5>();
    }
}
// the CTA's part of its unit's keys
struct TileWork {
    int s, h, lo, hi, nb;                                   // keys lo .. hi - 1 in nb blocks
};
__device__ __forceinline__ uint32_t tile_at(int row, int chunk) { return row * 128 + ((chunk ^ (row & 7)) << 4); }
// what a producer warp has written is handed to the tensor core
__device__ __forceinline__ void tile_publish(uint32_t bar) {
    fence_proxy_async_smem();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

// ---- producers: bf16 states ---------------------------------------------------------------------------------
template <int DH> struct TileStates {
    static constexpr bool KV4 = false;
    static constexpr float UP = 1.0f;
    StateKeys<bf16, DH> K;
    __device__ __forceinline__ void produce(const BatchD &B, const TileWork &w, uint8_t *smem, const TileBars &bars, bool &ok) const {
        using C = TileCfg<DH>;
        constexpr int CPR = DH / 8, NT = C::PW * 32, RS = NT / CPR, N = (C::KB + RS - 1) / RS;      // 16-byte pieces of a row; threads; rows a step, steps
        constexpr int FLY = 5;                                        // items (K of block 0, V of block 0, K ...) whose copies are in flight
        const int t = threadIdx.x, piece = t % CPR, row0 = t / CPR, lane = t & 31;
        // this thread's pieces of a block: from its first row on, in steps (few instructions a copy: a producer warp has a scheduler's
        // slots to itself for the tenth part of the time, and no latency to hide behind)
        uint32_t to[N];
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = smem_u32(smem) + (piece >> 3) * (C::KB * 128) + tile_at(row0 + i * RS, piece & 7);
        const long long first = w.s * K.seq_stride + w.h * K.head_stride + (long long)(w.lo + row0) * K.key_stride + piece * 8;
        const bf16 *from[2] = {K.k + first, K.v + first};
        const long long step = RS * K.key_stride, on = C::KB * K.key_stride;
        const unsigned char *mask = K.mask ? K.mask + (size_t)w.s * K.n_keys : nullptr;
        // What the mask says of this thread's rows of a block, and of key t of it (loaded a block ahead); the bits of these that are there.
        uint32_t raw[N + 1];
        auto look = [&](int b) {
            const int p0 = w.lo + b * C::KB;
#pragma unroll
            for (int i = 0; i <= N; ++i) {
                const int row = i < N ? row0 + i * RS : t, p = p0 + row;
                raw[i] = p < w.hi && row < C::KB;
                if (mask && raw[i]) raw[i] = mask[p];
            }
        };
        auto there = [&]() -> uint32_t {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i <= N; ++i) m |= (uint32_t)(raw[i] != 0) << (i < N ? i : 31);
            return m;
        };
        int done = 0, item = 0;                                       // published, begun
        auto publish = [&]() {
            const int st = (done >> 1) % C::NST;
            tile_publish(done & 1 ? bars.v_full(st) : bars.k_full(st)), ++done;
        };
        look(0);
        for (int b = 0; b < w.nb && ok; ++b) {
            const int st = b % C::NST, par = (b / C::NST - 1) & 1;
            const uint32_t bits = there();
            look(b + 1);
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                const uint32_t empty = kv ? bars.v_empty(st) : bars.k_empty(st);
                // (nothing is held back while waiting: what frees this stage may need it)
                while (b >= C::NST && !__all_sync(0xffffffffu, tile_test(empty, par))) {
                    if (done < item) {
                        cp_async_wait_upto(item - done - 1);
                        publish();
                    } else {
                        ok = __all_sync(0xffffffffu, tile_wait(empty, par));
                        break;
                    }
                }
                if (!ok) break;
                const uint32_t dst = (kv ? C::AT_V : C::AT_K) + st * C::BLK;
                const bf16 *src = from[kv];
#pragma unroll
                for (int i = 0; i < N; ++i, src += step) {
                    if (C::KB % RS && row0 + i * RS >= C::KB) break;
                    const bool here = bits >> i & 1;
                    cp_async16(dst + to[i], here ? src : K.k, here ? 16 : 0);
                }
                from[kv] += on;
                cp_async_commit();
                if (!kv) {
                    const uint32_t m = __ballot_sync(0xffffffffu, bits >> 31);
                    uint32_t *M = reinterpret_cast<uint32_t *>(smem + C::AT_MASK) + b % C::NM * 8 + (t >> 5);
                    if (lane == 0) M[0] = m, M[4] = 0, mbar_arrive(bars.m_full(b % C::NM));
                }
                // (the first block is wanted at once)
                ++item;
                if (item - done > (item < 2 * FLY ? 2 : FLY)) {
                    cp_async_wait_upto(item - done - 1);
                    publish();
                }
            }
        }
        while (ok && done < item) {
            cp_async_wait_upto(item - done - 1);
            publish();
        }
    }
};

// ---- producers: 4-bit pages ---------------------------------------------------------------------------------
template <int DH> struct TileKv4 {
    static constexpr bool KV4 = true;
    static constexpr float UP = KV4_UP;                     // what scores and results are to be multiplied by
    Kv4Keys<DH> K;
    // a thread's share of a block: 64 (DH 32: 32) dims of a key of K and of V
    static constexpr int NW = DH == 32 ? 4 : 8, SUBS = DH == 128 ? 2 : 1;
    struct Regs {
        uint32_t c[NW], w;                                  // codes, words
    };
    static __device__ __forceinline__ uint32_t load_words(const uint16_t *words, long long place, int sub) {
        if (DH == 32) return __ldg(words + place);
        return __ldg(reinterpret_cast<const uint32_t *>(words + place * (DH / 32)) + sub);
    }
    static __device__ __forceinline__ void load(Regs &r, const void *codes, const uint16_t *words, long long place, int sub) {
        if (place < 0) {
#pragma unroll
            for (int i = 0; i < NW; ++i) r.c[i] = 0;
            r.w = 0;
            return;
        }
        const uint4 *p = reinterpret_cast<const uint4 *>((const uint8_t *)codes + (size_t)place * (DH / 2)) + sub * 2;
#pragma unroll
        for (int i = 0; i < NW / 4; ++i) {
            const uint4 v = __ldg(p + i);
            r.c[4 * i] = v.x, r.c[4 * i + 1] = v.y, r.c[4 * i + 2] = v.z, r.c[4 * i + 3] = v.w;
        }
        r.w = load_words(words, place, sub);
    }
    // (a key that is not there has step 0: its row is zeros)
    static __device__ __forceinline__ void convert(const Regs &r, uint8_t *blk, int row, bool check) {
        const Kv4Scale lower(r.w & 0xffffu, r.w & 0xffffu, check), upper(r.w >> 16, r.w >> 16, check);
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const Kv4Scale &s = i < 4 ? lower : upper;
            *reinterpret_cast<uint4 *>(blk + tile_at(row, i)) = make_uint4(s.pair(r.c[i], 0), s.pair(r.c[i], 1), s.pair(r.c[i], 2), s.pair(r.c[i], 3));
        }
    }
    __device__ __forceinline__ void produce(const BatchD &B, const TileWork &w, uint8_t *smem, const TileBars &bars, bool &ok) const {
        using C = TileCfg<DH>;
        const int t = threadIdx.x, key = t / SUBS, sub = t % SUBS, lane = t & 31;
        // This thread's key of the block that is looked up next: token, entry of the table, offset in the page.  (From block to block by
        // additions: two divisions a block were a sixth of a producer's instructions.)
        const int P = K.P.page_tokens, L = B.table_len, dq = C::KB / P % L, dr = C::KB % P;
        const int *table = B.table + (size_t)w.s * L;
        int p = w.lo + key, off = p % P, pg = p / P % L;
        auto look_up = [&]() -> long long {
            long long at = -1;
            if (p < w.hi && key < C::KB) {
                const int page = __ldg(table + pg);
                if ((unsigned)page < (unsigned)K.P.n_pages) at = ((long long)page * K.P.heads + w.h) * P + off;
            }
            p += C::KB, off += dr, pg += dq;
            if (off >= P) off -= P, ++pg;
            if (pg >= L) pg -= L;
            return at;
        };
        Regs k[2], v[2];
        uint32_t there[2];
        {
            const long long a = look_up(), b = look_up();
            load(k[0], K.P.k, K.P.k_scale, a, sub), load(v[0], K.P.v, K.P.v_scale, a, sub);
            load(k[1], K.P.k, K.P.k_scale, b, sub), load(v[1], K.P.v, K.P.v_scale, b, sub);
            there[0] = __ballot_sync(0xffffffffu, a >= 0), there[1] = __ballot_sync(0xffffffffu, b >= 0);
        }
        long long next = look_up();
        // block b, whose codes are in k and v, into the rings; those of block b + 2 take their place
        auto block = [&](int b, Regs &k, Regs &v, uint32_t &there) {
            const int st = b % C::NST, par = (b / C::NST - 1) & 1;
            const uint32_t m = there;
            const long long place = next;
            there = __ballot_sync(0xffffffffu, place >= 0);
            next = look_up();
            // Values whose step is not finite go in as zeros (a product with the 0 of a row that does not see them would be NaN), a bit for
            // each of their keys.
            const bool bad0 = kv4_not_finite(v.w), bad1 = DH > 32 && kv4_not_finite(v.w >> 16);
            uint32_t bad = __ballot_sync(0xffffffffu, bad0 || bad1);
            if (bad0) v.w &= 0xffff0000u;
            if (bad1) v.w &= 0xffffu;
            if (b >= C::NST) ok = __all_sync(0xffffffffu, tile_wait(bars.k_empty(st), par));
            if (!ok) return;
            if (key < C::KB) convert(k, smem + C::AT_K + st * C::BLK + sub * (C::KB * 128), key, true);
            load(k, K.P.k, K.P.k_scale, place, sub);
            if (SUBS == 2) {
                // two lanes to a key, 16 keys to a warp
                bad |= bad >> 1;
                auto every_other = [](uint32_t x) {
                    x &= 0x55555555u;
                    x = (x | x >> 1) & 0x33333333u, x = (x | x >> 2) & 0x0F0F0F0Fu, x = (x | x >> 4) & 0x00FF00FFu;
                    return (x | x >> 8) & 0xFFFFu;
                };
                uint16_t *M = reinterpret_cast<uint16_t *>(smem + C::AT_MASK) + b % C::NM * 16 + (t >> 5);
                const uint32_t m16 = every_other(m), b16 = every_other(bad);
                if (lane == 0) M[0] = (uint16_t)m16, M[8] = (uint16_t)b16, mbar_arrive(bars.m_full(b % C::NM));
            } else if (lane == 0) {
                uint32_t *M = reinterpret_cast<uint32_t *>(smem + C::AT_MASK) + b % C::NM * 8 + (t >> 5);
                M[0] = m, M[4] = bad, mbar_arrive(bars.m_full(b % C::NM));
            }
            tile_publish(bars.k_full(st));
            if (b >= C::NST) ok = __all_sync(0xffffffffu, tile_wait(bars.v_empty(st), par));
            if (!ok) return;
            if (key < C::KB) convert(v, smem + C::AT_V + st * C::BLK + sub * (C::KB * 128), key, false);
            load(v, K.P.v, K.P.v_scale, place, sub);
            tile_publish(bars.v_full(st));
        };
        for (int b = 0; b < w.nb && ok; b += 2) {
            block(b, k[0], v[0], there[0]);
            if (ok && b + 1 < w.nb) block(b + 1, k[1], v[1], there[1]);
        }
    }
};

// S of a block whose sums have outgrown m, or that finds a row without one: the
// row's maximum over the keys that it sees, m and what has been summed so far adjusted to it, then P.
// seen: bits of the keys that the row sees; n: the group's jobs before this one.
template <int DH>
static __device__ __forceinline__ void tile_slow(uint32_t tS, uint32_t tO, const uint32_t *seen, float c, float down, int n,
                                              uint32_t pv_done, float &m_io, float &l_io, bool &ok) {
    using C = TileCfg<DH>;
    constexpr int KB = C::KB;
    float m = m_io, l = l_io, top = -INFINITY;
    // (by columns, in loops: a whole row in registers is no faster, and its registers are missing elsewhere)
    auto bits = [&](int i) { return (i < 32 ? seen[0] : i < 64 ? seen[1] : seen[2]) >> (i & 31); };
#pragma unroll 1
    for (int i = 0; i < KB; i += 16) {
        float x[16];
        tmem_ld16(tS + i, reinterpret_cast<uint32_t *>(x));
        const uint32_t s = bits(i);
        tmem_ld_wait();
        loaded16(x);
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, s >> e & 1 ? x[e] : -INFINITY);
    }
    // (m starts at -inf: the first score that is seen sets it)
    const bool rise = top * c > m * c + 8.0f || (m == -INFINITY && top != -INFINITY);
    if (__any_sync(0xffffffffu, rise)) {
        const float f = !rise ? 1.0f : m == -INFINITY ? 0.f : few_exp2((m - top) * c);
        if (rise) m = top;
        l *= f;
        if (n) {
            ok = ok && tile_wait(pv_done, ((n - 1) >> 1) & 1);         // O is at rest
            __syncwarp();
            tc_fence_after();
#pragma unroll 1
            for (int i = 0; i < DH; i += 16) {
                float o[16];
                tmem_ld16(tO + i, reinterpret_cast<uint32_t *>(o));
                tmem_ld_wait();
                loaded16(o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] *= f;               // (f may be 0: a value that is not finite stays one)
                tmem_st16(tO + i, reinterpret_cast<uint32_t *>(o));
            }
        }
    }
    const float mc = m == -INFINITY ? 0.f : fmaf(m, c, down);
    float sum = 0.f;
#pragma unroll 1
    for (int i = 0; i < KB; i += 16) {
        float x[16];
        tmem_ld16(tS + i, reinterpret_cast<uint32_t *>(x));
        const uint32_t s = bits(i);
        tmem_ld_wait();
        loaded16(x);
        uint32_t pk[8];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            const float a = s >> e & 1 ? few_exp2(fmaf(x[e], c, -mc)) : 0.f, b = s >> (e + 1) & 1 ? few_exp2(fmaf(x[e + 1], c, -mc)) : 0.f;
            sum += a + b, pk[e / 2] = bf16_pair(a, b);
        }
        tmem_st8(tS + i / 2, pk);                                      // (behind what is still to be read)
    }
    m_io = m, l_io = l + sum;
}
// One pass over S against the m that there is, 16 columns at a time with the next load in flight (xa: the first ones).  MASKED: keys that the
// row does not see count for nothing.  down: taken off the exponents.  False: a sum has outgrown m (most: the most that it may be), and S is as it was.
template <int DH, bool MASKED>
static __device__ __forceinline__ bool tile_fast(uint32_t tS, float *xa, const uint32_t *seen, float c, float down, float most, float m, float &l) {
    constexpr int KB = TileCfg<DH>::KB;
    const float mc = m == -INFINITY ? 0.f : fmaf(m, c, down);
    float2 ls[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    float xb[8];
    uint32_t pk[KB / 2];
    tmem_ld_wait();
    loaded16(xa);
    tmem_ld8(tS + 16, reinterpret_cast<uint32_t *>(xb));
#pragma unroll
    for (int i = 0; i < KB; i += 8) {
        // columns 0 .. 15 are in xa; then xb, xa (first half), xb ...
        float *x = i < 16 ? xa + i : (i >> 3) & 1 ? xa : xb;
        if (i >= 16) {
            tmem_ld_wait();
            loaded8(x);
            if (i + 8 < KB) tmem_ld8(tS + i + 8, reinterpret_cast<uint32_t *>((i >> 3) & 1 ? xb : xa));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float2 s = make_float2(x[2 * u], x[2 * u + 1]);
            if (MASKED) {
                const uint32_t bits = seen[i >> 5] >> (i & 31);
                s.x = bits >> (2 * u) & 1 ? s.x : -INFINITY, s.y = bits >> (2 * u + 1) & 1 ? s.y : -INFINITY;
            }
            const float2 e = ffma2(s, make_float2(c, c), make_float2(-mc, -mc));
            const float2 p = make_float2(few_exp2(e.x), few_exp2(e.y));
            ls[u & 1] = fadd2(ls[u & 1], p);
            pk[i / 2 + u] = bf16_pair(p.x, p.y);
        }
    }
    const float2 l2 = fadd2(ls[0], ls[1]);
    const float sum = l2.x + l2.y;
    if (!__all_sync(0xffffffffu, sum < most)) return false;
    l += sum;
#pragma unroll
    for (int i = 0; i < KB / 2; i += 8) tmem_st8(tS + i, pk + i);
    return true;
}

// D (+)= A B^T with descriptors whose upper halves are constants
__device__ __forceinline__ void tile_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        ".reg .b64 da, db;\n"
        "mov.b64 da, {%1, %5};\n"
        "mov.b64 db, {%2, %5};\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n"
        "}\n" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"((1024 >> 4) | 1 << 14 | 2 << 29)
        : "memory");
}
__device__ __forceinline__ void tile_mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        ".reg .b64 db;\n"
        "mov.b64 db, {%2, %5};\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n"
        "}\n" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"((1024 >> 4) | 1 << 14 | 2 << 29)
        : "memory");
}
// All products of a CTA, by one thread.  G groups; one: a single tile, whose blocks they share out.  (With a thread for each kind, S waits
// for the completion of the P V before it: the same times.)
template <int DH> static __device__ __forceinline__ bool tile_issue(const TileBars &bars, uint32_t base, uint32_t tmem, int jobs, int G, bool one) {
    using C = TileCfg<DH>;
    constexpr int KB = C::KB, SUB = C::SUB, NB = C::NB, NST = C::NST;
    constexpr uint32_t idesc_s = umma_idesc_bf16(128, KB), idesc_pv = umma_idesc_bf16(128, DH) | (1u << 16);       // V: MN-major
    // (a cluster's addresses hold the CTA's rank above bit 23; V's other 64 dims are KB rows on: the leading offset)
    const uint32_t at = base & 0x3ffffu, dQ = (at + C::AT_Q) >> 4, dK = (at + C::AT_K) >> 4, dV = (at + C::AT_V) >> 4 | (KB * 128 >> 4) << 16;
    bool ok = tile_wait(bars.q_full(), 0);
    // S is issued NB jobs ahead of P V, right behind the P V that reads the accumulator's last P: the tensor pipe takes one
    // thread's instructions in order
    int is = 0, gs = 0, js = 0, ks = 0, klap = 0;           // next S: accumulator, group, job, stage of K and how often its ring has gone round
    auto scores = [&]() {
        if (one || gs == 0) ok = ok && tile_wait(bars.k_full(ks), klap & 1);
        if (!ok) return;
        tc_fence_after();
        const uint32_t q = dQ + (one ? 0 : gs) * (C::Q_BYTES >> 4), k = dK + ks * (C::BLK >> 4), d = tmem + is * KB;
#pragma unroll
        for (int i = 0; i < DH / 16; ++i)
            tile_mma_ss(d, q + (i >> 2) * (128 * 128 >> 4) + 2 * (i & 3), k + (i >> 2) * (KB * 128 >> 4) + 2 * (i & 3), idesc_s, i != 0);
        umma_commit(bars.s_full(is));
        if (one || gs == G - 1) {
            umma_commit(bars.k_empty(ks));
            if (++ks == NST) ks = 0, ++klap;
        }
        ++js;
        if (++is == NB) is = 0;
        if (++gs == G) gs = 0;
    };
    while (js < NB && js < jobs && ok) scores();
    int ip = 0, par = 0, g = 0, n = 0, vs = 0, vlap = 0;    // next P V: accumulator, its phase, group, its jobs so far, stage of V
    for (int j = 0; j < jobs && ok; ++j) {
        if (one || g == 0) ok = ok && tile_wait(bars.v_full(vs), vlap & 1);
        ok = ok && tile_wait(bars.p_full(ip), par);
        if (!ok) break;
        tc_fence_after();
        const uint32_t d = tmem + C::TM_O + g * 64 * SUB, a = tmem + ip * KB, v = dV + vs * (C::BLK >> 4);
        tile_mma_ts(d, a, v, idesc_pv, n != 0);
#pragma unroll
        for (int i = 1; i < KB / 16; ++i) tile_mma_ts(d, a + 8 * i, v + i * (2048 >> 4), idesc_pv, 1);
        umma_commit(bars.pv_done(g, n));
        if (one || g == G - 1) {
            umma_commit(bars.v_empty(vs));
            if (++vs == NST) vs = 0, ++vlap;
        }
        if (++ip == NB) ip = 0, par ^= 1;
        if (++g == G) g = 0, ++n;
        if (js < jobs) scores();
    }
    return ok;
}

// Grid: x = split x (heads of keys), y = sequences, z = tiles (of `tiles` x 128 rows: 1 or NG).
template <typename Src, int DH>
__global__ void __launch_bounds__(TILE_THREADS, 1) k_attn_tile(const BatchD B, const AttnRows A, const Src src, int split, int tiles) {
    using C = TileCfg<DH>;
    constexpr int KB = C::KB, SUB = C::SUB, NG = C::NG, NB = C::NB;
    extern __shared__ uint8_t tile_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(tile_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ uint32_t s_tmem;
    __shared__ int s_expired;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % split, s = blockIdx.y, r0 = blockIdx.z * tiles * 128;
    const int2 sr = B.rows(s);
    const int len = src.K.length(B, s);
    const TileBars bars = {smem_u32(smem + C::AT_BAR)};
    if (threadIdx.x == 0) bars.init(C::PW, 4 * NG), s_expired = 0;
    const int rows = min(sr.y, B.max_rows) * A.share;
    if (r0 >= rows) return;                                 // (the whole cluster)
    __syncthreads();
    const int nr = min(tiles * 128, rows - r0);
    // Job j: block j / T, tile and group j % T; with one tile block j, group j % NG.
    const int T = (nr + 127) / 128, G = T == 1 ? NG : T;
    TileWork w;
    w.s = s, w.h = blockIdx.x / split;
    if (warp >= C::SM0) {
        // softmax warps: the row's queries, into the operand of its tile; with one tile, the groups share them out
        // (a row's pieces by neighbouring lanes: a row to a lane took 3000 clocks for three tiles)
        constexpr int CPR = DH / 8, RPI = 32 / CPR;
        const int g = (warp - C::SM0) >> 2, piece = lane % CPR;
        const uint32_t sq = smem_u32(smem + C::AT_Q) + (T == 1 ? 0 : g) * C::Q_BYTES + (piece >> 3) * (128 * 128);
        if (g < G)
            for (int i = T == 1 ? g : 0; i < CPR; i += T == 1 ? NG : 1) {
                const int trow = (warp & 3) * 32 + i * RPI + lane / CPR, r = (T == 1 ? 0 : g * 128) + trow;
                const int2 at = A.split(r0 + min(r, nr - 1));
                const bf16 *q = (const bf16 *)A.q + (long long)(sr.x + at.x) * A.q_stride + (w.h * A.share + at.y) * DH + piece * 8;
                cp_async16(sq + tile_at(trow, piece & 7), q, r < nr ? 16 : 0);
            }
        cp_async_commit();
    }
    {
        const KeyRange first = src.K.range(B, len, sr.y, A.split(r0).x), last = src.K.range(B, len, sr.y, A.split(r0 + nr - 1).x);
        const int all = max(0, (last.hi - first.lo + KB - 1) / KB), per = (all + split - 1) / split;
        w.lo = first.lo + min(all, rank * per) * KB;
        w.nb = max(0, min(all - rank * per, per));
        w.hi = min(last.hi, w.lo + w.nb * KB);
    }
    const int jobs = w.nb * T;
    const bool merge = split > 1 || (T == 1 && jobs >= 2);  // a row's result is in several groups
    uint32_t tmem = 0;
    if (warp >= C::PW) {
        // (the producers are on their way; the others wait for tensor memory)
        if (warp == C::PW) {
            tmem_alloc(smem_u32(&s_tmem), 512);
            tmem_relinquish();
        }
        tc_fence_before();
        asm volatile("bar.sync 2, %0;" ::"n"(TILE_THREADS - 32 * C::PW) : "memory");
        tc_fence_after();
        tmem = s_tmem;
    }
    bool ok = true;

    if (warp < C::SM0) {
        // ---------------- producers ----------------
        if (warp < C::PW && jobs) src.produce(B, w, smem, bars, ok);
        // ---------------- issuer of the products ----------------
        if (warp == C::PW && jobs) {
            // (what the products' operands come from is the same in all lanes, and the compiler has to know it: with operands moved to uniform
            // registers one by one they took 720 clocks a job for 620)
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), base = __shfl_sync(0xffffffffu, smem_u32(smem), 0);
            const int n_jobs = __shfl_sync(0xffffffffu, jobs, 0), n_g = __shfl_sync(0xffffffffu, G, 0);
            const bool one = __shfl_sync(0xffffffffu, T, 0) == 1;
            if (elect_one()) ok = tile_issue<DH>(bars, base, tm, n_jobs, n_g, one);
        }
        if (!ok) s_expired = 1;
    } else {
        // ---------------- softmax: a thread per row ----------------
        const int g = (warp - C::SM0) >> 2, quad = warp & 3, trow = quad * 32 + lane, r = (T == 1 ? 0 : g * 128) + trow;
        const uint32_t lane_off = (uint32_t)(quad * 32) << 16, tO = tmem + C::TM_O + g * 64 * SUB + lane_off;
        const bool some = __any_sync(0xffffffffu, r < nr);             // the warp has rows
        const float c = 1.4426950408889634f * rsqrtf((float)DH) * Src::UP;
        float down = 0.f, most = (float)(1ull << TILE_GROWTH_KV4);     // (4-bit values are below 1 here)
        if constexpr (!Src::KV4) {
            const int bits = sum_bits(TILE_GROWTH, (src.K.n_keys + KB - 1) / KB);
            down = (float)bits, most = exp2f(TILE_GROWTH - down);      // (read as operands from the arguments: cross_streams8 129 us for 127)
        }
        const KeyRange kr = src.K.range(B, len, sr.y, A.split(r0 + min(r, nr - 1)).x);
        cp_async_wait<0>();
        tile_publish(bars.q_full());
        float m = -INFINITY, l = 0.f;                                  // m: reference, in units of scores
        int n = 0;                                                     // the group's jobs so far
        for (int j = g; g < G && j < jobs; j += G, ++n) {
            const int b = T == 1 ? j : n, buf = j % NB;
            const uint32_t tS = tmem + buf * KB + lane_off;
            ok = ok && tile_wait2(bars.m_full(b % C::NM), (b / C::NM) & 1, bars.s_full(buf), (j / NB) & 1);
            __syncwarp();
            tc_fence_after();
            if (some) {                                                // (of rows that are not there P may be anything)
                float xa[16];
                tmem_ld16(tS, reinterpret_cast<uint32_t *>(xa));       // (of use where the fast path is taken)
                const uint4 mask = *reinterpret_cast<const uint4 *>(smem + C::AT_MASK + b % C::NM * 32);
                const uint4 bad = *reinterpret_cast<const uint4 *>(smem + C::AT_MASK + b % C::NM * 32 + 16);
                const int p0 = w.lo + b * KB;
                const bool whole = (mask.x & mask.y) == 0xffffffffu && (mask.z & C::M2) == C::M2 && !(bad.x | bad.y | (C::M2 ? bad.z : 0u)) &&
                                   p0 >= kr.lo && p0 + KB <= kr.hi;
                const bool all_whole = __all_sync(0xffffffffu, whole);
                uint32_t seen[3] = {0xffffffffu, 0xffffffffu, 0xffffffffu}, any = 1;
                if (!all_whole) {
                    const uint32_t there[3] = {mask.x, mask.y, mask.z}, bads[3] = {bad.x, bad.y, bad.z};
                    const int a = kr.lo - p0, e = kr.hi - p0;          // keys a .. e - 1 of the block
                    any = 0;
#pragma unroll
                    for (int k = 0; k < (KB + 31) / 32; ++k) {
                        const int a1 = min(max(a - 32 * k, 0), 32), e1 = min(max(e - 32 * k, 0), 32);
                        seen[k] = (e1 == 32 ? 0xffffffffu : (1u << e1) - 1) & ~(a1 == 32 ? 0xffffffffu : (1u << a1) - 1) & there[k];
                        any |= seen[k];
                        if (seen[k] & bads[k]) l = NAN;                // the row sees a value that is not finite
                    }
                }
                if (__any_sync(0xffffffffu, m == -INFINITY)) {
                    // a row without m (nothing has been summed for it): the largest of the first scores will do, if it sees one of them
                    tmem_ld_wait();
                    loaded16(xa);
                    float top = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 16; ++e) top = fmaxf(top, seen[0] >> e & 1 ? xa[e] : -INFINITY);
                    if (m == -INFINITY) m = top;
                }
                bool done = false;
                if (__all_sync(0xffffffffu, m != -INFINITY || !any))
                    done = all_whole ? tile_fast<DH, false>(tS, xa, seen, c, down, most, m, l) : tile_fast<DH, true>(tS, xa, seen, c, down, most, m, l);
                if (!done) {
                    tmem_ld_wait();
                    tile_slow<DH>(tS, tO, seen, c, down, n, bars.pv_done(g, n - 1), m, l, ok);
                }
                tmem_st_wait();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bars.p_full(buf));
        }
        if (n) ok = ok && tile_wait(bars.pv_done(g, n - 1), ((n - 1) >> 1) & 1);
        __syncwarp();
        tc_fence_after();
        if (!ok) s_expired = 1;
        if (merge) asm volatile("bar.sync 1, %0;" ::"n"(NG * 128) : "memory");    // queries and rings are at rest
        const int2 at = A.split(r0 + r);
        bf16 *out = (bf16 *)A.out + ((long long)(sr.x + at.x) * A.heads + w.h * A.share + at.y) * DH;
        const float expired = s_expired || !ok ? NAN : 0.f;
        if (merge ? g < G : some && (T > 1 ? g < T : g == 0)) {
            const float inv = (l == 0.f ? 0.f : Src::UP / l) + expired;
            uint8_t *state = smem + g * C::STATE;
#pragma unroll 1
            for (int i = 0; i < DH; i += 32) {
                float o[32];
                tmem_ld32(tO + i, reinterpret_cast<uint32_t *>(o));
                tmem_ld_wait();
                loaded32(o);
                if (merge) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        *reinterpret_cast<float4 *>(state + ((i / 4 + e) * 128 + trow) * 16) =
                            n ? make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
                } else if (r < nr) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t v[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) v[u] = n ? bf16_pair(o[8 * e + 2 * u] * inv, o[8 * e + 2 * u + 1] * inv) : bf16_pair(expired, expired);
                        *reinterpret_cast<uint4 *>(out + i + 8 * e) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                }
            }
            if (merge) *reinterpret_cast<float2 *>(state + 128 * DH * 4 + trow * 8) = make_float2(n ? m * c : -INFINITY, l + expired);
        }
        if (merge && T == 1) {
            // The groups' states of the one tile become one, over the first (a third or half of the columns to a group), or the result.  They count
            // in the groups' order; one without scores has zeros, and none is left out: a value that is not finite counts however small its factor.
            asm volatile("bar.sync 1, %0;" ::"n"(NG * 128) : "memory");
            float f[NG], mx = -INFINITY, sum = 0.f;
            float2 ml[NG];
#pragma unroll
            for (int k = 0; k < NG; ++k) ml[k] = *reinterpret_cast<const float2 *>(smem + k * C::STATE + 128 * DH * 4 + trow * 8), mx = fmaxf(mx, ml[k].x);
#pragma unroll
            for (int k = 0; k < NG; ++k) f[k] = ml[k].x == -INFINITY ? 0.f : few_exp2(ml[k].x - mx), sum = fmaf(ml[k].y, f[k], sum);
            const float inv = sum == 0.f ? 0.f : Src::UP / sum;
            for (int i = g; i < DH / 8; i += NG) {
                float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < NG; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float4 o = *reinterpret_cast<const float4 *>(smem + k * C::STATE + ((2 * i + e) * 128 + trow) * 16);
                        v[4 * e] = fmaf(o.x, f[k], v[4 * e]), v[4 * e + 1] = fmaf(o.y, f[k], v[4 * e + 1]);
                        v[4 * e + 2] = fmaf(o.z, f[k], v[4 * e + 2]), v[4 * e + 3] = fmaf(o.w, f[k], v[4 * e + 3]);
                    }
                if (split > 1) {
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        *reinterpret_cast<float4 *>(smem + ((2 * i + e) * 128 + trow) * 16) = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
                } else if (r < nr) {
                    *reinterpret_cast<uint4 *>(out + 8 * i) = make_uint4(bf16_pair(v[0] * inv, v[1] * inv), bf16_pair(v[2] * inv, v[3] * inv),
                                                                         bf16_pair(v[4] * inv, v[5] * inv), bf16_pair(v[6] * inv, v[7] * inv));
                }
            }
            if (g == 0) *reinterpret_cast<float2 *>(smem + NG * C::STATE + trow * 8) = make_float2(mx, sum);
        }
    }
    __syncwarp();
    cp_async_wait<0>();
    tc_fence_before();
    if (split > 1) {
        cluster_sync_all();
        // The CTAs' states.  Row words of four columns, 8 rows x 4 of them to a warp (32 bytes of a row, and every bank once); each CTA of a
        // cluster takes every split-th of these.  A word's loads are in flight together (one after the other they were 5 to 9 us of a call).
        const uint32_t st0 = smem_u32(smem);
        const int n_words = T * 16 * (DH / 16);
        for (int i = rank * 16 + warp; i < n_words; i += split * 16) {
            const int tile = i / (16 * (DH / 16)), in = i % (16 * (DH / 16));
            const int trow = (in / (DH / 16)) * 8 + (lane & 7), col4 = (in % (DH / 16)) * 4 + (lane >> 3), r = tile * 128 + trow;
            if (r >= nr) continue;
            const uint32_t at_ml = st0 + (T == 1 ? NG * C::STATE : tile * C::STATE + 128 * DH * 4) + trow * 8;
            const uint32_t at_o = st0 + tile * C::STATE + (col4 * 128 + trow) * 16;
            float2 ml[TILE_SPLIT];
            float4 o[TILE_SPLIT];
            float mx = -INFINITY, sum = 0.f;
#pragma unroll
            for (int k = 0; k < TILE_SPLIT; ++k) {
                ml[k] = make_float2(-INFINITY, 0.f), o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (k < split) ml[k] = ld_cluster_f2(cluster_map(at_ml, k)), o[k] = ld_cluster_f4(cluster_map(at_o, k));
            }
#pragma unroll
            for (int k = 0; k < TILE_SPLIT; ++k) mx = fmaxf(mx, ml[k].x);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int k = 0; k < TILE_SPLIT; ++k) {
                const float f = ml[k].x == -INFINITY ? 0.f : few_exp2(ml[k].x - mx);
                sum = fmaf(ml[k].y, f, sum);
                v.x = fmaf(o[k].x, f, v.x), v.y = fmaf(o[k].y, f, v.y), v.z = fmaf(o[k].z, f, v.z), v.w = fmaf(o[k].w, f, v.w);
            }
            const float inv = sum == 0.f ? 0.f : Src::UP / sum;
            const int2 at = A.split(r0 + r);
            bf16 *out = (bf16 *)A.out + ((long long)(sr.x + at.x) * A.heads + w.h * A.share + at.y) * DH + col4 * 4;
            *reinterpret_cast<uint2 *>(out) = make_uint2(bf16_pair(v.x * inv, v.y * inv), bf16_pair(v.z * inv, v.w * inv));
        }
        cluster_sync_all();                                 // nobody leaves while its state is read
    } else {
        __syncthreads();
    }
    if (warp == C::PW) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// How the work is laid out: tiles of a CTA (1 or NG), CTAs of a cluster that their keys are split over.
struct TilePlan {
    int tiles, split;
};
// Times in clocks, as measured with all SMs busy: a job (a key block of a tile) takes a CTA's pipes JOB, a block its producers LOAD (few rows
// are bound by that); a CTA has a beginning and an end (FIXED, and MERGE where there are states to merge); waves go by how many clusters the
// device holds at once.  16 heads x 64, 336 rows behind 5376 keys in 4-bit pages: a tile to a CTA in 2 pieces 42.7 us, three tiles in 1, 4, 6 and
// 8 (two waves) 108, 42.7, 35.2, 65; 512 encoder states: a tile in 1, 2 and 4 pieces 17.7, 15.7, 29.7, three tiles in 6 20.7.
template <int DH, bool KV4, typename F> static TilePlan tile_plan(long long units, long long rows, long long keys, int n_sm, F &&clusters) {
    constexpr int kb = TileCfg<DH>::KB, ng = TileCfg<DH>::NG;
    constexpr long long JOB = (DH == 128 ? 17 : 10) * kb, LOAD = (DH == 128 ? (KV4 ? 34 : 37) : KV4 ? 27 : 19) * kb, FIXED = 9000, MERGE = 3000;
    const long long blocks = (keys + kb - 1) / kb, t1 = (rows + 127) / 128;
    TilePlan best = {1, 1};
    long long least = -1;
    for (int tiles = 1; tiles <= ng; tiles += ng - 1)
        for (int split = 1; split <= TILE_SPLIT; ++split) {
            const long long fit = split == 1 ? n_sm : clusters(split);
            if (fit < 1 || (split > 1 && blocks < 2 * split)) break;
            const long long mine = t1 < tiles ? t1 : tiles, job = JOB * mine, per = (blocks + split - 1) / split;
            const long long cost = (units * ((t1 + tiles - 1) / tiles) + fit - 1) / fit *
                                   (per * (job > LOAD ? job : LOAD) + FIXED + (split > 1 || mine == 1 ? MERGE : 0));
            if (least < 0 || cost < least) least = cost, best = {tiles, split};
        }
    return best;
}

template <typename Src, int DH>
static int launch_attn_tile(const BatchD &B, const AttnRows &A, const Src &src, int kv_heads, long long keys, int dev, int n_sm, cudaStream_t st) {
    using C = TileCfg<DH>;
    auto kern = k_attn_tile<Src, DH>;
    static OncePerDevice once;
    static int fit[NFD_PAGED_DEVICES][TILE_SPLIT + 1];
    if (!once.run(dev, [&] {
            if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) != cudaSuccess) return false;
            for (int split = 2; split <= TILE_SPLIT; ++split) fit[dev][split] = clusters_that_fit(kern, split, TILE_THREADS, C::SMEM);
            return true;
        }))
        return NFD_E_CUDA;
    const long long rows = (long long)B.max_rows * A.share;
    const TilePlan pl = tile_plan<DH, Src::KV4>((long long)kv_heads * B.n_seqs, rows, keys, n_sm, [&](int k) { return fit[dev][k]; });
    const long long nz = (rows + 128 * pl.tiles - 1) / (128 * pl.tiles);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kv_heads * pl.split, B.n_seqs, (unsigned)nz), cfg.blockDim = dim3(TILE_THREADS), cfg.dynamicSmemBytes = C::SMEM, cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension, at.val.clusterDim.x = pl.split, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at, cfg.numAttrs = pl.split > 1;
    if (cudaLaunchKernelEx(&cfg, kern, B, A, src, pl.split, pl.tiles) != cudaSuccess) {
        cudaGetLastError();
        return NFD_E_CUDA;
    }
    return NFD_OK;
}
