// Attention of a few rows to many keys, on 4-bit pages, bf16 pages, bf16 states or the rows of packed prompts: single tokens, short speculations, a row or two of a
// decoder against an encoder's states.
//
// A unit of work is (sequence, head of keys, up to 8 NR rows: rows x heads that share it).  The bound is the stream of K and V, and with
// 4-bit pages the instructions that make bf16 numbers of codes; a unit is split over the CTAs of a
// cluster and their warps, each of which takes chunks of KC keys in turn, with a ring of its own in shared memory that
// cp.async fills NST - 1 chunks ahead, an online softmax of its own, and no barrier until the end.  Then the warps of a CTA merge through
// shared memory and the CTAs of a cluster through distributed shared memory, in a fixed order, each writing its share of the result: no
// working memory in HBM, one launch.
//
// Both products have the keys' operand on the 16-wide side of mma.m16n8k16 and the rows on the 8-wide side:
//     S^T = K Q^T   (16 keys x 8 rows),   O^T += V^T P^T   (16 dims x 8 rows)
// so that what a key costs does not grow with the 16 rows of a tile (with the rows on that side: twice the products and twice the registers
// for rows that are not there).  P^T changes sides by movmatrix.  The inner index of either product may be permuted as long as both of its
// operands are, so that a lane's share of a key is a run of its row (for S) and a lane's share of a value a run of dims
// (for O); 4-bit codes become bf16 numbers in registers (Kv4Scale).  P is rounded to one bf16 number, as in the kernel for many rows.
// Measured: one row, 16 heads x 64, behind 5712 tokens in 4-bit pages 10.0 us (pieces, merge and launch; 6.6 MB); eight sequences of up to 32768
// tokens, 24 heads on 8 x 128, 84.5 us (185 MB, 2.2 TB/s: nothing is saturated, 48 % of the issue slots, 28 % of the copy rate; latency, and lengths that
// differ); bf16 states, eight rows, 16 heads x 64 against 4096 25.4 us (134 MB, 5.3 TB/s);
// bf16 pages, 16 sequences of one row behind up to 16384 tokens, 24 heads on 8 x 128, 128 to 139 us (701 MB, 5.0 to 5.5 TB/s).
#pragma once
#include "nfd_attn_rows.cuh"
#include "nfd_sm100.cuh"

#define FEW_WARPS 8
#define FEW_SORTED 128              // sequences that are taken longest first, at most
#define FEW_PIECE (768 << 10)       // of a long sequence, at least
// Rows of a unit that this kernel takes.  Measured against the kernel for many rows, us: 16 heads x 64 behind 5712 tokens in 4-bit pages, 24, 64 and
// 100 rows 16.9, 17.5, 26.2 here and 21.2, 21.7, 22.6 there; 4 x 16 heads against 512 states 8.3, 9.5, 17.4 and 10.3, 10.5, 11.4;
// head dimension 128, eight sequences of 4 heads of keys behind 8192, 32 rows 46.4 and 50.1, 96 rows 151 and 51.
constexpr int few_most(int dh) { return dh == 128 ? 32 : 64; }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void *src, uint32_t bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void *src, uint32_t bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int n> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(n) : "memory"); }

__device__ __forceinline__ void mma_bf16(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// an 8 x 8 matrix of 16-bit numbers, a pair of a row to a lane, the other way round
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float few_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A warp's chunk of keys in shared memory, for 4-bit pages: codes of K and V, their words, and which keys are there.
template <int DH> struct FewKv4 {
    static constexpr bool KV4 = true, RANGES = false, SORTED = false;
    static constexpr int WARPS = FEW_WARPS;
    static constexpr float UP = KV4_UP;                     // what scores and results are to be multiplied by
    static __device__ __forceinline__ float down() { return 0.f; }        // taken off the exponents (sum_bits; values below 1 need nothing)
    static constexpr int KC = 32;
    static constexpr int NST = 3;                           // (with 4, head dimension 128 leaves one CTA to an SM: 138 us for 101)
    static constexpr int RB = DH / 2;                       // bytes of a row of codes
    static constexpr int WB = DH == 128 ? 8 : 4;            // bytes of a key's words (DH 32: a word and its neighbour)
    static constexpr int PR = RB / 16;                      // 16-byte pieces of a row
    static constexpr int STAGE = 2 * KC * (RB + WB) + 16;
    Kv4Keys<DH> K;
    // Key `lane` of the chunk that is looked up next: entry of the table, offset in the page; how far they move from chunk to chunk (additions
    // instead of two divisions a chunk).
    const int *table;
    int pg, off, dq, dr;
    long long place;                                        // of key `lane` of the chunk that is filled next

    __device__ __forceinline__ void start(const BatchD &B, int s, int h, int first, int step) {
        const int P = K.P.page_tokens, L = B.table_len, p = first + (threadIdx.x & 31);
        table = B.table + (size_t)s * L;
        off = p % P, pg = p / P % L, dr = step % P, dq = step / P % L;
    }
    __device__ __forceinline__ void look_up(const BatchD &B, int s, int h, int base, int hi) {
        const int P = K.P.page_tokens, L = B.table_len;
        place = -1;
        if (base + (int)(threadIdx.x & 31) < hi) {
            const int page = __ldg(table + pg);
            if ((unsigned)page < (unsigned)K.P.n_pages) place = ((long long)page * K.P.heads + h) * P + off;
        }
        off += dr, pg += dq;
        if (off >= P) off -= P, ++pg;
        if (pg >= L) pg -= L;
    }
    // the copies of a chunk; its places have been looked up
    __device__ __forceinline__ void fill(uint8_t *stage, uint32_t st, const BatchD &B, int s, int h, int base, int hi) {
        const int lane = threadIdx.x & 31;
        uint32_t *meta = reinterpret_cast<uint32_t *>(stage + 2 * KC * (RB + WB));
        const uint32_t there = __ballot_sync(0xffffffffu, place >= 0), odd = __ballot_sync(0xffffffffu, place & 1);
        if (lane == 0) meta[0] = there, meta[1] = odd;
#pragma unroll
        for (int j = 0; j < PR; ++j) {
            const int src = j * (32 / PR) + lane / PR, piece = lane % PR;
            const long long at = __shfl_sync(0xffffffffu, place, src);
            const size_t off = at >= 0 ? (size_t)at * RB + piece * 16 : 0;
            const uint32_t d = st + src * RB + piece * 16, n = at >= 0 ? 16 : 0;
            cp_async16(d, (const uint8_t *)K.P.k + off, n);
            cp_async16(d + KC * RB, (const uint8_t *)K.P.v + off, n);
        }
        const long long at = place >= 0 ? place : 0;
        const uint32_t d = st + 2 * KC * RB + lane * WB, n = place >= 0;
        if (DH == 128) {
            cp_async8(d, K.P.k_scale + at * 4, n * 8);
            cp_async8(d + KC * WB, K.P.v_scale + at * 4, n * 8);
        } else if (DH == 64) {
            cp_async4(d, K.P.k_scale + at * 2, n * 4);
            cp_async4(d + KC * WB, K.P.v_scale + at * 2, n * 4);
        } else {
            // one word a key: the aligned pair it is in, or, where it is the pair's first, only itself
            const uint32_t m = n ? 2 + 2 * (uint32_t)(at & 1) : 0;
            cp_async4(d, K.P.k_scale + (at & ~1LL), m);
            cp_async4(d + KC * WB, K.P.v_scale + (at & ~1LL), m);
        }
    }
    static __device__ __forceinline__ uint32_t mask(const uint8_t *stage) { return *reinterpret_cast<const uint32_t *>(stage + 2 * KC * (RB + WB)); }
    // Values whose step is not finite become zeros (a product with the 0 of a row that does not see them would be NaN); a bit for each
    // of their keys.
    static __device__ __forceinline__ uint32_t take_out(uint8_t *stage) {
        const int lane = threadIdx.x & 31;
        uint32_t *w = reinterpret_cast<uint32_t *>(stage + 2 * KC * RB + KC * WB + lane * WB);
        bool mine = false;
#pragma unroll
        for (int j = 0; j < WB / 4; ++j) {
            const uint32_t v = w[j];
            const bool b0 = kv4_not_finite(v), b1 = kv4_not_finite(v >> 16);
            if (DH == 32) mine |= reinterpret_cast<const uint32_t *>(stage + 2 * KC * (RB + WB))[1] >> lane & 1 ? b1 : b0;
            else mine |= b0 || b1;
        }
        const uint32_t bad = __ballot_sync(0xffffffffu, mine);
        if (bad) {
            if (mine)
                for (int j = 0; j < WB / 4; ++j) w[j] = 0;
            __syncwarp();
        }
        return bad;
    }
    static __device__ __forceinline__ uint32_t word(const uint8_t *w, int key, int group, const uint8_t *stage) {
        if (DH == 32) {
            const uint32_t *meta = reinterpret_cast<const uint32_t *>(stage + 2 * KC * (RB + WB));
            return *reinterpret_cast<const uint16_t *>(w + key * WB + 2 * (meta[1] >> key & 1));
        }
        return *reinterpret_cast<const uint16_t *>(w + key * WB + 2 * group);
    }
    // dims of Q that go with this lane's pair i of product step st
    static __device__ __forceinline__ int q_dim(int step, int c) { return c * (DH / 4) + 4 * step; }
    // B operand of S for the key of this lane: DH / 16 steps of two registers
    static __device__ __forceinline__ void k_frag(const uint8_t *stage, int key, int c, uint32_t *b) {
        constexpr int NW = DH / 32;                         // words of codes of a lane
        const uint32_t *src = reinterpret_cast<const uint32_t *>(stage + key * RB) + c * NW;
        uint32_t w[NW];
        if constexpr (NW == 4) {
            const uint4 v = *reinterpret_cast<const uint4 *>(src);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else if constexpr (NW == 2) {
            const uint2 v = *reinterpret_cast<const uint2 *>(src);
            w[0] = v.x, w[1] = v.y;
        } else {
            w[0] = *src;
        }
        const uint32_t sc = word(stage + 2 * KC * RB, key, c * (DH / 4) / 32, stage);
        const Kv4Scale scale(sc, sc, true);
#pragma unroll
        for (int i = 0; i < NW; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) b[4 * i + j] = scale.pair(w[i], j);
    }
    // dims of the result that this lane's n-th column of product tile t is
    static __device__ __forceinline__ int o_dim(int t, int n) {
        if (DH == 32) return 8 * (n >> 1) + 2 * t + (n & 1);
        return (n * (DH / 64) + t / 8) * 8 + 2 * (t & 3) + ((t >> 2) & 1);
    }
    // B operand of O for keys k0 (+4): DH / 8 tiles, one register each
    static __device__ __forceinline__ void v_frag(const uint8_t *stage, int k0, int n, uint32_t *b) {
        const uint8_t *v = stage + KC * RB, *w = stage + 2 * KC * RB + KC * WB;
        const int g = n * (DH / 8) / 32;
        const Kv4Scale scale(word(w, k0, g, stage), word(w, k0 + 4, g, stage), false);    // (take_out; checked, 3 to 5 % of a call)
        if constexpr (DH == 32) {
            const uint32_t x = *reinterpret_cast<const uint16_t *>(v + k0 * RB + n * 2) |
                               (uint32_t)*reinterpret_cast<const uint16_t *>(v + (k0 + 4) * RB + n * 2) << 16;
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = scale.pair(x, j);
        } else {
            constexpr int NW = DH / 64;
            uint32_t x[NW], y[NW];
            if constexpr (NW == 2) {
                const uint2 p = *reinterpret_cast<const uint2 *>(v + k0 * RB + n * 8), q = *reinterpret_cast<const uint2 *>(v + (k0 + 4) * RB + n * 8);
                x[0] = p.x, x[1] = p.y, y[0] = q.x, y[1] = q.y;
            } else {
                x[0] = *reinterpret_cast<const uint32_t *>(v + k0 * RB + n * 4), y[0] = *reinterpret_cast<const uint32_t *>(v + (k0 + 4) * RB + n * 4);
            }
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                const uint32_t even = __byte_perm(x[i], y[i], 0x5410), odd = __byte_perm(x[i], y[i], 0x7632);
#pragma unroll
                for (int j = 0; j < 4; ++j) b[8 * i + j] = scale.pair(even, j), b[8 * i + 4 + j] = scale.pair(odd, j);
            }
        }
    }
};

// The same for bf16 numbers.  Rows are swizzled in 16-byte pieces so that neither operand's reads meet in a bank.
template <int DH> struct FewBf16 {
    static constexpr bool KV4 = false;
    static constexpr float UP = 1.0f;
    static constexpr int KC = DH == 32 ? 32 : 16;
    static constexpr int NST = DH == 128 ? 3 : 4;
    static constexpr int RB = 2 * DH, PR = RB / 16;
    static constexpr int STAGE = 2 * KC * RB + 16;
    float bits;
    __device__ __forceinline__ float down() const { return bits; }
    static __device__ __forceinline__ uint32_t at_k(int key, int piece) { return key * RB + (piece ^ (key & 7 & (PR - 1))) * 16; }
    static __device__ __forceinline__ uint32_t at_v(int key, int piece) { return KC * RB + key * RB + (piece ^ (2 * key & 7 & (PR - 1))) * 16; }
    static __device__ __forceinline__ uint32_t mask(const uint8_t *stage) { return *reinterpret_cast<const uint32_t *>(stage + 2 * KC * RB); }
    static __device__ __forceinline__ uint32_t take_out(uint8_t *) { return 0; }
    static __device__ __forceinline__ int q_dim(int step, int c) { return 8 * (c + 4 * (step / 2)) + 4 * (step % 2); }
    static __device__ __forceinline__ void k_frag(const uint8_t *stage, int key, int c, uint32_t *b) {
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) {
            const uint4 v = *reinterpret_cast<const uint4 *>(stage + at_k(key, c + 4 * j));
            b[4 * j] = v.x, b[4 * j + 1] = v.y, b[4 * j + 2] = v.z, b[4 * j + 3] = v.w;
        }
    }
    static __device__ __forceinline__ int o_dim(int t, int n) { return DH == 32 ? 4 * n + t : 8 * (n + 8 * (t / 8)) + t % 8; }
    static __device__ __forceinline__ void v_frag(const uint8_t *stage, int k0, int n, uint32_t *b) {
        if constexpr (DH == 32) {
            const uint2 x = *reinterpret_cast<const uint2 *>(stage + at_v(k0, n >> 1) + 8 * (n & 1));
            const uint2 y = *reinterpret_cast<const uint2 *>(stage + at_v(k0 + 4, n >> 1) + 8 * (n & 1));
            b[0] = __byte_perm(x.x, y.x, 0x5410), b[1] = __byte_perm(x.x, y.x, 0x7632);
            b[2] = __byte_perm(x.y, y.y, 0x5410), b[3] = __byte_perm(x.y, y.y, 0x7632);
        } else {
#pragma unroll
            for (int i = 0; i < DH / 64; ++i) {
                const uint4 x = *reinterpret_cast<const uint4 *>(stage + at_v(k0, n + 8 * i)), y = *reinterpret_cast<const uint4 *>(stage + at_v(k0 + 4, n + 8 * i));
                const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    b[8 * i + 2 * j] = __byte_perm(xs[j], ys[j], 0x5410), b[8 * i + 2 * j + 1] = __byte_perm(xs[j], ys[j], 0x7632);
            }
        }
    }
};

// States of an encoder: all rows see the same keys.
template <int DH> struct FewStates : FewBf16<DH> {
    using F = FewBf16<DH>;
    static constexpr bool RANGES = false, SORTED = false;
    static constexpr int WARPS = FEW_WARPS;
    static constexpr int KC = F::KC, RB = F::RB, PR = F::PR;
    StateKeys<bf16, DH> K;
    uint32_t there;                                         // of the chunk that is filled next
    __device__ __forceinline__ void start(const BatchD &, int, int, int, int) {}
    __device__ __forceinline__ void look_up(const BatchD &B, int s, int h, int base, int hi) {
        const int p = base + (threadIdx.x & 31);
        bool t = p < hi && (threadIdx.x & 31) < KC;
        if (t && K.mask) t = K.mask[(size_t)s * K.n_keys + p];
        there = __ballot_sync(0xffffffffu, t);
    }
    __device__ __forceinline__ void fill(uint8_t *stage, uint32_t st, const BatchD &B, int s, int h, int base, int hi) {
        const int lane = threadIdx.x & 31;
        if (lane == 0) *reinterpret_cast<uint32_t *>(stage + 2 * KC * RB) = there;
        const long long seq = s * K.seq_stride + h * K.head_stride;
#pragma unroll
        for (int j = 0; j < KC * PR / 32; ++j) {
            const int key = (j * 32 + lane) / PR, piece = lane % PR;
            const bool t = there >> key & 1;
            const long long off = t ? seq + (base + key) * K.key_stride + piece * 8 : 0;
            cp_async16(st + F::at_k(key, piece), K.k + off, t ? 16 : 0);
            cp_async16(st + F::at_v(key, piece), K.v + off, t ? 16 : 0);
        }
    }
};

// Bf16 pages and the rows of packed prompts: the rows of a unit do not all see the same keys, and what a row does not see may be anything.
template <typename Keys, int DH> struct FewRows : FewBf16<DH> {
    using F = FewBf16<DH>;
    static constexpr bool RANGES = true, SORTED = Keys::HOLES;         // (of packed prompts no row sees more than a few)
    // two CTAs to an SM: one merges while the other streams (with eight warps 16 sequences of up to 16384 tokens, 24 heads on 8 x 128, took 178, 176, 170 and
    // 199 us in 1, 2, 4 and 8 pieces, where few_split_rows has its figures)
    static constexpr int WARPS = 4;
    static constexpr int KC = F::KC, RB = F::RB, PR = F::PR;
    Keys K;
    typename Keys::Cursor cur;
    long long place;                                        // of key `lane` of the chunk that is filled next
    __device__ __forceinline__ void start(const BatchD &B, int s, int h, int first, int step) { cur = K.cursor(B, s, B.rows(s).x, first + (threadIdx.x & 31), step); }
    __device__ __forceinline__ void look_up(const BatchD &B, int s, int h, int base, int hi) {
        const int lane = threadIdx.x & 31;
        place = K.next(cur, B, h, lane < KC && base + lane < hi);
    }
    __device__ __forceinline__ void fill(uint8_t *stage, uint32_t st, const BatchD &B, int s, int h, int base, int hi) {
        const int lane = threadIdx.x & 31;
        const uint32_t there = __ballot_sync(0xffffffffu, place >= 0);
        if (lane == 0) *reinterpret_cast<uint32_t *>(stage + 2 * KC * RB) = there;
#pragma unroll
        for (int j = 0; j < KC * PR / 32; ++j) {
            const int key = (j * 32 + lane) / PR, piece = lane % PR;
            const long long r = __shfl_sync(0xffffffffu, place, key);
            cp_async16(st + F::at_k(key, piece), K.k_row(r < 0 ? 0 : r, h) + piece * 8, r < 0 ? 0 : 16);
            cp_async16(st + F::at_v(key, piece), K.v_row(r < 0 ? 0 : r, h) + piece * 8, r < 0 ? 0 : 16);
        }
    }
    // Values of a chunk that are not finite become zeros (a product with the 0 of a row that does not see them would be NaN), after add(key, dim,
    // value) has been called for each of the dims of this lane: o_dim(t, n) of all t.
    template <typename Add> static __device__ __forceinline__ void take_out_values(uint8_t *stage, int n, Add &&add) {
        const int lane = threadIdx.x & 31;
        uint32_t keys = 0;
#pragma unroll 1
        for (int j = 0; j < KC * PR / 32; ++j) {
            const int key = (j * 32 + lane) / PR;
            const uint4 x = *reinterpret_cast<const uint4 *>(stage + F::at_v(key, lane % PR));
            if ((finite_bits(x.x) & finite_bits(x.y) & finite_bits(x.z) & finite_bits(x.w)) != 0xffffffffu) keys |= 1u << key;
        }
        keys = __reduce_or_sync(0xffffffffu, keys);
        if (!keys) return;
        for (uint32_t left = keys; left; left &= left - 1) {
            const int key = __ffs(left) - 1;
#pragma unroll 1
            for (int t = 0; t < DH / 8; ++t) {
                const int d = F::o_dim(t, n);
                const uint32_t x = *reinterpret_cast<const uint16_t *>(stage + F::at_v(key, d / 8) + d % 8 * 2);
                if ((x & 0x7F80u) == 0x7F80u) add(key, t, __uint_as_float(x << 16));
            }
        }
        __syncwarp();
#pragma unroll 1
        for (int j = 0; j < KC * PR / 32; ++j) {
            uint4 *v = reinterpret_cast<uint4 *>(stage + F::at_v((j * 32 + lane) / PR, lane % PR));
            const uint4 x = *v;
            *v = make_uint4(x.x & finite_bits(x.x), x.y & finite_bits(x.y), x.z & finite_bits(x.z), x.w & finite_bits(x.w));
        }
        __syncwarp();
    }
};

template <typename Src, int DH, int NR> struct FewCfg {
    static constexpr int ROWS = 8 * NR;
    static constexpr int STATE = ROWS * (DH + 2) * 4;                             // O, m, l of a warp or a CTA
    static constexpr int RING = (Src::NST * Src::STAGE + 15) / 16 * 16;
    static constexpr int WARP = RING > STATE ? RING : STATE;                      // a warp's ring, then its state
    static constexpr int SMEM = Src::WARPS * WARP + STATE;
    static_assert(SMEM <= 232448 - 1024, "shared memory of a CTA");
};

// The sequence of place `i` where they go by the tokens that they hold, the longest first: what takes longest begins first.  (For a whole warp; own: room for
// FEW_SORTED words that nobody else uses.  16 sequences of up to 16384 tokens, 24 heads on 8 x 128, 157 -> 139 us.)
static __device__ __forceinline__ int few_longest(const BatchD &B, int i, uint32_t *own) {
    if (B.n_seqs == 1 || B.n_seqs > FEW_SORTED) return i;
    constexpr int N = FEW_SORTED / 32;
    const int lane = threadIdx.x & 31;
    uint32_t word[N];                                       // length (as far as 24 bits go) and sequence: no two alike
    int most = 0, least = INT_MAX, before[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        word[k] = before[k] = 0;
        if (k * 32 + lane < B.n_seqs) {
            const int n = B.tokens(k * 32 + lane);
            most = max(most, n), least = min(least, n), word[k] = (uint32_t)min(n, 1 << 24) * FEW_SORTED + FEW_SORTED - 1 - (k * 32 + lane);
        }
        own[k * 32 + lane] = word[k];
    }
    __syncwarp();                                           // (before the words are read, or, where all are as long, overwritten)
    if (__reduce_max_sync(0xffffffffu, most) == __reduce_min_sync(0xffffffffu, least)) return i;
#pragma unroll 4
    for (int j = 0; j < B.n_seqs; j += 4) {
        const uint4 w = *reinterpret_cast<const uint4 *>(own + j);          // (zeros behind the last)
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k * 32 < B.n_seqs) before[k] += (w.x > word[k]) + (w.y > word[k]) + (w.z > word[k]) + (w.w > word[k]);
    }
    __syncwarp();                                           // (the words may be overwritten)
    int s = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t here = __ballot_sync(0xffffffffu, k * 32 + lane < B.n_seqs && before[k] == i);
        if (here) s = k * 32 + __ffs(here) - 1;
    }
    return s;
}

// grid: (CTAs of a cluster x heads of keys, sequences, tiles of 8 NR rows).  (States: their ring leaves one CTA to an SM, and so it may have all registers: not
// told so, the compiler spilled in 80.)
template <typename Src, int DH, int NR>
__global__ void __launch_bounds__(32 * Src::WARPS, Src::KV4 ? 0 : Src::RANGES ? 2 : 1) k_attn_few(const BatchD B, const AttnRows A, Src src, int split) {
    using F = FewCfg<Src, DH, NR>;
    constexpr int KC = Src::KC, NST = Src::NST, NS = DH / 16, KT = KC / 16, ROWS = F::ROWS;
    // S in two chains of products for a single tile of rows (states, eight rows against 4096 26.9 us for 25.9; with 4-bit pages and head
    // dimension 64 it gains nothing)
    constexpr bool TWO = NR == 1 && NS >= 4 && (!Src::KV4 || DH == 128);
    extern __shared__ __align__(16) uint8_t few_smem[];
    __shared__ int2 s_range[ROWS];                                                // keys that a row sees
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = lane & 3, n = lane >> 2;
    uint8_t *ring = few_smem + warp * F::WARP;
    int s = blockIdx.y;
    if constexpr (Src::SORTED) s = few_longest(B, s, reinterpret_cast<uint32_t *>(ring));
    const int rank = blockIdx.x % split, h = blockIdx.x / split, r0 = blockIdx.z * ROWS;
    const int2 sr = B.rows(s);
    const int len = src.K.length(B, s);
    const int rows = min(sr.y, B.max_rows) * A.share;                             // of the whole unit; row r: row r / share, head h * share + r % share
    if (r0 >= rows) return;                                                       // (the whole cluster)
    const int nr = min(ROWS, rows - r0);
    const KeyRange first = src.K.range(B, len, sr.y, A.split(r0).x), last = src.K.range(B, len, sr.y, A.split(r0 + nr - 1).x);
    // (bounds rise with the row, but for rows of tokens below 0, which see nothing: 0, 0)
    const int lo = first.lo, hi = last.hi;

    const uint32_t ring_s = smem_u32(ring);
    const int step = split * Src::WARPS * KC;
    int next = lo + (rank * Src::WARPS + warp) * KC;                               // next chunk to fill
    int base = next;
    src.start(B, s, h, next, step);
    src.look_up(B, s, h, next, hi);
#pragma unroll
    for (int i = 0; i < NST - 1; ++i) {
        if (next < hi) {
            src.fill(ring + i * Src::STAGE, ring_s + i * Src::STAGE, B, s, h, next, hi);
            next += step;
            src.look_up(B, s, h, next, hi);
        }
        cp_async_commit();
    }
    if (threadIdx.x < ROWS) {
        const KeyRange r = src.K.range(B, len, sr.y, A.split(r0 + min((int)threadIdx.x, nr - 1)).x);
        s_range[threadIdx.x] = make_int2(r.lo, r.hi);
    }
    // queries: row n of every tile of 8, in the order of K's inner index
    uint32_t qb[NR][NS][2];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        const int2 at = A.split(r0 + min(8 * t + n, nr - 1));
        const bf16 *q = (const bf16 *)A.q + (long long)(sr.x + at.x) * A.q_stride + (h * A.share + at.y) * DH;
#pragma unroll
        for (int st = 0; st < NS; ++st) {
            const uint2 v = *reinterpret_cast<const uint2 *>(q + Src::q_dim(st, c));
            qb[t][st][0] = v.x, qb[t][st][1] = v.y;
        }
    }
    const float cs = 1.4426950408889634f * rsqrtf((float)DH) * Src::UP;
    // this lane's rows: 2 c and 2 c + 1 of every tile of 8
    float o[NR][NS][4], m[NR][2], l[NR][2];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        m[t][0] = m[t][1] = -INFINITY, l[t][0] = l[t][1] = 0.f;
#pragma unroll
        for (int i = 0; i < NS; ++i) o[t][i][0] = o[t][i][1] = o[t][i][2] = o[t][i][3] = 0.f;
    }
    __syncthreads();
    int st = 0;
    for (; base < hi; base += step) {
        {
            const int f = st == 0 ? NST - 1 : st - 1;
            if (next < hi) {
                src.fill(ring + f * Src::STAGE, ring_s + f * Src::STAGE, B, s, h, next, hi);
                next += step;
                src.look_up(B, s, h, next, hi);
            }
            cp_async_commit();
        }
        cp_async_wait<NST - 1>();
        __syncwarp();
        uint8_t *stage = ring + st * Src::STAGE;
        const uint32_t all = KC == 32 ? 0xffffffffu : (1u << KC) - 1, there = Src::mask(stage), bad = Src::take_out(stage);
        float x[KT][NR][4];
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            // row i of half j of tile u is key 16 u + 8 j + i / 2 + 4 (i % 2): a lane's four keys of a product with V are 4 apart
            uint32_t a[2][2 * NS];
            Src::k_frag(stage, 16 * u + (n >> 1) + 4 * (n & 1), c, a[0]);
            Src::k_frag(stage, 16 * u + 8 + (n >> 1) + 4 * (n & 1), c, a[1]);
#pragma unroll
            for (int t = 0; t < NR; ++t) {
                float odd[4] = {0.f, 0.f, 0.f, 0.f};
                x[u][t][0] = x[u][t][1] = x[u][t][2] = x[u][t][3] = 0.f;
#pragma unroll
                for (int k = 0; k < NS; ++k) {
                    const uint32_t ak[4] = {a[0][2 * k], a[1][2 * k], a[0][2 * k + 1], a[1][2 * k + 1]};
                    mma_bf16(TWO && k & 1 ? odd : x[u][t], ak, qb[t][k][0], qb[t][k][1]);
                }
                if (TWO)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[u][t][e] += odd[e];
            }
        }
        if constexpr (Src::RANGES) {
            if (base < s_range[nr - 1].x || base + KC > s_range[0].y)
                Src::take_out_values(stage, n, [&](int key, int d, float v) {
                    const int p = base + key;
#pragma unroll
                    for (int t = 0; t < NR; ++t)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int2 kr = s_range[8 * t + 2 * c + e];
                            if (p < kr.x || p >= kr.y) continue;
#pragma unroll
                            for (int i = 0; i < NS; ++i) {
                                if (d == 2 * i) o[t][i][e] += v;
                                if (d == 2 * i + 1) o[t][i][2 + e] += v;
                            }
                        }
                });
        }
        // x[u][t]: keys n' and n' + 8 (0, 1 and 2, 3) of tile u, rows 2 c and 2 c + 1 (0, 2 and 1, 3)
        if ((there & all) != all || bad || base < s_range[nr - 1].x || base + KC > s_range[0].y) {
#pragma unroll
            for (int t = 0; t < NR; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int2 kr = s_range[8 * t + 2 * c + e];
#pragma unroll
                    for (int u = 0; u < KT; ++u)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int key = 16 * u + 8 * j + (n >> 1) + 4 * (n & 1), p = base + key;
                            const bool seen = (there >> key & 1) && p >= kr.x && p < kr.y;
                            if (!seen) x[u][t][2 * j + e] = -INFINITY;
                            else if (bad >> key & 1) l[t][e] = NAN;               // the row sees a value that is not finite
                        }
                }
        }
        // the rows' maxima; the reference m follows only where one rose by more than 8 (a factor of 256), and what was summed before with it
        float mn[NR][2];
        bool rise = false;
#pragma unroll
        for (int t = 0; t < NR; ++t)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float v = m[t][e];
#pragma unroll
                for (int u = 0; u < KT; ++u) v = fmaxf(v, fmaxf(x[u][t][e], x[u][t][2 + e]));
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
                mn[t][e] = v, rise |= v * cs > m[t][e] * cs + 8.0f;
            }
        if (__any_sync(0xffffffffu, rise)) {
#pragma unroll
            for (int t = 0; t < NR; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (!(mn[t][e] * cs > m[t][e] * cs + 8.0f)) continue;
                    const float f = few_exp2((m[t][e] - mn[t][e]) * cs);
                    m[t][e] = mn[t][e], l[t][e] *= f;
#pragma unroll
                    for (int i = 0; i < NS; ++i) o[t][i][e] *= f, o[t][i][2 + e] *= f;
                }
        }
        uint32_t p[KT][NR][2];                                                    // P^T: keys 2 c.., row n
#pragma unroll
        for (int t = 0; t < NR; ++t) {
            const float m0 = m[t][0] == -INFINITY ? 0.f : fmaf(m[t][0], cs, src.down()), m1 = m[t][1] == -INFINITY ? 0.f : fmaf(m[t][1], cs, src.down());
#pragma unroll
            for (int u = 0; u < KT; ++u)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float a = few_exp2(fmaf(x[u][t][2 * j], cs, -m0)), b = few_exp2(fmaf(x[u][t][2 * j + 1], cs, -m1));
                    l[t][0] += a, l[t][1] += b;
                    p[u][t][j] = transpose8(bf16_pair(a, b));
                }
        }
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            // (columns 2 c and 2 c + 1 of a half are keys c and c + 4 of it)
            uint32_t b0[2 * NS], b1[2 * NS];
            Src::v_frag(stage, 16 * u + c, n, b0);
            Src::v_frag(stage, 16 * u + 8 + c, n, b1);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const uint32_t a[4] = {b0[2 * i], b0[2 * i + 1], b1[2 * i], b1[2 * i + 1]};
#pragma unroll
                for (int t = 0; t < NR; ++t) mma_bf16(o[t][i], a, p[u][t][0], p[u][t][1]);
            }
        }
        __syncwarp();                                                             // the stage may be filled again
        if (++st == NST) st = 0;
    }
    cp_async_wait<0>();
    __syncwarp();
    // this warp's state into its (drained) ring: O by rows, then m and l of the rows
    float *S = reinterpret_cast<float *>(ring);
#pragma unroll
    for (int t = 0; t < NR; ++t) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[t][e] += __shfl_xor_sync(0xffffffffu, l[t][e], d);
            const int r = 8 * t + 2 * c + e;
            if (n == 0) S[ROWS * DH + 2 * r] = m[t][e] * cs, S[ROWS * DH + 2 * r + 1] = l[t][e];
#pragma unroll
            for (int i = 0; i < NS; ++i) S[r * DH + Src::o_dim(2 * i, n)] = o[t][i][e], S[r * DH + Src::o_dim(2 * i + 1, n)] = o[t][i][2 + e];
        }
    }
    __syncthreads();
    // the CTA's
    float *T = reinterpret_cast<float *>(few_smem + Src::WARPS * F::WARP);
    auto write = [&](int r, int d, float4 v, float sum) {
        const int2 at = A.split(r0 + r);
        const float inv = sum == 0.f ? 0.f : Src::UP / sum;
        bf16 *out = (bf16 *)A.out + ((long long)(sr.x + at.x) * A.heads + h * A.share + at.y) * DH + d;
        *reinterpret_cast<uint2 *>(out) = make_uint2(bf16_pair(v.x * inv, v.y * inv), bf16_pair(v.z * inv, v.w * inv));
    };
    for (int i = threadIdx.x; i < nr * (DH / 4); i += 32 * Src::WARPS) {
        const int r = i / (DH / 4), d = i % (DH / 4) * 4;
        float mx = -INFINITY;
#pragma unroll
        for (int w = 0; w < Src::WARPS; ++w) mx = fmaxf(mx, reinterpret_cast<const float *>(few_smem + w * F::WARP)[ROWS * DH + 2 * r]);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < Src::WARPS; ++w) {
            const float *W = reinterpret_cast<const float *>(few_smem + w * F::WARP);
            const float mw = W[ROWS * DH + 2 * r], f = mw == -INFINITY ? 0.f : few_exp2(mw - mx);
            const float4 x = *reinterpret_cast<const float4 *>(W + r * DH + d);
            sum = fmaf(W[ROWS * DH + 2 * r + 1], f, sum);
            v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
        }
        if (split == 1) {
            write(r, d, v, sum);
        } else {
            *reinterpret_cast<float4 *>(T + r * DH + d) = v;
            if (d == 0) T[ROWS * DH + 2 * r] = mx, T[ROWS * DH + 2 * r + 1] = sum;
        }
    }
    if (split == 1) return;
    // the cluster's: every CTA a share of the row words
    cluster_sync_all();
    const uint32_t Ts = smem_u32(T);
    for (int i = rank + split * threadIdx.x; i < nr * (DH / 4); i += split * 32 * Src::WARPS) {
        const int r = i / (DH / 4), d = i % (DH / 4) * 4;
        float mx = -INFINITY;
        for (int k = 0; k < split; ++k) mx = fmaxf(mx, ld_cluster_f2(cluster_map(Ts + (ROWS * DH + 2 * r) * 4, k)).x);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        float sum = 0.f;
        for (int k = 0; k < split; ++k) {
            const float2 ml = ld_cluster_f2(cluster_map(Ts + (ROWS * DH + 2 * r) * 4, k));
            const float4 x = ld_cluster_f4(cluster_map(Ts + (r * DH + d) * 4, k));
            const float f = ml.x == -INFINITY ? 0.f : few_exp2(ml.x - mx);
            sum = fmaf(ml.y, f, sum);
            v.x = fmaf(x.x, f, v.x), v.y = fmaf(x.y, f, v.y), v.z = fmaf(x.z, f, v.z), v.w = fmaf(x.w, f, v.w);
        }
        write(r, d, v, sum);
    }
    cluster_sync_all();                                                           // nobody leaves while its state is read
}

// CTAs of a cluster that a unit is split over: as many as let the device hold all units' clusters at once (fit[i]: clusters of 2^i CTAs), and
// no more than give every warp a chunk or two; sixteen where they get three and more.  (16 heads x 64, 24 rows behind 5712 tokens, one CTA to an
// SM: in 8 pieces, of which the device holds 14 at once, 23 us, in 4 pieces 15.  One row: in 8 pieces 10.8, in 16 11.8; 24 heads on 8 behind 32768
// tokens 39 and 33.)
static int few_split(long long units, long long keys, int kc, const int *fit, int warps = FEW_WARPS) {
    const long long chunks = (keys + kc - 1) / kc;
    int i = 0;
    while (i < 4 && units <= fit[i + 1] && chunks > (long long)(i == 3 ? 48 : 1 << i) * warps) ++i;
    return 1 << i;
}
// With bf16 pages and small CTAs (two to an SM) up to four pieces are doubled where the halves are still long (FEW_PIECE bytes of K and V): what the device does
// not hold at once evens out sequences of different lengths.  (One row, 1, 2, 4, 8 and 16 pieces, us.  24 heads on 8 x 128: 16 sequences of up to 16384
// tokens 217, 164, 139, 164 (8); 8 of up to 32768 409, 223, 162, 139, 158, all as long 416, 231, 217, 217, 250; 5 of up to 16384 207, 115, 80, 64, 78, all
// as long 211, 117, 90, 102, 94, of 8192 111, 66, 51, 66, 64.  16 heads x 64: 4 of up to 32768 307, 172, 115, 90, 102; 4 of 8192 84, 53, 43, 53, 61; 9 of
// up to 16384 162, 108, 90, 100, 129, of 8192 88, 76, 84, 82, 109.)
static int few_split_rows(long long units, long long keys, int kc, int dh, const int *fit, int warps) {
    const int split = few_split(units, keys, kc, fit, warps);
    return split <= 4 && keys * dh * 4 >= 2LL * split * FEW_PIECE ? 2 * split : split;
}

template <typename Src, int DH, int NR>
static int launch_attn_few_nr(const BatchD &B, const AttnRows &A, const Src &src, int kv_heads, long long keys, int dev, int n_sm, cudaStream_t st) {
    using F = FewCfg<Src, DH, NR>;
    auto kern = k_attn_few<Src, DH, NR>;
    static OncePerDevice once;
    static int fit[NFD_PAGED_DEVICES][5];
    if (!once.run(dev, [&] {
            if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, F::SMEM) != cudaSuccess ||
                cudaFuncSetAttribute(kern, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
                return false;
            for (int i = 1; i < 5; ++i) fit[dev][i] = clusters_that_fit(kern, 1 << i, 32 * Src::WARPS, F::SMEM);
            return true;
        }))
        return NFD_E_CUDA;
    const long long tiles = ((long long)B.max_rows * A.share + F::ROWS - 1) / F::ROWS;
    const long long units = (long long)kv_heads * B.n_seqs * tiles;
    const int split = Src::RANGES ? few_split_rows(units, keys, Src::KC, DH, fit[dev], Src::WARPS) : few_split(units, keys, Src::KC, fit[dev]);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(kv_heads * split, B.n_seqs, (unsigned)tiles), cfg.blockDim = dim3(32 * Src::WARPS), cfg.dynamicSmemBytes = F::SMEM, cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension, at.val.clusterDim.x = split, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at, cfg.numAttrs = split > 1;
    if (cudaLaunchKernelEx(&cfg, kern, B, A, src, split) != cudaSuccess) {
        cudaGetLastError();
        return NFD_E_CUDA;
    }
    return NFD_OK;
}
template <typename Src, int DH>
static int launch_attn_few(const BatchD &B, const AttnRows &A, const Src &src, int kv_heads, long long keys, int dev, int n_sm, cudaStream_t st) {
    if ((long long)B.max_rows * A.share <= 8) return launch_attn_few_nr<Src, DH, 1>(B, A, src, kv_heads, keys, dev, n_sm, st);
    if (DH == 128 || (long long)B.max_rows * A.share <= 16) return launch_attn_few_nr<Src, DH, 2>(B, A, src, kv_heads, keys, dev, n_sm, st);
    return launch_attn_few_nr<Src, DH, DH == 128 ? 2 : 4>(B, A, src, kv_heads, keys, dev, n_sm, st);
}
