// Attention of many rows under the block-wise causal mask on tcgen05 / TMEM, to bf16 pages or to the rows of packed prompts.
//
// The rows of a sequence that share a head of keys (rows x heads that share it) are cut into tiles of 128; a CTA takes as many of them as it has softmax
// groups (two with head dimension 128, three below), which share every copied block of keys, or one, whose blocks its groups take in turn.  Each group has
// an accumulator for S and one for O, m and l of its own:
//     S = Q K^T     UMMA 128 x KB x DH, operands in shared memory, accumulator in tensor memory
//     P = exp2(S c - m)   one thread per row: S to registers, exponentials, P as bf16 over the S it came from
//     O += P V      UMMA 128 x head_dim x KB, P from tensor memory, V as it lies (MN-major)
// P is rounded to bf16 because that product's operands are of one type, V's; its relative error of 2^-9 a key is of the size of V's own.  Sums, m and O are fp32.
// m is the largest of the first 16 scores that a row sees, and no other maximum is taken: a probability is exact to the same number of bits whatever its
// size.  Where a sum of a row passes 2^50 after all (or is NaN), or a row has no m yet, the warp takes its keys again, S being untouched so far: the
// maximum first, and where it has risen by more than 8 (a factor of 256) it becomes m and the row's O is rescaled in tensor memory.  What P grows to, O
// does, and values may be as large as bf16 goes, so that P is scaled down by as much as all blocks together can grow (sum_bits), in the exponent.
//
// A tile walks the blocks that its own rows see, and no others; in a block that only some rows see the others' scores become -inf.  There P is 0, which
// keeps keys out and not values: 0 x NaN is NaN.  So in blocks that not all rows of a CTA see, the producers take values that are not finite out of V and
// note where; a row that does see one adds it to its result at the end.
//
// Producer warps come first.  One or two of them fill a ring of K and V blocks in turn by TMA, a lane looking up the place of each box of keys, and the others look
// through values where that is needed; where pages do not consist of boxes (or with head dimension 32) all of them copy by cp.async, a lane looking up the
// place of each key (four chunks of 512 rows behind 15872, 16 heads on 4 x 128: 380 us so, 246 us by TMA).  The next warp issues the products, the last ones are the softmax
// groups.  Which keys of a block are there is told beside K, a bit each, in a ring of its own.
//
// A unit (sequence, head of keys, tiles) with many keys and few others beside it is split over the CTAs of a cluster, which merge through distributed
// shared memory in a fixed order.  Every wait on a barrier in memory is bounded; after one that ran out the rows are NaN.  (The cluster's own barrier needs
// no bound: every CTA comes to it, its other waits being bounded, or has left as a whole cluster.)
//
// What bounds it.  With head dimension 128 the tensor pipe: two causal prompts of 8192 rows, 16 heads on 4, take 462 us alone (1190 TFLOP/s) and 537 us after
// many of their kind, when the clock has fallen (1020).  With 64 a block is 10 short products, which their one thread issues in 600 to 700 clocks, and the
// chain S, P, O of each group (four prompts of 5376 rows in frames of 336, 16 heads: 346 us; the exponentials alone would take 211): hence three groups there,
// whose chains overlap; with 128 tensor memory holds two.  Groups with an issuing thread each, or that wait for their turn at the pipes, were slower.
// Short prompts are their CTAs' beginning (5 to 7 thousand clocks) and end (5).
#pragma once
#include "nfd_attn_tile.cuh"
#include <cuda.h>

#define BLOCK_THREADS 512
#define BLOCK_SPLIT 8               // most CTAs of a cluster
#define BLOCK_SORTED 128            // sequences whose tiles are dealt out deepest first
#define BLOCK_POLY 2                // pairs of eight whose exponentials are polynomials
#define BLOCK_GROWTH 50             // bits that a sum may grow by before m follows it

template <int DH> struct BlockCfg {
    static constexpr int SUB = DH == 128 ? 2 : 1;          // 64-dim parts of a row
    static constexpr int NG = DH == 128 ? 2 : 3;           // softmax groups
    static constexpr int KB = DH == 128 ? 128 : 96;        // keys of a block
    static constexpr int PARTS = DH == 128 ? 2 : 1;        // a block's P goes to its product in so many parts
    static constexpr int HK = KB / PARTS;
    static constexpr int PW = DH == 128 ? 4 : 3, KPW = KB / PW;        // producer warps, keys of each; the next one is the issuer
    static constexpr int SM0 = 16 - 4 * NG;                // first softmax warp
    static constexpr int REGS_LOW = DH == 128 ? 56 : 80, REGS_SOFTMAX = DH == 128 ? 200 : 144;      // registers of a thread: 4 x 128 to share out
    static constexpr int NST = DH == 128 ? 5 : 12;         // stages of the ring: K and V of the first block, of the second ...
    static constexpr int FLY = DH == 128 ? 3 : 5;          // of which the copies are in flight
    static constexpr int NM = 16;                          // masks
    static constexpr int Q_BYTES = SUB * 128 * 128;        // a tile's queries
    static constexpr int BLK = SUB * KB * 128;             // a block of K or V
    static constexpr int AT_Q = 0, AT_R = NG * Q_BYTES, AT_MASK = AT_R + NST * BLK, AT_BAR = AT_MASK + NM * 16, SMEM = AT_BAR + 544 + 1024;
    static constexpr int TM_O = NG * KB;                   // S of group g, and over it P, at g KB; O at TM_O + g 64 SUB
    static constexpr int STATE = 128 * DH * 4 + 128 * 8;   // a group's state, over queries and ring: O as [DH / 4][128] float4, then [128] (m, l)
    static_assert(TM_O + NG * 64 * SUB <= 512 && NG * STATE + 128 * 8 <= AT_MASK && SMEM <= 232448, "tensor and shared memory");
    static_assert(SMEM > 232448 / 2, "a CTA has an SM, and its tensor memory, to itself: nobody in a cluster waits for what another cluster holds");
    static_assert(NG + NST / 2 + 1 <= NM, "K runs so many blocks ahead of the softmax");
    static_assert((SM0 / 4) * REGS_LOW + NG * REGS_SOFTMAX <= 512 && PW < SM0, "registers; warps");
    static_assert(KPW * (DH / 8) % 32 == 0 && KPW <= 32 && KPW % 8 == 0 && HK % 32 == 0, "copies; bits of a warp's keys are whole bytes; S by 32 columns");
};

struct BlockBars {
    uint32_t b;
    __device__ __forceinline__ uint32_t full(int s) const { return b + 8 * s; }                  // stages (up to 12)
    __device__ __forceinline__ uint32_t empty(int s) const { return b + 96 + 8 * s; }
    __device__ __forceinline__ uint32_t m_full(int s) const { return b + 192 + 8 * s; }          // masks (16)
    __device__ __forceinline__ uint32_t s_full(int g) const { return b + 320 + 8 * g; }          // groups (up to 3)
    __device__ __forceinline__ uint32_t p_full(int g, int part) const { return b + 344 + 16 * g + 8 * part; }
    // of a group's even and odd parts: a warp may be done with one before the product of the one before it is
    __device__ __forceinline__ uint32_t pv_done(int g, int n) const { return b + 392 + 16 * g + 8 * (n & 1); }
    __device__ __forceinline__ uint32_t q_full() const { return b + 440; }
    __device__ __forceinline__ uint32_t landed(int s) const { return b + 448 + 8 * s; }          // stages: values that are looked through before they are used
    // (a barrier to a thread: one after the other they took a thousand clocks)
    __device__ __forceinline__ void init(int producers, int groups) const {
        const int i = threadIdx.x;
        if (i < 12) mbar_init(full(i), producers);
        else if (i < 24) mbar_init(empty(i - 12), 1);
        else if (i < 36) mbar_init(landed(i - 24), 1);
        else if (i < 52) mbar_init(m_full(i - 36), producers);
        else if (i < 55) mbar_init(s_full(i - 52), 1);
        else if (i < 61) mbar_init(p_full((i - 55) >> 1, (i - 55) & 1), 4);
        else if (i < 67) mbar_init(pv_done((i - 61) >> 1, i - 61), 1);
        else if (i == 67) mbar_init(q_full(), 4 * groups);
        if (i < 68) fence_mbar_init();
    }
};

// What a CTA works on: keys lo .. hi - 1 of a sequence in nb blocks; keys that not all rows see: those below edge_lo, those from edge_hi on.
template <int NG> struct BlockWork {
    int s, h, first_row, lo, hi, nb, edge_lo, edge_hi;
    bool turns;                                             // the groups take one tile's blocks in turn
    int b0[NG], b1[NG];                                     // otherwise each has a tile, and takes blocks b0 .. b1 - 1
    // are there rows of the CTA that do not see all of block b (of KB keys)
    __device__ __forceinline__ bool edge(int b, int KB) const { return lo + b * KB < edge_lo || lo + b * KB + KB > edge_hi; }
    // does group g take block b; which of its jobs is that; is it the first, the last to take it
    __device__ __forceinline__ bool takes(int g, int b) const { return turns ? b % NG == g : b >= b0[g] && b < b1[g]; }
    __device__ __forceinline__ int job(int g, int b) const { return turns ? b / NG : b - b0[g]; }
    __device__ __forceinline__ bool first(int g, int b) const {
        bool f = true;
#pragma unroll
        for (int k = 0; k < NG; ++k) f = f && !(k < g && takes(k, b));
        return f;
    }
    __device__ __forceinline__ bool last(int g, int b) const {
        bool f = true;
#pragma unroll
        for (int k = 0; k < NG; ++k) f = f && !(k > g && takes(k, b));
        return f;
    }
};
template <int n> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(n)); }
template <int n> __device__ __forceinline__ void leave_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(n)); }

// ---- keys that TMA brings ------------------------------------------------------------------------------------
// Pages: tensor [pages x heads][page_tokens][DH], a box of `rows` keys (a power of two that a page consists of, so that no box crosses its end).
template <int DH> struct PageBoxes : PageKeys<bf16, DH> {
    static constexpr bool TMA = true;
    static constexpr int COPIERS = 2;                       // warps that issue copies
    CUtensorMap maps[2];
    int rows;
    __device__ __forceinline__ int box() const { return rows; }
    __device__ __forceinline__ int begin(int lo) const { return lo & -rows; }
    // offset in its page and page of the next box (page -1: it is not there)
    __device__ __forceinline__ int2 next_box(typename PageKeys<bf16, DH>::Cursor &c, const BatchD &B, int h, bool there) const {
        const int T = this->P.page_tokens, L = B.table_len;
        int2 at = make_int2(c.off, -1);
        if (there) {
            const int page = __ldg(c.table + c.pg);
            if ((unsigned)page < (unsigned)this->P.n_pages) at.y = page * this->P.heads + h;
        }
        c.off += c.dr, c.pg += c.dq;
        if (c.off >= T) c.off -= T, ++c.pg;
        if (c.pg >= L) c.pg -= L;
        return at;
    }
    // (a page behind the last one is filled in as zeros)
    __device__ __forceinline__ void load(int kv, uint32_t dst, uint32_t bar, int part, int, int2 at) const {
        tma_load_3d(dst, &maps[kv], bar, 64 * part, at.x, at.y < 0 ? this->P.n_pages * this->P.heads : at.y);
    }
};
// The rows of packed prompts: tensor [rows][heads x DH], a box of a block's keys (what lies behind a sequence's end is the next one's, and masked).
template <int DH> struct PackedBoxes : PackedKeys<bf16, DH> {
    static constexpr bool TMA = true;
    static constexpr int COPIERS = 1;
    CUtensorMap maps[2];
    __device__ __forceinline__ int box() const { return BlockCfg<DH>::KB; }
    __device__ __forceinline__ int begin(int lo) const { return lo; }
    __device__ __forceinline__ int2 next_box(typename PackedKeys<bf16, DH>::Cursor &c, const BatchD &, int, bool) const {
        const int row = c.row;
        c.row += c.step;
        return make_int2(row, 0);
    }
    __device__ __forceinline__ void load(int kv, uint32_t dst, uint32_t bar, int part, int h, int2 at) const {
        tma_load_2d(dst, &maps[kv], bar, h * DH + 64 * part, at.x);
    }
};

// ---- producers ----------------------------------------------------------------------------------------------
// Values of a piece of a block that are not finite become zeros; was there one?
__device__ __forceinline__ bool block_take_out(uint8_t *at) {
    uint4 *v = reinterpret_cast<uint4 *>(at);
    const uint4 x = *v;
    const uint4 f = make_uint4(finite_bits(x.x), finite_bits(x.y), finite_bits(x.z), finite_bits(x.w));
    if ((f.x & f.y & f.z & f.w) == 0xffffffffu) return false;
    *v = make_uint4(x.x & f.x, x.y & f.y, x.z & f.z, x.w & f.w);
    return true;
}
// By TMA, a warp for K (first 0) and one for V of pages, one for both of packed rows: a lane's copy of a block is a box of 64 dims and `box` keys, looked up on
// the way.  (An issued box takes some 80 clocks, its operands going into uniform registers one by one; one thread for all of them, by shuffles, was slower
// still.  Four chunks of 512 rows behind 15872, 16 heads on 4 x 128, in pages of 8, 16 and 64 tokens, by one warp 401, 283, 246 us, by two 258, 248, 246.
// Packed rows are a box to a block, which one thread copies (two prompts of 8192, 467 us by two lanes, 461 so), and look through more values: four prompts
// of 5376 rows in frames of 336, 16 heads x 64, by one warp 344, by two 352.)
template <int DH, typename Keys>
static __device__ __forceinline__ void block_copy(const Keys &K, const BatchD &B, const BlockWork<BlockCfg<DH>::NG> &w, int first, uint8_t *smem, const BlockBars &bars, bool &ok) {
    using C = BlockCfg<DH>;
    constexpr int STEP = Keys::COPIERS;                      // every so many items (K and V in turn) are this warp's
    const int lane = threadIdx.x & 31, box = K.box(), groups = C::KB / box, part = lane / groups, group = lane - part * groups;
    const bool mine = part < C::SUB;
    const uint32_t to = smem_u32(smem) + C::AT_R + part * (C::KB * 128) + group * box * 128;
    int p = w.lo + group * box;
    auto cur = K.cursor(B, w.s, w.first_row, p, C::KB);
    auto look_up = [&]() -> int2 {
        const int2 at = K.next_box(cur, B, w.h, mine && p < w.hi);
        p += C::KB;
        return at;
    };
    int2 next = look_up();
    int st = first, item = first;
    uint32_t par = 1;                                        // (the first lap waits for nothing)
    for (int b = 0; b < w.nb && ok; ++b) {
        const int2 at = next;
        if (Keys::HOLES && first == 0) {
            const uint32_t there = __ballot_sync(0xffffffffu, at.y >= 0);
            uint8_t *M = smem + C::AT_MASK + b % C::NM * 16;
            if (lane < C::KB / 8) M[lane] = there >> (lane * 8 / box) & 1 ? 0xFF : 0;
            __syncwarp();
            if (lane == 0) mbar_arrive(bars.m_full(b % C::NM));
        }
        next = look_up();
#pragma unroll
        for (int i = 0; i < 2; i += STEP, item += STEP) {
            const int kv = STEP == 2 ? first : i;
            ok = __all_sync(0xffffffffu, tile_wait(bars.empty(st), par));
            if (!ok) break;
            const uint32_t bar = kv && w.edge(b, C::KB) ? bars.landed(st) : bars.full(st);
            if constexpr (Keys::HOLES) {
                if (lane == 0) mbar_expect_tx(bar, C::BLK);
                __syncwarp();
                if (mine) K.load(kv, to + st * C::BLK, bar, part, w.h, at);
            } else {
                // (one box: its place is the same in all lanes, and one thread copies it)
                const uint32_t dst = __shfl_sync(0xffffffffu, to, 0) + st * C::BLK;
                const int2 from = make_int2(__shfl_sync(0xffffffffu, at.x, 0), 0);
                if (elect_one()) {
                    mbar_expect_tx(bar, C::BLK);
#pragma unroll
                    for (int half = 0; half < C::SUB; ++half) K.load(kv, dst + half * (C::KB * 128), bar, half, w.h, from);
                }
            }
            if ((st += STEP) >= C::NST) st -= C::NST, par ^= 1;
        }
    }
    // Nobody leaves with copies in flight, whoever has given up waiting: of the last NST items, this warp's.  (After a wait that ran out a stage may
    // have been filled once more by the other warp, its earlier copies having landed before, and its barrier be a phase on: that wait runs out, too.)
    for (int i = item - STEP; i >= max(0, item - first - C::NST); i -= STEP) ok = tile_wait(bars.full(i % C::NST), (i / C::NST) & 1) && ok;
}
// and the other producer warps look through the values of blocks that not all rows see
template <int DH, int COPIERS> static __device__ __forceinline__ void block_look_through(const BlockWork<BlockCfg<DH>::NG> &w, uint8_t *smem, const BlockBars &bars, int *bad, bool &ok) {
    using C = BlockCfg<DH>;
    uint32_t laps = 0;                                       // phases of the stages' barriers
    for (int b = 0; b < w.nb; ++b) {                         // (all of it, whatever runs out: the threads meet at a barrier)
        if (!w.edge(b, C::KB)) continue;
        const int st = (2 * b + 1) % C::NST;
        if (ok) ok = tile_wait(bars.landed(st), laps >> st & 1);
        laps ^= 1u << st;
        bool some = false;
        for (int i = (threadIdx.x - 32 * COPIERS) * 16; i < C::BLK; i += (C::PW - COPIERS) * 32 * 16) some |= block_take_out(smem + C::AT_R + st * C::BLK + i);
        if (some) atomicMin(bad, w.lo + b * C::KB), atomicMax(bad + 1, w.lo + b * C::KB + C::KB);
        fence_proxy_async_smem();
        asm volatile("bar.sync 4, %0;" ::"n"((C::PW - COPIERS) * 32) : "memory");
        if (threadIdx.x == 32 * COPIERS) mbar_arrive(bars.full(st));
    }
}
// By cp.async, all of them.
template <int DH, typename Keys>
static __device__ __forceinline__ void block_produce(const Keys &K, const BatchD &B, const BlockWork<BlockCfg<DH>::NG> &w, uint8_t *smem, const BlockBars &bars, int *bad, bool &ok) {
    using C = BlockCfg<DH>;
    constexpr int CPR = DH / 8, N = C::KPW * CPR / 32;       // 16-byte pieces of a row; a lane's of a block
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane % CPR, sub = lane / CPR;
    // (rows sub, sub + RPI, ... of the warp's, whose first is a multiple of 8: bits of the row above sub only flip bits of the piece)
    constexpr int RPI = 32 / CPR;
    const uint32_t to0 = (piece >> 3) * (C::KB * 128) + tile_at(warp * C::KPW + sub, piece & 7);
    auto to = [&](int i) -> uint32_t { return (to0 ^ ((i * RPI & 7) << 4)) + i * RPI * 128; };
    int p = w.lo + warp * C::KPW + lane;
    auto cur = K.cursor(B, w.s, w.first_row, p, C::KB);
    auto look_up = [&]() -> long long {
        const long long row = K.next(cur, B, w.h, lane < C::KPW && p < w.hi);
        p += C::KB;
        return row;
    };
    long long next = look_up();
    int done = 0, item = 0;                                  // published, begun
    auto publish = [&]() {
        const int st = done % C::NST, p0 = w.lo + (done >> 1) * C::KB;
        cp_async_wait_upto(item - done - 1);
        if ((done & 1) && w.edge(done >> 1, C::KB)) {
            bool some = false;
#pragma unroll
            for (int i = 0; i < N; ++i) some |= block_take_out(smem + C::AT_R + st * C::BLK + to(i));
            if (some) atomicMin(bad, p0), atomicMax(bad + 1, p0 + C::KB);
        }
        tile_publish(bars.full(st)), ++done;
    };
    for (int b = 0; b < w.nb && ok; ++b) {
        const long long row = next;
        const uint32_t there = __ballot_sync(0xffffffffu, row >= 0);
        next = look_up();
        // (rows of 64 bytes and more: memory has fewer than 2^32 - 1 of them)
        constexpr uint32_t NONE = 0xffffffffu;
        uint32_t rows[N];
#pragma unroll
        for (int i = 0; i < N; ++i) rows[i] = __shfl_sync(0xffffffffu, (uint32_t)row, i * RPI + sub);
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            const int st = item % C::NST;
            if (item >= C::NST) {
                const uint32_t par = (item / C::NST - 1) & 1;
                // (nothing is held back while waiting: what frees this stage may need it)
                while (!__all_sync(0xffffffffu, tile_test(bars.empty(st), par))) {
                    if (done < item) {
                        publish();
                    } else {
                        ok = __all_sync(0xffffffffu, tile_wait(bars.empty(st), par));
                        break;
                    }
                }
                if (!ok) break;
            }
            const uint32_t dst = smem_u32(smem) + C::AT_R + st * C::BLK;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const bf16 *src = (kv ? K.v_row(rows[i] == NONE ? 0 : rows[i], w.h) : K.k_row(rows[i] == NONE ? 0 : rows[i], w.h)) + piece * 8;
                cp_async16(dst + to(i), src, rows[i] == NONE ? 0 : 16);
            }
            cp_async_commit();
            if (Keys::HOLES && !kv) {
                uint8_t *M = smem + C::AT_MASK + b % C::NM * 16 + warp * (C::KPW / 8);
                if (lane < C::KPW / 8) M[lane] = (uint8_t)(there >> (8 * lane));
                __syncwarp();
                if (lane == 0) mbar_arrive(bars.m_full(b % C::NM));
            }
            // (the first block is wanted at once)
            ++item;
            if (item - done > (item < 2 * C::FLY ? 2 : C::FLY)) publish();
        }
    }
    while (ok && done < item) publish();
}

// ---- issuer -------------------------------------------------------------------------------------------------
// All products of a CTA, by one thread: block by block, for either group P V of its block and then S of the one that takes the same accumulator next
// (the tensor pipe takes one thread's instructions in order).  Nothing here branches on whether a wait has run out (what follows then is computed from whatever is
// there, and thrown away): with control flow that is the same for all lanes the operands stay in uniform registers.  Otherwise, moved there one by one for
// every product, they cost more than the products.
template <int DH> static __device__ __forceinline__ bool block_issue(const BlockWork<BlockCfg<DH>::NG> &w, const BlockBars &bars, uint32_t base, uint32_t tmem) {
    using C = BlockCfg<DH>;
    constexpr int KB = C::KB, SUB = C::SUB, NST = C::NST, NG = C::NG;
    constexpr uint32_t idesc_s = umma_idesc_bf16(128, KB), idesc_pv = umma_idesc_bf16(128, DH) | (1u << 16);       // V: MN-major
    // (a cluster's addresses hold the CTA's rank above bit 23; V's other 64 dims are KB rows on: the leading offset)
    const uint32_t at = base & 0x3ffffu, dQ = (at + C::AT_Q) >> 4, dR = (at + C::AT_R) >> 4, lead = (KB * 128 >> 4) << 16;
    bool ok = tile_wait(bars.q_full(), 0);
    auto wait = [&](uint32_t bar, uint32_t parity) {
        if (ok) ok = tile_wait(bar, parity);
    };
    auto scores = [&](int g, int b, int st, uint32_t par) {  // stage of the block's K and its phase
        if (w.first(g, b)) wait(bars.full(st), par);
        tc_fence_after();
        const uint32_t q = dQ + (w.turns ? 0 : g) * (C::Q_BYTES >> 4), k = dR + st * (C::BLK >> 4), d = tmem + g * KB;
#pragma unroll
        for (int e = 0; e < (DH + 15) / 16; ++e)
            tile_mma_ss(d, q + (e >> 2) * (128 * 128 >> 4) + 2 * (e & 3), k + (e >> 2) * (KB * 128 >> 4) + 2 * (e & 3), idesc_s, e != 0);
        umma_commit(bars.s_full(g));
        if (w.last(g, b)) umma_commit(bars.empty(st));
    };
    const int ahead = w.turns ? NG : 1;                      // blocks
    int sk = 0, sv = 1;                                      // stages of the next K and the next V, and their phases
    uint32_t pk = 0, pv = 0;
    auto on = [&](int &st, uint32_t &par) {
        st += 2;
        if (st >= NST) st -= NST, par ^= 1;
    };
    for (int b = 0; b < ahead && b < w.nb; ++b) {
#pragma unroll
        for (int g = 0; g < NG; ++g)
            if (w.takes(g, b)) scores(g, b, sk, pk);
        on(sk, pk);
    }
    for (int b = 0; b < w.nb; ++b) {
        const uint32_t v = (dR + sv * (C::BLK >> 4)) | lead;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            if (w.takes(g, b)) {
                if (w.first(g, b)) wait(bars.full(sv), pv);
                const int n = w.job(g, b);
                const uint32_t d = tmem + C::TM_O + g * 64 * SUB, a = tmem + g * KB;
#pragma unroll
                for (int part = 0; part < C::PARTS; ++part) {
                    wait(bars.p_full(g, part), n & 1);
                    tc_fence_after();
                    constexpr int E = C::HK / 16;
#pragma unroll
                    for (int e = part * E; e < (part + 1) * E; ++e) tile_mma_ts(d, a + 8 * e, v + e * (2048 >> 4), idesc_pv, n != 0 || e != 0);
                    umma_commit(bars.pv_done(g, n * C::PARTS + part));
                }
                if (w.last(g, b)) umma_commit(bars.empty(sv));
            }
            if (b + ahead < w.nb && w.takes(g, b + ahead)) scores(g, b + ahead, sk, pk);
        }
        on(sk, pk), on(sv, pv);
    }
    return ok;
}

// ---- softmax ------------------------------------------------------------------------------------------------
// A part of a block whose sums have outgrown m, or that finds a row without one: the row's maximum over the keys that it sees, m and what has been
// summed so far adjusted to it, then P.  seen: bits of the keys that the row sees; n: the group's parts before this one; pv_done: of the last of them.
template <int DH>
static __device__ __forceinline__ void block_slow(uint32_t tS, uint32_t tP, uint32_t tO, const uint32_t *seen, float c, float down, int n, uint32_t pv_done,
                                               float &m_io, float &l_io, bool &ok) {
    constexpr int HK = BlockCfg<DH>::HK;
    float m = m_io, l = l_io, top = -INFINITY;
    constexpr int W = HK / 32;
    auto bits = [&](int i) { return (i < 32 ? seen[0] : i < 64 ? seen[1] : seen[W - 1]) >> (i & 31); };
#pragma unroll 1
    for (int i = 0; i < HK; i += 16) {
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
    for (int i = 0; i < HK; i += 16) {
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
        tmem_st8(tP + i / 2, pk);                                      // (behind what is still to be read)
    }
    m_io = m, l_io = l + sum;
}
// subnormal numbers to 0
__device__ __forceinline__ float2 flush2(float2 a) {
    unsigned long long ra, rd;
    asm("mov.b64 %0, {%1, %2};" : "=l"(ra) : "f"(a.x), "f"(a.y));
    asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(rd) : "l"(ra), "l"(0ull));
    float2 d;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(d.x), "=f"(d.y) : "l"(rd));
    return d;
}
// 2^x, x = s c - mc, of two numbers on the fp32 pipes: x = n + f with n whole, a polynomial of degree 3 in f (fitted for the least relative error on [-1/2, 1/2],
// 1.0e-4; P is rounded to bf16, 2^-9 = 2e-3, anyway), n added to the exponent, which must not leave its field.  So x, which is the other columns' to the bit, goes on
// as 127 - 253.4 u with u cut off at 0 and 1 by the instruction that makes it (a minimum and a maximum in its place cost 2 % of a call): below 2^-126 the
// result is 0, and from 2^127 on, and of NaN, whose u is 0, it is 2^127, so that the part's sum has outgrown m.  The steps of u are 1.5e-5 of x.  p has 2^127 in its
// coefficients, n is counted from there.
__device__ __forceinline__ float2 block_exp2_poly(float2 s, float c, float mc) {
    constexpr float top = 127.0f, range = 253.4f;                      // (127 - 253.4 = -126 - 0.4: n = -126, p < 1, a subnormal number)
    const float magic = 12582912.0f, one = 1.7014118346046923e38f;     // 1.5 x 2^23: an ulp is 1; 2^127
    const float2 x = ffma2(s, make_float2(c, c), make_float2(-mc, -mc));
    const float2 u = make_float2(__saturatef(fmaf(x.x, -1.0f / range, top / range)), __saturatef(fmaf(x.y, -1.0f / range, top / range)));
    const float2 t = ffma2(u, make_float2(-range, -range), make_float2(magic, magic)), n = ffma2(t, make_float2(-1.0f, -1.0f), make_float2(magic, magic));
    const float2 f = ffma2(u, make_float2(-range, -range), n);         // (n: the whole part's negative)
    float2 p = ffma2(f, make_float2(0.05517166852951050f * one, 0.05517166852951050f * one), make_float2(0.2426111251115799f * one, 0.2426111251115799f * one));
    p = ffma2(p, f, make_float2(0.6932609677314758f * one, 0.6932609677314758f * one));
    p = ffma2(p, f, make_float2(0.9999280571937561f * one, 0.9999280571937561f * one));
    p = make_float2(__int_as_float(__float_as_int(p.x) + (__float_as_int(t.x) << 23)), __int_as_float(__float_as_int(p.y) + (__float_as_int(t.y) << 23)));
    return flush2(p);
}
// sixteen scores to P, as pairs, and their sum.  BLOCK_POLY of eight pairs go to the fp32 pipes.  With none, one, two, three and four: two prompts of 8192 rows, 16
// heads on 4 x 128, 485, 463, 457, 449 and 473 us; four of 5376 in frames of 336, 16 heads x 64, 369, 348, 344, 354 and 377; four of 4096, 16 heads x 32, each in
// one frame, 362, 340, 336, 354 and 383.
template <bool MASKED> __device__ __forceinline__ void block_exp16(const float *x, uint32_t bits, float c, float mc, uint32_t *pk, float2 (&ls)[2]) {
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        float2 s = make_float2(x[2 * u], x[2 * u + 1]);
        if (MASKED) s.x = bits >> (2 * u) & 1 ? s.x : -INFINITY, s.y = bits >> (2 * u + 1) & 1 ? s.y : -INFINITY;
        const float2 e = ffma2(s, make_float2(c, c), make_float2(-mc, -mc));
        const float2 p = !MASKED && ((u + 1) * BLOCK_POLY / 8 != u * BLOCK_POLY / 8) ? block_exp2_poly(s, c, mc) : make_float2(few_exp2(e.x), few_exp2(e.y));
        ls[u & 1] = fadd2(ls[u & 1], p);
        pk[u] = bf16_pair(p.x, p.y);
    }
}
// One pass over a part of S against the m that there is, 16 columns at a time with the next load in flight (xa: the first ones, on their way).  MASKED: keys
// that the row does not see count for nothing; ready: whether there is an m, or nothing to see.  False: a sum has outgrown m (most: the most that it may
// be), and S is as it was.
template <int DH, bool MASKED>
static __device__ __forceinline__ bool block_fast(uint32_t tS, uint32_t tP, float (&xa)[16], const uint32_t *seen, bool ready, float c, float mc, float most, float &l) {
    constexpr int HK = BlockCfg<DH>::HK;
    float xb[16];
    float2 ls[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    uint32_t pk[HK / 2];
#pragma unroll
    for (int i = 0; i < HK; i += 16) {
        float (&x)[16] = i / 16 % 2 ? xb : xa;
        tmem_ld_wait();
        loaded16(x);
        if (i + 16 < HK) tmem_ld16(tS + i + 16, reinterpret_cast<uint32_t *>(i / 16 % 2 ? xa : xb));
        block_exp16<MASKED>(x, MASKED ? seen[i / 32] >> (i & 16) : 0, c, mc, pk + i / 2, ls);
    }
    const float2 l2 = fadd2(ls[0], ls[1]);
    const float sum = l2.x + l2.y;
    if (!__all_sync(0xffffffffu, sum < most && (!MASKED || ready))) return false;
    l += sum;
#pragma unroll
    for (int i = 0; i + 16 <= HK / 2; i += 16) tmem_st16(tP + i, pk + i);
    if (HK / 2 % 16) tmem_st8(tP + HK / 2 - 8, pk + HK / 2 - 8);
    return true;
}

// ---- which tiles a CTA takes --------------------------------------------------------------------------------
// Units of `tiles` x 128 rows that n rows of a sequence make.
__device__ __forceinline__ int block_units(int n, int share, int tiles) {
    const int t = (n * share + 127) >> 7;
    return tiles == 1 ? t : tiles == 2 ? (t + 1) >> 1 : (t + 2) / 3;
}
// Work item `slot` as (sequence, number of its unit); sequence -1: there is none.  The units that see the most keys come first, since what is dealt out last
// should be short: a unit's place is its depth in its sequence and, with pages, what the sequence holds before its rows (in units; about, but the same for
// every CTA).  Up to BLOCK_SORTED sequences there are as many items as units; otherwise, and for prompts of one length, as many as if all had max_rows.
// (24 sequences of up to 336 rows behind up to 33 frames, 16 heads x 64: 338 us by depth alone, 272 so; 12 of 512 behind up to 15872, 16 on 4 x 128: 377, 287.)
template <typename Keys> static __device__ __forceinline__ int2 block_unit(const Keys &K, const BatchD &B, int share, int tiles, int slot) {
    const int most = block_units(B.max_rows, share, tiles);
    if (B.n_seqs > BLOCK_SORTED || (!B.row_start && (!Keys::HOLES || B.n_seqs == 1))) {
        const int t = slot / B.n_seqs;
        return make_int2(t < most ? slot - t * B.n_seqs : -1, most - 1 - t);
    }
    const int lane = threadIdx.x & 31;
    constexpr int N = BLOCK_SORTED / 32;
    int t[N], at[N], all = 0, lo = INT_MAX, hi = 0;         // a sequence's units, the first one's place
#pragma unroll
    for (int i = 0; i < N; ++i) {
        t[i] = at[i] = 0;
        const int s = i * 32 + lane;
        if (i * 32 < B.n_seqs && s < B.n_seqs) {
            const int n = B.rows(s).y;
            t[i] = block_units(min(n, B.max_rows), share, tiles);
            if constexpr (Keys::HOLES) {
                const float before = fminf((float)max(K.length(B, s) - n, 0), ((float)K.mask.window + 1.0f) * (float)K.mask.frame_tokens);
                at[i] = (int)fminf(before * (float)share / (float)(128 * tiles), 268435456.0f);
            }
            if (t[i]) lo = min(lo, at[i]), hi = max(hi, at[i] + t[i] - 1);
        }
        all += t[i];
    }
    if (slot >= (int)__reduce_add_sync(0xffffffffu, (unsigned)all)) return make_int2(-1, 0);
    lo = Keys::HOLES ? __reduce_min_sync(0xffffffffu, lo) : 0, hi = Keys::HOLES ? __reduce_max_sync(0xffffffffu, hi) : most - 1;
    // the first place j with no more than `slot` units behind it
    auto behind = [&](int j) {
        int n = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) n += min(max(0, at[i] + t[i] - 1 - j), t[i]);
        return (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
    };
    while (lo < hi) {
        const int j = (lo + hi) >> 1;
        if (behind(j) <= slot) hi = j;
        else lo = j + 1;
    }
    int left = slot - behind(lo), s = -1, unit = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t m = __ballot_sync(0xffffffffu, lo >= at[i] && lo - at[i] < t[i]);
        const int n = __popc(m);
        if (s < 0 && left < n) {
            const bool me = (m >> lane & 1) && __popc(m & ((1u << lane) - 1)) == left;
            const int l = __ffs(__ballot_sync(0xffffffffu, me)) - 1;
            s = i * 32 + l, unit = lo - __shfl_sync(0xffffffffu, at[i], l);
        }
        left -= n;
    }
    return make_int2(s, unit);
}

// Grid: items x heads of keys x split (a cluster's CTAs).
template <int DH, typename Keys>
__global__ void __launch_bounds__(BLOCK_THREADS, 1) k_attn_block(const BatchD B, const AttnRows A, const __grid_constant__ Keys K, int kv_heads, int split, int tiles, FastDiv by_share, float down) {
    using C = BlockCfg<DH>;
    constexpr int KB = C::KB, SUB = C::SUB, NG = C::NG, HK = C::HK, PARTS = C::PARTS;
    extern __shared__ uint8_t block_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(block_raw) + 1023) & ~(uintptr_t)1023);
    __shared__ uint32_t s_tmem;
    __shared__ int s_expired, s_bad[2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = blockIdx.x % split, hs = blockIdx.x / split;
    const BlockBars bars = {smem_u32(smem + C::AT_BAR)};
    bars.init(Keys::TMA ? 1 : C::PW, NG);
    if (threadIdx.x == 96) s_expired = 0, s_bad[0] = INT_MAX, s_bad[1] = 0;
    const int slot = hs / kv_heads;
    const int2 unit = block_unit(K, B, A.share, tiles, slot);
    if (unit.x < 0) return;                                 // (the whole cluster)
    BlockWork<NG> w;
    w.s = unit.x, w.h = hs - slot * kv_heads;
    const int r0 = unit.y * tiles * 128;
    const int2 sr = B.rows(w.s);
    const int len = K.length(B, w.s);
    const int rows = min(sr.y, B.max_rows) * A.share;
    if (r0 >= rows) return;                                 // (the whole cluster)
    __syncthreads();
    const int nr = min(tiles * 128, rows - r0), T = (nr + 127) / 128;
    // row r of the CTA: row of the sequence, which of the heads
    auto split_row = [&](int r) {
        const int i = by_share.div(r0 + r);
        return make_int2(i, r0 + r - i * A.share);
    };
    w.first_row = sr.x;
    if (warp >= C::SM0) {
        // softmax warps: the row's queries, into the operand of its tile, a row's pieces by neighbouring lanes; of one tile each group a share
        constexpr int CPR = DH / 8, RPI = 32 / CPR;
        const int g = (warp - C::SM0) >> 2, piece = lane % CPR;
        const uint32_t sq = smem_u32(smem + C::AT_Q) + (T == 1 ? 0 : g) * C::Q_BYTES + (piece >> 3) * (128 * 128);
#pragma unroll 1
        for (int i = T == 1 ? g : g < T ? 0 : CPR; i < CPR; i += T == 1 ? NG : 1) {
            const int trow = (warp & 3) * 32 + i * RPI + lane / CPR, r = (T == 1 ? 0 : g * 128) + trow;
            const int2 at = split_row(min(r, nr - 1));
            const bf16 *q = (const bf16 *)A.q + (long long)(sr.x + at.x) * A.q_stride + (w.h * A.share + at.y) * DH + piece * 8;
            cp_async16(sq + tile_at(trow, piece & 7), q, r < nr ? 16 : 0);
        }
        cp_async_commit();
    }
    {
        // What the first and the last rows of the tiles see, a row to a lane.  (A CTA's beginning waits for its instructions: few of them, and loops.)
        const int g0 = lane >> 1, row = min(nr, g0 * 128 + (lane & 1 ? 128 : 1)) - 1;
        const KeyRange mine = K.range(B, len, sr.y, split_row(g0 < T ? row : nr - 1).x);
        int lo = __shfl_sync(0xffffffffu, mine.lo, 0);
        w.edge_lo = __shfl_sync(0xffffffffu, mine.lo, 2 * T - 1), w.edge_hi = __shfl_sync(0xffffffffu, mine.hi, 0);
        const int end = __shfl_sync(0xffffffffu, mine.hi, 2 * T - 1);
        if constexpr (Keys::TMA) lo = K.begin(lo);
        const int all = max(0, (end - lo + KB - 1) / KB), per = split == 1 ? all : (all + split - 1) / split;
        w.lo = lo + min(all, rank * per) * KB;
        w.nb = max(0, min(all - rank * per, per));
        w.turns = T == 1 && w.nb > 1;
        w.hi = min(end, w.lo + w.nb * KB);
        // (no block is left out between the tiles' ranges: rows see themselves, and those before them what comes before)
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const int a = __shfl_sync(0xffffffffu, mine.lo, 2 * g), e = __shfl_sync(0xffffffffu, mine.hi, 2 * g + 1);
            w.b0[g] = w.b1[g] = 0;
            if (!w.turns && g < T) {
                w.b1[g] = g == T - 1 ? w.nb : min(w.nb, max(0, e - w.lo + KB - 1) / KB);
                w.b0[g] = g == 0 ? 0 : min(max(0, a - w.lo) / KB, w.b1[g ? g - 1 : 0]);
            }
        }
    }
    const bool merge = split > 1 || w.turns;                // a row's result is in several groups
    uint32_t tmem = 0;
    if (warp >= C::PW) {
        // (the producers are on their way; the others wait for tensor memory)
        if (warp == C::PW) {
            tmem_alloc(smem_u32(&s_tmem), 512);
            tmem_relinquish();
        }
        tc_fence_before();
        asm volatile("bar.sync 2, %0;" ::"n"(BLOCK_THREADS - 32 * C::PW) : "memory");
        tc_fence_after();
        tmem = s_tmem;
    }
    bool ok = true;

    if (warp < C::SM0) {
        leave_registers<C::REGS_LOW>();
        if (warp < C::PW) {
            if constexpr (Keys::TMA) {
                if (warp < Keys::COPIERS) block_copy<DH>(K, B, w, warp, smem, bars, ok);
                else block_look_through<DH, Keys::COPIERS>(w, smem, bars, s_bad, ok);
            } else {
                if (w.nb) block_produce<DH>(K, B, w, smem, bars, s_bad, ok);
            }
            if (!ok) s_expired = 1;
            asm volatile("bar.arrive 1, %0;" ::"n"(NG * 128 + 32 * C::PW) : "memory");
        } else if (warp == C::PW && w.nb) {
            // (what the products' operands come from is the same in all lanes, and the compiler has to know it)
            const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), base = __shfl_sync(0xffffffffu, smem_u32(smem), 0);
            BlockWork<NG> u;
            u.nb = __shfl_sync(0xffffffffu, w.nb, 0), u.turns = __shfl_sync(0xffffffffu, (int)w.turns, 0);
#pragma unroll
            for (int g = 0; g < NG; ++g) u.b0[g] = __shfl_sync(0xffffffffu, w.b0[g], 0), u.b1[g] = __shfl_sync(0xffffffffu, w.b1[g], 0);
            if (elect_one()) {
                if (!block_issue<DH>(u, bars, base, tm)) s_expired = 1;
            }
        }
    } else {
        take_registers<C::REGS_SOFTMAX>();
        // ---------------- softmax: a thread per row ----------------
        const int g = (warp - C::SM0) >> 2, quad = warp & 3, trow = quad * 32 + lane, r = (T == 1 ? 0 : g * 128) + trow;
        const uint32_t lane_off = (uint32_t)(quad * 32) << 16, tO = tmem + C::TM_O + g * 64 * SUB + lane_off;
        const bool some = __any_sync(0xffffffffu, r < nr);             // the warp has rows
        const float c = 1.4426950408889634f * rsqrtf((float)DH);
        const float most = exp2f(BLOCK_GROWTH - down);
        const KeyRange kr = K.range(B, len, sr.y, split_row(min(r, nr - 1)).x);
        cp_async_wait<0>();
        tile_publish(bars.q_full());
        float m = -INFINITY, l = 0.f;                                  // m: reference, in units of scores
        int n = 0;                                                     // the group's jobs so far
        int b_first = g, b_end = w.nb;
        const int b_step = w.turns ? NG : 1;
#pragma unroll
        for (int k = 0; k < NG; ++k)
            if (!w.turns && g == k) b_first = w.b0[k], b_end = w.b1[k];
        uint32_t there[KB / 32];                                       // keys of the next block that are there
        auto look = [&](int b) {
            if constexpr (Keys::HOLES) {
                ok = ok && tile_wait(bars.m_full(b % C::NM), (b / C::NM) & 1);
                const uint32_t *mask = reinterpret_cast<const uint32_t *>(smem + C::AT_MASK + b % C::NM * 16);
#pragma unroll
                for (int k = 0; k < KB / 32; ++k) there[k] = mask[k];
            } else {
#pragma unroll
                for (int k = 0; k < KB / 32; ++k) there[k] = 0xffffffffu;
            }
        };
        for (int b = b_first; b < b_end; b += b_step, ++n) {
            const uint32_t tJ = tmem + g * KB + lane_off;
            // (the masks of a group's first block may be laps of their ring ahead; S says that they are there)
            if (n == 0) {
                ok = ok && tile_wait(bars.s_full(g), 0);
                look(b);
            }
            uint32_t every = 0xffffffffu;
#pragma unroll
            for (int k = 0; k < KB / 32; ++k) every &= there[k];
            const int p0 = w.lo + b * KB;
            const bool plain = __all_sync(0xffffffffu, every == 0xffffffffu && p0 >= kr.lo && p0 + KB <= kr.hi && m != -INFINITY) && some;
            if (n) ok = ok && tile_wait(bars.s_full(g), n & 1);
            __syncwarp();
            tc_fence_after();
#pragma unroll 1
            for (int part = 0; part < PARTS; ++part) {
                const uint32_t tS = tJ + part * HK, tP = tJ + part * (HK / 2);
                float x[16];
                if (some) tmem_ld16(tS, reinterpret_cast<uint32_t *>(x));
                if (plain) {                                           // all rows have an m and see all of these keys
                    if (!block_fast<DH, false>(tS, tP, x, there, true, c, fmaf(m, c, down), most, l))
                        block_slow<DH>(tS, tP, tO, there, c, down, n * PARTS + part, bars.pv_done(g, n * PARTS + part - 1), m, l, ok);
                } else if (some) {                                     // (of rows that are not there P may be anything)
                    const int a = kr.lo - p0 - part * HK, e = min(kr.hi - p0 - part * HK, HK);   // keys a .. e - 1 of the part
                    uint32_t seen[HK / 32], any = 0;
#pragma unroll
                    for (int k = 0; k < HK / 32; ++k) {
                        const int a1 = min(max(a - 32 * k, 0), 32), e1 = min(max(e - 32 * k, 0), 32);
                        seen[k] = (part ? there[KB / 32 - HK / 32 + k] : there[k]) & (e1 == 32 ? 0xffffffffu : (1u << e1) - 1) &
                                  ~(a1 == 32 ? 0xffffffffu : (1u << a1) - 1);
                        any |= seen[k];
                    }
                    tmem_ld_wait();
                    loaded16(x);
                    if (!__any_sync(0xffffffffu, any)) {               // none of the warp's rows sees any of these keys
                        const uint32_t zero[16] = {};
#pragma unroll
                        for (int k = 0; k < HK / 2; k += 8) tmem_st8(tP + k, zero);
                    } else {
                        if (__any_sync(0xffffffffu, m == -INFINITY)) {
                            // a row without m (nothing has been summed for it): the largest of the first scores will do, if it sees one of them
                            float top = -INFINITY;
#pragma unroll
                            for (int e = 0; e < 16; ++e) top = fmaxf(top, seen[0] >> e & 1 ? x[e] : -INFINITY);
                            if (m == -INFINITY) m = top;
                        }
                        if (!block_fast<DH, true>(tS, tP, x, seen, m != -INFINITY || !any, c, m == -INFINITY ? 0.f : fmaf(m, c, down), most, l))
                            block_slow<DH>(tS, tP, tO, seen, c, down, n * PARTS + part, bars.pv_done(g, n * PARTS + part - 1), m, l, ok);
                    }
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bars.p_full(g, part));
            }
            if (b + b_step < b_end) look(b + b_step);
        }
        const int parts = n * PARTS;
        if (n) ok = ok && tile_wait(bars.pv_done(g, parts - 1), ((parts - 1) >> 1) & 1);
        __syncwarp();
        tc_fence_after();
        if (!ok) s_expired = 1;
        asm volatile("bar.sync 1, %0;" ::"n"(NG * 128 + 32 * C::PW) : "memory");           // queries and ring are at rest, and what the producers found is told
        const float expired = s_expired || !ok ? NAN : 0.f;
        const int late_lo = max(s_bad[0], kr.lo), late_hi = min(s_bad[1], kr.hi);      // keys among which there are values that were taken out
        if (merge ? T == 1 || g < T : some && (T > 1 ? g < T : g == 0)) {
            const float inv = (l == 0.f ? 0.f : 1.0f / l) + expired;
            uint8_t *state = smem + g * C::STATE;
#pragma unroll 1
            for (int i = 0; i < DH; i += 32) {
                float o[32];
                tmem_ld32(tO + i, reinterpret_cast<uint32_t *>(o));
                tmem_ld_wait();
                loaded32(o);
                if (!n)
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = 0.f;
                for (int p = late_lo; p < late_hi && r < nr; ++p) {
                    auto cur = K.cursor(B, w.s, sr.x, p, 1);
                    const long long row = K.next(cur, B, w.h, true);
                    if (row < 0) continue;
                    const uint32_t *v = reinterpret_cast<const uint32_t *>(K.v_row(row, w.h) + i);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const uint32_t x = v[e], f = finite_bits(x);
                        o[2 * e] += f & 0xFFFFu ? 0.f : __uint_as_float(x << 16);
                        o[2 * e + 1] += f >> 16 ? 0.f : __uint_as_float(x & 0xffff0000u);
                    }
                }
                if (merge) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        *reinterpret_cast<float4 *>(state + ((i / 4 + e) * 128 + trow) * 16) = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                } else {
                    // over the tile's queries, as these lie
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t v[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) v[u] = bf16_pair(o[8 * e + 2 * u] * inv, o[8 * e + 2 * u + 1] * inv);
                        const int piece = i / 8 + e;
                        *reinterpret_cast<uint4 *>(smem + C::AT_Q + g * C::Q_BYTES + (piece >> 3) * (128 * 128) + tile_at(trow, piece & 7)) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                }
            }
            if (!merge) {
                // the warp's rows, a row's pieces by neighbouring lanes (a row to a lane, the stores took four times as long)
                __syncwarp();
                constexpr int CPR = DH / 8, RPI = 32 / CPR;
                const int piece = lane % CPR;
#pragma unroll 4
                for (int k = 0; k < CPR; ++k) {
                    const int row = quad * 32 + k * RPI + lane / CPR, rr = (T == 1 ? 0 : g * 128) + row;
                    if (rr >= nr) break;
                    const int2 at = split_row(rr);
                    bf16 *out = (bf16 *)A.out + ((long long)(sr.x + at.x) * A.heads + w.h * A.share + at.y) * DH + piece * 8;
                    *reinterpret_cast<uint4 *>(out) = *reinterpret_cast<const uint4 *>(smem + C::AT_Q + g * C::Q_BYTES + (piece >> 3) * (128 * 128) + tile_at(row, piece & 7));
                }
            }
            if (merge) *reinterpret_cast<float2 *>(state + 128 * DH * 4 + trow * 8) = make_float2(n ? m * c : -INFINITY, l + expired);
        }
        if (merge && T == 1) {
            // The groups' states of the one tile become one, over the first (a share of the columns to a group), or the result.  None is left out: a
            // value that is not finite counts however small its factor.
            asm volatile("bar.sync 3, %0;" ::"n"(NG * 128) : "memory");
            float f[NG], mx = -INFINITY, sum = 0.f;
            float2 ml[NG];
#pragma unroll
            for (int k = 0; k < NG; ++k) ml[k] = *reinterpret_cast<const float2 *>(smem + k * C::STATE + 128 * DH * 4 + trow * 8), mx = fmaxf(mx, ml[k].x);
#pragma unroll
            for (int k = 0; k < NG; ++k) f[k] = ml[k].x == -INFINITY ? 0.f : few_exp2(ml[k].x - mx), sum = fmaf(ml[k].y, f[k], sum);
            const float inv = sum == 0.f ? 0.f : 1.0f / sum;
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
                    const int2 at = split_row(r);
                    bf16 *out = (bf16 *)A.out + ((long long)(sr.x + at.x) * A.heads + w.h * A.share + at.y) * DH;
                    *reinterpret_cast<uint4 *>(out + 8 * i) = make_uint4(bf16_pair(v[0] * inv, v[1] * inv), bf16_pair(v[2] * inv, v[3] * inv),
                                                                         bf16_pair(v[4] * inv, v[5] * inv), bf16_pair(v[6] * inv, v[7] * inv));
                }
            }
            if (g == 0) *reinterpret_cast<float2 *>(smem + NG * C::STATE + trow * 8) = make_float2(mx, sum);
        }
        if (split > 1) {
            __syncwarp();
            cluster_sync_all();
            // The CTAs' states.  Row words of four columns, 8 rows x 4 of them to a warp (32 bytes of a row, and every bank once); each CTA of a
            // cluster takes every split-th of these.  Eight states' loads are in flight together: of several words where the CTAs are fewer (a word at a
            // time the merge of two CTAs took 17000 clocks).
            const uint32_t st0 = smem_u32(smem);
            const int n_words = T * 16 * (DH / 16), stride = split * 4 * NG;
            auto join = [&](auto most_ctas) {
                constexpr int S = decltype(most_ctas)::value, U = 8 / S;
                for (int i0 = rank * 4 * NG + warp - C::SM0; i0 < n_words; i0 += U * stride) {
                    float2 ml[U][S];
                    float4 o[U][S];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int i = min(i0 + u * stride, n_words - 1), tile = i / (16 * (DH / 16)), in = i % (16 * (DH / 16));
                        const int mrow = (in / (DH / 16)) * 8 + (lane & 7), col4 = (in % (DH / 16)) * 4 + (lane >> 3);
                        const uint32_t at_ml = st0 + (T == 1 ? NG * C::STATE : tile * C::STATE + 128 * DH * 4) + mrow * 8;
                        const uint32_t at_o = st0 + tile * C::STATE + (col4 * 128 + mrow) * 16;
#pragma unroll
                        for (int k = 0; k < S; ++k) {
                            ml[u][k] = make_float2(-INFINITY, 0.f), o[u][k] = make_float4(0.f, 0.f, 0.f, 0.f);
                            if (k < split) ml[u][k] = ld_cluster_f2(cluster_map(at_ml, k)), o[u][k] = ld_cluster_f4(cluster_map(at_o, k));
                        }
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int i = i0 + u * stride, tile = i / (16 * (DH / 16)), in = i % (16 * (DH / 16));
                        const int col4 = (in % (DH / 16)) * 4 + (lane >> 3), mr = tile * 128 + (in / (DH / 16)) * 8 + (lane & 7);
                        if (i >= n_words || mr >= nr) continue;
                        float mx = -INFINITY, sum = 0.f;
                        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int k = 0; k < S; ++k) mx = fmaxf(mx, ml[u][k].x);
#pragma unroll
                        for (int k = 0; k < S; ++k) {
                            const float f = ml[u][k].x == -INFINITY ? 0.f : few_exp2(ml[u][k].x - mx);
                            sum = fmaf(ml[u][k].y, f, sum);
                            v.x = fmaf(o[u][k].x, f, v.x), v.y = fmaf(o[u][k].y, f, v.y), v.z = fmaf(o[u][k].z, f, v.z), v.w = fmaf(o[u][k].w, f, v.w);
                        }
                        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
                        const int2 at = split_row(mr);
                        bf16 *out = (bf16 *)A.out + ((long long)(sr.x + at.x) * A.heads + w.h * A.share + at.y) * DH + col4 * 4;
                        *reinterpret_cast<uint2 *>(out) = make_uint2(bf16_pair(v.x * inv, v.y * inv), bf16_pair(v.z * inv, v.w * inv));
                    }
                }
            };
            if (split == 2) join(std::integral_constant<int, 2>());
            else if (split <= 4) join(std::integral_constant<int, 4>());
            else join(std::integral_constant<int, 8>());
            cluster_sync_all();                                 // nobody leaves while its state is read
        }
    }
    // (the other warps have too few registers for any of the above)
    __syncwarp();
    cp_async_wait<0>();
    tc_fence_before();
    if (split > 1) {
        if (warp < C::SM0) cluster_sync_all(), cluster_sync_all();
    } else {
        __syncthreads();
    }
    if (warp == C::PW) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// How the work is laid out: tiles of a CTA (1 or NG), CTAs of a cluster that their keys are split over, by times in clocks as measured with all SMs busy: a
// block of keys takes a CTA's pipes as long as its tiles say (JOB); a CTA has a beginning and an end (FIXED, and MERGE where there are states to merge).
// Units that see as many keys (mean = keys) go in waves of as many clusters as the device holds at once; where they differ the last ones are short, and what
// counts is the sum, or the longest.
template <int DH, typename Units, typename Clusters>
static TilePlan block_plan(long long rows, long long keys, long long mean, int n_sm, Units &&units, Clusters &&clusters) {
    constexpr int kb = BlockCfg<DH>::KB, ng = BlockCfg<DH>::NG;
    constexpr long long JOB[4] = {0, DH == 128 ? 1800 : 1350, DH == 128 ? 3250 : 2550, 2650}, FIXED = 9000, MERGE1 = 2000, MERGE = 7000;
    TilePlan best = {1, 1};
    long long least = -1;
    for (int tiles = 1; tiles <= ng; tiles += ng - 1)
        for (int split = 1; split <= BLOCK_SPLIT; ++split) {
            const long long fit = split == 1 ? n_sm : clusters(split), blocks = (keys + kb - 1) / kb, average = (mean + kb - 1) / kb;
            if (fit < 1 || (split > 1 && blocks < 2 * split)) break;
            const long long mine = rows < 128 * tiles ? (rows + 127) / 128 : tiles, rest = FIXED + (split > 1 ? MERGE : mine == 1 ? MERGE1 : 0);
            const long long longest = (blocks + split - 1) / split * JOB[mine] + rest, n = units(tiles);
            const long long sum = n * (average * JOB[mine] / split + rest) / fit + longest / 3;
            const long long cost = mean == keys ? (n + fit - 1) / fit * longest : sum > longest ? sum : longest;
            if (least < 0 || cost < least) least = cost, best = {tiles, split};
        }
    return best;
}

// A map of bf16 numbers for boxes of 64 x `rows`, swizzled as the products' operands are; dims and strides (bytes; of all but the first) from the innermost on.
static int block_map(CUtensorMap *map, const void *base, int rank, const cuuint64_t *dims, const cuuint64_t *strides, int rows) {
    typedef CUresult (*Encode)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                               CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<Encode> known;                      // (the same whichever thread stores it)
    Encode encode = known;
    if (!encode) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess || !fn || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return NFD_E_CUDA;
        }
        known = encode = (Encode)fn;
    }
    const cuuint32_t box[3] = {64, (cuuint32_t)rows, 1}, steps[3] = {1, 1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void *>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? NFD_OK : NFD_E_CUDA;
}

template <int DH, typename Keys>
static int launch_attn_block(const BatchD &B, const AttnRows &A, const Keys &K, int kv_heads, long long keys, int dev, int n_sm, cudaStream_t st) {
    using C = BlockCfg<DH>;
    auto kern = k_attn_block<DH, Keys>;
    static OncePerDevice once;
    static int fit[NFD_PAGED_DEVICES][BLOCK_SPLIT + 1];
    if (!once.run(dev, [&] {
            if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM) != cudaSuccess) return false;
            for (int split = 2; split <= BLOCK_SPLIT; ++split) fit[dev][split] = clusters_that_fit(kern, split, BLOCK_THREADS, C::SMEM);
            return true;
        }))
        return NFD_E_CUDA;
    const long long rows = (long long)B.max_rows * A.share, all_rows = (long long)B.n_rows * A.share;
    // units of a head: as many as the sequences' rows can make, or as if all had max_rows (block_unit)
    auto units = [&](int tiles) -> long long {
        const long long R = 128 * tiles, most = B.n_seqs * ((rows + R - 1) / R), real = all_rows / R + B.n_seqs;
        return B.row_start && B.n_seqs <= BLOCK_SORTED && real < most ? real : most;
    };
    // what a row sees on the average: of a prompt, as far as its window does not end before, half of it and half of its own frame
    long long mean = keys;
    if (!Keys::HOLES) {
        const long long frame = K.mask.frame_tokens, window = ((long long)K.mask.window + 1) * frame, n = B.max_rows;
        mean = n <= window ? (n + frame) / 2 : window - window * window / (2 * n) + frame / 2;
        mean = mean < keys ? mean : keys;
    }
    const TilePlan pl = block_plan<DH>(rows, keys, mean, n_sm, [&](int tiles) { return kv_heads * units(tiles); }, [&](int k) { return fit[dev][k]; });
    const long long grid = units(pl.tiles) * kv_heads * pl.split;
    if (grid > INT_MAX) return NFD_E_RANGE;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid), cfg.blockDim = dim3(BLOCK_THREADS), cfg.dynamicSmemBytes = C::SMEM, cfg.stream = st;
    cudaLaunchAttribute at;
    at.id = cudaLaunchAttributeClusterDimension, at.val.clusterDim.x = pl.split, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cfg.attrs = &at, cfg.numAttrs = pl.split > 1;
    // the parts that a row's keys are in, each of which may grow: the first key may lie anywhere in one (a window's, a ring's oldest, in boxes of a page)
    const long long row_keys = ((long long)K.mask.window + 1) * K.mask.frame_tokens;
    const float down = (float)sum_bits(BLOCK_GROWTH, parts_touched(keys < row_keys ? keys : row_keys, C::HK));
    FastDiv by_share;
    by_share.set(A.share);
    if (cudaLaunchKernelEx(&cfg, kern, B, A, K, kv_heads, pl.split, pl.tiles, by_share, down) != cudaSuccess) {
        cudaGetLastError();
        return NFD_E_CUDA;
    }
    return NFD_OK;
}

// The rows of a call to the kernel that suits the keys: by TMA where head dimension, pages and strides allow it.
template <int DH> static int attn_block(const BatchD &B, const AttnRows &A, const PageKeys<bf16, DH> &K, int kv_heads, long long keys, int dev, int n_sm, cudaStream_t st) {
    const long long planes = (long long)K.P.n_pages * K.P.heads;
    int rows = BlockCfg<DH>::KB & -BlockCfg<DH>::KB;        // the largest power of two that blocks and pages consist of
    while (K.P.page_tokens % rows) rows /= 2;
    if constexpr (DH >= 64) {
        if (rows >= 8 && planes < INT_MAX) {
            PageBoxes<DH> boxes;
            static_cast<PageKeys<bf16, DH> &>(boxes) = K;
            boxes.rows = rows;
            const cuuint64_t dims[3] = {DH, (cuuint64_t)K.P.page_tokens, (cuuint64_t)planes}, strides[2] = {DH * 2, (cuuint64_t)K.P.page_tokens * DH * 2};
            for (int i = 0; i < 2; ++i)
                if (const int r = block_map(&boxes.maps[i], i ? K.P.v : K.P.k, 3, dims, strides, rows)) return r;
            return launch_attn_block<DH>(B, A, boxes, kv_heads, keys, dev, n_sm, st);
        }
    }
    return launch_attn_block<DH>(B, A, K, kv_heads, keys, dev, n_sm, st);
}
template <int DH> static int attn_block(const BatchD &B, const AttnRows &A, const PackedKeys<bf16, DH> &K, int kv_heads, long long keys, int dev, int n_sm, cudaStream_t st) {
    if constexpr (DH >= 64) {
        PackedBoxes<DH> boxes;
        static_cast<PackedKeys<bf16, DH> &>(boxes) = K;
        const cuuint64_t dims[2] = {(cuuint64_t)kv_heads * DH, (cuuint64_t)B.n_rows};
        for (int i = 0; i < 2; ++i) {
            const cuuint64_t stride = (cuuint64_t)(i ? K.v_stride : K.k_stride) * 2;
            if (stride >= 1ull << 40) return NFD_E_RANGE;
            if (const int r = block_map(&boxes.maps[i], i ? K.v : K.k, 2, dims, &stride, BlockCfg<DH>::KB)) return r;
        }
        return launch_attn_block<DH>(B, A, boxes, kv_heads, keys, dev, n_sm, st);
    } else {
        return launch_attn_block<DH>(B, A, K, kv_heads, keys, dev, n_sm, st);
    }
}
