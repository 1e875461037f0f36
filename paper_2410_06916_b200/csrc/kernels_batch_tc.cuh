// Attention of many query rows over the paged cache on the 5th-generation tensor cores (sm_100a): whole prompts, and the
// rows of all sequences against a prefix that they share.
//
//     O = softmax(scale Q K^T) V,   one pass over the keys with a running maximum m and sum l per query row.
//
// Tiles.  A CTA takes two tiles of 128 query rows of one kv head; a tile packs the G query heads of that kv head's group,
// TQ = 128 / G tokens of G heads, so that a key is read once for the whole group, short sequences still fill a tile and
// the causal edge cuts through few tokens.  Keys come in tiles of 128.  S = Q K^T (128 x 128, fp32) and O (128 x D, fp32)
// live in TMEM; the softmax warps overwrite S with the 16-bit probabilities P, which the second product reads as its
// A operand straight from TMEM.  With both tiles 2 (128 + D) of the 512 columns are in use.
//
// Overlap.  While the softmax of tile A runs, the tensor pipe works on tile B, and the other way round: per key tile the
// pipe has 2 x 4 x 128^3 multiply-adds (2048 cycles at D = 128) and each of the SM's four schedulers 2 warps x 128
// exponentials (2048 cycles of its special function unit), so neither may wait for the other.  P is handed over in two
// halves, so that its product starts while the second half is still being computed.
//
// Rescaling.  O is rescaled only when a row's maximum has grown by more than 2^8 since the last time (the probabilities
// are then at most 2^8, which both 16-bit types hold); a softmax warp does it itself, between the arrival of S and its own
// hand-over of P: S(j) is committed behind the product with P(j-1), so nothing else touches O then.
//
// P is rounded to the cache's type: a relative error of half a step per probability, of the size of the result's own
// rounding.  The second product has no mixed-type form, and two of them (P as hi + lo) would cost half as much again.
// With fp16 the probabilities carry a factor 2^7, which keeps those a millionth of the largest away from subnormals.
//
// Pages.  A key tile is fetched page by page with 4-D TMA boxes {64 dims, page slots, 1 plane, 1 page}, 128-byte swizzle;
// pages outside the pool and pages behind the end are asked for beyond the last page, which fills zeros.  V's slots behind
// the end within the last page are zeroed in shared memory, since 0 x NaN would reach O; K needs no such care, its scores
// are masked.  Every wait is bounded.
#pragma once
#include <type_traits>

#include "kernels_batch.cuh"
#include "kernels_gemm_tc.cuh"

namespace swk {

constexpr int BT_THREADS = 352;     // 2 x 4 softmax warps, a TMA warp for Q and K, the MMA warp, a TMA warp for V
constexpr int BT_KEYS = 128;        // keys per tile
constexpr int BT_ROWS = 128;        // packed query rows per tile
constexpr int BT_PAGE_RING = 16;    // page-validity words kept (more than the key tiles ever in flight)
// Pairs of every 16 whose exponentials are polynomials: 4 of 16 (8192 tokens: 909 us; 2 of 16 922, 5 of 16 920, none 2 % more).
constexpr unsigned BT_POLY = 0x1111u;
constexpr float BT_GROW = 8.f;      // growth of the maximum (in powers of two) that triggers a rescaling

enum { BT_PROMPT = 0, BT_PREFIX = 1, BT_OWN = 2 };

template <int HALVES> struct BtShape {                                // D up to 64 * HALVES
    static constexpr int DP = 64 * HALVES;
    static constexpr int SLOT_BYTES = BT_KEYS * 128 * HALVES;         // one K or V tile
    static constexpr int Q_BYTES = BT_ROWS * 128 * HALVES;            // one query tile
    static constexpr int SLOTS = HALVES == 2 ? 5 : 10;
    static constexpr int BAR_BYTES = 512;
    static constexpr int SMEM_BYTES = 1024 + 2 * Q_BYTES + SLOTS * SLOT_BYTES + BAR_BYTES;
};

struct BtArgs {
    AttnView a;
    int mode, block, rows_per_tile;                                   // rows_per_tile: tokens of a tile (TQ)
    int tiles;                                                        // tiles of a piece: 2, or 1 where pairs would leave SMs idle
    int wide_out;                                                     // out's rows are multiples of 32 bytes
    int splits;                                                       // BT_PREFIX: cuts of the prefix
    float* part_o;                                                    // [slot][row][head][DP] fp32, unnormalised
    float2* part_ml;                                                  // [slot][row][head]: maximum in powers of two, sum
    int part_slot;                                                    // BT_OWN: its slot
};

struct BtItem {
    int seq, kvh, t0;                                                 // t0: first token of the pair within the sequence
    SeqSpan sp;                                                       // (the prefix: all rows, nothing of its own)
    int first_tile, np, slot;                                         // np: prefix tiles counted from first_tile on (then own tiles)
    int tiles[2];                                                     // key tiles of tile A and of tile B
};

// The idx-th piece of work, found by a whole warp; false when there are fewer.
__device__ __forceinline__ bool bt_locate(const BatchView& b, const BtArgs& g, int idx, BtItem& it)
{
    const int lane = threadIdx.x & 31, Hk = g.a.n_kv_heads, TQ = g.rows_per_tile, pair_rows = g.tiles * TQ;
    const int prefix_tiles = (b.prefix_len + BT_KEYS - 1) / BT_KEYS;
    it.first_tile = 0;
    it.slot = g.part_slot;
    if (g.mode == BT_PREFIX) {
        const int n = min(max(b.row_start[b.n_seqs], 0), b.n_rows), pairs = (n + pair_rows - 1) / pair_rows;
        if (idx >= pairs * Hk * g.splits) return false;
        const int s = idx % g.splits, rest = idx / g.splits;
        it.seq = -1;
        it.sp = {0, n, 0, 0};
        it.kvh = rest % Hk;
        it.t0 = rest / Hk * pair_rows;
        it.slot = s;
        it.first_tile = (int)((long long)prefix_tiles * s / g.splits);
        it.np = (int)((long long)prefix_tiles * (s + 1) / g.splits) - it.first_tile;
        it.tiles[0] = it.np;
        it.tiles[1] = g.tiles > 1 && it.t0 + TQ < n ? it.np : 0;
        return true;
    }
    for (int base = 0; base < b.n_seqs; base += 32) {
        SeqSpan sp = {};
        if (base + lane < b.n_seqs) sp = seq_span(b, base + lane);
        const int mine = (sp.n + pair_rows - 1) / pair_rows * Hk;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(FULL_WARP, upto, o);
            if (lane >= o) upto += v;
        }
        const unsigned m = __ballot_sync(FULL_WARP, idx < upto);
        if (m == 0) {
            idx -= __shfl_sync(FULL_WARP, upto, 31);
            continue;
        }
        const int at = __ffs(m) - 1;
        it.seq = base + at;
        it.sp = span_of(sp, at);
        idx -= __shfl_sync(FULL_WARP, upto - mine, at);
        const int pairs = (it.sp.n + pair_rows - 1) / pair_rows;
        it.kvh = idx % Hk;
        it.t0 = (pairs - 1 - idx / Hk) * pair_rows;                   // the longest pieces of a sequence first
        it.np = g.mode == BT_OWN ? 0 : prefix_tiles;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int t_end = min(it.sp.n, it.t0 + (x + 1) * TQ);     // tokens of this tile end here
            const bool some = x < g.tiles && it.t0 + x * TQ < it.sp.n;
            const int seen = seen_own(it.sp, t_end - 1);
            it.tiles[x] = some ? it.np + (seen + BT_KEYS - 1) / BT_KEYS : 0;
        }
        return true;
    }
    return false;
}

// ------------------------------------------------------------------------------ PTX wrappers
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, int c4, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4) : "memory");
}
// The MMA warp runs its loop with all lanes, and one of them issues: the operands then stay in uniform registers, which the
// instructions want (issued from under a per-lane branch, each one first moved its descriptors over and took about 165 cycles,
// three times what the tensor pipe needs for it).
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(p));
    return p != 0;
}
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// Descriptor of a V tile as the B operand [keys][dims], dims contiguous ("MN-major"): 64-dim groups one box apart, groups
// of 8 keys 1024 bytes apart, 128-byte swizzle.
__device__ __forceinline__ uint64_t tc_smem_desc_mn(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)((BT_KEYS * 128) >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float (&r)[32])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
                 "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
                   "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]),
                   "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]),
                   "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&u)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::"r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]),
                   "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld8(uint32_t addr, float (&r)[8])
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]) : "r"(addr));
}
__device__ __forceinline__ void tmem_st8(uint32_t addr, const float (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                 ::"f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "r"(addr) : "memory");
}
// The registers a load fills are operands of the wait, so that nothing reads them before it.
template <int N> __device__ __forceinline__ void tmem_wait_ld(float (&r)[N])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; i += 8)
        asm volatile("" : "+f"(r[i]), "+f"(r[i + 1]), "+f"(r[i + 2]), "+f"(r[i + 3]), "+f"(r[i + 4]), "+f"(r[i + 5]), "+f"(r[i + 6]), "+f"(r[i + 7]));
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// two fp32 operations in one instruction
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair2(float a, float b) { f32x2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ void split2(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) { f32x2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) { f32x2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ float max3(float a, float b, float c) { float r; asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
__device__ __forceinline__ float max2_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }   // NaN if any is
__device__ __forceinline__ float max3_nan(float a, float b, float c) { float r; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c)); return r; }
// 32 bytes at once: a full sector per lane, where lanes write rows of their own (p 32-byte aligned)
__device__ __forceinline__ void store32(void* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f, uint32_t g, uint32_t h)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e), "r"(f), "r"(g), "r"(h) : "memory");
}
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ unsigned batch_waits_over;                                 // bounded waits that ran out since the library was loaded (modulo 2^32); never cleared

// A wait of one role, by a whole warp: bounded, and over when another role has given up.  waits[0]: a role has given up;
// waits[1]: the limit, in 1024 cycles.  The lanes must take the same answer (the warp goes on to shuffles and barriers of its
// own) although each looks for itself: a lane leaves without success only BT_QUIET cycles after the giving up was
// known, by when nothing on the SM moves any more, and with a last look that then shows all lanes the same.  A block that gave
// up keeps its memory until what it asked for has landed (bt_give_up).
constexpr long long BT_QUIET = 2000000LL;                             // about a millisecond
__device__ __forceinline__ bool bt_try(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __noinline__ bool bt_wait_long(uint32_t bar, uint32_t parity, volatile int* waits)
{
    const long long t0 = clock64(), limit = (long long)waits[1] << 10;
    long long over = 0;                                               // when this lane knew
    for (uint32_t it = 0;; ++it) {
        if (bt_try(bar, parity)) return true;
        if ((it & 63u) != 63u) continue;
        const long long now = clock64();
        if (over) {
            if (now - over > BT_QUIET) return bt_try(bar, parity);
        } else if (waits[0]) {
            over = now;
        } else if (now - t0 > limit) {
            over = now;
            waits[0] = 1;
            atomicAdd(&batch_waits_over, 1u);
        }
    }
}
__device__ __forceinline__ bool bt_wait(uint32_t bar, uint32_t parity, volatile int* waits)
{
    for (int it = 0; it < 4; ++it)
        if (bt_try(bar, parity)) return true;
    return bt_wait_long(bar, parity, waits);
}
// The end of a block, behind a barrier of all its threads: copies, products and answers still on their way after a wait that
// ran out land before its memory is given back.
__device__ __forceinline__ void bt_give_up(volatile int* waits)
{
    if (!waits[0]) return;
    const long long t0 = clock64();
    while (clock64() - t0 < BT_QUIET) { }
}

// ------------------------------------------------------------------------------ which piece next
// Pieces differ in length (causal edges, ragged sequences), so whole prompts are launched one block per piece and a block that
// is done takes over the next block not yet launched (cluster launch control): pieces go out in order, to whoever is free,
// with the pipeline kept full.  (Dealt out in turn: 5003 ragged rows 158 us, 8192 rows 915.)  A call with a shared prefix splits
// the SMs between two launches instead (taking over there: 8 x 32 rows behind 3000 124 -> 112 us, 20 x 16 behind 1000 63 -> 73).
// The K warp asks for the next piece while the current one runs; the answer is read by every warp at its own pace from a ring of
// two.
__device__ __forceinline__ void bt_ask_piece(uint32_t answer, uint32_t bar)
{
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(bar) : "memory");
}
__device__ __forceinline__ int bt_answer(uint32_t answer)             // the block taken over, or -1: none is left
{
    uint32_t taken, x = 0;
    asm volatile("{\n\t.reg .b128 h;\n\t.reg .pred p;\n\t.reg .b32 y, z, w;\n\t"
                 "ld.shared.b128 h, [%2];\n\t"
                 "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
                 "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, y, z, w}, h;\n\t}"
                 : "=r"(taken), "=&r"(x) : "r"(answer) : "memory");
    return taken ? (int)x : -1;
}
template <bool PART> struct BtPieces {
    uint32_t answers, full, empty;                                    // two answers of 16 bytes, their barriers
    volatile int* waits;
    int idx, n;
    __device__ __forceinline__ void begin() { idx = blockIdx.x; n = 0; }
    // K warp, before it starts on a piece
    __device__ __forceinline__ bool ask()
    {
        if (PART) return true;
        const uint32_t at = n & 1, turn = (n >> 1) & 1;
        if (!bt_wait(empty + 8u * at, turn ^ 1u, waits)) return false;
        if (elect_one()) {
            mbar_expect_tx(full + 8u * at, 16u);
            bt_ask_piece(answers + 16u * at, full + 8u * at);
        }
        return true;
    }
    // every warp, behind a piece: false when there is none left (or a wait ran out: ok becomes false)
    __device__ __forceinline__ bool next(bool& ok)
    {
        if (PART) {
            idx += gridDim.x;
            return true;
        }
        const uint32_t at = n & 1, turn = (n >> 1) & 1;
        ok = bt_wait(full + 8u * at, turn, waits);
        if (!ok) return false;
        idx = bt_answer(answers + 16u * at);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(empty + 8u * at);
        ++n;
        return idx >= 0;
    }
};

// Bit i: key 32 q + i of a tile is shown to a row that sees the tile's keys below `seen`, and lies on a page of the pool.
__device__ __forceinline__ unsigned bt_shown(unsigned pages, int page_shift, int seen, int q)
{
    unsigned w = 0;
    if (page_shift >= 5) {
        w = (pages >> ((32 * q) >> page_shift)) & 1u ? 0xFFFFFFFFu : 0u;
    } else {
        const int slots = 1 << page_shift;                            // 8 or 16
        const unsigned one = (1u << slots) - 1u;
        unsigned bits = pages >> ((32 * q) >> page_shift);
        for (int at = 0; at < 32; at += slots, bits >>= 1)
            if (bits & 1u) w |= one << at;
    }
    const int n = seen - 32 * q;
    return n >= 32 ? w : n <= 0 ? 0u : w & ((1u << n) - 1u);
}

// 2^x for two values on the multiply-add pipe, x in about [-126, 127] (below, and for NaN: 2^-126): x = n + f with n the nearest integer,
// 2^f as a polynomial, n added to its exponent.  The coefficients minimise the largest relative error on [-1/2, 1/2] (a linear
// programme over 2001 Chebyshev points): 7.5e-5 for degree 3, which is a fiftieth of half a step of bf16; 2.6e-6 for degree 4, with
// which fp16's half step is 180 times as large.
template <typename T> __device__ __forceinline__ void ex2_poly(float x0, float x1, float& y0, float& y1)
{
    const float round = 12582912.f;                                   // 1.5 * 2^23: adding it leaves the nearest integer in the low bits
    const f32x2 x = pair2(fmaxf(x0, -126.f), fmaxf(x1, -126.f));
    const f32x2 t = add2(x, pair2(round, round));
    const f32x2 f = fma2(add2(t, pair2(-round, -round)), pair2(-1.f, -1.f), x);
    f32x2 p;
    if (std::is_same<T, __half>::value) {
        p = fma2(pair2(0.009567738510668278f, 0.009567738510668278f), f, pair2(0.05591749772429466f, 0.05591749772429466f));
        p = fma2(p, f, pair2(0.24024811387062073f, 0.24024811387062073f));
        p = fma2(p, f, pair2(0.6931219100952148f, 0.6931219100952148f));
        p = fma2(p, f, pair2(0.9999992251396179f, 0.9999992251396179f));
    } else {
        p = fma2(pair2(0.0551714189350605f, 0.0551714189350605f), f, pair2(0.24261116981506348f, 0.24261116981506348f));
        p = fma2(p, f, pair2(0.6932610273361206f, 0.6932610273361206f));
        p = fma2(p, f, pair2(0.9999280571937561f, 0.9999280571937561f));
    }
    float p0, p1, t0, t1;
    split2(p, p0, p1);
    split2(t, t0, t1);
    y0 = __int_as_float(__float_as_int(p0) + (__float_as_int(t0) << 23));
    y1 = __int_as_float(__float_as_int(p1) + (__float_as_int(t1) << 23));
}

// 32 scores -> probabilities (16 bits each, two to a register), their sum added up.  POLY: which of the 16 pairs take the
// polynomial instead of the special function unit.
template <typename T, unsigned POLY>
__device__ __forceinline__ void bt_weights(const float (&s)[32], f32x2 c2, f32x2 off2, f32x2 (&sum)[2], uint32_t (&p)[16])
{
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float p0, p1;
        split2(fma2(pair2(s[2 * i], s[2 * i + 1]), c2, off2), p0, p1);
        if ((POLY >> i) & 1u) {
            ex2_poly<T>(p0, p1, p0, p1);
        } else {
            p0 = ex2(p0);
            p1 = ex2(p1);
        }
        sum[i & 1] = add2(sum[i & 1], pair2(p0, p1));
        p[i] = pack2(p0, p1, T());
    }
}
__device__ __forceinline__ float bt_highest(const float (&s)[32])      // NaN if any is
{
    float x0 = s[0], x1 = s[1];
#pragma unroll
    for (int i = 2; i < 30; i += 4) {
        x0 = max3_nan(x0, s[i], s[i + 1]);
        x1 = max3_nan(x1, s[i + 2], s[i + 3]);
    }
    return max2_nan(max3_nan(x0, s[30], s[31]), x1);
}
// P of half h of the keys is in TMEM: the MMA warp may use it.
__device__ __forceinline__ void bt_hand_over(uint32_t p_bar, int h)
{
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(p_bar + 8u * h);
}
// Scores are weighed as 2^(c s + off), off = BIAS - c m rounded once, in one multiply-add.  Where c m is large its rounding is too
// (half a step of 2^30 is 32: a factor of 2^32 on all weights of the row, which no 16 bits hold), so beyond BT_FAR a row subtracts m
// from its scores first, an addition per score.  Below it the factor is at most 2^(2^-11).
constexpr float BT_FAR = 16384.f;
// The weights of a key tile with such rows, from the scores in TMEM on: their sum.  Rare; called from one place outside the
// softmax's common path, which keeps its registers (two calls inside it: 512 tokens 13.1 -> 13.8 us; in line: 8192 tokens 3 % more).
template <typename T>
__device__ __noinline__ float bt_weights_far(uint32_t s_at, uint32_t p_bar, float c, float m, int seen, unsigned pages, int page_shift)
{
    constexpr float BIAS = std::is_same<T, __half>::value ? 7.f : 0.f;
    float off = BIAS - (m == -INFINITY ? 0.f : m * c);
    const bool far = fabsf(off) > BT_FAR;
    const float by = far ? m : 0.f;
    if (far) off = BIAS;
    const f32x2 c2 = pair2(c, c), off2 = pair2(off, off);
    f32x2 sum[2] = {0ull, 0ull};
#pragma unroll 1
    for (int h = 1; h >= 0; --h) {                                    // the upper half of the keys goes first; both of its quarters are read before P overwrites them
        float a[32], b[32];
        uint32_t p[16];
        tmem_ld32(s_at + 64 * h, a);
        tmem_ld32(s_at + 64 * h + 32, b);
        tmem_wait_ld(a);
        tmem_wait_ld(b);
        const unsigned shown[2] = {bt_shown(pages, page_shift, seen, 2 * h), bt_shown(pages, page_shift, seen, 2 * h + 1)};
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            a[i] = (shown[0] >> i) & 1u ? a[i] - by : -INFINITY;
            b[i] = (shown[1] >> i) & 1u ? b[i] - by : -INFINITY;
        }
        bt_weights<T, 0u>(a, c2, off2, sum, p);
        tmem_st16(s_at + 64 + 32 * h, p);
        bt_weights<T, 0u>(b, c2, off2, sum, p);
        tmem_st16(s_at + 80 + 32 * h, p);
        bt_hand_over(p_bar, h);
    }
    float l0, l1;
    split2(add2(sum[0], sum[1]), l0, l1);
    return l0 + l1;
}
// Whether a row's maximum has outgrown what its sums are scaled by.
__device__ __forceinline__ bool bt_outgrown(float top, float m, float c) { return top > m && (m == -INFINITY || (top - m) * c > BT_GROW); }

// Such rows get the new maximum, their sums and (behind the first tile) O rescaled.  The others of the warp keep theirs: a row's
// bits do not depend on its neighbours' scores nor on the unused rows of a tile, which hold anything.  (They do depend on where the
// tile's causal edge lies: a tile with hidden keys takes no polynomials.)
template <int DP> __device__ __forceinline__ void bt_rescale(uint32_t o_at, float c, float top, bool mine, bool first, float& m, float& l)
{
    const float m_new = mine ? top : m, shrink = mine ? ex2((m - m_new) * c) : 1.f;
    l *= shrink;
    m = m_new;
    if (first) return;
#pragma unroll 1
    for (int i = 0; i < DP; i += 8) {                                 // rare; few registers beside the scores
        float o[8];
        tmem_ld8(o_at + i, o);
        tmem_wait_ld(o);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] *= shrink;
        tmem_st8(o_at + i, o);
    }
}
// The softmax warps' part of one key tile: S in, P out (over the upper half of S), the row's maximum m and sum l brought up to
// date.  s_at, o_at: this warp's lanes of S and O; p_bar: the two hand-over barriers.  Scores come a quarter (32 keys) at a
// time; the upper half of the keys goes first.
// MASKED: some keys are hidden from some rows.  False: m and O are up to date, but the weights are bt_weights_far's to make.
template <typename T, int DP, bool MASKED>
__device__ __forceinline__ bool bt_softmax(uint32_t s_at, uint32_t o_at, uint32_t p_bar, float c, int seen, unsigned pages, int page_shift, bool first, float& m, float& l)
{
    constexpr unsigned POLY = MASKED ? 0u : BT_POLY;                  // (the polynomial gives a hidden key 2^-126, not 0)
    auto hide = [&](int q, float (&s)[32]) {
        if (!MASKED) return;
        const unsigned shown = bt_shown(pages, page_shift, seen, q);
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (!((shown >> i) & 1u)) s[i] = -INFINITY;
    };
    constexpr float BIAS = std::is_same<T, __half>::value ? 7.f : 0.f;
    float s0[32], s1[32], s2[32], s3[32];
    tmem_ld32(s_at, s0);
    tmem_wait_ld(s0);
    tmem_ld32(s_at + 32, s1);
    hide(0, s0);
    float top = bt_highest(s0);
    tmem_wait_ld(s1);
    tmem_ld32(s_at + 64, s2);
    hide(1, s1);
    top = max2_nan(top, bt_highest(s1));
    tmem_wait_ld(s2);
    tmem_ld32(s_at + 96, s3);
    hide(2, s2);
    top = max2_nan(top, bt_highest(s2));
    tmem_wait_ld(s3);
    hide(3, s3);
    top = max2_nan(top, bt_highest(s3));
    // A score of NaN or +infinity makes the row NaN, through l: the polynomial below would give such a key, and every key beside an
    // infinite score, a weight near zero.
    if (!(top < INFINITY)) l = __int_as_float(0x7FFFFFFF);
    const bool grown = bt_outgrown(top, m, c);
    if (__any_sync(FULL_WARP, grown)) bt_rescale<DP>(o_at, c, top, grown, first, m, l);
    const float off = BIAS - (m == -INFINITY ? 0.f : m * c);
    if (__any_sync(FULL_WARP, fabsf(off) > BT_FAR)) return false;
    const f32x2 c2 = pair2(c, c), off2 = pair2(off, off);
    f32x2 sum[2] = {0ull, 0ull};
    uint32_t p[16];
    tmem_ld32(s_at, s0);
    bt_weights<T, POLY>(s2, c2, off2, sum, p);
    tmem_st16(s_at + 96, p);
    bt_weights<T, POLY>(s3, c2, off2, sum, p);
    tmem_st16(s_at + 112, p);
    bt_hand_over(p_bar, 1);
    tmem_wait_ld(s0);
    tmem_ld32(s_at + 32, s1);
    hide(0, s0);
    bt_weights<T, POLY>(s0, c2, off2, sum, p);
    tmem_st16(s_at + 64, p);
    tmem_wait_ld(s1);
    hide(1, s1);
    bt_weights<T, POLY>(s1, c2, off2, sum, p);
    tmem_st16(s_at + 80, p);
    bt_hand_over(p_bar, 0);
    float l0, l1;
    split2(add2(sum[0], sum[1]), l0, l1);
    l += l0 + l1;
    return true;
}

// A row's result to the output (a function of its own: inlined, its registers crowd out the softmax's).  Every lane takes
// part in the reading; `live` lanes store.
template <typename T, int COLS> __device__ __noinline__ void bt_store_out(uint32_t o_at, T* dst, int dims, bool some, bool live, bool wide, float l)
{
    const float inv = l == 0.f ? 0.f : 1.f / l;                       // 0: the row sees nothing
#pragma unroll 1
    for (int i = 0; i < COLS; i += 32) {
        float o[32];
        if (some) {
            tmem_ld32(o_at + i, o);
            tmem_wait_ld(o);
        }
        if (live) {
            uint32_t v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = l == 0.f ? 0u : pack2(o[2 * e] * inv, o[2 * e + 1] * inv, T());
            if (wide) {
#pragma unroll
                for (int e = 0; e < 16; e += 8)
                    if (i + 2 * e < dims) store32(dst + i + 2 * e, v[e], v[e + 1], v[e + 2], v[e + 3], v[e + 4], v[e + 5], v[e + 6], v[e + 7]);
            } else {
#pragma unroll
                for (int e = 0; e < 16; e += 4)
                    if (i + 2 * e < dims) *reinterpret_cast<uint4*>(dst + i + 2 * e) = make_uint4(v[e], v[e + 1], v[e + 2], v[e + 3]);
            }
        }
    }
}

// ------------------------------------------------------------------------------ the kernel
// grid: one block per piece (PART: persistent blocks that take pieces blockIdx.x, + gridDim.x, ...); block = 352.
// PART: leaves parts in the workspace (BT_PREFIX, BT_OWN) rather than results (BT_PROMPT).
template <typename T, int HALVES, bool PART>
__global__ void __launch_bounds__(BT_THREADS, 1)
attn_batch_tc_kernel(const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ CUtensorMap map_q, BatchView b, BtArgs g)
{
    typedef BtShape<HALVES> S;
    constexpr int DP = S::DP;
    constexpr bool HALF = std::is_same<T, __half>::value;
    constexpr uint32_t TYPE = HALF ? 0u : 1u;                         // operand format of both products
    constexpr uint32_t IDESC_QK = (1u << 4) | (TYPE << 7) | (TYPE << 10) | ((uint32_t)(BT_KEYS >> 3) << 17) | ((uint32_t)(BT_ROWS >> 4) << 24);
    constexpr uint32_t IDESC_PV = (1u << 4) | (TYPE << 7) | (TYPE << 10) | (1u << 16) | ((uint32_t)(DP >> 3) << 17) | ((uint32_t)(BT_ROWS >> 4) << 24);
    constexpr float BIAS = HALF ? 7.f : 0.f;

    pdl_trigger();
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_sh = base, ring = base + 2 * S::Q_BYTES, bars = ring + S::SLOTS * S::SLOT_BYTES;
    auto full = [&](int s) { return bars + 8u * s; };
    auto empty = [&](int s) { return bars + 8u * (S::SLOTS + s); };
    const uint32_t b2 = bars + 16u * S::SLOTS;
    auto q_full = [&](int x) { return b2 + 8u * x; };
    auto q_empty = [&](int x) { return b2 + 16u + 8u * x; };
    auto s_full = [&](int x) { return b2 + 32u + 8u * x; };
    auto p_ready = [&](int x, int h) { return b2 + 48u + 8u * (2 * x + h); };
    auto o_full = [&](int x) { return b2 + 80u + 8u * x; };
    const uint32_t landed = b2 + 96u;
    const uint32_t piece_bars = b2 + 104u, answers = bars + S::BAR_BYTES - 32u;   // answers: 16-byte aligned
    __shared__ uint32_t tmem_base_sh;
    __shared__ int waits_sh[2];
    __shared__ unsigned page_bits[BT_PAGE_RING];                      // bit p: page p of that key tile lies in the pool
    volatile int* waits = waits_sh;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = g.a.n_heads / g.a.n_kv_heads, TQ = g.rows_per_tile;
    if (warp == 9) {
        if (lane == 0) {
            for (int s = 0; s < S::SLOTS; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
            for (int x = 0; x < 2; ++x) {
                mbar_init(q_full(x), 1); mbar_init(q_empty(x), 1); mbar_init(s_full(x), 1); mbar_init(o_full(x), 1);
                mbar_init(p_ready(x, 0), 4); mbar_init(p_ready(x, 1), 4);
            }
            mbar_init(landed, 1);
            for (int i = 0; i < 2; ++i) { mbar_init(piece_bars + 8u * i, 1); mbar_init(piece_bars + 16u + 8u * i, 11); }
            waits[0] = 0;
            waits[1] = g.a.wait_kcycles;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_sh)), "r"(512));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (tid == 256) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_kv) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base_sh;
    BtPieces<PART> pieces = {answers, piece_bars, piece_bars + 16u, waits, 0, 0};
    pieces.begin();
    bool more_pieces = true;
    auto s_col = [&](int x) { return tmem + 128u * x; };              // S, then P, of tile x
    auto o_col = [&](int x) { return tmem + 256u + 128u * x; };

    if (warp == 8 || warp == 10) {
        // ---------------------------------------------------------------- TMA: one warp for the queries and K tiles, one for V tiles
        // The ring holds K and V tiles in turn.  A box costs its issuing lane some 90 cycles: with pages of 16, the 32 boxes of a
        // key tile's K and V would take one warp about as long as the products.
        const int kv = warp == 10;
        const int per_tile = BT_KEYS >> b.page_shift;                 // pages per key tile, 1..16
        uint32_t slot = kv, turn = 0, q_turn[2] = {0, 0}, landed_turn = 0;   // turn: parity of the ring's current pass
        int tile_no = 0;
        bool ok = true;
        BtItem it;
        for (; ok && more_pieces; more_pieces = ok && pieces.next(ok)) {
            if (kv == 0) ok = pieces.ask();
            if (!ok) break;
            if (!bt_locate(b, g, pieces.idx, it)) { if (PART) break; continue; }
            const int n_tiles = max(it.tiles[0], it.tiles[1]);
            const int plane = (g.block * 2 + kv) * g.a.n_kv_heads + it.kvh;
            if (kv == 0) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (!ok || it.tiles[x] == 0) continue;
                    ok = bt_wait(q_empty(x), q_turn[x] ^ 1u, waits);
                    q_turn[x] ^= 1u;
                    if (ok && elect_one()) {
                        mbar_expect_tx(q_full(x), (uint32_t)(TQ * G * 128 * HALVES));
                        for (int hf = 0; hf < HALVES; ++hf)
                            tma_load_3d(q_sh + x * S::Q_BYTES + hf * (BT_ROWS * 128), &map_q, 64 * hf, it.kvh * G, it.sp.r0 + it.t0 + x * TQ, q_full(x));
                    }
                }
            }
            // lane p: page p of the next tile, looked up a tile ahead
            auto look_up = [&](int j) {
                const bool shared_part = j < it.np;
                const int key0 = (shared_part ? it.first_tile + j : j - it.np) * BT_KEYS;
                const int left = (shared_part ? b.prefix_len : it.sp.len) - key0;
                int page = -1;
                if (j < n_tiles && lane < per_tile && (lane << b.page_shift) < left) {
                    const int at = (key0 >> b.page_shift) + lane;
                    page = shared_part ? b.prefix_pages[at] : b.page_table[(size_t)it.seq * b.table_stride + at];
                }
                return page;
            };
            int next_page = look_up(0);
            for (int j = 0; ok && j < n_tiles; ++j, ++tile_no) {
                const bool good = (unsigned)next_page < (unsigned)b.n_pages;
                const int page = good ? next_page : b.n_pages;        // beyond the last page: zeros
                const unsigned pages = __ballot_sync(FULL_WARP, good);
                next_page = look_up(j + 1);
                const bool shared_part = j < it.np;
                const int left = (shared_part ? b.prefix_len - (it.first_tile + j) * BT_KEYS : it.sp.len - (j - it.np) * BT_KEYS);   // keys of this tile that exist
                const int tail = left & (b.page_size - 1);            // slots of the last page that hold something
                // a V tile with unwritten slots: they are zeroed before the product may read them
                const bool mend = kv == 1 && left < BT_KEYS && tail != 0 && ((pages >> (left >> b.page_shift)) & 1u);
                ok = bt_wait(empty(slot), turn ^ 1u, waits);
                if (!ok) break;
                const uint32_t bar = mend ? landed : full(slot), dst = ring + slot * S::SLOT_BYTES;
                const bool asks = !(g.a.withhold && kv == 0 && tile_no == 0);
                if (elect_one()) {
                    if (kv == 0) page_bits[tile_no & (BT_PAGE_RING - 1)] = pages;
                    if (asks) mbar_expect_tx(bar, (uint32_t)S::SLOT_BYTES);
                }
                __syncwarp();
                for (int p = 0; asks && p < per_tile; ++p) {
                    const int pg = __shfl_sync(FULL_WARP, page, p);
                    if (elect_one()) {
#pragma unroll
                        for (int hf = 0; hf < HALVES; ++hf) tma_load_4d(dst + hf * (BT_KEYS * 128) + (p << b.page_shift) * 128, &map_kv, 64 * hf, 0, plane, pg, bar);
                    }
                }
                if (mend) {
                    ok = bt_wait(landed, landed_turn, waits);
                    landed_turn ^= 1u;
                    if (!ok) break;
                    const int row1 = ((left >> b.page_shift) + 1) << b.page_shift;
                    for (int i = lane; i < (row1 - left) * 8 * HALVES; i += 32) {
                        const int row = left + i / (8 * HALVES), piece = i % (8 * HALVES);
                        const uint32_t a = dst + (piece >> 3) * (BT_KEYS * 128) + row * 128 + (piece & 7) * 16;    // whole rows: the swizzle stays inside
                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(a), "r"(0) : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(full(slot));
                }
                slot += 2;
                if (slot >= S::SLOTS) { slot -= S::SLOTS; turn ^= 1u; }
            }
        }
    } else if (warp == 9) {
        // ---------------------------------------------------------------- tensor pipe
        uint32_t slot = 0, turn = 0, q_turn[2] = {0, 0}, p_turn[2] = {0, 0};
        bool ok = true;
        BtItem it;
        for (; ok && more_pieces; more_pieces = ok && pieces.next(ok)) {
            if (!bt_locate(b, g, pieces.idx, it)) { if (PART) break; continue; }
            const int n_tiles = max(it.tiles[0], it.tiles[1]);
            auto commit = [&](uint32_t bar) { if (elect_one()) tc_commit(bar); };
            auto scores = [&](int x, uint32_t k_sh) {                 // S(x) = Q(x) K^T
                if (elect_one()) {
                    const uint64_t qd = tc_smem_desc(q_sh + x * S::Q_BYTES), kd = tc_smem_desc(k_sh);
                    uint32_t q_lo = (uint32_t)qd, k_lo = (uint32_t)kd;
                    asm volatile("" : "+r"(q_lo), "+r"(k_lo));        // (kept from being precomputed for all steps, slots and tiles)
#pragma unroll
                    for (int k = 0; k < 4 * HALVES; ++k) {            // 16 dims a step: 32 bytes, 64 dims a box
                        const uint32_t step = ((k >> 2) * (BT_KEYS * 128) + (k & 3) * 32) >> 4;
                        tc_mma(s_col(x), (qd >> 32 << 32) | (q_lo + step), (kd >> 32 << 32) | (k_lo + step), IDESC_QK, k > 0);
                    }
                    tc_commit(s_full(x));
                }
            };
            auto weigh = [&](int x, uint32_t v_sh, bool first) {      // O(x) (+)= P(x) V
                const uint64_t vd = tc_smem_desc_mn(v_sh);
#pragma unroll
                for (int h = 1; h >= 0; --h) {                        // the upper half of the keys is ready first
                    if (!bt_wait(p_ready(x, h), p_turn[x], waits)) return false;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int k = 4 * h; k < 4 * h + 4; ++k)       // 16 keys a step: 8 columns of P, 2048 bytes of V
                            tc_mma_ts(o_col(x), s_col(x) + 64 + 8 * k, vd + (uint64_t)(k * (2048 >> 4)), IDESC_PV, !first || k != 4);
                    }
                }
                p_turn[x] ^= 1u;
                return true;
            };
#pragma unroll
            for (int x = 0; x < 2; ++x)
                if (ok && it.tiles[x]) { ok = bt_wait(q_full(x), q_turn[x], waits); q_turn[x] ^= 1u; }
            if (ok && n_tiles > 0) {
                ok = bt_wait(full(slot), turn, waits);
                tc_fence_after();
                if (ok) {
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (it.tiles[x]) {
                            scores(x, ring + slot * S::SLOT_BYTES);
                            if (it.tiles[x] == 1) commit(q_empty(x));
                        }
                    commit(empty(slot));
                    if (++slot == S::SLOTS) { slot = 0; turn ^= 1u; }
                }
            }
            for (int j = 0; ok && j < n_tiles; ++j) {
                const uint32_t v_slot = slot, v_turn = turn;
                if (++slot == S::SLOTS) { slot = 0; turn ^= 1u; }
                ok = bt_wait(full(v_slot), v_turn, waits);
                const bool more = j + 1 < n_tiles;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (ok && j < it.tiles[x]) {
                        ok = weigh(x, ring + v_slot * S::SLOT_BYTES, j == 0);
                        if (ok && j + 1 == it.tiles[x]) commit(o_full(x));
                    }
                    if (ok && x == 1) commit(empty(v_slot));
                    if (ok && j + 1 < it.tiles[x]) {
                        ok = bt_wait(full(slot), turn, waits);
                        if (ok) {
                            tc_fence_after();
                            scores(x, ring + slot * S::SLOT_BYTES);
                            if (j + 2 == it.tiles[x]) commit(q_empty(x));
                        }
                    }
                }
                if (ok && more) {
                    commit(empty(slot));
                    if (++slot == S::SLOTS) { slot = 0; turn ^= 1u; }
                }
            }
        }
    } else if (warp < 8) {
        // ---------------------------------------------------------------- softmax: a thread owns one packed query row
        const int x = warp >> 2, rho = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = s_col(x) + lanes, o_at = o_col(x) + lanes;
        const int tok = rho / G, head_in = rho - tok * G;
        const unsigned all_pages = 0xFFFFu >> (16 - (BT_KEYS >> b.page_shift));
        uint32_t s_turn = 0, o_turn = 0;
        int tile_no = 0;
        bool ok = true;
        BtItem it;
        for (; ok && more_pieces; more_pieces = ok && pieces.next(ok)) {
            if (!bt_locate(b, g, pieces.idx, it)) { if (PART) break; continue; }
            const int n_tiles = max(it.tiles[0], it.tiles[1]), mine = it.tiles[x];
            const int t = it.t0 + x * TQ + tok;                       // token within the sequence
            const bool live = x < g.tiles && tok < TQ && t < it.sp.n && (g.mode == BT_PREFIX || t < g.a.max_rows);
            // scores in powers of two; rows of the tile that belong to no token hold anything and must not ask for rescaling or the like
            const float c = live ? g.a.scale * 1.4426950408889634f : 0.f;
            const int own_seen = seen_own(it.sp, t);                  // own keys that this row sees
            const int all_see = seen_own(it.sp, it.t0 + x * TQ);      // ... that every row of the tile sees
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < mine; ++j) {
                ok = bt_wait(s_full(x), s_turn, waits);
                if (!ok) break;
                s_turn ^= 1u;
                tc_fence_after();
                const int key0 = (j < it.np ? it.first_tile + j : j - it.np) * BT_KEYS;
                const int seen = j < it.np ? b.prefix_len - key0 : own_seen - key0;       // this row sees keys below this
                const unsigned pages = page_bits[(tile_no + j) & (BT_PAGE_RING - 1)];
                const bool masked = key0 + BT_KEYS > (j < it.np ? b.prefix_len : all_see) || pages != all_pages;
                const bool done = masked ? bt_softmax<T, DP, true>(s_at, o_at, p_ready(x, 0), c, seen, pages, b.page_shift, j == 0, m, l)
                                         : bt_softmax<T, DP, false>(s_at, o_at, p_ready(x, 0), c, seen, pages, b.page_shift, j == 0, m, l);
                if (!done) l += bt_weights_far<T>(s_at, p_ready(x, 0), c, m, seen, pages, b.page_shift);
            }
            tile_no += n_tiles;
            if (!ok) break;
            if (mine > 0) {
                ok = bt_wait(o_full(x), o_turn, waits);
                if (!ok) break;
                o_turn ^= 1u;
                tc_fence_after();
            }
            if (m == -INFINITY && l == l) l = 0.f;                    // no score but -infinity: what the polynomial made of them does not count
            const int row = it.sp.r0 + t, head = it.kvh * G + head_in;
            if (PART) {
                const size_t at = ((size_t)it.slot * b.n_rows + row) * g.a.n_heads + head;
                if (live) g.part_ml[at] = make_float2(m * c - BIAS, l);
#pragma unroll 1
                for (int i = 0; i < DP; i += 32) {
                    float o[32];
                    if (mine > 0) {
                        tmem_ld32(o_at + i, o);
                        tmem_wait_ld(o);
                    }
                    if (live && l != 0.f) {
                        float* dst = g.part_o + at * DP + i;
#pragma unroll
                        for (int e = 0; e < 32; e += 8)
                            store32(dst + e, __float_as_uint(o[e]), __float_as_uint(o[e + 1]), __float_as_uint(o[e + 2]), __float_as_uint(o[e + 3]),
                                    __float_as_uint(o[e + 4]), __float_as_uint(o[e + 5]), __float_as_uint(o[e + 6]), __float_as_uint(o[e + 7]));
                    }
                }
            } else {
                T* dst = reinterpret_cast<T*>(g.a.out) + ((size_t)row * g.a.n_heads + head) * g.a.head_dim;
                bt_store_out<T, DP>(o_at, dst, g.a.head_dim, mine > 0, live, g.wide_out != 0, l);
            }
            tc_fence_before();                                        // O is read: the next piece's product may overwrite it
        }
    }
    __syncthreads();
    bt_give_up(waits);
    pdl_wait();                                           // (a launch before this one in the same call ends first)
    if (warp == 9) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512));
    }
}

} // namespace swk
