// Attention of few query rows per sequence over the paged cache (decoding steps, verified drafts, scoring windows): every
// cached K,V byte is read once and meets at most 64 query rows, so the kernel is bound by HBM; what it must get right is
// to keep enough bytes in flight on every SM, whatever the lengths of the sequences, and to lose no time between them.
//
// Work.  A piece of work ("item") is one kv head of one sequence, or of the prefix with the rows of all sequences (when
// those are few enough to fit a tile; otherwise the many-row kernel next door takes the prefix).  Items are numbered in
// units of 16 MT keys, and the units are cut into equal ranges, one per worker: every worker streams the same number of
// bytes, and a single long sequence is split over all of them.  A worker leaves one partial result per item it touches -
// unnormalised sums, their maximum, the sum of probabilities - in slot item + worker (both grow together, so no two
// meet); the joining kernel adds the slots of an item in order, so results do not depend on timing.
//
// A worker is MT warps that share the keys and split the query rows (16 each); a CTA holds 8 / MT workers.  No two warps
// hold parts of the same sum, so the end of an item costs its stores and nothing else (with a unit's keys split over four
// warps, joining them through shared memory took 1.8 us per item, more than a short item's stream).  Each worker's first
// warp asks for the next unit with TMA as soon as one is used up: three units of 8 MT KB per worker, 192 KB per SM, are in
// flight, four times what covers HBM's latency at 44 GB/s per SM.
// Products are mma.sync.m16n8k16.  (tcgen05 needs 128 rows a tile; at 16 to 64 rows the tensor pipe is idle most of the
// time either way.)  P is rounded to the cache's type as in the many-row kernel, fp16 with the same factor 2^7.
#pragma once
#include "kernels_batch_tc.cuh"

namespace swk {

constexpr int BD_WARPS = 8, BD_THREADS = 32 * BD_WARPS;
// Most packed query rows (tokens x heads of a group) of an item (12 sequences of 63: 35 us here, 41 with the many-row kernel).
constexpr int BD_MAX_ROWS = 64;

template <int HALVES, int MT> struct BdShape {
    static constexpr int DP = 64 * HALVES;
    static constexpr int KEYS = 16 * MT;                          // keys per unit
    static constexpr int WORKERS = BD_WARPS / MT;                       // of a CTA
    static constexpr int TILE_BYTES = KEYS * 128 * HALVES;        // K or V of a unit
    static constexpr int STAGES = HALVES == 2 ? 3 : 6;
    static constexpr int RING_BYTES = WORKERS * STAGES * 2 * TILE_BYTES;
    static constexpr int Q_BYTES = 16 * 128 * HALVES;             // a warp's queries
    static constexpr int SMEM_BYTES = 1024 + RING_BYTES + BD_WARPS * Q_BYTES;
};

struct BdArgs {
    AttnView a;
    int block, prefix_here;                               // prefix_here: the prefix is part of this launch's items
    int whole_boxes, planes;                              // a box holds K and V with all dims (head_dim 64 or 128); planes of the pool then
    float* part_o;                                        // [item + worker][16 MT][DP]
    float2* part_ml;                                      // [item + worker][16 MT]
    int* item_first;                                      // [item]: first and last worker that holds units of it
    int* item_last;
};

template <int KEYS> __device__ __forceinline__ int bd_units(const SeqSpan& s) { return s.n > 0 ? (s.len + KEYS - 1) / KEYS : 0; }

// A walk over a worker's units by a whole warp; all lanes hold the same values, except that lane i keeps the span of sequence
// base + i, so that going on to the next sequence costs a trip to memory once in 32.
struct BdWalk {
    int item, seq, kvh, unit, units;                      // seq -1: the prefix
    SeqSpan sp;
    int base;
    SeqSpan ahead;
};
__device__ __forceinline__ SeqSpan bd_span(const BatchView& b, BdWalk& w, int seq)
{
    if (seq < w.base || seq >= w.base + 32) {
        const int i = seq + (threadIdx.x & 31);
        w.base = seq;
        w.ahead = {};
        if (i < b.n_seqs) w.ahead = seq_span(b, i);
    }
    const int at = seq - w.base;
    return span_of(w.ahead, at);
}
template <int KEYS> __device__ __forceinline__ void bd_enter(const BatchView& b, const BdArgs& g, BdWalk& w)
{
    while (w.seq < b.n_seqs) {                            // skips sequences without units; the caller has units left
        w.sp = bd_span(b, w, w.seq);
        w.units = bd_units<KEYS>(w.sp);
        if (w.units > 0) break;
        ++w.seq;
    }
    w.item = (g.prefix_here ? g.a.n_kv_heads : 0) + w.seq * g.a.n_kv_heads + w.kvh;
}
template <int KEYS> __device__ __forceinline__ void bd_start(const BatchView& b, const BdArgs& g, int prefix_units, long long u, BdWalk& w)
{
    const int Hk = g.a.n_kv_heads, lane = threadIdx.x & 31;
    w.base = -64;
    if (u < (long long)prefix_units * Hk) {
        w.seq = -1;
        w.kvh = (int)(u / prefix_units);
        w.unit = (int)(u - (long long)w.kvh * prefix_units);
        w.units = prefix_units;
        w.item = w.kvh;
        w.sp = {0, min(max(b.row_start[b.n_seqs], 0), b.n_rows), b.prefix_len, 0};
        return;
    }
    u -= (long long)prefix_units * Hk;
    w.seq = 0;
    for (int base = 0; base < b.n_seqs; base += 32) {
        w.base = base;
        w.ahead = {};
        if (base + lane < b.n_seqs) w.ahead = seq_span(b, base + lane);
        const int mine = bd_units<KEYS>(w.ahead) * Hk;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(FULL_WARP, upto, o);
            if (lane >= o) upto += v;
        }
        const unsigned m = __ballot_sync(FULL_WARP, u < upto);
        if (m == 0) {
            u -= __shfl_sync(FULL_WARP, upto, 31);
            continue;
        }
        const int at = __ffs(m) - 1;
        u -= __shfl_sync(FULL_WARP, upto - mine, at);
        w.seq = base + at;
        break;
    }
    w.sp = bd_span(b, w, w.seq);
    w.units = bd_units<KEYS>(w.sp);
    w.kvh = (int)(u / w.units);
    w.unit = (int)(u - (long long)w.kvh * w.units);
    w.item = (g.prefix_here ? Hk : 0) + w.seq * Hk + w.kvh;
}
template <int KEYS> __device__ __forceinline__ void bd_next(const BatchView& b, const BdArgs& g, BdWalk& w)   // to the next unit; the caller has one left
{
    if (++w.unit < w.units) return;
    w.unit = 0;
    ++w.item;
    if (++w.kvh < g.a.n_kv_heads) return;
    w.kvh = 0;
    ++w.seq;
    bd_enter<KEYS>(b, g, w);
}

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// byte offset of 16-byte piece `piece` (8 dims) of row `row` in a 128-byte-swizzled tile of `rows` rows per 64-dim half
__device__ __forceinline__ uint32_t swizzled(int row, int piece, int rows)
{
    return (uint32_t)((piece >> 3) * rows * 128 + row * 128 + (((piece & 7) ^ (row & 7)) << 4));
}

template <typename T, int HALVES, int MT>
__global__ void __launch_bounds__(BD_THREADS, 1) attn_batch_dec_kernel(const __grid_constant__ CUtensorMap map_kv, BatchView b, BdArgs g)
{
    typedef BdShape<HALVES, MT> S;
    constexpr int DP = S::DP, KEYS = S::KEYS, R = 16 * MT;
    constexpr float BIAS = std::is_same<T, __half>::value ? 7.f : 0.f;
    pdl_trigger();

    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    __shared__ __align__(8) unsigned long long bars[S::WORKERS * S::STAGES * 2];
    __shared__ unsigned page_bits[S::WORKERS * S::STAGES];
    __shared__ int sums[BD_THREADS / 32];
    __shared__ int waits_sh[2];
    volatile int* waits = waits_sh;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, Hk = g.a.n_kv_heads, G = g.a.n_heads / Hk;
    const int wk = warp / MT, mt = warp % MT, gq = lane >> 2, t = lane & 3;
    auto full = [&](int s) { return smem_u32(&bars[wk * S::STAGES + s]); };
    auto empty = [&](int s) { return smem_u32(&bars[(S::WORKERS + wk) * S::STAGES + s]); };
    if (tid == 0) {
        for (int s = 0; s < S::WORKERS * S::STAGES; ++s) { mbar_init(smem_u32(&bars[s]), 1); mbar_init(smem_u32(&bars[S::WORKERS * S::STAGES + s]), MT); }
        waits[0] = 0;
        waits[1] = g.a.wait_kcycles;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_kv) : "memory");
    }
    // units of the whole batch (the host has made sure that they fit an int)
    const int prefix_units = g.prefix_here ? (b.prefix_len + KEYS - 1) / KEYS : 0;
    int own = 0;
    for (int i = tid; i < b.n_seqs; i += BD_THREADS) own += bd_units<KEYS>(seq_span(b, i));
    own = __reduce_add_sync(FULL_WARP, own);
    if (lane == 0) sums[warp] = own;
    __syncthreads();
    long long U = prefix_units;
#pragma unroll
    for (int w = 0; w < BD_THREADS / 32; ++w) U += sums[w];
    U *= Hk;
    // never more workers than units: the workers between an item's first and its last then all hold units of it
    const int all = gridDim.x * S::WORKERS, workers = (int)(U < (long long)all ? U : (long long)all), me = blockIdx.x * S::WORKERS + wk;
    const long long u0 = me < workers ? U * me / workers : 0, u1 = me < workers ? U * (me + 1) / workers : 0;
    const int count = (int)(u1 - u0);

    if (count > 0) {
        const uint32_t stages = base + wk * S::STAGES * 2 * S::TILE_BYTES;
        const float c = g.a.scale * 1.4426950408889634f;
        const int box_rows = min(b.page_size, KEYS), box_shift = min(b.page_shift, 31 - __clz(KEYS));
        const int per_unit = KEYS >> box_shift;                           // boxes (pages, or part of one) per unit, 1..8
        const unsigned all_boxes = (1u << per_unit) - 1u;
        BdWalk w;
        bd_start<KEYS>(b, g, prefix_units, u0, w);

        // ---- the fetching side, by the worker's first warp: `wf` is the next unit to ask for, its page ids are looked up already
        // Shared memory: box after box [K, V][64-dim half][slot][64 dims]
        const uint32_t box_half = box_rows * 128, box_v = HALVES * box_half, box_bytes = 2 * box_v;
        BdWalk wf = w;
        int asked = 0, f_stage = 0, next_page = 0;                        // next_page: lane p: page of box p of unit `asked`
        uint32_t f_turn = 0;
        auto look_up = [&]() {
            next_page = -1;                                               // beyond the end: no page
            const int key0 = wf.unit * KEYS;
            if (lane < per_unit && lane * box_rows < wf.sp.len - key0) {
                const int at = (key0 + lane * box_rows) >> b.page_shift;
                next_page = wf.seq < 0 ? b.prefix_pages[at] : b.page_table[(size_t)wf.seq * b.table_stride + at];
            }
        };
        auto ask = [&]() {                                                // asks for unit `asked`; its stage is free
            const bool good = (unsigned)next_page < (unsigned)b.n_pages;
            const int page = good ? next_page : b.n_pages;                // beyond the last page: zeros
            const unsigned pages = __ballot_sync(FULL_WARP, good) & all_boxes;
            const bool asks = !(g.a.withhold && asked == 0);
            if (elect_one()) {
                page_bits[wk * S::STAGES + f_stage] = pages;
                if (asks) mbar_expect_tx(full(f_stage), 2u * S::TILE_BYTES);
            }
            __syncwarp();
            // one lane asks for all boxes in turn (from lanes of their own they go out one by one as well), at some 90 cycles each
            const uint32_t dst = stages + f_stage * 2 * S::TILE_BYTES;
            const int plane = g.block * 2 * Hk + wf.kvh;
            for (int p = 0; asks && p < per_unit; ++p) {
                const int pageu = __shfl_sync(FULL_WARP, page, p), slot0 = (wf.unit * KEYS + p * box_rows) & (b.page_size - 1);
                if (elect_one()) {
                    if (g.whole_boxes) {
                        tma_load_5d(dst + p * box_bytes, &map_kv, 0, slot0, 0, 0, pageu == b.n_pages ? g.planes : pageu * (g.planes / b.n_pages) + plane, full(f_stage));
                    } else {
#pragma unroll
                        for (int x = 0; x < 2 * HALVES; ++x)
                            tma_load_4d(dst + p * box_bytes + x * box_half, &map_kv, 64 * (x % HALVES), slot0, plane + (x / HALVES) * Hk, pageu, full(f_stage));
                    }
                }
            }
            if (wf.unit == 0 || wf.unit + 1 == wf.units) {
                if (wf.unit == 0) g.item_first[wf.item] = me;             // (all lanes write the same)
                if (wf.unit + 1 == wf.units) g.item_last[wf.item] = me;
            }
            if (++f_stage == S::STAGES) { f_stage = 0; f_turn ^= 1u; }
            if (++asked < count) {
                bd_next<KEYS>(b, g, wf);
                look_up();
            }
        };
        if (mt == 0) {
            look_up();
            for (int i = 0; i < S::STAGES && asked < count; ++i) ask();
        }
        // This lane's rows in a unit: ldmatrix takes 8 rows of 8 lanes each; the eight-row groups of K and of V it starts from.
        const uint32_t k_lane = (lane & 7) * 128, k_piece = (lane >> 3) & 1, v_piece = lane >> 4;
        uint32_t k_grp[MT], v_grp[MT];
#pragma unroll
        for (int n = 0; n < MT; ++n) {
            const int kr = 16 * n + ((lane >> 4) << 3), vr = 16 * n + (((lane >> 3) & 1) << 3);
            k_grp[n] = (kr >> box_shift) * box_bytes + (kr & (box_rows - 1)) * 128 + k_lane;
            v_grp[n] = (vr >> box_shift) * box_bytes + (vr & (box_rows - 1)) * 128 + k_lane + box_v;
        }
        auto piece_at = [&](uint32_t piece) { return (piece >> 3) * box_half + (((piece & 7) ^ (lane & 7)) << 4); };

        uint32_t turn = 0;
        int stage = 0;
        bool ok = true, fresh = true;                                     // fresh: first unit of an item here
        uint32_t qf[4 * HALVES][4];
        float o[8 * HALVES][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        const int rho[2] = {16 * mt + gq, 16 * mt + gq + 8};              // this thread's two packed rows, their tokens
        const int tok[2] = {rho[0] / G, rho[1] / G};
        const uint32_t q_sh = base + S::RING_BYTES + warp * S::Q_BYTES;
        auto fetch_q = [&](const BdWalk& item) {                          // this warp's 16 rows of an item's queries; dead rows zero
#pragma unroll
            for (int i = 0; i < 4 * HALVES; ++i) {
                const int row = (i * 32 + lane) / (8 * HALVES), piece = (i * 32 + lane) % (8 * HALVES), r = 16 * mt + row, tk = r / G;
                const bool live = r < item.sp.n * G && 8 * piece < g.a.head_dim;
                const T* q = reinterpret_cast<const T*>(g.a.q) + (size_t)(item.sp.r0 + (live ? tk : 0)) * g.a.q_row_stride +
                             (size_t)(item.kvh * G + (live ? r - tk * G : 0)) * g.a.q_head_stride + (live ? 8 * piece : 0);
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(q_sh + swizzled(row, piece, 16)), "l"(q), "r"(live ? 16 : 0) : "memory");
            }
        };
        fetch_q(w);
        for (int k = 0; k < count; ++k) {
            if (fresh) {
                // queries into fragments; those of the next item set off for shared memory
                asm volatile("cp.async.wait_all;" ::: "memory");
                __syncwarp();
#pragma unroll
                for (int ks = 0; ks < 4 * HALVES; ++ks) ldsm4(qf[ks], q_sh + swizzled(lane & 15, 2 * ks + (lane >> 4), 16));
                __syncwarp();
                if (count - k > w.units - w.unit) {
                    BdWalk wn = w;
                    wn.unit = wn.units - 1;
                    bd_next<KEYS>(b, g, wn);
                    fetch_q(wn);
                }
#pragma unroll
                for (int nt = 0; nt < 8 * HALVES; ++nt) o[nt][0] = o[nt][1] = o[nt][2] = o[nt][3] = 0.f;
                m[0] = m[1] = -INFINITY;
                l[0] = l[1] = 0.f;
            }
            ok = bt_wait(full(stage), turn, waits);
            if (!ok) break;
            const uint32_t kv_sh = stages + stage * 2 * S::TILE_BYTES;
            const int key0 = w.unit * KEYS, left = w.sp.len - key0;
            if (left < KEYS && (left & (box_rows - 1)) != 0) {
                // slots behind the end may hold anything: V's become zero before they are read
                const int end = (left | (box_rows - 1)) + 1;
                for (int i = lane; i < (end - left) * 8 * HALVES; i += 32) {
                    const int row = left + i / (8 * HALVES), piece = i % (8 * HALVES);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};"      // whole rows: the swizzle stays inside
                                 ::"r"(kv_sh + (row >> box_shift) * box_bytes + box_v + (piece >> 3) * box_half + (row & (box_rows - 1)) * 128 + (piece & 7) * 16), "r"(0) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            float s[KEYS / 8][4];
#pragma unroll
            for (int n = 0; n < KEYS / 8; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
            for (int ks = 0; ks < 4 * HALVES; ++ks)
#pragma unroll
                for (int n = 0; n < KEYS / 16; ++n) {
                    uint32_t kf[4];                                       // keys 16 n .. + 15 x dims 16 ks .. + 15
                    ldsm4(kf, kv_sh + k_grp[n] + piece_at(2 * ks + k_piece));
                    mma16816(s[2 * n], qf[ks], kf[0], kf[1], T());
                    mma16816(s[2 * n + 1], qf[ks], kf[2], kf[3], T());
                }
            const unsigned pages = page_bits[wk * S::STAGES + stage];
            // own part: rows see keys up to their own position; the prefix: all rows see all of it
            int seen[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) seen[e] = w.seq < 0 ? left : min(left, w.sp.pos0 + tok[e] + 1 - key0);
            if (__any_sync(FULL_WARP, min(seen[0], seen[1]) < KEYS) || pages != all_boxes) {
#pragma unroll
                for (int n = 0; n < KEYS / 8; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = 8 * n + 2 * t + (e & 1);
                        if (key >= seen[e >> 1] || !((pages >> (key >> box_shift)) & 1u)) s[n][e] = -INFINITY;
                    }
            }
            float top[2] = {-INFINITY, -INFINITY}, off[2];
#pragma unroll
            for (int n = 0; n < KEYS / 8; ++n) {
                top[0] = max3(top[0], s[n][0], s[n][1]);
                top[1] = max3(top[1], s[n][2], s[n][3]);
            }
            // as in the many-row kernel, a row's sums are rescaled when its maximum has grown by more than 2^8
            bool moved[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                top[e] = fmaxf(top[e], __shfl_xor_sync(FULL_WARP, top[e], 1));
                top[e] = fmaxf(top[e], __shfl_xor_sync(FULL_WARP, top[e], 2));
                moved[e] = bt_outgrown(top[e], m[e], c);
            }
            if (__any_sync(FULL_WARP, moved[0] || moved[1])) {
                float shrink[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    shrink[e] = moved[e] ? ex2((m[e] - top[e]) * c) : 1.f;
                    if (moved[e]) m[e] = top[e];
                    l[e] *= shrink[e];
                }
#pragma unroll
                for (int nt = 0; nt < 8 * HALVES; ++nt) {
                    o[nt][0] *= shrink[0]; o[nt][1] *= shrink[0];
                    o[nt][2] *= shrink[1]; o[nt][3] *= shrink[1];
                }
            }
            bool far[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                off[e] = BIAS - (m[e] == -INFINITY ? 0.f : m[e] * c);
                far[e] = fabsf(off[e]) > BT_FAR;
            }
            if (__builtin_expect(__any_sync(FULL_WARP, far[0] || far[1]), 0)) {
                if (far[0]) off[0] = BIAS;
                if (far[1]) off[1] = BIAS;
#pragma unroll
                for (int n = 0; n < KEYS / 8; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n][e] -= far[e >> 1] ? m[e >> 1] : 0.f;
            }
#pragma unroll
            for (int n = 0; n < KEYS / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[n][e] = ex2(fmaf(s[n][e], c, off[e >> 1]));
                    l[e >> 1] += s[n][e];
                }
#pragma unroll
            for (int n = 0; n < KEYS / 16; ++n) {
                const uint32_t pf[4] = {pack2(s[2 * n][0], s[2 * n][1], T()), pack2(s[2 * n][2], s[2 * n][3], T()),
                                        pack2(s[2 * n + 1][0], s[2 * n + 1][1], T()), pack2(s[2 * n + 1][2], s[2 * n + 1][3], T())};
#pragma unroll
                for (int d = 0; d < 4 * HALVES; ++d) {                    // keys 16 n .. + 15 x dims 16 d .. + 15
                    uint32_t vf[4];
                    ldsm4_trans(vf, kv_sh + v_grp[n] + piece_at(2 * d + v_piece));
                    mma16816(o[2 * d], pf, vf[0], vf[1], T());
                    mma16816(o[2 * d + 1], pf, vf[2], vf[3], T());
                }
            }
            // ---- the stage is used up: ask for the unit that takes its place
            __syncwarp();
            if (MT > 1 && lane == 0) mbar_arrive(empty(stage));
            if (mt == 0 && asked < count) {
                if (MT > 1) ok = bt_wait(empty(f_stage), f_turn ^ 1u, waits);
                if (!ok) break;
                ask();
            }
            if (++stage == S::STAGES) { stage = 0; turn ^= 1u; }
            fresh = w.unit + 1 == w.units || k + 1 == count;
            if (fresh) {
                // ---- the item, or this worker's share of it, ends
                const size_t slot = (size_t)(w.item + me) * R;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[e] += __shfl_xor_sync(FULL_WARP, l[e], 1);
                    l[e] += __shfl_xor_sync(FULL_WARP, l[e], 2);
                    if (rho[e] < w.sp.n * G) {
                        float* out = g.part_o + (slot + rho[e]) * DP + 2 * t;
#pragma unroll
                        for (int nt = 0; nt < 8 * HALVES; ++nt) *reinterpret_cast<float2*>(out + 8 * nt) = make_float2(o[nt][2 * e], o[nt][2 * e + 1]);
                        if (t == 0) g.part_ml[slot + rho[e]] = make_float2(m[e] * c - BIAS, l[e]);
                    }
                }
            }
            if (k + 1 < count) bd_next<KEYS>(b, g, w);
        }
    }
    __syncthreads();
    bt_give_up(waits);
    pdl_wait();                                           // the launch before this one ends first: what follows waits for both
}

// ------------------------------------------------------------------------------ joining the parts
struct BjArgs {
    AttnView a;
    int dp, item_rows;                                    // item_rows: rows of a slot of the few-row kernel
    int prefix_here, own_here;                            // which parts the few-row kernel left
    int splits;                                           // parts of the many-row kernel: slots 0 .. splits - 1 of every row
    const float* many_o;
    const float2* many_ml;
    const float* few_o;
    const float2* few_ml;
    const int* item_first;
    const int* item_last;
    int workers;                                          // of the few-row kernel, at most
};

// out[row][h] = sum_i 2^(M_i - M) O_i / sum_i 2^(M_i - M) l_i over the parts of a row, in a fixed order: the many-row
// kernel's parts, then the prefix item's, then the own item's.
struct BjSum {
    float M, l;
    float4 acc;
};
// The first worker that left a part of an item, and how many did; none where a wait ran out before the entries were written (they
// are then whatever the workspace held).
__device__ __forceinline__ int bj_parts(const BjArgs& g, int item, int& first)
{
    const int f = g.item_first[item], l = g.item_last[item];
    const bool good = f >= 0 && f <= l && l < g.workers;
    first = good ? f : 0;
    return good ? l - f + 1 : 0;
}
struct BjKind {                                           // one kind of parts: how many, where the first one's sums and maximum are, what lies between two
    const float* o;
    const float2* ml;
    int n;
    long long stride;                                     // in (row, head)s
};

// WARPS warps per (row, head), each taking every WARPS-th part, lanes over dims.  A head costs four dependent trips to memory (its
// sequence, its items' first and last worker, its parts, the store) and one more for every batch of further parts.  Eight warps
// are for few rows, whose items are cut into many parts (one row, 64 heads, 148 parts each).
// grid = (rows, ceil(heads / (8 / WARPS))), block = 256.
template <typename T, int WARPS>
__global__ void __launch_bounds__(256, WARPS == 1 ? 4 : 3) attn_join_kernel(BatchView b, BjArgs g)
{
    constexpr int BJ_PARTS = WARPS == 1 ? 4 : 8;          // parts whose sums and maxima are fetched at once
    pdl_wait();
    const int row = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.y * (8 / WARPS) + warp / WARPS, turn = warp % WARPS;
    if (h >= g.a.n_heads) return;                         // (WARPS 8: all or none of a block)
    const int Hk = g.a.n_kv_heads, G = g.a.n_heads / Hk, kvh = h / G, hg = h - kvh * G;
    int f0 = 0, n0 = 0;
    if (g.prefix_here) n0 = bj_parts(g, kvh, f0);
    SeqSpan sp;
    const int seq = find_seq(b, row, sp);
    if (seq < 0 || row - sp.r0 >= g.a.max_rows) return;   // the same for the whole block
    const int own_item = (g.prefix_here ? Hk : 0) + seq * Hk + kvh;
    int f1 = 0, n1 = 0;
    if (g.own_here && sp.len > 0) n1 = bj_parts(g, own_item, f1);
    BjKind kinds[3];
    const size_t at[3] = {(size_t)row * g.a.n_heads + h, (size_t)(kvh + f0) * g.item_rows + row * G + hg, (size_t)(own_item + f1) * g.item_rows + (row - sp.r0) * G + hg};
#pragma unroll
    for (int j = 0; j < 3; ++j)
        kinds[j] = {(j ? g.few_o : g.many_o) + at[j] * g.dp + 4 * lane, (j ? g.few_ml : g.many_ml) + at[j], j == 0 ? g.splits : j == 1 ? n0 : n1,
                    j ? (long long)g.item_rows : (long long)b.n_rows * g.a.n_heads};
    const bool mine = 4 * lane < g.dp;
    const int parts = g.splits + n0 + n1;
    BjSum s = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    for (int p0 = turn; p0 < parts; p0 += BJ_PARTS * WARPS) {
        float2 x[BJ_PARTS];
        float4 v[BJ_PARTS];
#pragma unroll
        for (int i = 0; i < BJ_PARTS; ++i) {
            int part = p0 + i * WARPS;
            x[i] = make_float2(-INFINITY, 0.f);
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (part < parts) {
                const bool many = part < kinds[0].n, prefix = !many && part < kinds[0].n + kinds[1].n;
                const BjKind& k = many ? kinds[0] : prefix ? kinds[1] : kinds[2];
                const long long off = (part - (many ? 0 : prefix ? kinds[0].n : kinds[0].n + kinds[1].n)) * k.stride;
                x[i] = k.ml[off];
                if (mine) v[i] = *reinterpret_cast<const float4*>(k.o + off * g.dp);
            }
        }
        float top = s.M;
#pragma unroll
        for (int i = 0; i < BJ_PARTS; ++i) top = x[i].y != 0.f ? fmaxf(top, x[i].x) : top;
        const float shrink = s.M == top ? 1.f : ex2(s.M - top);
        s.l *= shrink;
        s.acc.x *= shrink; s.acc.y *= shrink; s.acc.z *= shrink; s.acc.w *= shrink;
        s.M = top;
#pragma unroll
        for (int i = 0; i < BJ_PARTS; ++i) {
            if (x[i].y == 0.f) continue;                  // an empty part: its sums were not written
            const float f = ex2(x[i].x - top);
            s.l += x[i].y * f;
            s.acc.x += f * v[i].x; s.acc.y += f * v[i].y; s.acc.z += f * v[i].z; s.acc.w += f * v[i].w;
        }
    }
    if (WARPS > 1) {
        __shared__ float4 acc_sh[8][32];
        __shared__ float2 ml_sh[8];
        acc_sh[warp][lane] = s.acc;
        if (lane == 0) ml_sh[warp] = make_float2(s.M, s.l);
        __syncthreads();
        if (warp > 0) return;
        s = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
#pragma unroll
        for (int w = 0; w < WARPS; ++w) s.M = fmaxf(s.M, ml_sh[w].x);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            if (ml_sh[w].y == 0.f) continue;
            const float f = ex2(ml_sh[w].x - s.M);
            const float4 v = acc_sh[w][lane];
            s.l += f * ml_sh[w].y;
            s.acc.x += f * v.x; s.acc.y += f * v.y; s.acc.z += f * v.z; s.acc.w += f * v.w;
        }
    }
    const float inv = s.l == 0.f ? 0.f : 1.f / s.l;       // 0: the row sees nothing
    if (4 * lane < g.a.head_dim) {
        T* out = reinterpret_cast<T*>(g.a.out) + ((size_t)row * g.a.n_heads + h) * g.a.head_dim + 4 * lane;
        *reinterpret_cast<uint2*>(out) = make_uint2(pack2(s.acc.x * inv, s.acc.y * inv, T()), pack2(s.acc.z * inv, s.acc.w * inv, T()));
    }
}

} // namespace swk
