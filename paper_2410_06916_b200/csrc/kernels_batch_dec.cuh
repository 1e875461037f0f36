// Attention of few query rows per sequence over the paged cache (decoding steps, verified drafts, scoring windows): every
// cached K,V byte is read once and meets at most 64 query rows, so the kernel is bound by HBM; what it must get right is
// to keep enough bytes in flight on every SM, whatever the lengths of the sequences.
//
// Work.  A piece of work ("item") is one kv head of one sequence, or of the prefix with the rows of all sequences (when
// those are few enough to fit a tile; otherwise the many-row kernel next door takes the prefix).  Items are numbered in
// units of 64 keys, and the units are cut into gridDim.x equal ranges, one per persistent CTA: each SM streams the same
// number of bytes, and a single long sequence is split over all of them.  A CTA leaves one partial result per item it
// touches - unnormalised sums, their maximum, the sum of probabilities - in slot item + CTA (both grow together, so no two
// meet); the joining kernel adds the slots of an item in order, so results do not depend on timing.
//
// A CTA is a TMA warp that fills a ring of five 64-key stages (160 KB in flight per SM; 44 KB would cover HBM's latency at
// 44 GB/s per SM, the rest covers the ends of items) and two groups of four warps that take stages in turn.
// Products are mma.sync.m16n8k16: a group's warps split MT row tiles x 4 / MT key ranges.  (tcgen05 needs 128 rows a
// tile; at 16 to 64 rows the tensor pipe is idle most of the time either way.)  P is rounded to the cache's type as in the
// many-row kernel, fp16 with the same factor 2^7.
#pragma once
#include "kernels_batch_tc.cuh"

namespace swk {

constexpr int BD_THREADS = 288;                           // 8 consumer warps, the TMA warp
constexpr int BD_KEYS = 64;                               // keys per unit
constexpr int BD_AHEAD = 4;                               // units by which page ids are looked up ahead of their use
constexpr int BD_MAX_ROWS = 64;                           // packed query rows (tokens x heads of a group) of an item

template <int HALVES> struct BdShape {
    static constexpr int DP = 64 * HALVES;
    static constexpr int TILE_BYTES = BD_KEYS * 128 * HALVES;     // K or V of a unit
    static constexpr int STAGES = HALVES == 2 ? 5 : 10;
    static constexpr int O_STRIDE = DP + 4;                       // floats per row of a warp's merged output
    static constexpr int MERGE_BYTES = 4 * 16 * O_STRIDE * 4;
    static constexpr int smem_bytes(int mt) { return 1024 + STAGES * 2 * TILE_BYTES + 2 * mt * 16 * 128 * HALVES + MERGE_BYTES; }
};

struct BdArgs {
    AttnView a;
    int block, prefix_here;                               // prefix_here: the prefix is part of this launch's items
    int rows_per_box;                                     // tokens of a query box (16 MT / G)
    float* part_o;                                        // [item + CTA][16 MT][DP]
    float2* part_ml;                                      // [item + CTA][16 MT]
    int* item_first;                                      // [item]: first and last CTA that holds units of it
    int* item_last;
};

__device__ __forceinline__ int bd_units(const SeqSpan& s) { return s.n > 0 ? (s.len + BD_KEYS - 1) / BD_KEYS : 0; }

// A walk over a CTA's units by a whole warp; all lanes hold the same values, except that lane i keeps the span of sequence
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
        w.ahead = {0, 0, 0};
        if (i < b.n_seqs) w.ahead = seq_span(b, i);
    }
    const int at = seq - w.base;
    return {__shfl_sync(FULL_WARP, w.ahead.r0, at), __shfl_sync(FULL_WARP, w.ahead.n, at), __shfl_sync(FULL_WARP, w.ahead.len, at)};
}
__device__ __forceinline__ void bd_enter(const BatchView& b, const BdArgs& g, BdWalk& w)
{
    while (w.seq < b.n_seqs) {                            // skips sequences without units; the caller has units left
        w.sp = bd_span(b, w, w.seq);
        w.units = bd_units(w.sp);
        if (w.units > 0) break;
        ++w.seq;
    }
    w.item = (g.prefix_here ? g.a.n_kv_heads : 0) + w.seq * g.a.n_kv_heads + w.kvh;
}
__device__ __forceinline__ void bd_start(const BatchView& b, const BdArgs& g, int prefix_units, long long u, BdWalk& w)
{
    const int Hk = g.a.n_kv_heads, lane = threadIdx.x & 31;
    w.base = -64;
    if (u < (long long)prefix_units * Hk) {
        w.seq = -1;
        w.kvh = (int)(u / prefix_units);
        w.unit = (int)(u - (long long)w.kvh * prefix_units);
        w.units = prefix_units;
        w.item = w.kvh;
        w.sp.r0 = 0;
        w.sp.n = min(max(b.row_start[b.n_seqs], 0), b.n_rows);
        w.sp.len = b.prefix_len;
        return;
    }
    u -= (long long)prefix_units * Hk;
    w.seq = 0;
    for (int base = 0; base < b.n_seqs; base += 32) {
        w.base = base;
        w.ahead = {0, 0, 0};
        if (base + lane < b.n_seqs) w.ahead = seq_span(b, base + lane);
        const int mine = bd_units(w.ahead) * Hk;
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
    w.units = bd_units(w.sp);
    w.kvh = (int)(u / w.units);
    w.unit = (int)(u - (long long)w.kvh * w.units);
    w.item = (g.prefix_here ? Hk : 0) + w.seq * Hk + w.kvh;
}
__device__ __forceinline__ void bd_next(const BatchView& b, const BdArgs& g, BdWalk& w)   // to the next unit; the caller has one left
{
    if (++w.unit < w.units) return;
    w.unit = 0;
    ++w.item;
    if (++w.kvh < g.a.n_kv_heads) return;
    w.kvh = 0;
    ++w.seq;
    bd_enter(b, g, w);
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
__global__ void __launch_bounds__(BD_THREADS, 1)
attn_batch_dec_kernel(const __grid_constant__ CUtensorMap map_kv, const __grid_constant__ CUtensorMap map_q, BatchView b, BdArgs g)
{
    typedef BdShape<HALVES> S;
    constexpr int DP = S::DP, R = 16 * MT, WK = 4 / MT, KW = BD_KEYS / WK;   // key ranges of a group, keys per warp
    constexpr int Q_BYTES = R * 128 * HALVES;
    constexpr float BIAS = std::is_same<T, __half>::value ? 7.f : 0.f;
    pdl_trigger();

    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_sh = base + S::STAGES * 2 * S::TILE_BYTES;
    float* merge = reinterpret_cast<float*>(smem_raw + (q_sh + 2 * Q_BYTES - smem_u32(smem_raw)));   // [4][16][O_STRIDE]
    __shared__ __align__(8) unsigned long long bars[2 * S::STAGES + 4];
    __shared__ float2 ml_sh[4][16];
    __shared__ unsigned page_bits[S::STAGES];
    __shared__ int sums[BD_THREADS / 32];
    __shared__ int abort_flag;
    volatile int* abort_sh = &abort_flag;
    auto full = [&](int s) { return smem_u32(&bars[s]); };
    auto empty = [&](int s) { return smem_u32(&bars[S::STAGES + s]); };
    auto q_full = [&](int s) { return smem_u32(&bars[2 * S::STAGES + s]); };
    auto q_empty = [&](int s) { return smem_u32(&bars[2 * S::STAGES + 2 + s]); };

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, Hk = g.a.n_kv_heads;
    if (tid == 0) {
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 4); }
        for (int s = 0; s < 2; ++s) { mbar_init(q_full(s), 1); mbar_init(q_empty(s), 8); }
        abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_kv) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
    }
    // units of the whole batch (the host has made sure that they fit an int)
    const int prefix_units = g.prefix_here ? (b.prefix_len + BD_KEYS - 1) / BD_KEYS : 0;
    int own = 0;
    for (int i = tid; i < b.n_seqs; i += BD_THREADS) own += bd_units(seq_span(b, i));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) own += __shfl_xor_sync(FULL_WARP, own, o);
    if (lane == 0) sums[warp] = own;
    __syncthreads();
    long long U = prefix_units;
#pragma unroll
    for (int w = 0; w < BD_THREADS / 32; ++w) U += sums[w];
    U *= Hk;
    // never more CTAs than units: the CTAs between an item's first and its last then all hold units of it
    const int ctas = (int)(U < (long long)gridDim.x ? U : (long long)gridDim.x), cta = blockIdx.x;
    const long long u0 = cta < ctas ? U * cta / ctas : 0, u1 = cta < ctas ? U * (cta + 1) / ctas : 0;
    const int count = (int)(u1 - u0);

    if (count > 0 && warp == 8) {
        // ---------------------------------------------------------------- TMA
        BdWalk w, wa;                                                     // the unit being fetched; one whose page ids are being fetched
        bd_start(b, g, prefix_units, u0, w);
        wa = w;
        const int per_unit = max(1, BD_KEYS >> b.page_shift);             // pages per unit, 1..8
        const int kv = lane >> 4, pg = (lane & 15) / HALVES, half = (lane & 15) % HALVES;
        const bool boxed = pg < per_unit;
        const int box_rows = min(b.page_size, BD_KEYS);
        const uint32_t box_at = kv * S::TILE_BYTES + half * (BD_KEYS * 128) + pg * box_rows * 128;
        // Page ids come BD_AHEAD units before they are needed: a trip to memory takes as long as a unit streams.
        auto page_of = [&]() {
            int page = b.n_pages;                                         // beyond the last page: zeros
            const int key0 = wa.unit * BD_KEYS;
            if (boxed && pg * box_rows < wa.sp.len - key0) {
                const int at = (key0 >> b.page_shift) + pg;
                page = wa.seq < 0 ? b.prefix_pages[at] : b.page_table[(size_t)wa.seq * b.table_stride + at];
            }
            return page;
        };
        int ids[BD_AHEAD];
#pragma unroll
        for (int i = 0; i < BD_AHEAD; ++i) {
            ids[i] = i < count ? page_of() : b.n_pages;
            if (i + 1 < count) bd_next(b, g, wa);
        }
        uint32_t turn = 0, q_turn = 0;
        int stage = 0, qb = 0;
        bool ok = true, fresh = true;                                     // fresh: first unit of a segment
        for (int k = 0; ok && k < count; ++k) {
            if (fresh && lane == 0) {
                ok = bt_wait(q_empty(qb), q_turn ^ 1u, abort_sh);
                if (ok) {
                    mbar_expect_tx(q_full(qb), (uint32_t)(g.rows_per_box * (g.a.n_heads / Hk) * 128 * HALVES));
                    for (int hf = 0; hf < HALVES; ++hf)
                        tma_load_3d(q_sh + qb * Q_BYTES + hf * (R * 128), &map_q, 64 * hf, w.kvh * (g.a.n_heads / Hk), w.sp.r0, q_full(qb));
                    if (w.unit == 0) g.item_first[w.item] = blockIdx.x;
                }
            }
            const int key0 = w.unit * BD_KEYS;
            int page = ids[0];
#pragma unroll
            for (int i = 0; i + 1 < BD_AHEAD; ++i) ids[i] = ids[i + 1];
            if (k + BD_AHEAD < count) {
                ids[BD_AHEAD - 1] = page_of();
                if (k + BD_AHEAD + 1 < count) bd_next(b, g, wa);
            }
            const bool good = (unsigned)page < (unsigned)b.n_pages;
            if (!good) page = b.n_pages;
            const unsigned bits = __ballot_sync(FULL_WARP, boxed && good && half == 0 && kv == 0);
            unsigned pages = 0;
#pragma unroll
            for (int p = 0; p < 16 / HALVES; ++p) pages |= ((bits >> (p * HALVES)) & 1u) << p;
            if (lane == 0) {
                ok = ok && bt_wait(empty(stage), turn ^ 1u, abort_sh);
                if (ok) {
                    page_bits[stage] = pages;
                    mbar_expect_tx(full(stage), 2u * S::TILE_BYTES);
                }
            }
            ok = __shfl_sync(FULL_WARP, ok ? 1 : 0, 0) != 0;
            if (!ok) break;
            if (boxed)
                tma_load_4d(base + stage * 2 * S::TILE_BYTES + box_at, &map_kv, 64 * half, key0 & (b.page_size - 1) & ~(box_rows - 1),
                            (g.block * 2 + kv) * Hk + w.kvh, page, full(stage));
            if (++stage == S::STAGES) { stage = 0; turn ^= 1u; }
            if (fresh) { qb ^= 1; if (qb == 0) q_turn ^= 1u; }
            fresh = w.unit + 1 == w.units;
            if (fresh && lane == 0) g.item_last[w.item] = blockIdx.x;
            if (k + 1 < count) bd_next(b, g, w);
        }
        if (!ok && lane == 0) {                                           // copies still on their way land before the block ends
            const long long t0 = clock64();
            while (clock64() - t0 < 2000000LL) { }
        }
    } else if (count > 0) {
        // ---------------------------------------------------------------- consumers
        const int group = warp >> 2, w4 = warp & 3, mt = w4 / WK, kr = w4 % WK, gq = lane >> 2, t = lane & 3;
        const int G = g.a.n_heads / Hk;
        const float c = g.a.scale * 1.4426950408889634f;
        BdWalk w;
        bd_start(b, g, prefix_units, u0, w);
        uint32_t turn = 0, q_turn = 0;
        int stage = 0, qb = 0;
        bool ok = true;
        uint32_t qf[4 * HALVES][4];
        float o[8 * HALVES][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        int row_tok[2];                                                   // token of this thread's two rows (within the item)
#pragma unroll
        for (int e = 0; e < 2; ++e) row_tok[e] = (16 * mt + gq + 8 * e) / G;
        bool fresh = true;
        // after a wait that ran out a warp goes on without waiting or computing: the barriers below count on all eight
        for (int k = 0; k < count; ++k) {
            if (fresh) {
                ok = ok && bt_wait(q_full(qb), q_turn, abort_sh);
#pragma unroll
                for (int ks = 0; ks < 4 * HALVES; ++ks)                   // rows 16 mt .. + 15, dims 16 ks .. + 15
                    ldsm4(qf[ks], q_sh + qb * Q_BYTES + swizzled(16 * mt + (lane & 15), 2 * ks + (lane >> 4), R));
                __syncwarp();
                if (lane == 0) mbar_arrive(q_empty(qb));
                qb ^= 1;
                if (qb == 0) q_turn ^= 1u;
#pragma unroll
                for (int nt = 0; nt < 8 * HALVES; ++nt) o[nt][0] = o[nt][1] = o[nt][2] = o[nt][3] = 0.f;
                m[0] = m[1] = -INFINITY;
                l[0] = l[1] = 0.f;
            }
            if ((k & 1) == group) ok = ok && bt_wait(full(stage), turn, abort_sh);
            if ((k & 1) == group && ok) {
                const uint32_t k_sh = base + stage * 2 * S::TILE_BYTES, v_sh = k_sh + S::TILE_BYTES;
                const int key0 = w.unit * BD_KEYS, left = w.sp.len - key0, first = kr * KW;
                if (first < left) {
                    if (left < first + KW && (left & (min(b.page_size, BD_KEYS) - 1)) != 0) {
                        // slots behind the end may hold anything: this warp's rows of V become zero before it reads them
                        for (int i = lane; i < (first + KW - left) * 8 * HALVES; i += 32) {
                            const int row = left + i / (8 * HALVES), piece = i % (8 * HALVES);
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(v_sh + swizzled(row, piece, BD_KEYS)), "r"(0) : "memory");
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    float s[KW / 8][4];
#pragma unroll
                    for (int n = 0; n < KW / 8; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
#pragma unroll
                    for (int ks = 0; ks < 4 * HALVES; ++ks)
#pragma unroll
                        for (int n = 0; n < KW / 16; ++n) {
                            uint32_t kf[4];                               // keys 16 n .. + 15 x dims 16 ks .. + 15
                            ldsm4(kf, k_sh + swizzled(first + 16 * n + (lane & 7) + ((lane >> 4) << 3), 2 * ks + ((lane >> 3) & 1), BD_KEYS));
                            mma16816(s[2 * n], qf[ks], kf[0], kf[1], T());
                            mma16816(s[2 * n + 1], qf[ks], kf[2], kf[3], T());
                        }
                    const unsigned pages = page_bits[stage];
                    const unsigned all = 0xFFu >> (8 - max(1, BD_KEYS >> b.page_shift));
                    // own part: rows see keys up to their own position; the prefix: all rows see all of it
                    int seen[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) seen[e] = w.seq < 0 ? left : w.sp.len - w.sp.n + row_tok[e] + 1 - key0;
                    if (min(seen[0], seen[1]) < first + KW || left < first + KW || pages != all) {
#pragma unroll
                        for (int n = 0; n < KW / 8; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int key = first + 8 * n + 2 * t + (e & 1);
                                if (key >= min(seen[e >> 1], left) || !((pages >> (key >> min(b.page_shift, 6))) & 1u)) s[n][e] = -INFINITY;
                            }
                    }
                    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int n = 0; n < KW / 8; ++n) {
                        top[0] = fmaxf(top[0], fmaxf(s[n][0], s[n][1]));
                        top[1] = fmaxf(top[1], fmaxf(s[n][2], s[n][3]));
                    }
                    float off[2];
                    bool moved = false;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        top[e] = fmaxf(top[e], __shfl_xor_sync(FULL_WARP, top[e], 1));
                        top[e] = fmaxf(top[e], __shfl_xor_sync(FULL_WARP, top[e], 2));
                        moved = moved || top[e] > m[e];
                    }
                    if (__any_sync(FULL_WARP, moved)) {
                        float shrink[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float m_new = fmaxf(m[e], top[e]);
                            shrink[e] = m_new == m[e] ? 1.f : ex2((m[e] - m_new) * c);
                            m[e] = m_new;
                            l[e] *= shrink[e];
                        }
#pragma unroll
                        for (int nt = 0; nt < 8 * HALVES; ++nt) {
                            o[nt][0] *= shrink[0]; o[nt][1] *= shrink[0];
                            o[nt][2] *= shrink[1]; o[nt][3] *= shrink[1];
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 2; ++e) off[e] = BIAS - (m[e] == -INFINITY ? 0.f : m[e] * c);
#pragma unroll
                    for (int n = 0; n < KW / 8; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            s[n][e] = ex2(fmaf(s[n][e], c, off[e >> 1]));
                            l[e >> 1] += s[n][e];
                        }
#pragma unroll
                    for (int n = 0; n < KW / 16; ++n) {
                        uint32_t pf[4] = {pack2(s[2 * n][0], s[2 * n][1], T()), pack2(s[2 * n][2], s[2 * n][3], T()),
                                          pack2(s[2 * n + 1][0], s[2 * n + 1][1], T()), pack2(s[2 * n + 1][2], s[2 * n + 1][3], T())};
#pragma unroll
                        for (int d = 0; d < 4 * HALVES; ++d) {            // keys 16 n .. + 15 x dims 16 d .. + 15
                            uint32_t vf[4];
                            ldsm4_trans(vf, v_sh + swizzled(first + 16 * n + (lane & 15), 2 * d + (lane >> 4), BD_KEYS));
                            mma16816(o[2 * d], pf, vf[0], vf[1], T());
                            mma16816(o[2 * d + 1], pf, vf[2], vf[3], T());
                        }
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(empty(stage));
            }
            if (++stage == S::STAGES) { stage = 0; turn ^= 1u; }
            fresh = w.unit + 1 == w.units || k + 1 == count;
            if (fresh) {
                // ---- the segment ends: join the eight warps' sums, in a fixed order, and leave them in the segment's slot
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    l[e] += __shfl_xor_sync(FULL_WARP, l[e], 1);
                    l[e] += __shfl_xor_sync(FULL_WARP, l[e], 2);
                }
                float* mine = merge + w4 * 16 * S::O_STRIDE;
                if (group == 1) {
#pragma unroll
                    for (int nt = 0; nt < 8 * HALVES; ++nt) {
                        *reinterpret_cast<float2*>(mine + gq * S::O_STRIDE + 8 * nt + 2 * t) = make_float2(o[nt][0], o[nt][1]);
                        *reinterpret_cast<float2*>(mine + (gq + 8) * S::O_STRIDE + 8 * nt + 2 * t) = make_float2(o[nt][2], o[nt][3]);
                    }
                    if (t == 0) { ml_sh[w4][gq] = make_float2(m[0], l[0]); ml_sh[w4][gq + 8] = make_float2(m[1], l[1]); }
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (group == 0) {
                    float f0[2], f1[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float2 other = ml_sh[w4][gq + 8 * e];
                        const float m_new = fmaxf(m[e], other.x);
                        f0[e] = m[e] == m_new ? 1.f : ex2((m[e] - m_new) * c);
                        f1[e] = other.x == m_new ? 1.f : ex2((other.x - m_new) * c);
                        m[e] = m_new;
                        l[e] = l[e] * f0[e] + other.y * f1[e];
                    }
                    __syncwarp();
#pragma unroll
                    for (int nt = 0; nt < 8 * HALVES; ++nt) {
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float2* at = reinterpret_cast<float2*>(mine + (gq + 8 * e) * S::O_STRIDE + 8 * nt + 2 * t);
                            const float2 other = *at;
                            *at = make_float2(o[nt][2 * e] * f0[e] + other.x * f1[e], o[nt][2 * e + 1] * f0[e] + other.y * f1[e]);
                        }
                    }
                    if (t == 0) { ml_sh[w4][gq] = make_float2(m[0], l[0]); ml_sh[w4][gq + 8] = make_float2(m[1], l[1]); }
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                const int live = min(w.sp.n * G, R);
                const size_t slot = (size_t)(w.item + (int)blockIdx.x) * R;
                for (int i = tid; i < live * (DP / 4); i += 256) {
                    const int r = i / (DP / 4), d = (i % (DP / 4)) * 4, w0 = (r >> 4) * WK;
                    float top = -INFINITY;
#pragma unroll
                    for (int j = 0; j < WK; ++j) top = fmaxf(top, ml_sh[w0 + j][r & 15].x);
                    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                    float sum = 0.f;
#pragma unroll
                    for (int j = 0; j < WK; ++j) {
                        const float2 ml = ml_sh[w0 + j][r & 15];
                        const float f = ml.x == top ? 1.f : ex2((ml.x - top) * c);
                        const float4 v = *reinterpret_cast<const float4*>(merge + ((w0 + j) * 16 + (r & 15)) * S::O_STRIDE + d);
                        acc.x += f * v.x; acc.y += f * v.y; acc.z += f * v.z; acc.w += f * v.w;
                        sum += f * ml.y;
                    }
                    *reinterpret_cast<float4*>(g.part_o + (slot + r) * DP + d) = acc;
                    if (d == 0) g.part_ml[slot + r] = make_float2(top * c - BIAS, sum);
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
            }
            if (k + 1 < count) bd_next(b, g, w);
        }
    }
    pdl_wait();                                           // the launch before this one ends first: what follows waits for both
}

// ------------------------------------------------------------------------------ joining the parts
struct BjArgs {
    AttnView a;
    int dp, item_rows;                                    // item_rows: rows of a slot of the few-row kernel (16 MT)
    int prefix_here, own_here;                            // which parts the few-row kernel left
    int splits;                                           // parts of the many-row kernel: slots 0 .. splits - 1 of every row
    const float* many_o;
    const float2* many_ml;
    const float* few_o;
    const float2* few_ml;
    const int* item_first;
    const int* item_last;
};

// out[row][h] = sum_i 2^(M_i - M) O_i / sum_i 2^(M_i - M) l_i over the parts of a row, in a fixed order.  One warp per
// (row, head), lanes over dims; the parts' maxima are fetched 32 at a time.  grid = (rows, ceil(heads / 4)), block = 128.
template <typename T>
__global__ void __launch_bounds__(128) attn_join_kernel(BatchView b, BjArgs g)
{
    pdl_wait();
    const int row = blockIdx.x, lane = threadIdx.x & 31, h = blockIdx.y * 4 + (threadIdx.x >> 5);
    if (h >= g.a.n_heads) return;
    SeqSpan sp;
    const int seq = find_seq(b, row, sp);
    if (seq < 0 || row - sp.r0 >= g.a.max_rows) return;
    const int Hk = g.a.n_kv_heads, G = g.a.n_heads / Hk, kvh = h / G, hg = h - kvh * G;
    // parts 0 .. n0: the many-row kernel's; then the prefix item's; then the own item's
    int first[2] = {0, 0}, n[2] = {0, 0}, item[2], rho[2];
    item[0] = kvh;
    rho[0] = row * G + hg;
    if (g.prefix_here) { first[0] = g.item_first[kvh]; n[0] = g.item_last[kvh] - first[0] + 1; }
    item[1] = (g.prefix_here ? Hk : 0) + seq * Hk + kvh;
    rho[1] = (row - sp.r0) * G + hg;
    if (g.own_here && bd_units(sp) > 0) { first[1] = g.item_first[item[1]]; n[1] = g.item_last[item[1]] - first[1] + 1; }
    const int parts = g.splits + n[0] + n[1];
    auto place = [&](int i, const float2*& ml, const float*& o) {
        if (i < g.splits) {
            const size_t at = ((size_t)i * b.n_rows + row) * g.a.n_heads + h;
            ml = g.many_ml + at;
            o = g.many_o + at * g.dp;
        } else {
            const int j = i - g.splits < n[0] ? 0 : 1;
            const int cta = first[j] + i - g.splits - (j ? n[0] : 0);
            const size_t at = (size_t)(item[j] + cta) * g.item_rows + rho[j];
            ml = g.few_ml + at;
            o = g.few_o + at * g.dp;
        }
    };
    float M = -INFINITY, l = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    const bool mine = 4 * lane < g.dp;
    for (int p0 = 0; p0 < parts; p0 += 32) {
        float2 ml = make_float2(-INFINITY, 0.f);
        const float2* pml;
        const float* po;
        if (p0 + lane < parts) {
            place(p0 + lane, pml, po);
            ml = *pml;
        }
        if (ml.y == 0.f) ml.x = -INFINITY;                // an empty part: its sums were not written
        const float M_new = fmaxf(M, warp_max(ml.x));
        const float shrink = M == M_new ? 1.f : exp2f(M - M_new);
        const float f = ml.y == 0.f ? 0.f : exp2f(ml.x - M_new);
        l = l * shrink + warp_sum(ml.y * f);
        acc.x *= shrink; acc.y *= shrink; acc.z *= shrink; acc.w *= shrink;
        M = M_new;
        const int m = min(32, parts - p0);
#pragma unroll 4
        for (int i = 0; i < m; ++i) {
            const float fi = __shfl_sync(FULL_WARP, f, i);
            if (fi == 0.f) continue;                      // the same for the whole warp
            place(p0 + i, pml, po);
            if (mine) {
                const float4 v = *reinterpret_cast<const float4*>(po + 4 * lane);
                acc.x += fi * v.x; acc.y += fi * v.y; acc.z += fi * v.z; acc.w += fi * v.w;
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;           // 0: the row sees nothing
    if (4 * lane < g.a.head_dim) {
        T* out = reinterpret_cast<T*>(g.a.out) + ((size_t)row * g.a.n_heads + h) * g.a.head_dim + 4 * lane;
        *reinterpret_cast<uint2*>(out) = make_uint2(pack2(acc.x * inv, acc.y * inv, T()), pack2(acc.z * inv, acc.w * inv, T()));
    }
}

} // namespace swk
