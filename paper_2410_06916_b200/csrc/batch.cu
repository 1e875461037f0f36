// Batches of sequences over one paged K,V cache: argument checks, launch shapes and entry points of swift_rope_table,
// swift_kv_append, swift_prompt_attention and swift_prefix_attention.  No context and no state between calls.
// This translation unit gets its own copies of the shared device code (separate namespace).
#define swk swk_batch
#include "kernels_batch_dec.cuh"
#include "batch_host.cuh"

thread_local char swift_batch_error_text[512] = "";

namespace {

// what the tensor-core kernels take; the rest is computed in fp32 arithmetic
inline bool tensor_core_shape(const swift_paged_kv* kv) { return kv->dtype != SWIFT_F32 && kv->head_dim % 8 == 0 && kv->head_dim <= 128; }
swift_status check_attention(const swift_paged_kv* kv, const swift_row_batch* b, const swift_attention_args* a, BatchView* bv, AttnView* av)
{
    swift_status st = check_batch(kv, b, bv);
    if (st != SWIFT_OK) return st;
    if (!a) return fail_batch(SWIFT_EINVAL, "null arguments");
    if (a->block < 0 || a->block >= kv->n_blocks) return fail_batch(SWIFT_EINVAL, "block %d outside 0..%d", a->block, kv->n_blocks - 1);
    if (a->n_heads < 1 || a->n_heads > MAX_HEADS || a->n_heads % kv->n_kv_heads)
        return fail_batch(SWIFT_EINVAL, "n_heads %d is not a multiple of the cache's %d (at most %d)", a->n_heads, kv->n_kv_heads, MAX_HEADS);
    if (!(a->scale > 0.f) || !std::isfinite(a->scale * 2.f)) return fail_batch(SWIFT_EINVAL, "scale must be positive and below 2^127");
    if (b->n_rows > 0) {
        const int es = type_size(kv->dtype);
        if (!a->q.ptr || !a->out) return fail_batch(SWIFT_EINVAL, "null q or out");
        const int unit = tensor_core_shape(kv) ? 16 : es;
        if (!aligned(a->q.ptr, unit) || !aligned(a->out, unit) || a->q.row_stride * es % unit || a->q.head_stride * es % unit)
            return fail_batch(SWIFT_EINVAL, "q, its strides and out must be multiples of %d bytes", unit);
        if (a->q.row_stride < 0 || a->q.head_stride < 0) return fail_batch(SWIFT_EINVAL, "negative strides");
    }
    av->q = a->q.ptr;
    av->q_row_stride = a->q.row_stride;                   // a stride over a single row or head means nothing
    av->q_head_stride = a->q.head_stride;
    av->pool = block_base(kv, a->block);
    av->page_elems = 2 * kv_elems(kv) * kv->n_blocks;
    av->kv_elems = kv_elems(kv);
    av->out = a->out;
    av->n_heads = a->n_heads;
    av->n_kv_heads = kv->n_kv_heads;
    av->head_dim = kv->head_dim;
    av->max_rows = b->n_rows;
    av->scale = a->scale;
    av->wait_kcycles = (int)(TC_WAIT_CYCLES >> 10);
    av->withhold = 0;
    return SWIFT_OK;
}

// [page][block, K/V, kv head][slot][dim]; a box is one plane's slots of a page, at most a tile of them
swift_status make_kv_map(const swift_paged_kv* kv, int most_slots, CUtensorMap* out)
{
    const cuuint64_t D2 = 2ull * kv->head_dim, planes = 2ull * kv->n_blocks * kv->n_kv_heads;
    const cuuint64_t dims[4] = {(cuuint64_t)kv->head_dim, (cuuint64_t)kv->page_size, planes, (cuuint64_t)kv->n_pages};
    const cuuint64_t strides[3] = {D2, D2 * kv->page_size, D2 * kv->page_size * planes};
    const cuuint32_t box[4] = {64, (cuuint32_t)(kv->page_size < most_slots ? kv->page_size : most_slots), 1, 1};
    return make_map(out, kv->dtype, kv->pool, 4, dims, strides, box);
}

// The same pool for head_dim 64 or 128, seen as [plane][K, V][64-dim half][slot][64 dims] with overlapping planes (plane + n_kv_heads
// holds the V of plane's K): one box brings a page's K and V for a kv head.
swift_status make_kv_whole_map(const swift_paged_kv* kv, int most_slots, CUtensorMap* out)
{
    const cuuint64_t D2 = 2ull * kv->head_dim, halves = kv->head_dim / 64, plane = D2 * kv->page_size;
    const cuuint64_t dims[5] = {64, (cuuint64_t)kv->page_size, halves, 2, 2ull * kv->n_blocks * kv->n_kv_heads * kv->n_pages};
    const cuuint64_t strides[4] = {D2, 128, plane * kv->n_kv_heads, plane};
    const cuuint32_t box[5] = {64, (cuuint32_t)(kv->page_size < most_slots ? kv->page_size : most_slots), (cuuint32_t)halves, 2, 1};
    return make_map(out, kv->dtype, kv->pool, 5, dims, strides, box);
}

// [row][head][dim]; a box is one tile: the heads of a group for rows_per_tile rows
swift_status make_q_map(const swift_paged_kv* kv, const BatchView& bv, const AttnView& av, int rows_per_tile, CUtensorMap* out)
{
    const cuuint64_t dims[3] = {(cuuint64_t)kv->head_dim, (cuuint64_t)av.n_heads, (cuuint64_t)bv.n_rows};
    const cuuint64_t strides[2] = {2ull * av.q_head_stride, 2ull * av.q_row_stride};
    const cuuint32_t box[3] = {64, (cuuint32_t)(av.n_heads / av.n_kv_heads), (cuuint32_t)rows_per_tile};
    return make_map(out, kv->dtype, av.q, 3, dims, strides, box);
}

template <typename T, int HALVES, bool PART>
cudaError_t launch_tc(const CUtensorMap& kv_map, const CUtensorMap& q_map, const BatchView& bv, const BtArgs& g, int grid, cudaStream_t s, bool after_previous)
{
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = allow_smem(attn_batch_tc_kernel<T, HALVES, PART>, BtShape<HALVES>::SMEM_BYTES, done);
    if (e != cudaSuccess) return e;
    return launch(attn_batch_tc_kernel<T, HALVES, PART>, dim3(grid), BT_THREADS, BtShape<HALVES>::SMEM_BYTES, s, after_previous, kv_map, q_map, bv, g);
}

template <bool PART>
cudaError_t launch_tc_any(bool bf16, bool wide, const CUtensorMap& kv_map, const CUtensorMap& q_map, const BatchView& bv, const BtArgs& g, int grid,
                          cudaStream_t s, bool after)
{
    if (bf16) return wide ? launch_tc<__nv_bfloat16, 2, PART>(kv_map, q_map, bv, g, grid, s, after) : launch_tc<__nv_bfloat16, 1, PART>(kv_map, q_map, bv, g, grid, s, after);
    return wide ? launch_tc<__half, 2, PART>(kv_map, q_map, bv, g, grid, s, after) : launch_tc<__half, 1, PART>(kv_map, q_map, bv, g, grid, s, after);
}

// The many-row kernel in one of its three modes on at most `most` SMs; items: an upper bound of its pieces of work.
swift_status run_tc(const swift_paged_kv* kv, const BatchView& bv, const BtArgs& g, long long items, int most, cudaStream_t s, bool after_previous)
{
    CUtensorMap kv_map, q_map;
    swift_status st = make_kv_map(kv, BT_KEYS, &kv_map);
    if (st == SWIFT_OK) st = make_q_map(kv, bv, g.a, g.rows_per_tile, &q_map);
    if (st != SWIFT_OK) return st;
    const int grid = (int)(items < most ? items : most);          // prompts: `most` does not limit, blocks take over one another's pieces
    const bool wide = kv->head_dim > 64, bf16 = kv->dtype == SWIFT_BF16;
    const cudaError_t e = g.mode == BT_PROMPT ? launch_tc_any<false>(bf16, wide, kv_map, q_map, bv, g, grid, s, after_previous)
                                              : launch_tc_any<true>(bf16, wide, kv_map, q_map, bv, g, grid, s, after_previous);
    if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
    return SWIFT_OK;
}

swift_status run_prompt(const swift_paged_kv* kv, const BatchView& bv, const AttnView& av, int block, cudaStream_t s)
{
    BtArgs g = {};
    g.a = av;
    g.mode = BT_PROMPT;
    g.block = block;
    g.rows_per_tile = BT_ROWS / (av.n_heads / av.n_kv_heads);
    g.wide_out = aligned(av.out, 32) && av.head_dim % 16 == 0;
    // A pair of tiles takes little longer than one tile (each works while the other waits), so pieces are pairs unless even
    // single tiles leave no SM more than one (512 tokens of 32 heads: 14.7 us with single tiles, 16.5 with pairs).
    g.tiles = piece_bound(bv, av.n_kv_heads, g.rows_per_tile) <= multiprocessors() ? 1 : 2;
    return run_tc(kv, bv, g, piece_bound(bv, av.n_kv_heads, g.tiles * g.rows_per_tile), 0x7FFFFFFF, s, false);
}

// ------------------------------------------------------------------------------ few rows per sequence
// How swift_prefix_attention runs a batch, from sizes the host knows.
struct PrefixPlan {
    bool rows;                  // fp32 arithmetic: no tensor-core form
    bool prompt;                // too many rows for the few-row kernel, and no prefix or none worth sharing: each sequence by itself
    bool few, prefix_few;       // the few-row kernel takes the sequences' own parts; and the prefix
    int group, dp, mt, grid, pre_grid;   // grid: CTAs of the few-row kernel; pre_grid: of the prefix's
    long long items;
    int splits;                 // cuts of the prefix by the many-row kernel (0: it has no prefix work)
    int slots;                  // parts per row that the many-row kernel leaves: splits, and the own part if it takes it
    size_t many_o, many_ml, few_o, few_ml, first, last, bytes;   // offsets in the workspace
};

swift_status plan_prefix(const swift_paged_kv* kv, const BatchView& bv, int n_heads, int max_rows, PrefixPlan* p)
{
    *p = PrefixPlan();
    const int Hk = kv->n_kv_heads, sms = multiprocessors();
    if (max_rows > bv.n_rows) max_rows = bv.n_rows;
    p->group = n_heads / Hk;
    p->dp = kv->head_dim > 64 ? 128 : 64;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t o = at; at += (n + 255) / 256 * 256; return o; };
    p->rows = !tensor_core_shape(kv) || p->group > BT_ROWS;
    if (!p->rows) {
        const long long own = (long long)max_rows * p->group, all = (long long)bv.n_rows * p->group;
        p->few = own <= BD_MAX_ROWS;
        p->mt = own <= 16 ? 1 : own <= 32 ? 2 : 4;
        // the prefix too, if the rows of all sequences fit the same tile (a larger tile for the prefix alone slows the own parts: 10
        // sequences x 5 rows, 40 heads: 43 us against 27 with the many-row kernel beside it)
        p->prefix_few = p->few && bv.prefix_len > 0 && all <= 16 * p->mt;
        p->prompt = !p->few && bv.prefix_len == 0;
        if (bv.prefix_len > 0 && !p->prefix_few && !p->prompt) {
            // The prefix is tensor work, the sequences' own parts are HBM work: both kernels run at once, on SMs of their own, and
            // the share of SMs and the cuts of the prefix are chosen for the earliest common end.  Costs in microseconds: a key
            // tile of a pair of query tiles 1.75, a piece's set-up and write-back 8; own parts at 44 GB/s per SM up to 6 TB/s, 4 an item,
            // their lengths (which only the device knows) taken as 0.6 of the page table's width, and never more than 5/6 of the
            // SMs for them.  (64 continuations of 8192 positions, 64 heads on 8, about 750 own positions: 86 us one after the other.)
            const int tiles = ceil_div(bv.prefix_len, BT_KEYS), TQ = BT_ROWS / p->group;
            const long long pairs = (long long)ceil_div(bv.n_rows, 2 * TQ) * Hk;
            const double own_bytes = 0.6 * bv.n_seqs * bv.max_len * Hk * kv->head_dim * 4.0;
            double best = 0;
            for (int share = 2; share <= 12; ++share) {               // twelfths of the SMs
                const int g = sms * share / 12, rest = g == sms ? sms : sms - g;
                if (!p->few && g < sms) continue;
                const double stream_us = own_bytes / (rest * 44e3 < 6e6 ? rest * 44e3 : 6e6), item_us = 4.0 * ceil_div((long long)bv.n_seqs * Hk, rest * (BD_WARPS / p->mt));
                const double own_us = p->few ? 3.0 + (stream_us > item_us ? stream_us : item_us) : 0.0;
                for (int waves = 1; waves <= 4; ++waves) {            // as many cuts as fill that many waves
                    long long c = (long long)waves * g / pairs;
                    c = c < 1 ? 1 : c > tiles ? tiles : c > 64 ? 64 : c;
                    const double pre_us = ceil_div(pairs * c, g) * (ceil_div(tiles, c) * 1.75 + 8.0);
                    const double cost = (g == sms ? pre_us + own_us : pre_us > own_us ? pre_us : own_us) + c;    // every cut is read again by the join
                    if (p->splits == 0 || cost < best) {
                        best = cost;
                        p->splits = (int)c;
                        p->pre_grid = g;
                    }
                }
            }
        }
        if (!p->few && !p->prompt) {
            // Rows that fill tiles anyway gain nothing from a shared prefix but a better split over the SMs, and pay for writing and
            // joining parts: by the same costs, whichever form ends earlier.
            const int TQ2 = 2 * (BT_ROWS / p->group), own_tiles = ceil_div((long long)(0.6 * bv.max_len), BT_KEYS), tiles = ceil_div(bv.prefix_len, BT_KEYS);
            const long long seqs = bv.n_seqs < bv.n_rows ? bv.n_seqs : bv.n_rows, own_pieces = seqs * ceil_div(max_rows, TQ2) * Hk;
            const double one = ceil_div(own_pieces, sms) * ((tiles + own_tiles) * 1.75 + 8.0);
            const double shared = ceil_div((long long)ceil_div(bv.n_rows, TQ2) * Hk * p->splits, sms) * (ceil_div(tiles, p->splits) * 1.75 + 8.0) +
                                  ceil_div(own_pieces, sms) * (own_tiles * 1.75 + 8.0) + 5.0 + (double)bv.n_rows * n_heads * (p->splits + 1.5) * p->dp * 4 / 5e6;
            if (one < shared) {
                p->prompt = true;
                p->splits = 0;
            }
        }
        p->slots = p->splits + (!p->few && !p->prompt ? 1 : 0);
        const size_t many = (size_t)p->slots * bv.n_rows * n_heads;
        p->many_o = take(many * p->dp * 4);
        p->many_ml = take(many * 8);
        if (p->few) {
            p->items = (long long)(bv.n_seqs + (p->prefix_few ? 1 : 0)) * Hk;
            p->grid = p->splits > 0 && p->pre_grid < sms ? sms - p->pre_grid : sms;
            const int keys = 16 * p->mt;
            const long long units = ((long long)bv.n_seqs * ceil_div(bv.max_len, keys) + ceil_div(bv.prefix_len, keys)) * Hk;
            if (units > 0x7FFFFFFFll) return fail_batch(SWIFT_EUNSUPPORTED, "a page table of %d x %d for %d kv heads is beyond 2^31 units of work", bv.n_seqs, bv.table_stride, Hk);
            const size_t rows_all = (size_t)(p->items + (long long)p->grid * (BD_WARPS / p->mt)) * 16 * p->mt;
            p->few_o = take(rows_all * p->dp * 4);
            p->few_ml = take(rows_all * 8);
            p->first = take((size_t)p->items * 4);
            p->last = take((size_t)p->items * 4);
        }
    }
    p->bytes = at > 256 ? at : 256;
    return SWIFT_OK;
}

template <typename T, int HALVES, int MT>
cudaError_t launch_dec(const CUtensorMap& kv_map, const BatchView& bv, const BdArgs& g, int grid, cudaStream_t s, bool after_previous)
{
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = allow_smem(attn_batch_dec_kernel<T, HALVES, MT>, BdShape<HALVES, MT>::SMEM_BYTES, done);
    if (e != cudaSuccess) return e;
    return launch(attn_batch_dec_kernel<T, HALVES, MT>, dim3(grid), BD_THREADS, BdShape<HALVES, MT>::SMEM_BYTES, s, after_previous, kv_map, bv, g);
}

template <typename T>
cudaError_t launch_dec_any(const PrefixPlan& p, const CUtensorMap& kv_map, const BatchView& bv, const BdArgs& g, cudaStream_t s, bool after)
{
    if (p.dp == 128) {
        if (p.mt == 1) return launch_dec<T, 2, 1>(kv_map, bv, g, p.grid, s, after);
        if (p.mt == 2) return launch_dec<T, 2, 2>(kv_map, bv, g, p.grid, s, after);
        return launch_dec<T, 2, 4>(kv_map, bv, g, p.grid, s, after);
    }
    if (p.mt == 1) return launch_dec<T, 1, 1>(kv_map, bv, g, p.grid, s, after);
    if (p.mt == 2) return launch_dec<T, 1, 2>(kv_map, bv, g, p.grid, s, after);
    return launch_dec<T, 1, 4>(kv_map, bv, g, p.grid, s, after);
}

template <typename T>
cudaError_t launch_join(const PrefixPlan& p, const BatchView& bv, const BjArgs& j, cudaStream_t s)
{
    // An item has about (workers / items + 1) parts of the few-row kernel: with more than eight of them the eight warps of a block
    // share a head, else each takes one (one row behind 16000 positions: 23 us with eight warps per head, 69 with one; 64 rows
    // behind 750 on average: 64 and 47).
    const bool cut = p.few && (long long)p.grid * (BD_WARPS / p.mt) > 8 * p.items;
    return cut ? launch(attn_join_kernel<T, 8>, dim3(bv.n_rows, j.a.n_heads), 256, 0, s, true, bv, j)
               : launch(attn_join_kernel<T, 1>, dim3(bv.n_rows, ceil_div(j.a.n_heads, 8)), 256, 0, s, true, bv, j);
}

swift_status run_prefix(const swift_paged_kv* kv, const BatchView& bv, const AttnView& av, int block, const PrefixPlan& p, unsigned char* ws, cudaStream_t s)
{
    bool before = false;                                  // a kernel of this call has been launched
    BtArgs t = {};
    t.a = av;
    t.block = block;
    t.rows_per_tile = BT_ROWS / p.group;
    t.tiles = 2;
    t.part_o = reinterpret_cast<float*>(ws + p.many_o);
    t.part_ml = reinterpret_cast<float2*>(ws + p.many_ml);
    if (p.splits > 0) {
        t.mode = BT_PREFIX;
        t.splits = p.splits;
        const swift_status st = run_tc(kv, bv, t, (long long)ceil_div(bv.n_rows, 2 * t.rows_per_tile) * av.n_kv_heads * p.splits, p.pre_grid, s, before);
        if (st != SWIFT_OK) return st;
        before = true;
    }
    BjArgs j = {};
    j.a = av;
    j.dp = p.dp;
    j.item_rows = 16 * p.mt;
    j.prefix_here = p.prefix_few;
    j.own_here = p.few;
    j.splits = p.slots;
    j.many_o = t.part_o;
    j.many_ml = t.part_ml;
    j.few_o = reinterpret_cast<float*>(ws + p.few_o);
    j.few_ml = reinterpret_cast<float2*>(ws + p.few_ml);
    j.item_first = reinterpret_cast<int*>(ws + p.first);
    j.item_last = reinterpret_cast<int*>(ws + p.last);
    j.workers = p.grid * (BD_WARPS / p.mt);
    cudaError_t e = cudaSuccess;
    if (p.few) {
        BdArgs g = {};
        g.a = av;
        g.block = block;
        g.prefix_here = p.prefix_few;
        g.part_o = reinterpret_cast<float*>(ws + p.few_o);
        g.part_ml = reinterpret_cast<float2*>(ws + p.few_ml);
        g.item_first = reinterpret_cast<int*>(ws + p.first);
        g.item_last = reinterpret_cast<int*>(ws + p.last);
        CUtensorMap kv_map;
        const long long planes = 2ll * kv->n_blocks * kv->n_kv_heads * kv->n_pages;
        g.whole_boxes = kv->head_dim % 64 == 0 && planes < 0x7FFFFFFFll;
        g.planes = g.whole_boxes ? (int)planes : 0;
        const swift_status st = g.whole_boxes ? make_kv_whole_map(kv, 16 * p.mt, &kv_map) : make_kv_map(kv, 16 * p.mt, &kv_map);
        if (st != SWIFT_OK) return st;
        e = kv->dtype == SWIFT_BF16 ? launch_dec_any<__nv_bfloat16>(p, kv_map, bv, g, s, before) : launch_dec_any<__half>(p, kv_map, bv, g, s, before);
    } else {
        t.mode = BT_OWN;
        t.part_slot = p.splits;
        const swift_status st = run_tc(kv, bv, t, piece_bound(bv, av.n_kv_heads, 2 * t.rows_per_tile), multiprocessors(), s, before);
        if (st != SWIFT_OK) return st;
    }
    if (e == cudaSuccess) {
        e = kv->dtype == SWIFT_BF16 ? launch_join<__nv_bfloat16>(p, bv, j, s) : launch_join<__half>(p, bv, j, s);
    }
    if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
    return SWIFT_OK;
}

cudaError_t launch_rows(const swift_paged_kv* kv, const BatchView& bv, const AttnView& av, cudaStream_t s)
{
    switch (kv->dtype) {
    case SWIFT_F32: return launch_fp32<float, float>(bv, av, s);
    case SWIFT_BF16: return launch_fp32<__nv_bfloat16, __nv_bfloat16>(bv, av, s);
    default: return launch_fp32<__half, __half>(bv, av, s);
    }
}

// What each stream's last report saw of its device's count of waits that ran out (batch_waits_over): the device's count is never
// cleared, so a report to one stream takes nothing from another, nor from a wait that runs out meanwhile.  Streams are known by
// their ids, which a process uses once.  When more streams report than there is room for, the one whose report is the oldest is
// forgotten and counts from 0 again: told twice rather than never.
class Reports {
public:
    bool changed(int dev, unsigned long long stream, unsigned count)
    {
        while (busy.test_and_set(std::memory_order_acquire)) { }      // a few comparisons long
        Entry* e = nullptr;
        for (int i = 0; i < ENTRIES; ++i)
            if (entries[i].age != 0 && entries[i].dev == dev && entries[i].stream == stream) e = &entries[i];
        if (!e) {
            e = &entries[0];
            for (int i = 1; i < ENTRIES; ++i)
                if (entries[i].age < e->age) e = &entries[i];
            e->dev = dev;
            e->stream = stream;
            e->seen = 0;
        }
        const bool news = e->seen != count;
        e->seen = count;
        e->age = ++clock;
        busy.clear(std::memory_order_release);
        return news;
    }
private:
    static constexpr int ENTRIES = 256;
    struct Entry { unsigned long long age, stream; int dev; unsigned seen; };     // age 0: free
    Entry entries[ENTRIES] = {};
    unsigned long long clock = 0;
    std::atomic_flag busy = ATOMIC_FLAG_INIT;
};
Reports g_reports;

swift_status prompt_attention(const swift_paged_kv* kv, const swift_row_batch* batch, const swift_attention_args* args, int probe_us, cudaStream_t s)
{
    BatchView bv;
    AttnView av;
    swift_status st = check_attention(kv, batch, args, &bv, &av);
    if (st != SWIFT_OK) return st;
    if (bv.n_rows == 0 || bv.n_seqs == 0) return SWIFT_OK;
    set_probe(&av, probe_us);
    if (!tensor_core_shape(kv) || av.n_heads / av.n_kv_heads > BT_ROWS) {
        const cudaError_t e = launch_rows(kv, bv, av, s);
        if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
        return SWIFT_OK;
    }
    return run_prompt(kv, bv, av, args->block, s);
}

swift_status prefix_attention(const swift_paged_kv* kv, const swift_row_batch* batch, const swift_attention_args* args, int max_rows,
                              swift_devbuf workspace, int probe_us, cudaStream_t s)
{
    BatchView bv;
    AttnView av;
    swift_status st = check_attention(kv, batch, args, &bv, &av);
    if (st != SWIFT_OK) return st;
    if (max_rows < 1) return fail_batch(SWIFT_EINVAL, "max_rows %d", max_rows);
    if (bv.n_rows == 0 || bv.n_seqs == 0) return SWIFT_OK;
    PrefixPlan p;
    st = plan_prefix(kv, bv, av.n_heads, max_rows, &p);
    if (st != SWIFT_OK) return st;
    if (!workspace.dptr || !aligned(workspace.dptr, 256)) return fail_batch(SWIFT_EINVAL, "the workspace must be 256-byte aligned device memory");
    if (workspace.bytes < p.bytes) return fail_batch(SWIFT_ECAPACITY, "workspace of %zu bytes, %zu needed", workspace.bytes, p.bytes);
    av.max_rows = max_rows;
    set_probe(&av, probe_us);
    if (p.rows) {
        const cudaError_t e = launch_rows(kv, bv, av, s);
        if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
        return SWIFT_OK;
    }
    if (p.prompt) return run_prompt(kv, bv, av, args->block, s);
    return run_prefix(kv, bv, av, args->block, p, reinterpret_cast<unsigned char*>(workspace.dptr), s);
}

} // namespace

extern "C" {

const char* swift_batch_error(void) { return swift_batch_error_text; }

swift_status swift_rope_table(const swift_rope_desc* d, float* table_dev, void* cuda_stream)
{
    if (!d || !table_dev) return fail_batch(SWIFT_EINVAL, "null description or table");
    if (!aligned(table_dev, 8)) return fail_batch(SWIFT_EINVAL, "the table must be 8-byte aligned");
    if (d->n_positions < 0 || d->n_positions > MAX_POSITIONS) return fail_batch(SWIFT_EINVAL, "n_positions %d", d->n_positions);
    if (d->rotary_dim < 2 || d->rotary_dim > 256 || d->rotary_dim % 2) return fail_batch(SWIFT_EINVAL, "rotary_dim %d is not even in 2..256", d->rotary_dim);
    if (!(d->theta > 0.0) || std::isinf(d->theta) || !(d->factor > 0.0) || std::isinf(d->factor) || !std::isfinite(d->magnitude))
        return fail_batch(SWIFT_EINVAL, "theta and factor must be positive and finite, magnitude finite");
    if (d->original_positions < 0) return fail_batch(SWIFT_EINVAL, "original_positions %d", d->original_positions);
    if (d->original_positions > 0 && !(std::isfinite(d->low_turns) && std::isfinite(d->high_turns) && d->low_turns < d->high_turns))
        return fail_batch(SWIFT_EINVAL, "low_turns must be below high_turns");
    if (d->n_positions == 0) return SWIFT_OK;
    RopeTableArgs a;
    a.table = reinterpret_cast<float2*>(table_dev);
    a.n_positions = d->n_positions;
    a.half = d->rotary_dim / 2;
    a.log_theta_step = 2.0 * std::log(d->theta) / d->rotary_dim;
    a.inv_factor = 1.0 / d->factor;
    a.turns_per_freq = d->original_positions / (2.0 * 3.14159265358979323846);
    a.low = d->low_turns;
    a.inv_range = d->original_positions > 0 ? 1.0 / (d->high_turns - d->low_turns) : 0.0;
    a.magnitude = d->magnitude;
    const long long threads = (long long)ceil_div(d->n_positions, RT_RUN) * a.half;
    const cudaError_t e = launch(rope_run_kernel, dim3((unsigned)((threads + 127) / 128)), 128, 0, (cudaStream_t)cuda_stream, false, a);
    if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
    return SWIFT_OK;
}

swift_status swift_kv_append(const swift_paged_kv* kv, const swift_row_batch* batch, const swift_append_args* x, void* cuda_stream)
{
    BatchView bv;
    swift_status st = check_batch(kv, batch, &bv);
    if (st != SWIFT_OK) return st;
    if (!x) return fail_batch(SWIFT_EINVAL, "null arguments");
    if (x->block < 0 || x->block >= kv->n_blocks) return fail_batch(SWIFT_EINVAL, "block %d outside 0..%d", x->block, kv->n_blocks - 1);
    if (x->n_heads < 0 || x->n_heads > MAX_HEADS) return fail_batch(SWIFT_EINVAL, "n_heads %d", x->n_heads);
    if (x->x_dtype != SWIFT_F32 && x->x_dtype != kv->dtype) return fail_batch(SWIFT_EUNSUPPORTED, "q, k, v must be fp32 or of the cache's type");
    st = check_append(kv, x);
    if (st != SWIFT_OK) return st;
    if (bv.n_rows == 0 || bv.n_seqs == 0) return SWIFT_OK;
    AppendView a;
    bool vecs[2];
    st = view_append(kv, x, kv->dtype, &a, vecs);
    if (st != SWIFT_OK) return st;
    const bool vec = vecs[0] && vecs[1];
    cudaStream_t s = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (kv->dtype == SWIFT_F32) e = launch_append<float, float>(bv, a, vec, s);
    else if (kv->dtype == SWIFT_BF16) e = x->x_dtype == SWIFT_F32 ? launch_append<float, __nv_bfloat16>(bv, a, vec, s) : launch_append<__nv_bfloat16, __nv_bfloat16>(bv, a, vec, s);
    else e = x->x_dtype == SWIFT_F32 ? launch_append<float, __half>(bv, a, vec, s) : launch_append<__half, __half>(bv, a, vec, s);
    if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
    return SWIFT_OK;
}

swift_status swift_prompt_attention(const swift_paged_kv* kv, const swift_row_batch* batch, const swift_attention_args* args, void* cuda_stream)
{
    return prompt_attention(kv, batch, args, 0, (cudaStream_t)cuda_stream);
}

size_t swift_prefix_workspace_bytes(const swift_paged_kv* kv, const swift_row_batch* batch, int32_t n_heads, int32_t max_rows)
{
    BatchView bv;
    if (check_batch(kv, batch, &bv) != SWIFT_OK) return 0;
    if (n_heads < 1 || n_heads > MAX_HEADS || n_heads % kv->n_kv_heads || max_rows < 1) {
        fail_batch(SWIFT_EINVAL, "n_heads %d, max_rows %d", n_heads, max_rows);
        return 0;
    }
    PrefixPlan p;
    return plan_prefix(kv, bv, n_heads, max_rows, &p) == SWIFT_OK ? p.bytes : 0;
}

swift_status swift_prefix_attention(const swift_paged_kv* kv, const swift_row_batch* batch, const swift_attention_args* args, int32_t max_rows,
                                    swift_devbuf workspace, void* cuda_stream)
{
    return prefix_attention(kv, batch, args, max_rows, workspace, 0, (cudaStream_t)cuda_stream);
}

swift_status swift_probe_batch_wait_limit(const swift_paged_kv* kv, const swift_row_batch* batch, const swift_attention_args* args, int32_t max_rows,
                                          swift_devbuf workspace, int32_t limit_us, void* cuda_stream)
{
    if (limit_us < 1 || limit_us > 100000) return fail_batch(SWIFT_EINVAL, "limit_us must be in 1..100000");
    if (max_rows < 0) return fail_batch(SWIFT_EINVAL, "max_rows %d", max_rows);
    if (kv && args && kv->n_kv_heads > 0 && (!tensor_core_shape(kv) || args->n_heads / kv->n_kv_heads > BT_ROWS))
        return fail_batch(SWIFT_EUNSUPPORTED, "fp32 arithmetic has no waits");
    if (max_rows == 0) return prompt_attention(kv, batch, args, limit_us, (cudaStream_t)cuda_stream);
    return prefix_attention(kv, batch, args, max_rows, workspace, limit_us, (cudaStream_t)cuda_stream);
}

swift_status swift_batch_sync(void* cuda_stream)
{
    unsigned count = 0;
    int dev = 0;
    unsigned long long id = 0;
    unsigned count8 = 0;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaStreamGetId(s, &id);
    if (e == cudaSuccess) e = cudaMemcpyFromSymbolAsync(&count, batch_waits_over, sizeof count, 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = swift_batch8_waits(&count8, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    count += count8;
    if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "the stream's work failed: %s", cudaGetErrorString(e));
    if (g_reports.changed(dev, id, count)) return fail_batch(SWIFT_ETIMEOUT, "a device-side wait of an attention call ran out of time");
    return SWIFT_OK;
}

} // extern "C"
