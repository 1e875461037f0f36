// Batches of sequences over a paged cache of 8-bit codes: argument checks, launch shapes and entry points of swift_coded_append,
// swift_coded_prompt_attention and swift_coded_prefix_attention.  No context and no state between calls.
// This translation unit gets its own copies of the shared device code (separate namespace).
#define swk swk_batch8
#include "kernels_batch8_tc.cuh"
#include "batch_host.cuh"

cudaError_t swift_batch8_waits(unsigned* count, cudaStream_t s)
{
    return cudaMemcpyFromSymbolAsync(count, batch_waits_over, sizeof *count, 0, cudaMemcpyDeviceToHost, s);
}

namespace {

swift_status check_cache8(const swift_coded_kv* c, const swift_row_batch* b, BatchView* bv)
{
    const swift_status st = check_batch(c ? &c->kv : nullptr, b, bv, true);
    if (st != SWIFT_OK) return st;
    if (!c->scales || !aligned(c->scales, 4)) return fail_batch(SWIFT_EINVAL, "the scales must be 4-byte aligned device memory");
    return SWIFT_OK;
}
inline float* block_scales(const swift_coded_kv* c, int block) { return c->scales + (size_t)block * 2 * c->kv.n_kv_heads; }
inline long long scale_page(const swift_coded_kv* c) { return 2ll * c->kv.n_blocks * c->kv.n_kv_heads; }

// what the tensor-core kernels take; the rest is computed in fp32 arithmetic
inline bool tensor_core_shape8(const swift_paged_kv* kv, int x_dtype, int n_heads)
{
    return x_dtype != SWIFT_F32 && kv->head_dim % 16 == 0 && kv->head_dim <= 128 && n_heads / kv->n_kv_heads <= BT_ROWS;
}

swift_status check_attention8(const swift_coded_kv* c, const swift_row_batch* b, const swift_attention_args* a, int x_dtype, BatchView* bv, AttnView* av)
{
    swift_status st = check_cache8(c, b, bv);
    if (st != SWIFT_OK) return st;
    const swift_paged_kv* kv = &c->kv;
    if (!a) return fail_batch(SWIFT_EINVAL, "null arguments");
    if (!type_known(x_dtype)) return fail_batch(SWIFT_EINVAL, "type %d of q and out unknown", x_dtype);
    if (a->block < 0 || a->block >= kv->n_blocks) return fail_batch(SWIFT_EINVAL, "block %d outside 0..%d", a->block, kv->n_blocks - 1);
    if (a->n_heads < 1 || a->n_heads > MAX_HEADS || a->n_heads % kv->n_kv_heads)
        return fail_batch(SWIFT_EINVAL, "n_heads %d is not a multiple of the cache's %d (at most %d)", a->n_heads, kv->n_kv_heads, MAX_HEADS);
    if (!(a->scale > 0.f) || !std::isfinite(a->scale * 2.f)) return fail_batch(SWIFT_EINVAL, "scale must be positive and below 2^127");
    if (b->n_rows > 0) {
        const int es = type_size(x_dtype);
        if (!a->q.ptr || !a->out) return fail_batch(SWIFT_EINVAL, "null q or out");
        const int unit = tensor_core_shape8(kv, x_dtype, a->n_heads) ? 16 : es;
        if (!aligned(a->q.ptr, unit) || !aligned(a->out, unit) || a->q.row_stride * es % unit || a->q.head_stride * es % unit)
            return fail_batch(SWIFT_EINVAL, "q, its strides and out must be multiples of %d bytes", unit);
        if (a->q.row_stride < 0 || a->q.head_stride < 0) return fail_batch(SWIFT_EINVAL, "negative strides");
    }
    av->q = a->q.ptr;
    av->q_row_stride = a->q.row_stride;
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
    av->scales = block_scales(c, a->block);
    av->scale_page = scale_page(c);
    return SWIFT_OK;
}

template <typename TC> cudaError_t launch_rows8(int x_dtype, const BatchView& bv, const AttnView& av, cudaStream_t s)
{
    switch (x_dtype) {
    case SWIFT_F32: return launch_fp32<float, TC>(bv, av, s);
    case SWIFT_BF16: return launch_fp32<__nv_bfloat16, TC>(bv, av, s);
    default: return launch_fp32<__half, TC>(bv, av, s);
    }
}
swift_status run_rows8(const swift_paged_kv* kv, int x_dtype, const BatchView& bv, const AttnView& av, cudaStream_t s)
{
    const cudaError_t e = kv->dtype == SWIFT_I8 ? launch_rows8<int8_t>(x_dtype, bv, av, s) : launch_rows8<__nv_fp8_e4m3>(x_dtype, bv, av, s);
    if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
    return SWIFT_OK;
}

// Pages that get rows, at most: each row adds one at most, and n rows of a sequence lie on n / page_size + 2 at most.
long long page_bound(const BatchView& bv)
{
    const long long some = bv.n_seqs < bv.n_rows ? bv.n_seqs : bv.n_rows, bound = bv.n_rows / bv.page_size + 2 * some;
    return bound < bv.n_rows ? bound : bv.n_rows;
}

template <typename TX, typename CODE, int PIECE, int LPH>
cudaError_t launch_append8_form(const BatchView& bv, Append8View& v, cudaStream_t s)
{
    v.pages = (int)page_bound(bv);
    if (PIECE == 8 && v.a.n_heads > 0) {
        // the queries, in blocks of the same launch: a row's heads to as many warps as make two waves of warps, as the 16-bit cache's append does
        const int batch = 32 / LPH * AP_UNROLL<TX>, most = ceil_div(v.a.n_heads, batch), wanted = ceil_div(148 * 40, bv.n_rows);
        v.q_chunks = wanted < most ? wanted : most;
        v.q_per_warp = ceil_div(ceil_div(v.a.n_heads, v.q_chunks), 32 / LPH) * (32 / LPH);
    }
    const long long kv_blocks = (long long)v.pages * 2 * v.a.n_kv_heads, q_blocks = ((long long)bv.n_rows * v.q_chunks + AP_THREADS / 32 - 1) / (AP_THREADS / 32);
    if (kv_blocks + q_blocks > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    return launch(append8_kernel<TX, CODE, PIECE, LPH>, dim3((unsigned)(kv_blocks + q_blocks)), AP_THREADS, 0, s, false, bv, v);
}
template <typename TX, typename CODE>
cudaError_t launch_append8(const BatchView& bv, Append8View& v, bool q_vec, bool kv_vec, cudaStream_t s)
{
    v.q_chunks = v.q_per_warp = 0;
    if (!q_vec || !kv_vec) {
        if (v.a.n_heads > 0) {
            AppendView q = v.a;                           // the queries alone, by the 16-bit cache's kernels
            q.n_kv_heads = 0;
            const cudaError_t e = launch_append<TX, TX>(bv, q, q_vec, s);
            if (e != cudaSuccess) return e;
        }
        return launch_append8_form<TX, CODE, 1, 32>(bv, v, s);
    }
    const int pieces = v.a.head_dim / 16;
    if (pieces <= 1) return launch_append8_form<TX, CODE, 8, 1>(bv, v, s);
    if (pieces <= 2) return launch_append8_form<TX, CODE, 8, 2>(bv, v, s);
    if (pieces <= 4) return launch_append8_form<TX, CODE, 8, 4>(bv, v, s);
    if (pieces <= 8) return launch_append8_form<TX, CODE, 8, 8>(bv, v, s);
    return launch_append8_form<TX, CODE, 8, 16>(bv, v, s);
}
template <typename TX>
cudaError_t launch_append8_any(int dtype, const BatchView& bv, Append8View& v, bool q_vec, bool kv_vec, cudaStream_t s)
{
    return dtype == SWIFT_I8 ? launch_append8<TX, int8_t>(bv, v, q_vec, kv_vec, s) : launch_append8<TX, __nv_fp8_e4m3>(bv, v, q_vec, kv_vec, s);
}

// ------------------------------------------------------------------------------ few rows per sequence
// [page][block, K/V, kv head][slot][dim] bytes, seen as [plane][K, V][slot][dim] with overlapping planes (plane + n_kv_heads holds the V
// of plane's K): one box brings a page's K and V for a kv head.  dp: bytes of a row in shared memory, 64 or 128; what lies beyond head_dim is 0.
// K and V apart (whole = false): for tiles of one of them, not swizzled.
swift_status make_codes_map(const swift_paged_kv* kv, int dp, int most_slots, bool whole, CUtensorMap* out)
{
    if (2ll * kv->n_blocks * kv->n_kv_heads * kv->n_pages > 0x7FFFFFFFll)
        return fail_batch(SWIFT_EUNSUPPORTED, "a pool of %d pages of %d heads is beyond 2^31 planes", kv->n_pages, 2 * kv->n_blocks * kv->n_kv_heads);
    const EncodeTiled encode = encoder();
    if (!encode) return fail_batch(SWIFT_ECUDA, "cuTensorMapEncodeTiled not available from the driver");
    const cuuint64_t row = kv->head_dim, plane = row * kv->page_size;
    const cuuint64_t dims[4] = {row, (cuuint64_t)kv->page_size, 2, 2ull * kv->n_blocks * kv->n_kv_heads * kv->n_pages};
    const cuuint64_t strides[3] = {row, plane * kv->n_kv_heads, plane};
    const cuuint32_t box[4] = {(cuuint32_t)dp, (cuuint32_t)(kv->page_size < most_slots ? kv->page_size : most_slots), whole ? 2u : 1u, 1}, one[4] = {1, 1, 1, 1};
    const CUresult r = encode(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, kv->pool, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              !whole ? CU_TENSOR_MAP_SWIZZLE_NONE : dp == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail_batch(SWIFT_EINVAL, "cuTensorMapEncodeTiled refused the tensor (code %d): a cache of odd size", (int)r);
    return SWIFT_OK;
}

// How swift_coded_prefix_attention runs a batch, from sizes the host knows: the choices of the 16-bit cache's plan, with this cache's
// bytes and rates.
struct Plan8 {
    bool rows;                  // fp32 arithmetic: no tensor-core form
    bool prompt;                // too many rows for the few-row kernel, and no prefix or none worth sharing: each sequence by itself
    bool few, prefix_few;       // the few-row kernel takes the sequences' own parts; and the prefix
    bool eight;                 // in its form for 8 rows
    int group, dp, mt, workers, grid, pre_grid;                    // grid: CTAs of the few-row kernel; pre_grid: of the prefix's
    long long items;
    int splits;                 // cuts of the prefix by the many-row kernel (0: it has no prefix work)
    int slots;                  // parts per row that the many-row kernel leaves: splits, and the own part if it takes it
    size_t many_o, many_ml, few_o, few_ml, first, last, bytes;   // offsets in the workspace
};
inline int unit_keys8(const Plan8& p) { return p.mt == 1 && !p.eight ? 32 : 64; }

swift_status plan_prefix8(const swift_coded_kv* c, const BatchView& bv, int n_heads, int max_rows, int x_dtype, Plan8* p)
{
    *p = Plan8();
    const swift_paged_kv* kv = &c->kv;
    const int Hk = kv->n_kv_heads, sms = multiprocessors();
    if (max_rows > bv.n_rows) max_rows = bv.n_rows;
    p->group = n_heads / Hk;
    p->dp = kv->head_dim > 64 ? 128 : 64;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t o = at; at += (n + 255) / 256 * 256; return o; };
    p->rows = !tensor_core_shape8(kv, x_dtype, n_heads);
    if (!p->rows) {
        // Costs in microseconds: a key tile of a pair of query tiles, a piece's set-up and write-back; own parts per SM and in all.
        constexpr double TILE = 1.9, PIECE = 9.0, SM_RATE = 30e3, RATE = 4.5e6;
        const long long own = (long long)max_rows * p->group, all = (long long)bv.n_rows * p->group;
        p->few = own <= BD_MAX_ROWS;
        p->mt = own <= 16 ? 1 : own <= 32 ? 2 : 4;
        p->prefix_few = p->few && bv.prefix_len > 0 && all <= 16 * p->mt;
        p->eight = p->few && own <= 8 && (!p->prefix_few || all <= 8);
        p->workers = 8 / p->mt;                           // of a CTA
        p->prompt = !p->few && bv.prefix_len == 0;
        if (bv.prefix_len > 0 && !p->prefix_few && !p->prompt) {
            // The prefix is tensor work, the sequences' own parts are HBM work: both kernels run at once on SMs of their own, and the share
            // of SMs and the cuts of the prefix are chosen for the earliest common end; own lengths (which only the device knows) are taken
            // as 0.6 of the page table's width, and never more than 5/6 of the SMs are for them.
            const int tiles = ceil_div(bv.prefix_len, BT_KEYS), TQ = BT_ROWS / p->group;
            const long long pairs = (long long)ceil_div(bv.n_rows, 2 * TQ) * Hk;
            const double own_bytes = 0.6 * bv.n_seqs * bv.max_len * Hk * kv->head_dim * 2.0;
            double best = 0;
            for (int share = 2; share <= 12; ++share) {               // twelfths of the SMs
                const int g = sms * share / 12, rest = g == sms ? sms : sms - g;
                if (!p->few && g < sms) continue;
                const double stream_us = own_bytes / (rest * SM_RATE < RATE ? rest * SM_RATE : RATE), item_us = 4.0 * ceil_div((long long)bv.n_seqs * Hk, rest * p->workers);
                const double own_us = p->few ? 3.0 + (stream_us > item_us ? stream_us : item_us) : 0.0;
                for (int waves = 1; waves <= 4; ++waves) {            // as many cuts as fill that many waves
                    long long n = (long long)waves * g / pairs;
                    n = n < 1 ? 1 : n > tiles ? tiles : n > 64 ? 64 : n;
                    const double pre_us = ceil_div(pairs * n, g) * (ceil_div(tiles, n) * TILE + PIECE);
                    const double cost = (g == sms ? pre_us + own_us : pre_us > own_us ? pre_us : own_us) + n;    // every cut is read again by the join
                    if (p->splits == 0 || cost < best) {
                        best = cost;
                        p->splits = (int)n;
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
            const double one = ceil_div(own_pieces, sms) * ((tiles + own_tiles) * TILE + PIECE);
            const double shared = ceil_div((long long)ceil_div(bv.n_rows, TQ2) * Hk * p->splits, sms) * (ceil_div(tiles, p->splits) * TILE + PIECE) +
                                  ceil_div(own_pieces, sms) * (own_tiles * TILE + PIECE) + 5.0 + (double)bv.n_rows * n_heads * (p->splits + 1.5) * p->dp * 4 / 5e6;
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
            const int keys = unit_keys8(*p);
            const long long units = ((long long)bv.n_seqs * ceil_div(bv.max_len, keys) + ceil_div(bv.prefix_len, keys)) * Hk;
            if (units > 0x7FFFFFFFll) return fail_batch(SWIFT_EUNSUPPORTED, "a page table of %d x %d for %d kv heads is beyond 2^31 units of work", bv.n_seqs, bv.table_stride, Hk);
            const size_t rows_all = (size_t)(p->items + (long long)p->grid * p->workers) * 16 * p->mt;
            p->few_o = take(rows_all * p->dp * 4);
            p->few_ml = take(rows_all * 8);
            p->first = take((size_t)p->items * 4);
            p->last = take((size_t)p->items * 4);
        }
    }
    p->bytes = at > 256 ? at : 256;
    return SWIFT_OK;
}

// ------------------------------------------------------------------------------ many rows
template <int HALVES, bool PART>
cudaError_t launch_tc8(const CUtensorMap& map, const BatchView& bv, const B8TcArgs& g, int grid, cudaStream_t s, bool after_previous)
{
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = allow_smem(attn_batch8_tc_kernel<HALVES, PART>, B8TcShape<HALVES>::SMEM_BYTES, done);
    if (e != cudaSuccess) return e;
    return launch(attn_batch8_tc_kernel<HALVES, PART>, dim3(grid), B8_THREADS, B8TcShape<HALVES>::SMEM_BYTES, s, after_previous, map, bv, g);
}
// The many-row kernel in one of its three modes on at most `most` SMs; items: an upper bound of its pieces of work.
swift_status run_tc8(const swift_paged_kv* kv, int x_dtype, const BatchView& bv, const BtArgs& t, long long items, int most, cudaStream_t s, bool after)
{
    const bool wide = kv->head_dim > 64;
    CUtensorMap map;
    const swift_status st = make_codes_map(kv, wide ? 128 : 64, BT_KEYS, false, &map);
    if (st != SWIFT_OK) return st;
    const B8TcArgs g = {t, kv->dtype == SWIFT_E4M3, x_dtype == SWIFT_BF16, kv->n_blocks};
    const int grid = (int)(items < most ? items : most);          // prompts: `most` does not limit, blocks take over one another's pieces
    const bool part = t.mode != BT_PROMPT;
    const cudaError_t e = wide ? (part ? launch_tc8<2, true>(map, bv, g, grid, s, after) : launch_tc8<2, false>(map, bv, g, grid, s, after))
                               : (part ? launch_tc8<1, true>(map, bv, g, grid, s, after) : launch_tc8<1, false>(map, bv, g, grid, s, after));
    if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
    return SWIFT_OK;
}
swift_status run_prompt8(const swift_paged_kv* kv, int x_dtype, const BatchView& bv, const AttnView& av, int block, cudaStream_t s)
{
    BtArgs g = {};
    g.a = av;
    g.mode = BT_PROMPT;
    g.block = block;
    g.rows_per_tile = BT_ROWS / (av.n_heads / av.n_kv_heads);
    g.tiles = piece_bound(bv, av.n_kv_heads, g.rows_per_tile) <= multiprocessors() ? 1 : 2;     // as for the 16-bit cache
    return run_tc8(kv, x_dtype, bv, g, piece_bound(bv, av.n_kv_heads, g.tiles * g.rows_per_tile), 0x7FFFFFFF, s, false);
}

template <typename QT, typename CODE, int DP, int MT, bool EIGHT = false>
cudaError_t launch_dec8(const CUtensorMap& map, const BatchView& bv, const BdArgs& g, int grid, cudaStream_t s, bool after_previous)
{
    typedef B8Shape<DP, MT, EIGHT> S;
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = allow_smem(attn_batch8_dec_kernel<QT, CODE, DP, MT, EIGHT>, S::SMEM_BYTES, done);
    if (e != cudaSuccess) return e;
    return launch(attn_batch8_dec_kernel<QT, CODE, DP, MT, EIGHT>, dim3(grid), 32 * S::WARPS, S::SMEM_BYTES, s, after_previous, map, bv, g);
}
template <typename QT, typename CODE, int DP>
cudaError_t launch_dec8_rows(const Plan8& p, const CUtensorMap& map, const BatchView& bv, const BdArgs& g, cudaStream_t s, bool after)
{
    if (p.eight) return launch_dec8<QT, CODE, DP, 1, true>(map, bv, g, p.grid, s, after);
    if (p.mt == 1) return launch_dec8<QT, CODE, DP, 1>(map, bv, g, p.grid, s, after);
    if (p.mt == 2) return launch_dec8<QT, CODE, DP, 2>(map, bv, g, p.grid, s, after);
    return launch_dec8<QT, CODE, DP, 4>(map, bv, g, p.grid, s, after);
}
template <typename QT, typename CODE>
cudaError_t launch_dec8_any(const Plan8& p, const CUtensorMap& map, const BatchView& bv, const BdArgs& g, cudaStream_t s, bool after)
{
    return p.dp == 128 ? launch_dec8_rows<QT, CODE, 128>(p, map, bv, g, s, after) : launch_dec8_rows<QT, CODE, 64>(p, map, bv, g, s, after);
}

template <typename T>
cudaError_t launch_join8(const Plan8& p, const BatchView& bv, const BjArgs& j, cudaStream_t s)
{
    const bool cut = p.few && (long long)p.grid * p.workers > 8 * p.items;       // as for the 16-bit cache
    return cut ? launch(attn_join_kernel<T, 8>, dim3(bv.n_rows, j.a.n_heads), 256, 0, s, true, bv, j)
               : launch(attn_join_kernel<T, 1>, dim3(bv.n_rows, ceil_div(j.a.n_heads, 8)), 256, 0, s, true, bv, j);
}

template <typename QT>
swift_status run_prefix8(const swift_coded_kv* c, int x_dtype, const BatchView& bv, const AttnView& av, int block, const Plan8& p, unsigned char* ws, cudaStream_t s)
{
    const swift_paged_kv* kv = &c->kv;
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
        const swift_status st = run_tc8(kv, x_dtype, bv, t, (long long)ceil_div(bv.n_rows, 2 * t.rows_per_tile) * av.n_kv_heads * p.splits, p.pre_grid, s, before);
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
    j.workers = p.grid * p.workers;
    cudaError_t e = cudaSuccess;
    if (p.few) {
        BdArgs g = {};
        g.a = av;
        g.block = block;
        g.prefix_here = p.prefix_few;
        g.planes = 2 * kv->n_blocks * kv->n_kv_heads * kv->n_pages;
        g.part_o = reinterpret_cast<float*>(ws + p.few_o);
        g.part_ml = reinterpret_cast<float2*>(ws + p.few_ml);
        g.item_first = reinterpret_cast<int*>(ws + p.first);
        g.item_last = reinterpret_cast<int*>(ws + p.last);
        CUtensorMap map;
        const swift_status st = make_codes_map(kv, p.dp, unit_keys8(p), true, &map);
        if (st != SWIFT_OK) return st;
        e = kv->dtype == SWIFT_I8 ? launch_dec8_any<QT, int8_t>(p, map, bv, g, s, before) : launch_dec8_any<QT, __nv_fp8_e4m3>(p, map, bv, g, s, before);
    } else {
        t.mode = BT_OWN;
        t.part_slot = p.splits;
        const swift_status st = run_tc8(kv, x_dtype, bv, t, piece_bound(bv, av.n_kv_heads, 2 * t.rows_per_tile), multiprocessors(), s, before);
        if (st != SWIFT_OK) return st;
    }
    if (e == cudaSuccess) e = launch_join8<QT>(p, bv, j, s);
    if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
    return SWIFT_OK;
}

swift_status prompt8(const swift_coded_kv* c, const swift_row_batch* batch, const swift_attention_args* args, int x_dtype, int probe_us, cudaStream_t s)
{
    BatchView bv;
    AttnView av;
    const swift_status st = check_attention8(c, batch, args, x_dtype, &bv, &av);
    if (st != SWIFT_OK) return st;
    if (bv.n_rows == 0 || bv.n_seqs == 0) return SWIFT_OK;
    set_probe(&av, probe_us);
    if (!tensor_core_shape8(&c->kv, x_dtype, av.n_heads)) return run_rows8(&c->kv, x_dtype, bv, av, s);
    return run_prompt8(&c->kv, x_dtype, bv, av, args->block, s);
}

swift_status prefix8(const swift_coded_kv* c, const swift_row_batch* batch, const swift_attention_args* args, int x_dtype, int max_rows,
                     swift_devbuf workspace, int probe_us, cudaStream_t s)
{
    BatchView bv;
    AttnView av;
    swift_status st = check_attention8(c, batch, args, x_dtype, &bv, &av);
    if (st != SWIFT_OK) return st;
    if (max_rows < 1) return fail_batch(SWIFT_EINVAL, "max_rows %d", max_rows);
    if (bv.n_rows == 0 || bv.n_seqs == 0) return SWIFT_OK;
    Plan8 p;
    st = plan_prefix8(c, bv, av.n_heads, max_rows, x_dtype, &p);
    if (st != SWIFT_OK) return st;
    if (!workspace.dptr || !aligned(workspace.dptr, 256)) return fail_batch(SWIFT_EINVAL, "the workspace must be 256-byte aligned device memory");
    if (workspace.bytes < p.bytes) return fail_batch(SWIFT_ECAPACITY, "workspace of %zu bytes, %zu needed", workspace.bytes, p.bytes);
    av.max_rows = max_rows;
    set_probe(&av, probe_us);
    if (p.rows) return run_rows8(&c->kv, x_dtype, bv, av, s);
    if (p.prompt) return run_prompt8(&c->kv, x_dtype, bv, av, args->block, s);
    unsigned char* ws = reinterpret_cast<unsigned char*>(workspace.dptr);
    return x_dtype == SWIFT_BF16 ? run_prefix8<__nv_bfloat16>(c, x_dtype, bv, av, args->block, p, ws, s)
                                 : run_prefix8<__half>(c, x_dtype, bv, av, args->block, p, ws, s);
}

} // namespace

extern "C" {

swift_status swift_coded_append(const swift_coded_kv* c, const swift_row_batch* batch, const swift_append_args* x, void* cuda_stream)
{
    BatchView bv;
    swift_status st = check_cache8(c, batch, &bv);
    if (st != SWIFT_OK) return st;
    const swift_paged_kv* kv = &c->kv;
    if (!x) return fail_batch(SWIFT_EINVAL, "null arguments");
    if (x->block < 0 || x->block >= kv->n_blocks) return fail_batch(SWIFT_EINVAL, "block %d outside 0..%d", x->block, kv->n_blocks - 1);
    if (x->n_heads < 0 || x->n_heads > MAX_HEADS) return fail_batch(SWIFT_EINVAL, "n_heads %d", x->n_heads);
    if (!type_known(x->x_dtype)) return fail_batch(SWIFT_EUNSUPPORTED, "q, k, v must be fp32, bf16 or fp16");
    st = check_append(kv, x);
    if (st != SWIFT_OK) return st;
    if (bv.n_rows == 0 || bv.n_seqs == 0) return SWIFT_OK;
    Append8View v;
    bool vec[2];
    st = view_append(kv, x, x->x_dtype, &v.a, vec);
    if (st != SWIFT_OK) return st;
    v.scales = block_scales(c, x->block);
    v.scale_page = scale_page(c);
    cudaStream_t s = (cudaStream_t)cuda_stream;
    cudaError_t e;
    if (x->x_dtype == SWIFT_F32) e = launch_append8_any<float>(kv->dtype, bv, v, vec[0], vec[1], s);
    else if (x->x_dtype == SWIFT_BF16) e = launch_append8_any<__nv_bfloat16>(kv->dtype, bv, v, vec[0], vec[1], s);
    else e = launch_append8_any<__half>(kv->dtype, bv, v, vec[0], vec[1], s);
    if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "kernel launch failed: %s", cudaGetErrorString(e));
    return SWIFT_OK;
}

swift_status swift_coded_prompt_attention(const swift_coded_kv* c, const swift_row_batch* batch, const swift_attention_args* args, int32_t x_dtype, void* cuda_stream)
{
    return prompt8(c, batch, args, x_dtype, 0, (cudaStream_t)cuda_stream);
}

size_t swift_coded_prefix_workspace_bytes(const swift_coded_kv* c, const swift_row_batch* batch, int32_t n_heads, int32_t max_rows, int32_t x_dtype)
{
    BatchView bv;
    if (check_cache8(c, batch, &bv) != SWIFT_OK) return 0;
    if (n_heads < 1 || n_heads > MAX_HEADS || n_heads % c->kv.n_kv_heads || max_rows < 1 || !type_known(x_dtype)) {
        fail_batch(SWIFT_EINVAL, "n_heads %d, max_rows %d, type %d", n_heads, max_rows, x_dtype);
        return 0;
    }
    Plan8 p;
    return plan_prefix8(c, bv, n_heads, max_rows, x_dtype, &p) == SWIFT_OK ? p.bytes : 0;
}

swift_status swift_coded_prefix_attention(const swift_coded_kv* c, const swift_row_batch* batch, const swift_attention_args* args, int32_t x_dtype,
                                        int32_t max_rows, swift_devbuf workspace, void* cuda_stream)
{
    return prefix8(c, batch, args, x_dtype, max_rows, workspace, 0, (cudaStream_t)cuda_stream);
}

swift_status swift_probe_coded_wait_limit(const swift_coded_kv* c, const swift_row_batch* batch, const swift_attention_args* args, int32_t x_dtype,
                                        int32_t max_rows, swift_devbuf workspace, int32_t limit_us, void* cuda_stream)
{
    if (limit_us < 1 || limit_us > 100000) return fail_batch(SWIFT_EINVAL, "limit_us must be in 1..100000");
    if (max_rows < 0) return fail_batch(SWIFT_EINVAL, "max_rows %d", max_rows);
    if (c && args && c->kv.n_kv_heads > 0 && !tensor_core_shape8(&c->kv, x_dtype, args->n_heads))
        return fail_batch(SWIFT_EUNSUPPORTED, "fp32 arithmetic has no waits");
    if (max_rows == 0) return prompt8(c, batch, args, x_dtype, limit_us, (cudaStream_t)cuda_stream);
    return prefix8(c, batch, args, x_dtype, max_rows, workspace, limit_us, (cudaStream_t)cuda_stream);
}

} // extern "C"
