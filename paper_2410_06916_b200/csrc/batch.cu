// Batches of sequences over one paged K,V cache: argument checks, launch shapes and entry points of swift_rope_table,
// swift_kv_append, swift_prompt_attention and swift_prefix_attention.  No context and no state between calls.
#include "../../include/swift.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>

// This translation unit gets its own copies of the shared device code (separate namespace).
#define swk swk_batch
#include "kernels_batch_dec.cuh"

using namespace swk;

namespace {

thread_local char g_batch_error[512] = "";

swift_status fail_batch(swift_status s, const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_batch_error, sizeof g_batch_error, fmt, ap);
    va_end(ap);
    return s;
}

constexpr int MAX_POSITIONS = 1 << 30;      // prefix_len and table_stride * page_size
constexpr int MAX_HEADS = 4096;

inline int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
inline bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }
inline int type_size(int dtype) { return dtype == SWIFT_F32 ? 4 : 2; }
inline bool type_known(int dtype) { return dtype == SWIFT_F32 || dtype == SWIFT_BF16 || dtype == SWIFT_F16; }

template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kernel)(KArgs...), dim3 grid, int block, size_t smem, cudaStream_t stream, bool after_previous, Args&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = after_previous ? 1 : 0;   // only between the kernels of one call
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

swift_status check_batch(const swift_paged_kv* kv, const swift_row_batch* b, BatchView* out)
{
    if (!kv || !b) return fail_batch(SWIFT_EINVAL, "null cache or batch");
    if (!kv->pool || !aligned(kv->pool, 16)) return fail_batch(SWIFT_EINVAL, "the pool must be 16-byte aligned device memory");
    if (!type_known(kv->dtype)) return fail_batch(SWIFT_EINVAL, "cache type %d unknown", kv->dtype);
    if (kv->n_pages < 1 || kv->n_blocks < 1 || kv->n_kv_heads < 1 || kv->n_kv_heads > MAX_HEADS)
        return fail_batch(SWIFT_EINVAL, "cache of %d pages, %d blocks, %d heads", kv->n_pages, kv->n_blocks, kv->n_kv_heads);
    if (kv->page_size < 8 || kv->page_size > 128 || (kv->page_size & (kv->page_size - 1)))
        return fail_batch(SWIFT_EINVAL, "page_size %d is not a power of two in 8..128", kv->page_size);
    if (kv->head_dim < 2 || kv->head_dim > 256 || kv->head_dim % 2) return fail_batch(SWIFT_EINVAL, "head_dim %d is not even in 2..256", kv->head_dim);
    if ((long long)kv->n_blocks * 2 * kv->n_kv_heads > (1 << 24)) return fail_batch(SWIFT_EINVAL, "too many heads in a page");
    if (b->n_seqs < 0 || b->n_rows < 0) return fail_batch(SWIFT_EINVAL, "n_seqs %d, n_rows %d", b->n_seqs, b->n_rows);
    if (b->n_seqs > SWIFT_MAX_SEQS) return fail_batch(SWIFT_ECAPACITY, "n_seqs %d above %d", b->n_seqs, (int)SWIFT_MAX_SEQS);
    if (b->n_seqs > 0 && (!b->row_start || !b->kv_len || !b->page_table)) return fail_batch(SWIFT_EINVAL, "null row_start, kv_len or page_table");
    if (b->table_stride < 1 || (long long)b->table_stride * kv->page_size > MAX_POSITIONS)
        return fail_batch(SWIFT_EINVAL, "table_stride %d outside 1..%d", b->table_stride, MAX_POSITIONS / kv->page_size);
    if (b->prefix_len < 0 || b->prefix_len > MAX_POSITIONS) return fail_batch(SWIFT_EINVAL, "prefix_len %d", b->prefix_len);
    if (b->prefix_len > 0 && !b->prefix_pages) return fail_batch(SWIFT_EINVAL, "null prefix_pages with prefix_len %d", b->prefix_len);
    out->n_seqs = b->n_seqs;
    out->n_rows = b->n_rows;
    out->table_stride = b->table_stride;
    out->prefix_len = b->prefix_len;
    out->page_size = kv->page_size;
    out->page_shift = __builtin_ctz(kv->page_size);
    out->n_pages = kv->n_pages;
    out->max_len = b->table_stride * kv->page_size;
    out->row_start = b->row_start;
    out->kv_len = b->kv_len;
    out->page_table = b->page_table;
    out->prefix_pages = b->prefix_pages;
    return SWIFT_OK;
}

// what the tensor-core kernels take; the rest is computed in fp32 arithmetic
inline bool tensor_core_shape(const swift_paged_kv* kv) { return kv->dtype != SWIFT_F32 && kv->head_dim % 8 == 0 && kv->head_dim <= 128; }
inline long long kv_elems(const swift_paged_kv* kv) { return (long long)kv->n_kv_heads * kv->page_size * kv->head_dim; }
inline const char* block_base(const swift_paged_kv* kv, int block)
{
    return reinterpret_cast<const char*>(kv->pool) + (size_t)block * 2 * kv_elems(kv) * type_size(kv->dtype);
}

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

// ------------------------------------------------------------------------------ tensor-core attention
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encoder()
{
    static const EncodeTiled fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) f = nullptr;
        return reinterpret_cast<EncodeTiled>(f);
    }();
    return fn;
}

// 16-bit tensor of `rank` dims, contiguous in the first; boxes start with 64 of them (128 bytes, one swizzle row).
swift_status make_map(CUtensorMap* out, int dtype, const void* base, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box)
{
    const EncodeTiled encode = encoder();
    if (!encode) return fail_batch(SWIFT_ECUDA, "cuTensorMapEncodeTiled not available from the driver");
    const cuuint32_t one[5] = {1, 1, 1, 1, 1};
    const CUresult r = encode(out, dtype == SWIFT_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, const_cast<void*>(base),
                              dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail_batch(SWIFT_EINVAL, "cuTensorMapEncodeTiled refused the tensor (code %d): strides of q beyond 2^40 bytes, or a cache of odd size", (int)r);
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

int multiprocessors()
{
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
    return n;
}

// A kernel's shared-memory size is set once per device.
template <typename K> cudaError_t allow_smem(K kernel, int bytes, std::atomic<unsigned long long>& done)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < 64 && (done.load() >> dev & 1))) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev);
    return e;
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

// Pieces of `rows` tokens of the modes that take each sequence by itself, at most.
long long piece_bound(const BatchView& bv, int n_kv_heads, int rows)
{
    if (bv.n_seqs == 1) return (long long)ceil_div(bv.n_rows, rows) * n_kv_heads;
    const long long some = bv.n_seqs < bv.n_rows ? bv.n_seqs : bv.n_rows;
    return (bv.n_rows / rows + some) * n_kv_heads;
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

template <typename T, int RPW, int NV> cudaError_t launch_fp32_form(const BatchView& bv, const AttnView& av, cudaStream_t s)
{
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = allow_smem(attn_fp32_kernel<T, RPW, NV>, af_smem_bytes(128 * NV, RPW), done);
    if (e != cudaSuccess) return e;
    const long long group = av.n_heads / av.n_kv_heads, some = bv.n_seqs < bv.n_rows ? bv.n_seqs : bv.n_rows;
    const long long pieces = (bv.n_rows * group / (4 * RPW) + some) * av.n_kv_heads;       // at most
    if (pieces > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    return launch(attn_fp32_kernel<T, RPW, NV>, dim3((unsigned)pieces), 128, af_smem_bytes(av.head_dim, RPW), s, false, bv, av);
}
template <typename T> cudaError_t launch_fp32(const BatchView& bv, const AttnView& av, cudaStream_t s)
{
    // 64 rows a block where sequences have the rows for it and the blocks still reach every SM, else 16 (fp32, 5003 ragged rows of 56
    // heads on 8: 3.9 ms with 64, 5.6 with 16; 160 rows of 32 heads: 52 and 42 us; 12 sequences x 63: 151 and 131).
    const long long packed = (long long)bv.n_rows * (av.n_heads / av.n_kv_heads);
    const bool many = packed > 32ll * bv.n_seqs && packed / 64 * av.n_kv_heads >= multiprocessors();
    if (av.head_dim > 128) return many ? launch_fp32_form<T, 16, 2>(bv, av, s) : launch_fp32_form<T, 4, 2>(bv, av, s);
    return many ? launch_fp32_form<T, 16, 1>(bv, av, s) : launch_fp32_form<T, 4, 1>(bv, av, s);
}
cudaError_t launch_rows(const swift_paged_kv* kv, const BatchView& bv, const AttnView& av, cudaStream_t s)
{
    switch (kv->dtype) {
    case SWIFT_F32: return launch_fp32<float>(bv, av, s);
    case SWIFT_BF16: return launch_fp32<__nv_bfloat16>(bv, av, s);
    default: return launch_fp32<__half>(bv, av, s);
    }
}

template <typename TX, typename TC>
cudaError_t launch_append(const BatchView& b, const AppendView& a, bool vec, cudaStream_t s)
{
    const int units = a.n_heads + 2 * a.n_kv_heads;
    // 16-byte pieces where sizes and alignment allow them (8192 rows of 80 heads: 70 us; element by element 248)
    if (!vec) return launch(append_any_kernel<TX, TC>, dim3(b.n_rows, ceil_div(units, AP_THREADS / 32)), AP_THREADS, 0, s, false, b, a);
    const int pieces = a.head_dim / 16;
    const int lph = pieces <= 1 ? 1 : pieces <= 2 ? 2 : pieces <= 4 ? 4 : pieces <= 8 ? 8 : 16;
    // A row's heads go to one warp where the rows alone make two waves of warps (20 per SM), else to as many warps as that takes, at
    // most one per batch of loads (8192 rows of 80 heads: 70 us with one warp per row, 84 with two blocks per row).
    const int batch = 32 / lph * AP_UNROLL<TX>, most = ceil_div(units, batch), wanted = ceil_div(148 * 40, b.n_rows);
    const int chunks = wanted < most ? wanted : most, per_warp = ceil_div(ceil_div(units, chunks), 32 / lph) * (32 / lph);
    const dim3 grid((unsigned)(((long long)b.n_rows * chunks + AP_THREADS / 32 - 1) / (AP_THREADS / 32)));
    switch (lph) {
    case 1: return launch(append_vec_kernel<TX, TC, 1>, grid, AP_THREADS, 0, s, false, b, a, per_warp, chunks);
    case 2: return launch(append_vec_kernel<TX, TC, 2>, grid, AP_THREADS, 0, s, false, b, a, per_warp, chunks);
    case 4: return launch(append_vec_kernel<TX, TC, 4>, grid, AP_THREADS, 0, s, false, b, a, per_warp, chunks);
    case 8: return launch(append_vec_kernel<TX, TC, 8>, grid, AP_THREADS, 0, s, false, b, a, per_warp, chunks);
    default: return launch(append_vec_kernel<TX, TC, 16>, grid, AP_THREADS, 0, s, false, b, a, per_warp, chunks);
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

// limit_us > 0: the probe of swift_probe_batch_wait_limit.
void set_probe(AttnView* av, int limit_us)
{
    if (limit_us <= 0) return;
    av->wait_kcycles = 2 * limit_us;                      // about 2 cycles per nanosecond
    av->withhold = 1;
}

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

const char* swift_batch_error(void) { return g_batch_error; }

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
    if (x->rope && (x->rotary_dim < 2 || x->rotary_dim > kv->head_dim || x->rotary_dim % 2 || x->rope_positions < 0 || !aligned(x->rope, 8)))
        return fail_batch(SWIFT_EINVAL, "rotary_dim %d is not even in 2..head_dim, or the table is not 8-byte aligned", x->rotary_dim);
    if ((x->q_gain || x->k_gain) && !(x->eps >= 0.f && std::isfinite(x->eps))) return fail_batch(SWIFT_EINVAL, "eps must be finite and not negative");
    if (bv.n_rows == 0 || bv.n_seqs == 0) return SWIFT_OK;
    if (!x->k.ptr || !x->v.ptr || (x->n_heads > 0 && (!x->q.ptr || !x->q_out))) return fail_batch(SWIFT_EINVAL, "null q, k, v or q_out");
    AppendView a;
    const int es = type_size(x->x_dtype), rd = x->rope ? x->rotary_dim : 0;
    const swift_rows* in[3] = {&x->q, &x->k, &x->v};
    bool vec = kv->head_dim % 16 == 0 && rd % 16 == 0 && (!x->rope || aligned(x->rope, 16)) && aligned(x->q_out, 16);
    // with pairs (i, i + R/2) the second piece starts at R/2: 16-byte loads need R/2 in whole pieces of 8, which R % 16 gives
    for (int w = 0; w < 3; ++w) {
        const bool used = w > 0 || x->n_heads > 0;
        a.x[w] = in[w]->ptr;
        a.row_stride[w] = in[w]->row_stride;
        a.head_stride[w] = in[w]->head_stride;
        if (used && !aligned(in[w]->ptr, es)) return fail_batch(SWIFT_EINVAL, "q, k, v must be aligned to their element size");
        if (used && (in[w]->row_stride < 0 || in[w]->head_stride < 0)) return fail_batch(SWIFT_EINVAL, "negative strides");
        vec = vec && (!used || (aligned(in[w]->ptr, 16) && in[w]->row_stride * es % 16 == 0 && in[w]->head_stride * es % 16 == 0));
    }
    if (x->n_heads > 0 && !aligned(x->q_out, type_size(kv->dtype))) return fail_batch(SWIFT_EINVAL, "q_out must be aligned to its element size");
    a.n_heads = x->n_heads;
    a.n_kv_heads = kv->n_kv_heads;
    a.head_dim = kv->head_dim;
    a.rotary_dim = rd;
    a.interleaved = x->interleaved != 0;
    a.rope_positions = x->rope_positions;
    a.gain[0] = x->q_gain;
    a.gain[1] = x->k_gain;
    if ((x->q_gain && !aligned(x->q_gain, 4)) || (x->k_gain && !aligned(x->k_gain, 4))) return fail_batch(SWIFT_EINVAL, "gains must be 4-byte aligned");
    vec = vec && aligned(x->q_gain, 16) && aligned(x->k_gain, 16);
    a.eps = x->eps;
    a.rope = reinterpret_cast<const float2*>(x->rope);
    a.positions = x->positions;
    a.q_out = x->q_out;
    a.pool = const_cast<char*>(block_base(kv, x->block));
    a.page_elems = 2 * kv_elems(kv) * kv->n_blocks;
    a.kv_elems = kv_elems(kv);
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
    cudaStream_t s = (cudaStream_t)cuda_stream;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaStreamGetId(s, &id);
    if (e == cudaSuccess) e = cudaMemcpyFromSymbolAsync(&count, batch_waits_over, sizeof count, 0, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) return fail_batch(SWIFT_ECUDA, "the stream's work failed: %s", cudaGetErrorString(e));
    if (g_reports.changed(dev, id, count)) return fail_batch(SWIFT_ETIMEOUT, "a device-side wait of an attention call ran out of time");
    return SWIFT_OK;
}

} // extern "C"
