// What the host sides of the batch operators share: errors, launches, checks of a batch, tensor maps.  Included by one translation unit
// for the 16- and 32-bit caches and one for the 8-bit ones, each behind its own copy of the device code.
#pragma once
#include "../../include/swift.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>

// the calling thread's last failure, whichever unit it happened in (batch.cu)
extern thread_local char swift_batch_error_text[512];
// waits that ran out in the 8-bit caches' kernels on the current device (batch8.cu); ordered behind the stream's work
cudaError_t swift_batch8_waits(unsigned* count, cudaStream_t s);

namespace {

using namespace swk;

swift_status fail_batch(swift_status s, const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(swift_batch_error_text, sizeof swift_batch_error_text, fmt, ap);
    va_end(ap);
    return s;
}

constexpr int MAX_POSITIONS = 1 << 30;      // prefix_len and table_stride * page_size
constexpr int MAX_HEADS = 4096;

inline int ceil_div(long long a, long long b) { return (int)((a + b - 1) / b); }
inline bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }
inline int type_size(int dtype) { return dtype == SWIFT_F32 ? 4 : dtype == SWIFT_I8 || dtype == SWIFT_E4M3 ? 1 : 2; }
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

// eight: the cache is to be an 8-bit one, else it must not be
swift_status check_batch(const swift_paged_kv* kv, const swift_row_batch* b, BatchView* out, bool eight = false)
{
    if (!kv || !b) return fail_batch(SWIFT_EINVAL, "null cache or batch");
    if (!kv->pool || !aligned(kv->pool, 16)) return fail_batch(SWIFT_EINVAL, "the pool must be 16-byte aligned device memory");
    if (!(eight ? kv->dtype == SWIFT_I8 || kv->dtype == SWIFT_E4M3 : type_known(kv->dtype))) return fail_batch(SWIFT_EINVAL, "cache type %d unknown", kv->dtype);
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

inline long long kv_elems(const swift_paged_kv* kv) { return (long long)kv->n_kv_heads * kv->page_size * kv->head_dim; }
inline const char* block_base(const swift_paged_kv* kv, int block)
{
    return reinterpret_cast<const char*>(kv->pool) + (size_t)block * 2 * kv_elems(kv) * type_size(kv->dtype);
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

// Pieces of `rows` tokens of the modes that take each sequence by itself, at most.
long long piece_bound(const BatchView& bv, int n_kv_heads, int rows)
{
    if (bv.n_seqs == 1) return (long long)ceil_div(bv.n_rows, rows) * n_kv_heads;
    const long long some = bv.n_seqs < bv.n_rows ? bv.n_seqs : bv.n_rows;
    return (bv.n_rows / rows + some) * n_kv_heads;
}

template <typename T, typename TC, int RPW, int NV> cudaError_t launch_fp32_form(const BatchView& bv, const AttnView& av, cudaStream_t s)
{
    static std::atomic<unsigned long long> done{0};
    const cudaError_t e = allow_smem(attn_fp32_kernel<T, TC, RPW, NV>, af_smem_bytes(128 * NV, RPW), done);
    if (e != cudaSuccess) return e;
    const long long group = av.n_heads / av.n_kv_heads, some = bv.n_seqs < bv.n_rows ? bv.n_seqs : bv.n_rows;
    const long long pieces = (bv.n_rows * group / (4 * RPW) + some) * av.n_kv_heads;       // at most
    if (pieces > 0x7FFFFFFFll) return cudaErrorInvalidConfiguration;
    return launch(attn_fp32_kernel<T, TC, RPW, NV>, dim3((unsigned)pieces), 128, af_smem_bytes(av.head_dim, RPW), s, false, bv, av);
}
template <typename T, typename TC> cudaError_t launch_fp32(const BatchView& bv, const AttnView& av, cudaStream_t s)
{
    // 64 rows a block where sequences have the rows for it and the blocks still reach every SM, else 16 (fp32, 5003 ragged rows of 56
    // heads on 8: 3.9 ms with 64, 5.6 with 16; 160 rows of 32 heads: 52 and 42 us; 12 sequences x 63: 151 and 131).
    const long long packed = (long long)bv.n_rows * (av.n_heads / av.n_kv_heads);
    const bool many = packed > 32ll * bv.n_seqs && packed / 64 * av.n_kv_heads >= multiprocessors();
    if (av.head_dim > 128) return many ? launch_fp32_form<T, TC, 16, 2>(bv, av, s) : launch_fp32_form<T, TC, 4, 2>(bv, av, s);
    return many ? launch_fp32_form<T, TC, 16, 1>(bv, av, s) : launch_fp32_form<T, TC, 4, 1>(bv, av, s);
}

// An append's arguments that do not depend on whether there are rows.
swift_status check_append(const swift_paged_kv* kv, const swift_append_args* x)
{
    if (x->rope && (x->rotary_dim < 2 || x->rotary_dim > kv->head_dim || x->rotary_dim % 2 || x->rope_positions < 0 || !aligned(x->rope, 8)))
        return fail_batch(SWIFT_EINVAL, "rotary_dim %d is not even in 2..head_dim, or the table is not 8-byte aligned", x->rotary_dim);
    if ((x->q_gain || x->k_gain) && !(x->eps >= 0.f && std::isfinite(x->eps))) return fail_batch(SWIFT_EINVAL, "eps must be finite and not negative");
    return SWIFT_OK;
}

// The others; q_dtype: of q_out.  vec: 16-byte pieces fit q, and k and v.
swift_status view_append(const swift_paged_kv* kv, const swift_append_args* x, int q_dtype, AppendView* a, bool (&vec)[2])
{
    if (!x->k.ptr || !x->v.ptr || (x->n_heads > 0 && (!x->q.ptr || !x->q_out))) return fail_batch(SWIFT_EINVAL, "null q, k, v or q_out");
    const int es = type_size(x->x_dtype), rd = x->rope ? x->rotary_dim : 0;
    const swift_rows* in[3] = {&x->q, &x->k, &x->v};
    // with pairs (i, i + R/2) the second piece starts at R/2: 16-byte loads need R/2 in whole pieces of 8, which R % 16 gives
    vec[0] = vec[1] = kv->head_dim % 16 == 0 && rd % 16 == 0 && (!x->rope || aligned(x->rope, 16));
    vec[0] = vec[0] && aligned(x->q_out, 16) && aligned(x->q_gain, 16);
    vec[1] = vec[1] && aligned(x->k_gain, 16);
    for (int w = 0; w < 3; ++w) {
        const bool used = w > 0 || x->n_heads > 0;
        a->x[w] = in[w]->ptr;
        a->row_stride[w] = in[w]->row_stride;
        a->head_stride[w] = in[w]->head_stride;
        if (used && !aligned(in[w]->ptr, es)) return fail_batch(SWIFT_EINVAL, "q, k, v must be aligned to their element size");
        if (used && (in[w]->row_stride < 0 || in[w]->head_stride < 0)) return fail_batch(SWIFT_EINVAL, "negative strides");
        bool& fits = vec[w > 0];
        fits = fits && (!used || (aligned(in[w]->ptr, 16) && in[w]->row_stride * es % 16 == 0 && in[w]->head_stride * es % 16 == 0));
    }
    if (x->n_heads > 0 && !aligned(x->q_out, type_size(q_dtype))) return fail_batch(SWIFT_EINVAL, "q_out must be aligned to its element size");
    a->n_heads = x->n_heads;
    a->n_kv_heads = kv->n_kv_heads;
    a->head_dim = kv->head_dim;
    a->rotary_dim = rd;
    a->interleaved = x->interleaved != 0;
    a->rope_positions = x->rope_positions;
    a->gain[0] = x->q_gain;
    a->gain[1] = x->k_gain;
    if ((x->q_gain && !aligned(x->q_gain, 4)) || (x->k_gain && !aligned(x->k_gain, 4))) return fail_batch(SWIFT_EINVAL, "gains must be 4-byte aligned");
    a->eps = x->eps;
    a->rope = reinterpret_cast<const float2*>(x->rope);
    a->positions = x->positions;
    a->q_out = x->q_out;
    a->pool = const_cast<char*>(block_base(kv, x->block));
    a->page_elems = 2 * kv_elems(kv) * kv->n_blocks;
    a->kv_elems = kv_elems(kv);
    return SWIFT_OK;
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


// limit_us > 0: the probe of swift_probe_batch_wait_limit.
void set_probe(AttnView* av, int limit_us)
{
    if (limit_us <= 0) return;
    av->wait_kcycles = 2 * limit_us;                      // about 2 cycles per nanosecond
    av->withhold = 1;
}

} // namespace
