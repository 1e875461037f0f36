// Batches of sequences over one paged cache: the shared row and page arithmetic, the rotary table, the pass between a
// layer's projection and its attention (norm + rotation + append), and attention in fp32 arithmetic for the types and head
// sizes the tensor-core kernels next door do not take.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace swk {

constexpr unsigned FULL_WARP = 0xFFFFFFFFu;

// ------------------------------------------------------------------------------ the batch as kernels see it
struct BatchView {
    int n_seqs, n_rows, table_stride, prefix_len;
    int page_size, page_shift, n_pages, max_len;          // max_len = table_stride * page_size
    const int* row_start;
    const int* kv_len;
    const int* page_table;
    const int* prefix_pages;
};
struct SeqSpan { int r0, n, len, pos0; };                 // first row, rows, cached positions that can be read (own), own position of row r0

__device__ __forceinline__ SeqSpan make_span(const BatchView& b, int start, int end, int len)
{
    SeqSpan s;
    s.r0 = min(max(start, 0), b.n_rows);
    s.n = min(max(end, s.r0), b.n_rows) - s.r0;
    s.len = min(max(len, 0), b.max_len);
    // From the lengths as given: a sequence longer than its table keeps its rows' positions, and those behind the table are left
    // out.  Positions behind max_len or far below 0 are alike, so the 64-bit difference may be clamped to an int.
    const long long pos0 = (long long)len - end + s.r0;
    s.pos0 = (int)max(-0x80000000ll, min(pos0, (long long)b.max_len));
    return s;
}
__device__ __forceinline__ SeqSpan seq_span(const BatchView& b, int i)
{
    return make_span(b, b.row_start[i], b.row_start[i + 1], b.kv_len[i]);
}

// lane `at`'s span, for the whole warp
__device__ __forceinline__ SeqSpan span_of(const SeqSpan& s, int at)
{
    return {__shfl_sync(FULL_WARP, s.r0, at), __shfl_sync(FULL_WARP, s.n, at), __shfl_sync(FULL_WARP, s.len, at), __shfl_sync(FULL_WARP, s.pos0, at)};
}
// how many of its sequence's cached positions row t sees
__device__ __forceinline__ int seen_own(const SeqSpan& s, int t) { return min(max(s.pos0 + t + 1, 0), s.len); }

// The sequence that holds row `row`, found by a whole warp: 32 row starts per step are compared at once, so a batch of up
// to 32 sequences costs one trip to memory (the spans' three numbers come with it) and one of 1024 two.  Returns -1 for
// padding rows.  All lanes get the result.
__device__ __forceinline__ int find_seq(const BatchView& b, int row, SeqSpan& span)
{
    const int lane = threadIdx.x & 31;
    int base = 0, n = b.n_seqs;                           // the last i in [base, base + n) with row_start[i] <= row
    while (n > 32) {
        const int step = (n + 31) >> 5;
        const int i = base + lane * step;
        const bool le = lane * step < n && b.row_start[i] <= row;
        const unsigned m = __ballot_sync(FULL_WARP, le);
        if (m == 0) return -1;
        const int at = 31 - __clz(m);
        n = min(step, n - at * step);
        base += at * step;
    }
    int start = 0, end = 0, len = 0;
    if (lane < n) {
        start = b.row_start[base + lane];
        end = b.row_start[base + lane + 1];
        len = b.kv_len[base + lane];
    }
    const unsigned m = __ballot_sync(FULL_WARP, lane < n && start <= row);
    if (m == 0) return -1;
    const int at = 31 - __clz(m);
    span = make_span(b, __shfl_sync(FULL_WARP, start, at), __shfl_sync(FULL_WARP, end, at), __shfl_sync(FULL_WARP, len, at));
    if (row < span.r0 || row >= span.r0 + span.n) return -1;
    return base + at;
}

__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(int8_t v) { return (float)v; }
__device__ __forceinline__ float to_float(__nv_fp8_e4m3 v) { return (float)v; }
__device__ __forceinline__ void store_val(__half* p, float v) { *p = __float2half_rn(v); }

__device__ __forceinline__ void load8(const float* p, float (&x)[8])      // from 16-byte loads
{
    const float4 a = reinterpret_cast<const float4*>(p)[0], c = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = c.x; x[5] = c.y; x[6] = c.z; x[7] = c.w;
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16)      // a in the low half
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[8])
{
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(x[0], x[1], T()), pack2(x[2], x[3], T()), pack2(x[4], x[5], T()), pack2(x[6], x[7], T()));
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8])
{
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// eight values as they lie in memory, to be widened when they are used
template <typename T> struct Raw8 { uint4 v; };
template <> struct Raw8<float> { float4 a, b; };
template <typename T> __device__ __forceinline__ void fetch8(const T* p, Raw8<T>& r) { r.v = __ldcs(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ void fetch8(const float* p, Raw8<float>& r)
{
    r.a = __ldcs(reinterpret_cast<const float4*>(p));
    r.b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
}
__device__ __forceinline__ void widen8(const Raw8<float>& r, float (&x)[8])
{
    x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w; x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}
__device__ __forceinline__ void widen8(const Raw8<__nv_bfloat16>& r, float (&x)[8])
{
    const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void widen8(const Raw8<__half>& r, float (&x)[8])
{
    const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

// ------------------------------------------------------------------------------ rotary table
constexpr int RT_RUN = 16;          // positions one thread writes

struct RopeTableArgs {
    float2* table;
    int n_positions, half;
    double log_theta_step;          // ln(theta) * 2 / rotary_dim
    double inv_factor, turns_per_freq, low, inv_range, magnitude;   // turns_per_freq = original_positions / (2 pi); 0: no parts
};

// table[p][i] = magnitude * (cos, sin)(p f_i).  A thread takes one pair i and RT_RUN positions: two 64-bit sincos, then a
// 64-bit rotation per position (its error grows by about 2^-53 a step, far below the fp32 result's half step).  Bound by
// the table's writes, which neighbouring threads make to neighbouring pairs.  block = 128, grid = ceil(half * runs / 128).
__global__ void __launch_bounds__(128) rope_run_kernel(RopeTableArgs a)
{
    const int runs = (a.n_positions + RT_RUN - 1) / RT_RUN;
    const long long idx = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (idx >= (long long)runs * a.half) return;
    const int run = (int)(idx / a.half), i = (int)(idx - (long long)run * a.half);
    double f = exp(-a.log_theta_step * (double)i);
    double keep = 0.0;
    if (a.turns_per_freq > 0.0) keep = fmin(1.0, fmax(0.0, (a.turns_per_freq * f - a.low) * a.inv_range));
    f = keep * f + (1.0 - keep) * f * a.inv_factor;
    const int p0 = run * RT_RUN, p1 = min(p0 + RT_RUN, a.n_positions);
    double s, c, ds, dc;
    sincos((double)p0 * f, &s, &c);
    sincos(f, &ds, &dc);
    s *= a.magnitude;
    c *= a.magnitude;
    float2* out = a.table + (size_t)p0 * a.half + i;
    for (int p = p0; p < p1; ++p, out += a.half) {
        *out = make_float2((float)c, (float)s);
        const double c1 = c * dc - s * ds;
        s = s * dc + c * ds;
        c = c1;
    }
}

// ------------------------------------------------------------------------------ norm + rotation + append
struct AppendView {
    const void* x[3];                                     // q, k, v
    long long row_stride[3], head_stride[3];
    int n_heads, n_kv_heads, head_dim, rotary_dim, interleaved, rope_positions;
    const float* gain[2];
    float eps;
    const float2* rope;
    const int* positions;
    void* q_out;
    void* pool;                                           // of this block: + block's offset within a page
    long long page_elems, kv_elems;                       // elements per page (all blocks), per K or V of a block
};

// One pair turned.  The contraction is spelt out so that both forms of the kernel give the same bits.
__device__ __forceinline__ void turn_pair(float x, float y, float2 cs, float& a, float& b)   // x, y by value: a, b may be they
{
    a = fmaf(x, cs.x, -__fmul_rn(y, cs.y));
    b = fmaf(y, cs.x, __fmul_rn(x, cs.y));
}

// What a row needs to know besides its data: where it goes and which table row turns it.  `slot` < 0: the row is left out.
struct RowPlace { long long kv_off; int slot, rope_row; };

__device__ __forceinline__ bool place_row(const BatchView& b, const AppendView& a, int row, RowPlace& p)
{
    SeqSpan sp;
    const int given = a.positions ? a.positions[row] : 0;
    const int seq = find_seq(b, row, sp);
    if (seq < 0) return false;
    const int own = sp.pos0 + (row - sp.r0);
    if (own < 0 || own >= b.max_len) return false;        // before the first position, or behind the page table
    const int page = b.page_table[(size_t)seq * b.table_stride + (own >> b.page_shift)];
    p.rope_row = a.positions ? given : b.prefix_len + own;
    if ((unsigned)page >= (unsigned)b.n_pages) return false;
    if (a.rope && (unsigned)p.rope_row >= (unsigned)a.rope_positions) return false;
    p.slot = own & (b.page_size - 1);
    p.kv_off = (long long)page * a.page_elems;
    return true;
}

// Vector form.  A group of LPH lanes (a power of two >= head_dim / 16) takes one head; a lane holds two pieces of 8 dims
// that a rotation pairs up: with pairs (i, i + R/2), piece c and the piece R/2 further on; with neighbouring pairs, or
// behind the rotated part, two pieces side by side.  So no value crosses lanes except the norm's sum.  A warp stays within
// one row: it locates the row once (three dependent trips to memory), keeps the row's 8 (cos, sin) pairs in registers (the
// gains come from L1 for every head: kept in registers too, 8192 rows of 80 heads took 78 us instead of 71), and goes
// through `per_warp` of its heads, two or four loads ahead, kept in the 16 bytes they have in memory until used.  Many rows:
// a whole row per warp, bound by HBM; few rows: as few heads per warp as one batch of loads holds, bound by the trips.  grid = ceil(rows x chunks / 4), block = 128.
constexpr int AP_THREADS = 128;
template <typename TX> constexpr int AP_UNROLL = sizeof(TX) == 2 ? 4 : 2;      // 32 registers of loads in flight

template <typename TX, typename TC, int LPH>
__device__ __forceinline__ void append_vec_rows(const BatchView& b, const AppendView& a, int per_warp, int chunks, unsigned block)
{
    constexpr int GROUPS = 32 / LPH, UNROLL = AP_UNROLL<TX>;
    const int lane = threadIdx.x & 31, c = lane & (LPH - 1), grp = lane / LPH;
    const long long job = (long long)block * (AP_THREADS / 32) + (threadIdx.x >> 5);
    const int row = (int)(job / chunks);
    if (row >= b.n_rows) return;
    const int D = a.head_dim, half = a.rotary_dim >> 1, pieces = D >> 4;
    const int u0 = (int)(job - (long long)row * chunks) * per_warp, units = min(u0 + per_warp, a.n_heads + 2 * a.n_kv_heads);
    const bool lane_live = c < pieces;
    int oa, ob;                                           // the two pieces' first dims
    bool turned;
    if (a.interleaved) {
        oa = 16 * c;
        ob = oa + 8;
        turned = oa < a.rotary_dim;                       // rotary_dim is a multiple of 16 here
    } else {
        const int rc = half >> 3;
        turned = c < rc;
        oa = turned ? 8 * c : a.rotary_dim + 16 * (c - rc);
        ob = turned ? oa + half : oa + 8;
    }
    auto which = [&](int u, int& h) {                     // 0 q, 1 k, 2 v; its head
        const int w = u < a.n_heads ? 0 : u < a.n_heads + a.n_kv_heads ? 1 : 2;
        h = w == 0 ? u : w == 1 ? u - a.n_heads : u - a.n_heads - a.n_kv_heads;
        return w;
    };
    Raw8<TX> ra[UNROLL], rb[UNROLL];
    auto fetch = [&](int first) {                         // heads first + grp, + GROUPS, ...
#pragma unroll
        for (int j = 0; j < UNROLL; ++j) {
            const int u = first + grp + j * GROUPS;
            ra[j] = {};
            rb[j] = {};
            if (lane_live && u < units) {
                int h;
                const int w = which(u, h);
                const TX* src = reinterpret_cast<const TX*>(a.x[w]) + row * a.row_stride[w] + h * a.head_stride[w];
                fetch8(src + oa, ra[j]);
                fetch8(src + ob, rb[j]);
            }
        }
    };
    fetch(u0);
    RowPlace place;
    if (!place_row(b, a, row, place)) return;             // the same for the whole warp
    float2 cs[8];
    turned = turned && a.rope != nullptr && lane_live;
    if (turned) {
        const float4* t = reinterpret_cast<const float4*>(a.rope + (size_t)place.rope_row * half + (a.interleaved ? oa >> 1 : oa));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float4 v = t[e];
            cs[2 * e] = make_float2(v.x, v.y);
            cs[2 * e + 1] = make_float2(v.z, v.w);
        }
    }
    const bool normed = a.gain[0] != nullptr || a.gain[1] != nullptr;
    for (int first = u0; first < units; first += UNROLL * GROUPS) {
#pragma unroll
        for (int j = 0; j < UNROLL; ++j) {
            if (first + j * GROUPS >= units) break;       // the same for the whole warp
            const int u = first + grp + j * GROUPS;
            int h;
            const int w = which(u, h);
            float xa[8], xb[8];
            widen8(ra[j], xa);
            widen8(rb[j], xb);
            if (normed) {
                float ss = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) ss += xa[e] * xa[e] + xb[e] * xb[e];
#pragma unroll
                for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(FULL_WARP, ss, o);
                const float* gain = w < 2 ? a.gain[w] : nullptr;
                if (gain != nullptr && lane_live) {
                    const float r = rsqrtf(ss / (float)D + a.eps);
                    float ga[8], gb[8];
                    load8(gain + oa, ga);
                    load8(gain + ob, gb);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        xa[e] *= r * ga[e];
                        xb[e] *= r * gb[e];
                    }
                }
            }
            if (!lane_live || u >= units) continue;
            if (turned && w < 2) {
                if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        turn_pair(xa[2 * e], xa[2 * e + 1], cs[e], xa[2 * e], xa[2 * e + 1]);
                        turn_pair(xb[2 * e], xb[2 * e + 1], cs[4 + e], xb[2 * e], xb[2 * e + 1]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) turn_pair(xa[e], xb[e], cs[e], xa[e], xb[e]);
                }
            }
            TC* dst = w == 0 ? reinterpret_cast<TC*>(a.q_out) + ((size_t)row * a.n_heads + h) * D
                             : reinterpret_cast<TC*>(a.pool) + place.kv_off + (w == 2 ? a.kv_elems : 0) + ((size_t)h * b.page_size + place.slot) * D;
            store8(dst + oa, xa);
            store8(dst + ob, xb);
        }
        if (first + UNROLL * GROUPS < units) fetch(first + UNROLL * GROUPS);
    }
}

template <typename TX, typename TC, int LPH>
__global__ void __launch_bounds__(AP_THREADS, 5) append_vec_kernel(BatchView b, AppendView a, int per_warp, int chunks)
{
    append_vec_rows<TX, TC, LPH>(b, a, per_warp, chunks, blockIdx.x);
}

// Scalar form: any even head_dim and rotary_dim, any alignment.  One warp per head of a row, lanes over pairs.
// grid = (rows, ceil(heads / 4)), block = 128.
template <typename TX, typename TC>
__global__ void __launch_bounds__(AP_THREADS) append_any_kernel(BatchView b, AppendView a)
{
    const int row = blockIdx.x, lane = threadIdx.x & 31, u = blockIdx.y * (AP_THREADS / 32) + (threadIdx.x >> 5);
    if (u >= a.n_heads + 2 * a.n_kv_heads) return;
    RowPlace place;
    if (!place_row(b, a, row, place)) return;
    const int w = u < a.n_heads ? 0 : u < a.n_heads + a.n_kv_heads ? 1 : 2;
    const int h = w == 0 ? u : w == 1 ? u - a.n_heads : u - a.n_heads - a.n_kv_heads, D = a.head_dim;
    const TX* src = reinterpret_cast<const TX*>(a.x[w]) + row * a.row_stride[w] + h * a.head_stride[w];
    TC* dst = w == 0 ? reinterpret_cast<TC*>(a.q_out) + ((size_t)row * a.n_heads + h) * D
                     : reinterpret_cast<TC*>(a.pool) + place.kv_off + (w == 2 ? a.kv_elems : 0) + ((size_t)h * b.page_size + place.slot) * D;
    const float* gain = w < 2 ? a.gain[w] : nullptr;
    float r = 1.f;
    if (gain) {
        float ss = 0.f;
        for (int i = lane; i < D; i += 32) { const float v = to_float(src[i]); ss += v * v; }
        r = rsqrtf(warp_sum(ss) / (float)D + a.eps);
    }
    const int R = (w < 2 && a.rope) ? a.rotary_dim : 0, half = a.rotary_dim >> 1;
    for (int i = lane; i < (R >> 1); i += 32) {
        const int ia = a.interleaved ? 2 * i : i, ib = a.interleaved ? 2 * i + 1 : i + half;
        float x = to_float(src[ia]), y = to_float(src[ib]);
        if (gain) { x *= r * gain[ia]; y *= r * gain[ib]; }
        const float2 cs = a.rope[(size_t)place.rope_row * half + i];
        turn_pair(x, y, cs, x, y);
        store_val(dst + ia, x);
        store_val(dst + ib, y);
    }
    for (int i = R + lane; i < D; i += 32) {
        float x = to_float(src[i]);
        if (gain) x *= r * gain[i];
        store_val(dst + i, x);
    }
}

// ------------------------------------------------------------------------------ attention in fp32 arithmetic
struct AttnView {
    const void* q;
    long long q_row_stride, q_head_stride;
    const void* pool;                                     // of this block
    long long page_elems, kv_elems;
    void* out;
    int n_heads, n_kv_heads, head_dim, max_rows;
    float scale;
    int wait_kcycles, withhold;                           // limit of the tensor-core kernels' waits in 1024 cycles; withhold: a copy is never asked for
    const float* scales;                                  // 8-bit caches: this block's [K, V][kv head] of page 0
    long long scale_page;                                 // and how far on the next page's are
};

// Any type and head size: fp32 caches, whose products the matrix instructions would round, and the sizes the tensor-core
// kernels do not take.  A block of four warps takes 4 RPW query rows of a kv head (tokens x heads of the group, so that a group
// shares its keys) and goes through the keys 32 at a time, widened to fp32 in shared memory.  Eight lanes share a row's scores
// and its running maximum and sum (RPW / 4 rows x 4 keys a lane); for the weighted sum of V a lane holds four dims (NV times) of
// all its warp's rows.  With RPW 16 both products make 8 multiply-adds per 16-byte load from shared memory, so the multiply-add
// rate bounds them (5003 ragged rows of 56 heads on 8, fp32: 3.9 ms, 25 TFLOP/s of the 96 GFLOP that count; keys staged one float
// at a time and 16 rows a block 10.9); RPW 4 is for batches too small to fill the SMs with that.  grid = pieces, block = 128.
constexpr int AF_KEYS = 32;
__host__ __device__ inline int af_stride(int head_dim) { return (head_dim + 3) / 4 * 4 + 4; }   // floats per staged row: 16-byte loads of eight rows fall into different banks
__host__ __device__ constexpr int af_p_stride(int rpw) { return rpw == 4 ? 4 : rpw + 4; }       // floats per key of a warp's weights: no bank conflicts
__host__ __device__ inline int af_smem_bytes(int head_dim, int rpw)
{
    return ((4 * rpw + 2 * AF_KEYS) * af_stride(head_dim) + 4 * AF_KEYS * af_p_stride(rpw)) * 4 + AF_KEYS * 16;
}

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
template <typename T> __device__ __forceinline__ float4 load4(const T* p)      // 16-bit types: 8 bytes
{
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    const T* e = reinterpret_cast<const T*>(&v);
    return make_float4(to_float(e[0]), to_float(e[1]), to_float(e[2]), to_float(e[3]));
}

__device__ __forceinline__ float4 load4(const int8_t* p)                      // 8-bit codes: 4 bytes
{
    const char4 v = *reinterpret_cast<const char4*>(p);
    return make_float4((float)v.x, (float)v.y, (float)v.z, (float)v.w);
}
__device__ __forceinline__ float4 load4(const __nv_fp8_e4m3* p) { return (float4)*reinterpret_cast<const __nv_fp8x4_e4m3*>(p); }

// T: of q and out; TC: of the cache.  8-bit codes become values, code x scale in fp32, as they are staged.
template <typename T, typename TC, int RPW, int NV>
__global__ void __launch_bounds__(128) attn_fp32_kernel(BatchView b, AttnView a)
{
    constexpr bool CODES = sizeof(TC) == 1;
    constexpr int ROWS = 4 * RPW, RT = RPW / 4, PS = af_p_stride(RPW);
    extern __shared__ __align__(16) float af_smem[];
    const int D = a.head_dim, ld = af_stride(D), G = a.n_heads / a.n_kv_heads, Hk = a.n_kv_heads, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    float* q_sh = af_smem;
    float* k_sh = q_sh + ROWS * ld;
    float* v_sh = k_sh + AF_KEYS * ld;
    float* p_sh = v_sh + AF_KEYS * ld + warp * AF_KEYS * PS;          // this warp's weights, [key][row]
    long long* at_sh = reinterpret_cast<long long*>(af_smem + (ROWS + 2 * AF_KEYS) * ld + 4 * AF_KEYS * PS);   // element offset of each key's K, -1: nothing there
    float2* scale_sh = reinterpret_cast<float2*>(at_sh + AF_KEYS);    // (codes) its scales, of K and of V
    // ---- this block's piece
    int idx = blockIdx.x, seq = -1;
    SeqSpan sp = {};
    for (int base = 0; base < b.n_seqs && seq < 0; base += 32) {
        SeqSpan mine = {};
        if (base + lane < b.n_seqs) mine = seq_span(b, base + lane);
        const int pieces = (mine.n * G + ROWS - 1) / ROWS * Hk;
        int upto = pieces;
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
        idx -= __shfl_sync(FULL_WARP, upto - pieces, at);
        seq = base + at;
        sp = span_of(mine, at);
    }
    if (seq < 0) return;                                  // the same for the whole block
    const int kvh = idx % Hk, rho0 = idx / Hk * ROWS, rows = min(ROWS, sp.n * G - rho0);
    const TC* head = reinterpret_cast<const TC*>(a.pool) + (size_t)kvh * b.page_size * D;
    // ---- queries; dead rows and the dims behind the last are zero
    for (int r = warp; r < ROWS; r += 4) {
        const int tok = (rho0 + r) / G;
        const T* src = reinterpret_cast<const T*>(a.q) + (long long)(sp.r0 + tok) * a.q_row_stride + (long long)(kvh * G + rho0 + r - tok * G) * a.q_head_stride;
        for (int d = lane; d < ld; d += 32) q_sh[r * ld + d] = r < rows && d < D ? to_float(src[d]) : 0.f;
    }
    for (int i = tid; i < 2 * AF_KEYS * (ld - D); i += 128) k_sh[i / (ld - D) * ld + D + i % (ld - D)] = 0.f;
    const int grp = lane >> 3, sub = lane & 7, row0 = warp * RPW;     // this lane's rows of scores: row0 + grp + 4 r
    int seen[RT];
    float m[RT], l[RT], o[RPW][4 * NV];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        seen[r] = b.prefix_len + seen_own(sp, min(rho0 + row0 + grp + 4 * r, sp.n * G - 1) / G);
        m[r] = -INFINITY;
        l[r] = 0.f;
    }
    const int last = min(rho0 + rows - 1, sp.n * G - 1) / G, total = b.prefix_len + seen_own(sp, last);   // what the last row sees
#pragma unroll
    for (int r = 0; r < RPW; ++r)
#pragma unroll
        for (int e = 0; e < 4 * NV; ++e) o[r][e] = 0.f;
    for (int p0 = 0; p0 < total; p0 += AF_KEYS) {
        __syncthreads();                                  // the tile before is used up
        if (tid < AF_KEYS) {
            long long at = -1;
            const int p = p0 + tid, own = p - b.prefix_len, pp = own < 0 ? p : own;
            if (p < total) {
                const int page = own < 0 ? b.prefix_pages[pp >> b.page_shift] : b.page_table[(size_t)seq * b.table_stride + (pp >> b.page_shift)];
                if ((unsigned)page < (unsigned)b.n_pages) {
                    at = (long long)page * a.page_elems + (long long)(pp & (b.page_size - 1)) * D;
                    if (CODES) {
                        const float* s = a.scales + page * a.scale_page + kvh;
                        scale_sh[tid] = make_float2(s[0], s[Hk]);
                    }
                }
            }
            at_sh[tid] = at;
        }
        __syncthreads();
        if (D % 4 == 0) {                                 // 16 (or 8) bytes a lane: pages and rows start on multiples of that
#pragma unroll 4
            for (int j = warp; j < AF_KEYS; j += 4) {
                const long long at = at_sh[j];
#pragma unroll
                for (int e = 0; e < NV; ++e) {
                    const int d = 4 * lane + 128 * e;
                    if (d >= D) break;
                    float4 kx = make_float4(0.f, 0.f, 0.f, 0.f), vx = kx;
                    if (at >= 0) {
                        kx = load4(head + at + d);
                        vx = load4(head + at + a.kv_elems + d);
                        if (CODES) {
                            const float2 s = scale_sh[j];
                            kx.x *= s.x; kx.y *= s.x; kx.z *= s.x; kx.w *= s.x;
                            vx.x *= s.y; vx.y *= s.y; vx.z *= s.y; vx.w *= s.y;
                        }
                    }
                    *reinterpret_cast<float4*>(k_sh + j * ld + d) = kx;
                    *reinterpret_cast<float4*>(v_sh + j * ld + d) = vx;
                }
            }
        } else {
            for (int j = warp; j < AF_KEYS; j += 4) {
                const long long at = at_sh[j];
                const float2 s = CODES && at >= 0 ? scale_sh[j] : make_float2(1.f, 1.f);
                for (int d = lane; d < D; d += 32) {
                    k_sh[j * ld + d] = at >= 0 ? (CODES ? to_float(head[at + d]) * s.x : to_float(head[at + d])) : 0.f;
                    v_sh[j * ld + d] = at >= 0 ? (CODES ? to_float(head[at + a.kv_elems + d]) * s.y : to_float(head[at + a.kv_elems + d])) : 0.f;
                }
            }
        }
        __syncthreads();
        if (row0 >= rows) continue;                       // the same for the whole warp
        float s[RT][4];                                   // keys sub, sub + 8, sub + 16, sub + 24
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[r][i] = 0.f;
#pragma unroll 2
        for (int d = 0; d < ld - 4; d += 4) {
            float4 y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = *reinterpret_cast<const float4*>(k_sh + (sub + 8 * i) * ld + d);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const float4 x = *reinterpret_cast<const float4*>(q_sh + (row0 + grp + 4 * r) * ld + d);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[r][i] = fmaf(x.x, y[i].x, fmaf(x.y, y[i].y, fmaf(x.z, y[i].z, fmaf(x.w, y[i].w, s[r][i]))));
            }
        }
        bool there[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) there[i] = at_sh[sub + 8 * i] >= 0;
        float shrink[RT];
        __syncwarp();                                     // the weights before are used up
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float top = m[r];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[r][i] = p0 + sub + 8 * i >= seen[r] || !there[i] ? -INFINITY : s[r][i] * a.scale;     // scaled behind the sum, as the other kernels do
                top = fmaxf(top, s[r][i]);
            }
#pragma unroll
            for (int x = 4; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(FULL_WARP, top, x));
            shrink[r] = m[r] == top ? 1.f : expf(m[r] - top);
            const float from = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = expf(s[r][i] - from);
                p_sh[(sub + 8 * i) * PS + grp + 4 * r] = e;
                sum += e;
            }
#pragma unroll
            for (int x = 4; x > 0; x >>= 1) sum += __shfl_xor_sync(FULL_WARP, sum, x);
            l[r] = l[r] * shrink[r] + sum;
            m[r] = top;
        }
        __syncwarp();
#pragma unroll
        for (int r = 0; r < RPW; ++r) {
            const float f = __shfl_sync(FULL_WARP, shrink[r >> 2], 8 * (r & 3));
#pragma unroll
            for (int e = 0; e < 4 * NV; ++e) o[r][e] *= f;
        }
        const int n = min(AF_KEYS, total - p0);
#pragma unroll 2
        for (int j = 0; j < n; ++j) {
            float4 v[NV];
#pragma unroll
            for (int e = 0; e < NV; ++e) {
                const int d = 4 * lane + 128 * e;
                v[e] = d < D ? *reinterpret_cast<const float4*>(v_sh + j * ld + d) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int r = 0; r < RPW; r += 4) {
                const float4 w = *reinterpret_cast<const float4*>(p_sh + j * PS + r);
                const float wr[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < NV; ++e) {
                        o[r + i][4 * e] = fmaf(wr[i], v[e].x, o[r + i][4 * e]);
                        o[r + i][4 * e + 1] = fmaf(wr[i], v[e].y, o[r + i][4 * e + 1]);
                        o[r + i][4 * e + 2] = fmaf(wr[i], v[e].z, o[r + i][4 * e + 2]);
                        o[r + i][4 * e + 3] = fmaf(wr[i], v[e].w, o[r + i][4 * e + 3]);
                    }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RPW; ++r) {
        const float sum = __shfl_sync(FULL_WARP, l[r >> 2], 8 * (r & 3));
        const int rr = row0 + r, t = (rho0 + rr) / G;
        if (rr >= rows || t >= a.max_rows) continue;
        T* out = reinterpret_cast<T*>(a.out) + ((size_t)(sp.r0 + t) * a.n_heads + kvh * G + rho0 + rr - t * G) * D;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;   // 0: the row sees nothing
#pragma unroll
        for (int e = 0; e < 4 * NV; ++e) {
            const int d = 4 * lane + 128 * (e >> 2) + (e & 3);
            if (d < D) store_val(out + d, o[r][e] * inv);
        }
    }
}

} // namespace swk
