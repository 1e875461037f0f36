// One token per row of logits: temperature, top-k, top-p and min-p, drawn with a given random number.
//
// Every filter keeps a run from the start of one order (logits falling, equal ones by rising id), so what all of them keep is known by
// the last token of the run, the cut: tokens are numbered by (logit, id) in that order as 64-bit integers, and a token is kept when
// its number is not above the cut's.  top-k's cut is where a count reaches k, top-p's where a sum of weights reaches its share, and the draw is
// a search for where a running sum in the order of ids passes uniform x total.
//
// Weights.  w = exp((l - max) / T) in 64 bits, as an integer in units of 2^-45: sums of up to 2^18 of them fit 63 bits and do not depend
// on the order of the additions, so the same logits give the same token whatever the number of blocks.  32-bit weights would not do:
// with 10^5 tokens a row has as many borders, and sums that are 10^-8 off would draw the neighbour in one row of a few hundred.
// exp: l - max times log2(e) / T is n / 256 + r; 2^(n / 256) is a table's entry and a shift, 2^r the exponential series up to the
// fourth power (|r ln 2| < 2^-9.5: the rest is below 2^-53).
//
// A cluster of up to eight blocks holds a row's logits in shared memory, read from HBM once.  A cut is found by a histogram of the weights over
// 512 bins of 1/16 in (max - l) / T, added up over the cluster; the tokens of the bin that it lies in (some hundred of them) are then gathered
// and ordered.  Bins with more than a list holds (equal logits, flat rows) are divided again by the tokens' numbers.
#pragma once
#include <cooperative_groups.h>

#include "kernels_batch.cuh"

namespace swk {

constexpr int SA_THREADS = 512, SA_WARPS = SA_THREADS / 32;
constexpr int SA_BINS = 512, SA_LIST = 512;               // one of each per thread
constexpr int SA_CHUNK = 128;                             // tokens whose kept weights are summed up for the draw
constexpr int SA_BLOCKS = 8;                              // of a cluster, at most
constexpr int SA_CHUNKS = 256;                            // of a block, at most
constexpr int SA_UNIT_BITS = 45;

typedef unsigned long long u64;

struct SampleView {
    const void* logits;
    long long row_stride;
    int n_rows, vocab, slice;                             // slice: tokens of a block, a multiple of SA_CHUNK
    const float* uniforms;
    const float* temperature;
    const int* top_k;
    const float* top_p;
    const float* min_p;
    float temperature_all, top_p_all, min_p_all;
    int top_k_all;
    int* tokens;
    float* probs;
};

struct SampleShared {
    double table[256];                                    // 2^(j / 256)
    u64 mass[SA_BINS];
    u64 list_at[2][SA_LIST], list_w[2][SA_LIST];          // [0]: this block's or the whole list's tokens, [1]: the other
    u64 chunk[SA_CHUNKS];
    u64 warps[SA_WARPS];
    u64 best, range[2], total, base, cut;
    unsigned count[SA_BINS];
    unsigned n_list, found, population, bad;
};

__device__ __forceinline__ u64 sa_number(float x, int id) // rising in the order of the tokens
{
    const unsigned b = __float_as_uint(x);
    return (u64)(b & 0x80000000u ? b : ~(b | 0x80000000u)) << 32 | (unsigned)id;
}

__device__ __forceinline__ u64 sa_warp_sum(u64 v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(FULL_WARP, v, o);
    return v;
}
__device__ __forceinline__ u64 sa_warp_scan(u64 v)        // inclusive
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const u64 x = __shfl_up_sync(FULL_WARP, v, o);
        if (lane >= o) v += x;
    }
    return v;
}
__device__ __forceinline__ u64 sa_block_scan(u64 v, SampleShared& sh, u64& all)   // inclusive over the block's threads
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    v = sa_warp_scan(v);
    __syncthreads();
    if (lane == 31) sh.warps[warp] = v;
    __syncthreads();
    all = 0;
    u64 before = 0;
#pragma unroll
    for (int w = 0; w < SA_WARPS; ++w) {
        const u64 x = sh.warps[w];
        if (w < warp) before += x;
        all += x;
    }
    return before + v;
}

struct SampleWeight {
    double top, rate;                                     // log2(e) 256 / T
    const double* table;
    // exp((x - top) / T) 2^45, in 64 bits; 0 where it rounds to 0
    __device__ __forceinline__ double operator()(float x) const
    {
        const double y = ((double)x - top) * rate;
        if (!(y > -256.0 * (SA_UNIT_BITS + 1))) return 0.0;
        const double round = 6755399441055744.0;          // 1.5 * 2^52: adding it leaves the nearest integer in the low bits
        const double t = y + round, r = (y - (t - round)) * (0.69314718055994530942 / 256.0);
        const int n = __double2loint(t);
        const double p = fma(fma(fma(fma(r, 1.0 / 24.0, 1.0 / 6.0), r, 0.5), r, 1.0), r, 1.0) * table[n & 255];
        return __hiloint2double(__double2hiint(p) + (((n >> 8) + SA_UNIT_BITS) << 20), __double2loint(p));
    }
    static __device__ __forceinline__ u64 whole(double w) { return (u64)__double_as_longlong(w + 4503599627370496.0) & 0xFFFFFFFFFFFFFull; }   // + 2^52
};

// grid = rows x blocks of a cluster, block = 512
template <typename T>
__global__ void __launch_bounds__(SA_THREADS) sample_kernel(SampleView s)
{
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int blocks = cluster.num_blocks(), rank = cluster.block_rank(), row = blockIdx.x / blocks;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    extern __shared__ __align__(16) unsigned char sa_smem[];
    SampleShared& sh = *reinterpret_cast<SampleShared*>(sa_smem);
    T* vals = reinterpret_cast<T*>(sa_smem + (sizeof(SampleShared) + 15) / 16 * 16);
    const int id0 = rank * s.slice, n = max(0, min(s.slice, s.vocab - id0));
    auto value = [&](int i) { return to_float(vals[i]) + 0.f; };          // (-0 as 0)
    auto other = [&](int r) { return cluster.map_shared_rank(&sh, r); };

    // ---- the logits, their largest and whether all are numbers below infinity
    float best = -INFINITY;
    int best_id = 0x7FFFFFFF;
    bool bad = false;
    {
        auto meet = [&](T v, int i) {
            const float x = to_float(v) + 0.f;
            bad |= !(x < INFINITY);
            if (x > best) { best = x; best_id = id0 + i; }
        };
        const T* src = reinterpret_cast<const T*>(s.logits) + row * s.row_stride + id0;
        constexpr int PER = 16 / sizeof(T);
        int i = tid * PER, done = 0;
        if (reinterpret_cast<uintptr_t>(src) % 16 == 0) {
            done = n / PER * PER;
            for (; i + 3 * SA_THREADS * PER < done; i += 4 * SA_THREADS * PER) {
                uint4 v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = __ldcs(reinterpret_cast<const uint4*>(src + i + j * SA_THREADS * PER));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    *reinterpret_cast<uint4*>(vals + i + j * SA_THREADS * PER) = v[j];
#pragma unroll
                    for (int e = 0; e < PER; ++e) meet(reinterpret_cast<const T*>(&v[j])[e], i + j * SA_THREADS * PER + e);
                }
            }
            for (; i < done; i += SA_THREADS * PER) {
                const uint4 v = __ldcs(reinterpret_cast<const uint4*>(src + i));
                *reinterpret_cast<uint4*>(vals + i) = v;
#pragma unroll
                for (int e = 0; e < PER; ++e) meet(reinterpret_cast<const T*>(&v)[e], i + e);
            }
        }
        for (i = done + tid; i < n; i += SA_THREADS) {
            const T v = src[i];
            vals[i] = v;
            meet(v, i);
        }
    }
    if (tid < 256) sh.table[tid] = exp2(tid / 256.0);
    if (tid == 0) sh.bad = 0;
    __syncthreads();
    if (bad) sh.bad = 1;
    u64 first = sa_number(best, best_id);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) first = min(first, __shfl_xor_sync(FULL_WARP, first, o));
    if (lane == 0) sh.warps[warp] = first;
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < SA_WARPS; ++w) first = min(first, sh.warps[w]);
        sh.best = first;
    }
    cluster.sync();
    for (int r = 0; r < blocks; ++r) {
        const u64 x = other(r)->best;
        first = r ? min(first, x) : x;
        bad |= other(r)->bad != 0;
    }
    const int first_id = (int)(unsigned)first;
    const float temperature = s.temperature ? s.temperature[row] : s.temperature_all, u = s.uniforms[row];
    const float top_p = s.top_p ? s.top_p[row] : s.top_p_all, min_p = s.min_p ? s.min_p[row] : s.min_p_all;
    const int top_k = s.top_k ? s.top_k[row] : s.top_k_all;
    const unsigned high = (unsigned)(first >> 32);
    const float top = __uint_as_float(high & 0x80000000u ? high : ~high & 0x7FFFFFFFu);
    bad |= top == -INFINITY || !(u >= 0.f && u < 1.f) || !(temperature >= 0.f && temperature < INFINITY) || top_p != top_p || !(min_p <= 1.f);
    if (bad || temperature == 0.f || top_k == 1 || top_p <= 0.f) {        // the same for the whole cluster
        if (rank == 0 && tid == 0) {
            s.tokens[row] = bad ? -1 : first_id;
            if (s.probs) s.probs[row] = bad ? 0.f : 1.f;
        }
        cluster.sync();                                   // no block ends while another reads its memory
        return;
    }
    const SampleWeight weight = {(double)top, 1.4426950408889634074 * 256.0 / (double)temperature, sh.table};
    const float bin_rate = 16.f / temperature;
    auto bin_of = [&](float x) { return min((int)((top - x) * bin_rate), SA_BINS - 1); };   // rises as x falls
    u64 cut = ~0ull;

    // ---- the first token at which the count (MASS: the sum of weights) of what is kept reaches a target becomes the cut
    auto shorten = [&](bool by_mass, u64 target) {
        u64 lo = 0, hi = cut, base = 0;                   // numbers that are searched; what lies before them
        int shift = -1, at = 0;                           // bins of numbers >> shift; -1: of values
        for (bool again = true; again;) {
            if (tid < SA_BINS) {
                sh.count[tid] = 0;
                sh.mass[tid] = 0;
            }
            __syncthreads();
            for (int i = tid; i < n; i += SA_THREADS) {
                const float x = value(i);
                const u64 num = sa_number(x, id0 + i);
                if (num < lo || num > hi) continue;
                const int bin = shift < 0 ? bin_of(x) : (int)((num - lo) >> shift);
                if (by_mass) {
                    const u64 w = SampleWeight::whole(weight(x));
                    if (w == 0) continue;
                    atomicAdd(&sh.mass[bin], w);
                }
                atomicAdd(&sh.count[bin], 1u);
            }
            cluster.sync();
            unsigned c = 0;
            u64 m = 0;
            for (int r = 0; r < blocks; ++r) {
                c += other(r)->count[tid];
                if (by_mass) m += other(r)->mass[tid];
            }
            const u64 mine = by_mass ? m : c;
            u64 all;
            const u64 upto = sa_block_scan(mine, sh, all);
            if (by_mass && target == 0) target = max((u64)ceil((double)top_p * (double)all), 1ull);   // (of the first histogram, which holds all that is kept)
            if (by_mass && target > base + all) target = base + all;
            if (base + upto - mine < target && target <= base + upto) {
                sh.found = tid;
                sh.base = base + upto - mine;
                sh.population = c;
            }
            cluster.sync();                               // (every block has read the others' bins)
            at = sh.found;
            base = sh.base;
            again = sh.population > SA_LIST;
            auto here = [&](float x, u64 num) { return num >= lo && num <= hi && (shift < 0 ? bin_of(x) == at : (int)((num - lo) >> shift) == at); };
            if (!again) {
                // ---- the bin's tokens, of all blocks
                if (tid == 0) sh.n_list = 0;
                __syncthreads();
                for (int i = tid; i < n; i += SA_THREADS) {
                    const float x = value(i);
                    const u64 num = sa_number(x, id0 + i);
                    if (!here(x, num)) continue;
                    u64 w = 1;
                    if (by_mass) w = SampleWeight::whole(weight(x));
                    if (w == 0) continue;
                    const unsigned k = atomicAdd(&sh.n_list, 1u);
                    sh.list_at[0][k] = num;
                    sh.list_w[0][k] = w;
                }
                cluster.sync();
                int total = 0;
                for (int r = 0; r < blocks; ++r) {
                    const int here_n = other(r)->n_list;
                    if (tid < here_n) {
                        sh.list_at[1][total + tid] = other(r)->list_at[0][tid];
                        sh.list_w[1][total + tid] = other(r)->list_w[0][tid];
                    }
                    total += here_n;
                }
                cluster.sync();
                // ---- fewer and fewer of them, until a warp can order them
                int from = 1;
                while (total > 32) {
                    u64 num = tid < total ? sh.list_at[from][tid] : ~0ull, w = tid < total ? sh.list_w[from][tid] : 0;
                    u64 least = num, most = tid < total ? num : 0;
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) {
                        least = min(least, __shfl_xor_sync(FULL_WARP, least, o));
                        most = max(most, __shfl_xor_sync(FULL_WARP, most, o));
                    }
                    if (tid == 0) { sh.range[0] = ~0ull; sh.range[1] = 0; sh.n_list = 0; }
                    sh.mass[tid] = 0;
                    __syncthreads();
                    if (lane == 0) { atomicMin(&sh.range[0], least); atomicMax(&sh.range[1], most); }
                    __syncthreads();
                    const u64 start = sh.range[0];
                    const int down = max(0, 64 - __clzll((long long)(sh.range[1] - start)) - 9);
                    const int bin = tid < total ? (int)((num - start) >> down) : 0;
                    if (tid < total) atomicAdd(&sh.mass[bin], w);
                    __syncthreads();
                    const u64 part = sh.mass[tid];
                    u64 sum;
                    const u64 end = sa_block_scan(part, sh, sum);
                    if (base + end - part < target && target <= base + end) {
                        sh.found = tid;
                        sh.base = base + end - part;
                    }
                    __syncthreads();
                    base = sh.base;
                    if (tid < total && bin == (int)sh.found) {
                        const unsigned k = atomicAdd(&sh.n_list, 1u);
                        sh.list_at[from ^ 1][k] = num;
                        sh.list_w[from ^ 1][k] = w;
                    }
                    __syncthreads();
                    total = sh.n_list;
                    from ^= 1;
                    __syncthreads();
                }
                if (warp == 0) {
                    const u64 num = lane < total ? sh.list_at[from][lane] : ~0ull, w = lane < total ? sh.list_w[from][lane] : 0;
                    u64 before = base;
                    for (int j = 0; j < 32; ++j) {
                        const u64 num_j = __shfl_sync(FULL_WARP, num, j), w_j = __shfl_sync(FULL_WARP, w, j);
                        if (num_j < num) before += w_j;
                    }
                    if (lane < total && before < target && target <= before + w) sh.cut = num;
                }
                __syncthreads();
                cut = sh.cut;
                __syncthreads();
            } else {
                // ---- too many for a list: the range of their numbers is divided in the next round
                u64 least = ~0ull, most = 0;
                for (int i = tid; i < n; i += SA_THREADS) {
                    const float x = value(i);
                    const u64 num = sa_number(x, id0 + i);
                    if (!here(x, num)) continue;
                    least = min(least, num);
                    most = max(most, num);
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
                    least = min(least, __shfl_xor_sync(FULL_WARP, least, o));
                    most = max(most, __shfl_xor_sync(FULL_WARP, most, o));
                }
                if (tid == 0) { sh.range[0] = ~0ull; sh.range[1] = 0; }
                __syncthreads();
                if (lane == 0) { atomicMin(&sh.range[0], least); atomicMax(&sh.range[1], most); }
                cluster.sync();
                lo = ~0ull;
                hi = 0;
                for (int r = 0; r < blocks; ++r) {
                    lo = min(lo, other(r)->range[0]);
                    hi = max(hi, other(r)->range[1]);
                }
                shift = max(0, 64 - __clzll((long long)(hi - lo)) - 9);
                cluster.sync();
            }
        }
    };
    if (top_k > 0 && top_k < s.vocab) shorten(false, (u64)top_k);
    if (top_p < 1.f) shorten(true, 0);

    // ---- the draw: kept weights by chunks of consecutive ids, then by blocks
    const double least = (double)min_p * (double)(1ull << SA_UNIT_BITS);
    auto kept = [&](int i) -> u64 {
        if (i >= n) return 0;
        const float x = value(i);
        if (sa_number(x, id0 + i) > cut) return 0;
        const double w = weight(x);
        return w >= least ? SampleWeight::whole(w) : 0;
    };
    const int chunks = (n + SA_CHUNK - 1) / SA_CHUNK;
    for (int c = warp; c < chunks; c += SA_WARPS) {
        u64 sum = 0;
#pragma unroll
        for (int j = 0; j < SA_CHUNK / 32; ++j) sum += kept(c * SA_CHUNK + 32 * j + lane);
        sum = sa_warp_sum(sum);
        if (lane == 0) sh.chunk[c] = sum;
    }
    __syncthreads();
    const u64 part = tid < chunks ? sh.chunk[tid] : 0;
    u64 mine;
    const u64 end = sa_block_scan(part, sh, mine);
    if (tid == 0) sh.total = mine;
    cluster.sync();
    u64 total = 0, before = 0;
    for (int r = 0; r < blocks; ++r) {
        const u64 x = other(r)->total;
        if (r < rank) before += x;
        total += x;
    }
    const u64 goal = (u64)((double)u * (double)total);    // the lowest id whose running sum is above it
    if (before <= goal && goal < before + mine) {
        if (before + end - part <= goal && goal < before + end) {
            sh.found = tid;
            sh.base = before + end - part;
        }
        __syncthreads();
        if (warp == 0) {
            u64 upto = sh.base;
            for (int j = 0; j < SA_CHUNK / 32; ++j) {
                const int i = sh.found * SA_CHUNK + 32 * j + lane;
                const u64 w = kept(i), incl = upto + sa_warp_scan(w);
                if (incl - w <= goal && goal < incl) {
                    s.tokens[row] = id0 + i;
                    if (s.probs) s.probs[row] = (float)((double)w / (double)total);
                }
                upto = __shfl_sync(FULL_WARP, incl, 31);
            }
        }
    }
    cluster.sync();                                       // no block ends while another reads its memory
}

} // namespace swk
