// ra_paged.cu -- the paged cache: host side of ra_paged_* and the kernels that write rows, read them back and
// choose pages by their bounds.
#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include <new>

#include "ra_internal.h"
#include "ra_paged.h"
#include "ra_ptx.cuh"

namespace ra {
namespace {

constexpr int kRowThreads = 256, kRowWarps = kRowThreads / 32;
constexpr unsigned kAll = 0xffffffffu;

// ---------------------------------------------------------------------------- which rows a CTA has
struct Slice {
    int b;         // sequence, -1: none
    int page;      // its page
    int off;       // first position within the page
    int n;         // rows
    int row0;      // their first row in the call's tensors
    bool fresh;    // the page begins with them
};

// Rows [row0, row0 + n) of sequence b end at its length.
__device__ __forceinline__ int sequence_rows(const PagedRowsParams& p, int b, int& row0, int& len)
{
    len = paged_len(p.c, b);
    row0 = p.rows[b];
    const int end = p.rows[b + 1];
    if (row0 < 0 || end < row0 || end > p.n_rows || end - row0 > len) {
        if (end != row0) atomicOr(p.c.err, kPagedErrInput);
        return 0;
    }
    return end - row0;
}

// A sequence's rows are cut at its page ends; slices are numbered through the batch, and a CTA finds its own: each thread
// counts a run of sequences, a scan numbers them, and the thread that has it looks it up (one-row calls: a slice per
// sequence).
__device__ __forceinline__ Slice find_slice(const PagedRowsParams& p, int slice)
{
    auto look_up = [&](int b, int i, int row0, int start, int len) {  // the sequence's page i, its rows from `start` on
        Slice s;
        const int lo = max(start, i << p.c.page_shift), hi = min(len, (i + 1) << p.c.page_shift);
        s.page = paged_page(p.c, b, i);
        s.off = lo - (i << p.c.page_shift);
        s.n = hi - lo;
        s.row0 = row0 + (lo - start);
        s.fresh = s.off == 0;
        s.b = s.page >= 0 ? b : -1;
        return s;
    };
    if (!p.rows) {
        const int len = paged_len(p.c, slice);
        if (len > 0) return look_up(slice, (len - 1) >> p.c.page_shift, slice, len - 1, len);
        return Slice{-1, 0, 0, 0, 0, false};
    }
    __shared__ Slice found;
    __shared__ int warp_sum[kRowWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (p.c.batch + blockDim.x - 1) / blockDim.x, b0 = min(tid * per, p.c.batch), b1 = min(b0 + per, p.c.batch);
    int mine = 0, row0 = 0, len = 0, n = 0, of = 0;
    for (int b = b0; b < b1; ++b) {
        n = sequence_rows(p, b, row0, len);
        of = n > 0 ? ((len - 1) >> p.c.page_shift) - ((len - n) >> p.c.page_shift) + 1 : 0;
        mine += of;
    }
    int inc = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(kAll, inc, o);
        if (lane >= o) inc += t;
    }
    if (lane == 31) warp_sum[warp] = inc;
    if (tid == 0) found.b = -1;
    __syncthreads();
    int at = inc - mine;
    for (int w = 0; w < warp; ++w) at += warp_sum[w];
    if (slice >= at && slice < at + mine)
        for (int b = b0; b < b1; ++b) {
            if (per > 1) {
                n = sequence_rows(p, b, row0, len);
                of = n > 0 ? ((len - 1) >> p.c.page_shift) - ((len - n) >> p.c.page_shift) + 1 : 0;
            }
            if (slice < at + of) {
                found = look_up(b, ((len - n) >> p.c.page_shift) + slice - at, row0, len - n, len);
                break;
            }
            at += of;
        }
    __syncthreads();
    return found;
}

// ---------------------------------------------------------------------------- formats
__device__ __forceinline__ uint32_t max_halves(uint32_t a) { return max(a & 0xffffu, a >> 16); }
// Largest |x| of 8 bf16 values, as the bits of a bf16 (an infinity or NaN is 0x7f80 or more).
__device__ __forceinline__ uint32_t amax_bits(const uint4& x)
{
    const uint32_t k = 0x7fff7fffu;
    return max_halves(__vmaxu2(__vmaxu2(x.x & k, x.y & k), __vmaxu2(x.z & k, x.w & k)));
}
// Smallest e >= least with amax <= top * 2^e for top = (1 + frac / 128) * 2^log (bf16 bits, finite).
__device__ __forceinline__ int scale_exp(uint32_t amax, int log, int frac, int least)
{
    return max((int)(amax >> 7) - 127 - log + ((int)(amax & 127u) > frac), least);
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // e in [-126, 127]

// 8 values to e4m3 codes (nearest, ties to even) at scale 2^-e, exact but for that rounding.
__device__ __forceinline__ uint2 to_codes(const uint4& x, float inv)
{
    auto two = [&](uint32_t a) {
        return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(bf16lo(a) * inv, bf16hi(a) * inv), __NV_SATFINITE, __NV_E4M3);
    };
    return make_uint2(two(x.x) | two(x.y) << 16, two(x.z) | two(x.w) << 16);
}
__device__ __forceinline__ uint32_t from_codes(uint32_t two, float scale)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    const __nv_bfloat162 r = __floats2bfloat162_rn(f.x * scale, f.y * scale);
    return *reinterpret_cast<const uint32_t*>(&r);
}

// What a CTA's first steps read: the tables, and of one-row calls the rows.
__device__ __forceinline__ void prefetch_start(const PagedRowsParams& p, int D)
{
    const PrefetchShare mine = prefetch_share(gridDim.x, gridDim.y, blockIdx.x, blockIdx.y, blockDim.x, threadIdx.x);
    const int i = mine.i, n = mine.n;
    if (i < 0) return;
    prefetch_sequences(p.c, i, n);
    if (p.rows) {
        prefetch_lines(p.rows, 4ll * (p.c.batch + 1), i, n);
    } else if (p.k_in) {
        prefetch_heads(p.k_in, p.row_stride, p.head_stride, p.c.KVH, D, p.c.batch, i, n);
        prefetch_heads(p.v_in, p.row_stride, p.head_stride, p.c.KVH, D, p.c.batch, i, n);
    }
}

// ---------------------------------------------------------------------------- write
// A CTA takes the rows of one page of up to 8 KV heads, a warp each; where there are too few of those for the SMs, of 2
// heads, `split` warps per head, each every split-th set of rows.  D / 8 lanes hold a row of 8 channels each; a warp's
// lower half takes K rows, the upper half the V rows beside them, kAtOnce sets of them under way (with 2, 4 and 8: 17k rows of
// 10 heads written in 8 bits in 27.4, 25.6 and 25.8 us and read back in 28.3, 20.0 and 19.3; 65k rows of 8 heads in bf16 in 45.1, 44.0
// and 42.9 and 45.2, 43.4 and 43.2; four warps a head over pages of 16 rows 32.2, 32.4 and 37.0).  What
// bounds it is memory, each row being read once and written once, and in 8 bits the instructions of the rounding (two thirds of
// the issue slots): those 17k rows, 132 MB, are written in 25 us, 0.78 of the copy rate.  Keeping bounds adds 16 comparisons a lane
// and row set and the page's own reduction: the same rows in 41 us in 8 bits and 39 in bf16 (27 without).
constexpr int kAtOnce = 4;

template <int FMT, int D>
struct RowPlace {  // what a lane does in every set
    using Geo = PagedGeo<FMT, D>;
    static constexpr int LPR = D / 8, RPW = 16 / LPR;  // lanes per row, rows per warp (K and V of each)
    int is_v, sub, c8, U, u_shift;
    __device__ __forceinline__ RowPlace(int lane, int page_shift)
    {
        is_v = lane >> 4;
        sub = (lane & 15) / LPR;
        c8 = lane % LPR;
        U = Geo::unit_rows(1 << page_shift);
        u_shift = 31 - __clz(U);
    }
    __device__ __forceinline__ long long head(const PagedView& c, int page, int h) const  // byte of the head's units
    {
        return ((long long)page * c.KVH + h) * ((1 << c.page_shift) >> u_shift) * Geo::unit_stride(U);
    }
    __device__ __forceinline__ int unit(int pos) const { return (pos >> u_shift) * Geo::unit_stride(U); }
    __device__ __forceinline__ int codes(int pos) const  // of this lane's channels in the unit
    {
        const int r = pos & (U - 1);
        return is_v * U * Geo::kRow + (FMT == RA_PAGED_FP8 ? Geo::chunk(r, c8 >> 1) + (c8 & 1) * 8 : Geo::chunk(r, c8));
    }
    __device__ __forceinline__ int scale(int pos) const { return 2 * U * Geo::kRow + is_v * U + (pos & (U - 1)); }
};

template <int FMT, int D, bool BOUNDS>
__global__ void __launch_bounds__(kRowThreads) paged_write_kernel(const PagedRowsParams p, const int split, const int heads)
{
    using Place = RowPlace<FMT, D>;
    constexpr int LPR = Place::LPR, RPW = Place::RPW;
    __shared__ float s_lo[BOUNDS ? kRowWarps : 1][D], s_hi[BOUNDS ? kRowWarps : 1][D];
    __shared__ int s_bad[kRowWarps];
    prefetch_start(p, D);
    pdl_wait();
    pdl_launch_dependents();
    const Slice sl = find_slice(p, blockIdx.x);
    if (sl.b < 0) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Place at(lane, p.c.page_shift);
    const int part = warp % split, h = blockIdx.y * heads + warp / split;  // `heads` of them per CTA
    const bool mine = h < p.c.KVH;
    float lo[8], hi[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lo[i] = INFINITY;
        hi[i] = -INFINITY;
    }
    bool bad = false;
    if (mine) {
        const uint16_t* src = (at.is_v ? p.v_in : p.k_in) + sl.row0 * p.row_stride + h * p.head_stride + at.c8 * 8;
        uint8_t* units = p.c.rows + at.head(p.c, sl.page, h);
        const int step = split * RPW;
        for (int r0 = part * RPW + at.sub; r0 - at.sub < sl.n; r0 += step * kAtOnce) {
            uint4 x[kAtOnce];
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int r = r0 + k * step;
                x[k] = r < sl.n ? __ldcs(reinterpret_cast<const uint4*>(src + r * p.row_stride)) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) {
                const int r = r0 + k * step, pos = sl.off + r;
                if (r - at.sub >= sl.n) break;  // (the warp)
                uint32_t a = 0;
                if (FMT == RA_PAGED_FP8 || BOUNDS) {
                    a = amax_bits(x[k]);
#pragma unroll
                    for (int o = 1; o < LPR; o <<= 1) a = max(a, __shfl_xor_sync(kAll, a, o));
                }
                if (r < sl.n) {
                    uint8_t* unit = units + at.unit(pos);
                    if constexpr (FMT == RA_PAGED_FP8) {
                        const bool nan = a >= 0x7f80u;
                        const int e = nan ? 0 : scale_exp(a, 8, 0x60, kFp8MinExp);
                        *reinterpret_cast<uint2*>(unit + at.codes(pos)) =
                            nan ? make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu) : to_codes(x[k], exp2i(-e));  // e4m3's NaN
                        if (at.c8 == 0) unit[at.scale(pos)] = (uint8_t)(e + 127);
                    } else {
                        *reinterpret_cast<uint4*>(unit + at.codes(pos)) = x[k];
                    }
                    if (BOUNDS && !at.is_v) {
                        bad = bad || a >= 0x7f80u;
                        const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            lo[2 * i] = fminf(lo[2 * i], bf16lo(w[i]));
                            hi[2 * i] = fmaxf(hi[2 * i], bf16lo(w[i]));
                            lo[2 * i + 1] = fminf(lo[2 * i + 1], bf16hi(w[i]));
                            hi[2 * i + 1] = fmaxf(hi[2 * i + 1], bf16hi(w[i]));
                        }
                    }
                }
            }
        }
    }
    if constexpr (!BOUNDS) return;
    // The page's bounds: over the rows of the head's warps, and over what the page held before.
    bad = __any_sync(kAll, bad);
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int o = LPR; o < 16; o <<= 1) {
            lo[i] = fminf(lo[i], __shfl_xor_sync(kAll, lo[i], o));
            hi[i] = fmaxf(hi[i], __shfl_xor_sync(kAll, hi[i], o));
        }
    if (lane < LPR)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s_lo[warp][at.c8 * 8 + i] = lo[i];
            s_hi[warp][at.c8 * 8 + i] = hi[i];
        }
    if (lane == 0) s_bad[warp] = bad;
    if (split > 1) __syncthreads();
    else __syncwarp();
    if (!mine || part != 0) return;
    const long long where = (long long)sl.page * p.c.KVH + h;
    uint16_t* run = p.c.lohi + where * 2 * D;
    constexpr int CPL = D / 32;  // channels per lane
    float l[CPL], g[CPL];
    uint32_t amax = 0;
    bool nan = !sl.fresh && p.c.lohi_exp[where] == kScaleNaN;
    for (int w = warp; w < warp + split; ++w) nan = nan || s_bad[w];
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
        const int d = lane * CPL + i;
        l[i] = s_lo[warp][d];
        g[i] = s_hi[warp][d];
        for (int w = warp + 1; w < warp + split; ++w) {
            l[i] = fminf(l[i], s_lo[w][d]);
            g[i] = fmaxf(g[i], s_hi[w][d]);
        }
        if (!sl.fresh) {
            l[i] = fminf(l[i], __uint_as_float((uint32_t)run[d] << 16));
            g[i] = fmaxf(g[i], __uint_as_float((uint32_t)run[D + d] << 16));
        }
        run[d] = (uint16_t)(__float_as_uint(l[i]) >> 16);  // exact: every bound is a bf16 value
        run[D + d] = (uint16_t)(__float_as_uint(g[i]) >> 16);
        amax = max(amax, max(__float_as_uint(fabsf(l[i])), __float_as_uint(fabsf(g[i]))) >> 16);
    }
    amax = __reduce_max_sync(kAll, amax);
    nan = nan || amax >= 0x7f80u;
    const int e = nan ? 0 : scale_exp(amax, 6, 0x7e, kInt8MinExp);
    if (lane == 0) p.c.lohi_exp[where] = nan ? kScaleNaN : (uint8_t)(e + 127);
    int8_t* out = p.c.lohi8 + where * 2 * D;
#pragma unroll
    for (int i = 0; i < CPL; ++i) {
        out[lane * CPL + i] = nan ? 0 : (int8_t)floorf(l[i] * exp2i(-e));
        out[D + lane * CPL + i] = nan ? 0 : (int8_t)ceilf(g[i] * exp2i(-e));
    }
}

// ---------------------------------------------------------------------------- read back
// The same division of the work; a code times its row's scale is exact in bf16.  Bound by memory (65k rows of 8 heads of 64
// channels in bf16, 268 MB moved: 43.6 us, 0.91 of the copy rate).
template <int FMT, int D>
__global__ void __launch_bounds__(kRowThreads) paged_read_kernel(const PagedRowsParams p, const int split, const int heads)
{
    using Place = RowPlace<FMT, D>;
    constexpr int RPW = Place::RPW;
    prefetch_start(p, D);
    pdl_wait();
    pdl_launch_dependents();
    const Slice sl = find_slice(p, blockIdx.x);
    if (sl.b < 0) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, step = split * RPW;
    const Place at(lane, p.c.page_shift);
    const int h = blockIdx.y * heads + warp / split;
    if (h >= p.c.KVH) return;
    uint16_t* dst = (at.is_v ? p.v_out : p.k_out) + sl.row0 * p.row_stride + h * p.head_stride + at.c8 * 8;
    const uint8_t* units = p.c.rows + at.head(p.c, sl.page, h);
    for (int r0 = warp % split * RPW + at.sub; r0 < sl.n; r0 += step * kAtOnce) {
        uint4 x[kAtOnce];
        float f[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int r = min(r0 + k * step, sl.n - 1), pos = sl.off + r;
            const uint8_t* unit = units + at.unit(pos);
            if constexpr (FMT == RA_PAGED_FP8) {
                const uint2 q = *reinterpret_cast<const uint2*>(unit + at.codes(pos));
                x[k].x = q.x;
                x[k].y = q.y;
                f[k] = __uint_as_float((uint32_t)unit[at.scale(pos)] << 23);
            } else {
                x[k] = *reinterpret_cast<const uint4*>(unit + at.codes(pos));
            }
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            const int r = r0 + k * step;
            if (r >= sl.n) break;
            if constexpr (FMT == RA_PAGED_FP8)
                x[k] = make_uint4(from_codes(x[k].x & 0xffffu, f[k]), from_codes(x[k].x >> 16, f[k]), from_codes(x[k].y & 0xffffu, f[k]),
                                  from_codes(x[k].y >> 16, f[k]));
            __stcs(reinterpret_cast<uint4*>(dst + r * p.row_stride), x[k]);
        }
    }
}

// ---------------------------------------------------------------------------- choosing pages
// A cluster per sequence and KV head (one CTA where there are many heads).  What bounds it is latency (one user's 516
// pages: 6 us, of which 1 us until the scores begin, 1.2 the scores, 1.5 the cluster's join, 1 the cut, 0.7 the list),
// then, in a batch, its longest head (143k pages, 37 MB: 15 us, where the bytes take 5.4).  Scores: D / 8 lanes read a
// page's bounds, 16 bytes each, 8 pages (D = 64: as many) under way per lane; products of 16-bit sums of queries and
// 8-bit bounds (the sum over the heads is taken before the pages are read, so their number costs nothing).  Then the first CTA
// finds the key that `top` pages reach, by histograms of 1024 bins over the keys that are left, from the range the keys
// span (two passes for scores that differ), and lists the pages in order.
constexpr int kSelThreads = 256, kSelWarps = kSelThreads / 32, kSelBins = 1024, kSelKeys = 8192, kSelMostCluster = 8;

__device__ __forceinline__ uint32_t order_key(float s)  // larger key: larger value
{
    const uint32_t u = __float_as_uint(s);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

template <int D>
__global__ void __launch_bounds__(kSelThreads, 4) paged_select_kernel(const PagedSelectParams p)
{
    constexpr int LPP = D / 8;               // lanes per page
    constexpr int PPL = 32 / LPP;            // pages per load of a warp
    constexpr int kLoads = 8, PPW = PPL * kLoads;  // pages a warp takes at a time
    constexpr int kTwins = LPP / kLoads;     // lanes that hold the same page
    __shared__ __align__(16) uint32_t s_q[D];  // channel pairs: negative parts of the queries (against lo), then positive (hi)
    __shared__ uint32_t s_keys[kSelKeys];
    __shared__ int s_hist[kSelBins];
    __shared__ uint32_t s_amax, s_least, s_most;
    __shared__ int s_special;
    __shared__ int s_warp[2][kSelWarps], s_bin, s_need, s_in_bin;
    const int rank = blockIdx.x % p.cluster, h = blockIdx.x / p.cluster, b = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        s_amax = s_most = 0;
        s_least = 0xffffffffu;
        s_special = 0;
    }
    prefetch_lines(p.c.lens + b, 4, tid, kSelThreads);
    prefetch_lines(p.c.table + (long long)b * p.c.table_stride, min(4ll * p.c.table_stride, 4096ll), tid, kSelThreads);
    prefetch_heads(p.q + b * p.q_row_stride + (long long)h * p.c.G * p.q_head_stride, 0, p.q_head_stride, p.c.G, D, 1, tid, kSelThreads);
    pdl_wait();
    pdl_launch_dependents();
    // what the first steps wait for, all under way at once: the length, the queries, the warp's first pages (of columns
    // the table has, looked at only if the length covers them)
    const uint16_t* q = p.q + b * p.q_row_stride + (long long)h * p.c.G * p.q_head_stride;
    uint32_t amax = 0;
    for (int i = tid; i < p.c.G * D / 8; i += kSelThreads)
        amax = max(amax, amax_bits(*reinterpret_cast<const uint4*>(q + i / (D / 8) * p.q_head_stride + i % (D / 8) * 8)));
    const int32_t* table = p.c.table + (long long)b * p.c.table_stride;
    const int first = (rank * kSelWarps + warp) * PPW, step = p.cluster * kSelWarps * PPW;
    const int local = lane % LPP / kTwins * PPL + lane / LPP;  // the page this lane holds, of the warp's
    int next = first + local < p.c.table_stride ? table[first + local] : -1;
    const int len = paged_len(p.c, b);
    const int n = (len + (1 << p.c.page_shift) - 1) >> p.c.page_shift;
    int32_t* sel = p.sel + ((long long)b * p.c.KVH + h) * p.top;
    if (n <= p.top) {  // (the whole cluster)
        if (rank == 0)
            for (int i = tid; i < p.top; i += kSelThreads) sel[i] = i < n ? i : -1;
        return;
    }
    // ---- the group's queries in 8 bits, summed over the heads
    amax = __reduce_max_sync(kAll, amax);
    __syncthreads();
    if (lane == 0) atomicMax(&s_amax, amax);
    __syncthreads();
    amax = s_amax;
    const bool finite = amax < 0x7f80u;  // queries that are not: every score is 0
    const float inv = finite ? exp2i(-scale_exp(amax, 6, 0x7e, kInt8MinExp)) : 0.f;
    if (tid < D / 2) {
        int up0 = 0, up1 = 0, down0 = 0, down1 = 0;
        for (int g = 0; g < p.c.G && finite; ++g) {
            const uint32_t two = *reinterpret_cast<const uint32_t*>(q + g * p.q_head_stride + 2 * tid);
            const int x = __float2int_rn(bf16lo(two) * inv), y = __float2int_rn(bf16hi(two) * inv);
            up0 += max(x, 0);
            up1 += max(y, 0);
            down0 += min(x, 0);
            down1 += min(y, 0);
        }
        s_q[tid] = (uint32_t)(down0 & 0xffff) | (uint32_t)down1 << 16;
        s_q[D / 2 + tid] = (uint32_t)up0 | (uint32_t)up1 << 16;
    }
    __syncthreads();
    // ---- scores
    uint32_t* keys = p.keys + ((long long)b * p.c.KVH + h) * p.max_pages;
    const bool in_smem = p.cluster == 1 && n <= kSelKeys;
    uint32_t qw[8];  // this lane's 16 bytes of a page's bounds: channels 16 (lane % LPP) .. of lo, then of hi
#pragma unroll
    for (int i = 0; i < 8; ++i) qw[i] = s_q[lane % LPP * 8 + i];
    // pages that are always taken have keys above any score's; the range is that of the scores
    constexpr uint32_t kAlways = 0xffffffffu, kNotFinite = 0xfffffffeu;
    uint32_t least = kAlways, most = 0;
    int special = 0;
    auto count = [&](uint32_t key) {
        if (key >= kNotFinite) {
            ++special;
        } else {
            least = min(least, key);
            most = max(most, key);
        }
    };
    for (int base = first; base < n; base += step) {
        const int mine = base + local;
        int row = -1, e = 0;  // of the bounds
        if (mine < n) {
            if (next < 0 || next >= p.c.pages) {
                atomicOr(p.c.err, kPagedErrInput);
            } else {
                row = next * p.c.KVH + h;
                e = p.c.lohi_exp[row];
            }
        }
        next = mine + step < n ? table[mine + step] : -1;  // (of the next pages, while these are read)
        uint4 x[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {  // the lane's group reads the pages its lanes hold, in turn
            const int from = __shfl_sync(kAll, row, lane / LPP * LPP + k * kTwins);
            x[k] = from >= 0 ? *reinterpret_cast<const uint4*>(p.c.lohi8 + (long long)from * (2 * D) + lane % LPP * 16) : make_uint4(0, 0, 0, 0);
        }
        int sum[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const uint32_t w[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
            sum[k] = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[k] = __dp2a_lo((int)qw[2 * i], (int)w[i], sum[k]);
                sum[k] = __dp2a_hi((int)qw[2 * i + 1], (int)w[i], sum[k]);
            }
        }
        // The sums over the group's lanes, halved as they go: each lane ends with the one of the page it holds.
#pragma unroll
        for (int o = LPP / 2, left = kLoads / 2; left; o >>= 1, left >>= 1) {
            const bool upper = lane & o;
#pragma unroll
            for (int k = 0; k < left; ++k)
                sum[k] = (upper ? sum[k + left] : sum[k]) + __shfl_xor_sync(kAll, upper ? sum[k] : sum[k + left], o);
        }
        if constexpr (kTwins == 2) sum[0] += __shfl_xor_sync(kAll, sum[0], 1);
        if (mine < n && lane % kTwins == 0) {
            const uint32_t key = mine < p.first || mine >= n - p.last ? kAlways
                                 : row < 0                            ? 0u
                                 : e == kScaleNaN                     ? kNotFinite
                                                                      : order_key((float)sum[0] * __uint_as_float((uint32_t)e << 23));
            (in_smem ? s_keys : keys)[mine] = key;
            if (p.cluster == 1) count(key);
        }
    }
    if (p.cluster > 1) {
        cluster_sync();
        if (rank) return;
        for (int i = tid; i < n; i += kSelThreads) {
            const uint32_t key = __ldcg(&keys[i]);
            if (n <= kSelKeys) s_keys[i] = key;
            count(key);
        }
    }
    const uint32_t* all = n <= kSelKeys ? s_keys : keys;
    least = __reduce_min_sync(kAll, least);
    most = __reduce_max_sync(kAll, most);
    special = __reduce_add_sync(kAll, special);
    if (lane == 0) {
        atomicMin(&s_least, least);
        atomicMax(&s_most, most);
        atomicAdd(&s_special, special);
    }
    __syncthreads();
    least = s_least;
    most = s_most;
    special = s_special;
    // ---- the cut: keys above `high` are taken, of those in [least, high] the `need` largest
    uint32_t high = most, cut = 0;
    int need = p.top - special, ties = 0;
    if (need <= 0) {  // among those
        need = p.top;
        least = kNotFinite;
        high = kAlways;
    }
    for (;;) {
        const int bits = 32 - __clz((high - least) | 1u), shift = max(0, bits - 10);  // 1024 bins from `least` on
        for (int i = tid; i < kSelBins; i += kSelThreads) s_hist[i] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kSelThreads) {
            const uint32_t key = all[i];
            if (key >= least && key <= high) atomicAdd(&s_hist[(key - least) >> shift], 1);
        }
        __syncthreads();
        // thread t: kSelBins / kSelThreads bins from the top down; keys in the bins above, from a scan
        constexpr int kOwn = kSelBins / kSelThreads;
        int in[kOwn], inc = 0;
#pragma unroll
        for (int k = 0; k < kOwn; ++k) {
            in[k] = s_hist[kSelBins - 1 - kOwn * tid - k];
            inc += in[k];
        }
        const int mine = inc;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(kAll, inc, o);
            if (lane >= o) inc += y;
        }
        if (lane == 31) s_warp[0][warp] = inc;
        __syncthreads();
        int above = inc - mine;
#pragma unroll
        for (int w = 0; w < kSelWarps; ++w) above += w < warp ? s_warp[0][w] : 0;
        if (above < need && above + mine >= need) {  // one thread
            int k = 0;
            while (above + in[k] < need) above += in[k++];
            s_bin = kSelBins - 1 - kOwn * tid - k;
            s_need = need - above;
            s_in_bin = in[k];
        }
        __syncthreads();
        need = s_need;
        const uint32_t low = least + ((uint32_t)s_bin << shift);
        const bool whole = s_in_bin == need;
        __syncthreads();
        if (whole || shift == 0) {  // all of the bin, or keys that are equal
            cut = low;
            ties = whole ? 0x7fffffff : need;
            break;
        }
        const uint32_t end = low + ((1u << shift) - 1u);
        high = end < low || end > high ? high : end;
        least = low;
    }
    // (a whole bin: every key from its low end on; one value: `ties` of it, the earliest)
    const bool whole = ties == 0x7fffffff;
    int taken = 0, equal = 0;
    for (int base = 0; base < n; base += kSelThreads) {
        const int i = base + tid;
        const uint32_t key = i < n ? all[i] : 0u;
        const bool above = i < n && (whole ? key >= cut : key > cut), eq = i < n && !whole && key == cut;
        const unsigned eq_mask = __ballot_sync(kAll, eq), above_mask = __ballot_sync(kAll, above);
        if (lane == 0) {
            s_warp[0][warp] = __popc(eq_mask);
            s_warp[1][warp] = __popc(above_mask);
        }
        __syncthreads();
        // ties that are taken come first of all ties, so both prefixes give the place
        int rank_eq = equal + __popc(eq_mask & ((1u << lane) - 1u)), at = taken + __popc(above_mask & ((1u << lane) - 1u));
#pragma unroll
        for (int w = 0; w < kSelWarps; ++w) {
            if (w < warp) {
                rank_eq += s_warp[0][w];
                at += s_warp[1][w];
            }
            equal += s_warp[0][w];
            taken += s_warp[1][w];
        }
        if (above) sel[at + min(rank_eq, whole ? 0 : ties)] = i;
        if (eq && rank_eq < ties) sel[at + rank_eq] = i;
        __syncthreads();
    }
}

template <int FMT, int D>
cudaError_t launch_rows(const PagedRowsParams& p, bool write, int sms, cudaStream_t s)
{
    // every slice has a row, and a sequence's rows touch at most n / page + 2 pages
    const long long most = ((long long)p.n_rows >> p.c.page_shift) + 2ll * p.c.batch;
    const unsigned pages = (unsigned)(most < p.n_rows ? most : p.n_rows);
    // several warps per head where there are few pages, of more than a row; the heads spread evenly over the CTAs.  With one and
    // four warps a head: 64 page heads of 64 rows written in 8 bits in 16.9 and 5.9 us, 4096 of 128 in bf16 in 49.5 and 44.0, 5120 of 64
    // in 8 bits in 48.5 and 46.8, 9728 in 88.0 and 84.4, 20480 in 174 and 173; of pages of 16 rows 9000 in bf16 in 22.7 and 21.9, but
    // 10660 in 8 bits in 25.6 and 32.4 (four rows a warp): so up to 9728 (64 x 152)
    const int split = p.rows && (long long)pages * p.c.KVH < 64ll * sms ? 4 : 1, fit = kRowWarps / split;
    const int ctas = (p.c.KVH + fit - 1) / fit, heads = (p.c.KVH + ctas - 1) / ctas;
    const dim3 grid(pages, ctas);
    const dim3 block(32 * heads * split);
    if (!write) return launch_pdl(paged_read_kernel<FMT, D>, grid, block, 0, s, p, split, heads);
    return p.c.lohi ? launch_pdl(paged_write_kernel<FMT, D, true>, grid, block, 0, s, p, split, heads)
                    : launch_pdl(paged_write_kernel<FMT, D, false>, grid, block, 0, s, p, split, heads);
}

cudaError_t launch_rows(int fmt, int D, const PagedRowsParams& p, bool write, int sms, cudaStream_t s)
{
    if (fmt == RA_PAGED_FP8) return D == 128 ? launch_rows<RA_PAGED_FP8, 128>(p, write, sms, s) : launch_rows<RA_PAGED_FP8, 64>(p, write, sms, s);
    return D == 128 ? launch_rows<RA_PAGED_BF16, 128>(p, write, sms, s) : launch_rows<RA_PAGED_BF16, 64>(p, write, sms, s);
}

}  // namespace

cudaError_t launch_paged_write(int fmt, int D, const PagedRowsParams& p, int sms, cudaStream_t s)
{
    return launch_rows(fmt, D, p, true, sms, s);
}
cudaError_t launch_paged_read(int fmt, int D, const PagedRowsParams& p, int sms, cudaStream_t s)
{
    return launch_rows(fmt, D, p, false, sms, s);
}
cudaError_t launch_paged_select(int D, PagedSelectParams p, int sms, cudaStream_t s)
{
    // a head's pages over several CTAs while all of them run at once, four on an SM (by CTAs a head, 1, 2, 4 and 8: one sequence of
    // 8 heads and 33k tokens 8.0, 7.5, 6.5 and 5.9 us; four such 8.9, 8.1, 7.2 and 7.2; 16 of up to 31k 13.2, 11.3, 10.8
    // and 13.3; 32 of up to 64k 15.2, 15.0, 16.5 and 21.6)
    p.cluster = 1;
    while (p.cluster < kSelMostCluster && 2 * p.cluster * p.c.KVH * p.c.batch <= 4 * sms) p.cluster *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.c.KVH * p.cluster, p.c.batch);
    cfg.blockDim = dim3(kSelThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = p.cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return D == 128 ? cudaLaunchKernelEx(&cfg, paged_select_kernel<128>, p) : cudaLaunchKernelEx(&cfg, paged_select_kernel<64>, p);
}

}  // namespace ra

// ================================================================================ host side
using namespace ra;

struct ra_paged {
    int L, H, KVH, G, D, page, page_shift, pages, max_batch, max_len, format, bounds;
    int device = -1, sms = 0;
    bool bound = false;
    size_t layer_rows = 0, layer_lohi = 0, layer_exp = 0;  // bytes of one layer
    size_t off_rows = 0, off_lohi = 0, off_lohi8 = 0, off_exp = 0, off_keys = 0, off_partial = 0, off_err = 0;
    size_t bytes = 0;
    uint8_t* arena = nullptr;
    int max_pages = 0;  // of one sequence
    char err[256] = "no error";
};

namespace {

thread_local char g_paged_error[256] = "no error";
constexpr int kPagedMaxSMs = 160;  // sizes the attention's scratch (the GB300 has 152)

int fail(ra_paged* c, int code, const char* fmt, ...) __attribute__((format(printf, 3, 4)));
int fail(ra_paged* c, int code, const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_paged_error, sizeof g_paged_error, fmt, ap);
    va_end(ap);
    if (c) memcpy(c->err, g_paged_error, sizeof c->err);
    return code;
}
int cuda_fail(ra_paged* c, cudaError_t e, const char* what) { return fail(c, RA_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e)); }

size_t up256(size_t x) { return (x + 255) / 256 * 256; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

template <int FMT, int D>
size_t page_bytes(int page)  // of one KV head
{
    using Geo = PagedGeo<FMT, D>;
    return (size_t)(page / Geo::unit_rows(page)) * Geo::unit_stride(Geo::unit_rows(page));
}
size_t page_bytes(int format, int D, int page)
{
    if (format == RA_PAGED_FP8) return D == 128 ? page_bytes<RA_PAGED_FP8, 128>(page) : page_bytes<RA_PAGED_FP8, 64>(page);
    return D == 128 ? page_bytes<RA_PAGED_BF16, 128>(page) : page_bytes<RA_PAGED_BF16, 64>(page);
}

int check_bound(ra_paged* c)
{
    if (!c) return fail(nullptr, RA_ERR_INVALID_ARG, "ctx is NULL");
    if (!c->bound) return fail(c, RA_ERR_STATE, "no device arena bound (call ra_paged_bind first)");
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev != c->device)
        return fail(c, RA_ERR_STATE, "current device %d is not the bound device %d", dev, c->device);
    return RA_OK;
}

// What every call on a layer shares: the layer, the batch and the sequences' tables.
int view(ra_paged* c, int layer, int batch, const int32_t* lens, const int32_t* table, int table_stride, PagedView& v)
{
    int rc;
    if ((rc = check_bound(c)) != RA_OK) return rc;
    if (layer < 0 || layer >= c->L) return fail(c, RA_ERR_INVALID_ARG, "layer %d out of [0, %d)", layer, c->L);
    if (batch < 1 || batch > c->max_batch) return fail(c, RA_ERR_INVALID_ARG, "batch %d out of [1, %d]", batch, c->max_batch);
    if (!lens || !table) return fail(c, RA_ERR_INVALID_ARG, "lens and table must not be NULL");
    if ((reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(table)) & 3u)
        return fail(c, RA_ERR_INVALID_ARG, "lens and table must be 4-byte aligned");
    if (table_stride < 1) return fail(c, RA_ERR_INVALID_ARG, "table_stride %d < 1", table_stride);
    v.rows = c->arena + c->off_rows + layer * c->layer_rows;
    v.lohi = c->bounds ? (uint16_t*)(c->arena + c->off_lohi + layer * c->layer_lohi) : nullptr;
    v.lohi8 = c->bounds ? (int8_t*)(c->arena + c->off_lohi8 + layer * (c->layer_lohi / 2)) : nullptr;
    v.lohi_exp = c->bounds ? c->arena + c->off_exp + layer * c->layer_exp : nullptr;
    v.err = (int32_t*)(c->arena + c->off_err);
    v.lens = lens;
    v.table = table;
    v.KVH = c->KVH;
    v.G = c->G;
    v.page_shift = c->page_shift;
    v.pages = c->pages;
    v.max_len = c->max_len;
    v.batch = batch;
    v.table_stride = table_stride;
    return RA_OK;
}

int check_strides(ra_paged* c, const char* what, long long row, long long head)
{
    if (row < 0 || head < 0 || row % 8 || head % 8)
        return fail(c, RA_ERR_INVALID_ARG, "%s strides (%lld, %lld) must be non-negative multiples of 8 elements", what, row, head);
    return RA_OK;
}

int rows_call(ra_paged* c, int layer, const void* k, const void* v, int64_t row_stride, int64_t head_stride, int batch,
              const int32_t* rows, int n_rows, const int32_t* lens, const int32_t* table, int table_stride, bool write, void* stream)
{
    PagedRowsParams p{};
    int rc = view(c, layer, batch, lens, table, table_stride, p.c);
    if (rc != RA_OK) return rc;
    if (n_rows < 0) return fail(c, RA_ERR_INVALID_ARG, "n_rows %d < 0", n_rows);
    if (!rows && n_rows != batch) return fail(c, RA_ERR_INVALID_ARG, "without rows, n_rows (%d) must be the batch (%d)", n_rows, batch);
    if (reinterpret_cast<uintptr_t>(rows) & 3u) return fail(c, RA_ERR_INVALID_ARG, "rows must be 4-byte aligned");
    if (n_rows == 0) return RA_OK;
    if (!k || !v || !aligned16(k) || !aligned16(v)) return fail(c, RA_ERR_INVALID_ARG, "k and v must be non-NULL and 16-byte aligned");
    if ((rc = check_strides(c, "k / v", row_stride, head_stride)) != RA_OK) return rc;
    if (!write && rows_overlap(row_stride, head_stride, n_rows, c->KVH, c->D))
        return fail(c, RA_ERR_INVALID_ARG, "rows read back would overlap (strides %lld, %lld)", (long long)row_stride, (long long)head_stride);
    if (write) {
        p.k_in = (const uint16_t*)k;
        p.v_in = (const uint16_t*)v;
    } else {
        p.k_out = (uint16_t*)const_cast<void*>(k);
        p.v_out = (uint16_t*)const_cast<void*>(v);
    }
    p.row_stride = row_stride;
    p.head_stride = head_stride;
    p.rows = rows;
    p.n_rows = n_rows;
    const cudaError_t e = write ? launch_paged_write(c->format, c->D, p, c->sms, (cudaStream_t)stream)
                                : launch_paged_read(c->format, c->D, p, c->sms, (cudaStream_t)stream);
    return e == cudaSuccess ? RA_OK : cuda_fail(c, e, write ? "paged write launch" : "paged read launch");
}

int attn_call(ra_paged* c, int layer, const uint16_t* q, int64_t q_row_stride, int64_t q_head_stride, uint16_t* out, float* lse,
              int batch, const int32_t* lens, const int32_t* table, int table_stride, const int32_t* sel, int top, float scale,
              void* stream, uint64_t probe_ns = 0, int probe_share = 0, int probe_tile = 0)
{
    PagedAttnParams p{};
    p.probe_ns = probe_ns;
    p.probe_share = probe_share;
    p.probe_tile = probe_tile;
    int rc = view(c, layer, batch, lens, table, table_stride, p.c);
    if (rc != RA_OK) return rc;
    if (!q || !out || !aligned16(q) || !aligned16(out)) return fail(c, RA_ERR_INVALID_ARG, "q and out must be non-NULL and 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(lse) & 3u) return fail(c, RA_ERR_INVALID_ARG, "lse must be 4-byte aligned");
    if ((rc = check_strides(c, "q", q_row_stride, q_head_stride)) != RA_OK) return rc;
    p.q = q;
    p.q_row_stride = q_row_stride;
    p.q_head_stride = q_head_stride;
    p.out = out;
    p.lse = lse;
    p.sel = sel;
    p.top = top;
    p.scale_log2 = (scale > 0.f ? scale : 1.0f / sqrtf((float)c->D)) * 1.4426950408889634f;
    p.partial = (float*)(c->arena + c->off_partial);
    const cudaError_t e = c->format == RA_PAGED_FP8 ? launch_paged_attn_fp8(c->D, p, c->sms, (cudaStream_t)stream)
                                                    : launch_paged_attn_bf16(c->D, p, c->sms, (cudaStream_t)stream);
    return e == cudaSuccess ? RA_OK : cuda_fail(c, e, "paged attention launch");
}

}  // namespace

extern "C" {

const char* ra_paged_last_error(const ra_paged* c) { return c ? c->err : g_paged_error; }

int ra_paged_create(ra_paged** out, int layers, int q_heads, int kv_heads, int head_dim, int page, int pages, int max_batch,
                    int max_len, int format, int bounds)
{
    if (!out) return fail(nullptr, RA_ERR_INVALID_ARG, "out is NULL");
    *out = nullptr;
    if (layers < 1 || q_heads < 1 || kv_heads < 1 || pages < 1 || max_batch < 1 || max_len < 1)
        return fail(nullptr, RA_ERR_INVALID_ARG, "layers, heads, pages, max_batch and max_len must be at least 1");
    if (q_heads % kv_heads) return fail(nullptr, RA_ERR_INVALID_ARG, "q_heads %d is not a multiple of kv_heads %d", q_heads, kv_heads);
    if (format != RA_PAGED_BF16 && format != RA_PAGED_FP8) return fail(nullptr, RA_ERR_INVALID_ARG, "unknown format %d", format);
    if (head_dim != 64 && head_dim != 128) return fail(nullptr, RA_ERR_UNSUPPORTED, "head_dim %d is not 64 or 128", head_dim);
    if (q_heads / kv_heads > kPagedMaxG)
        return fail(nullptr, RA_ERR_UNSUPPORTED, "%d query heads per KV head, more than %d", q_heads / kv_heads, kPagedMaxG);
    if (page != 16 && page != 32 && page != 64 && page != 128) return fail(nullptr, RA_ERR_UNSUPPORTED, "page %d is not 16, 32, 64 or 128", page);
    if (max_batch > RA_MAX_BATCH) return fail(nullptr, RA_ERR_UNSUPPORTED, "max_batch %d above %d", max_batch, RA_MAX_BATCH);
    if ((long long)pages * kv_heads > 0x7fffffff) return fail(nullptr, RA_ERR_UNSUPPORTED, "pages * kv_heads above 2^31 - 1");
    if (kv_heads > 65535 || layers > 65535) return fail(nullptr, RA_ERR_UNSUPPORTED, "more than 65535 layers or KV heads");
    if (max_len > 1 << 30) return fail(nullptr, RA_ERR_UNSUPPORTED, "max_len %d above 2^30", max_len);
    const int max_pages = (max_len - 1) / page + 1;
    if ((long long)max_batch * kv_heads * max_pages > (1ll << 30) / (page > 16 ? 4 : 1))
        return fail(nullptr, RA_ERR_UNSUPPORTED, "max_batch * kv_heads * max_len too large for 32-bit tile counts");
    if ((double)layers * pages * kv_heads * page * head_dim * 8.0 > 1e13) return fail(nullptr, RA_ERR_UNSUPPORTED, "cache of more than 10 TB");
    ra_paged* c = new (std::nothrow) ra_paged;
    if (!c) return fail(nullptr, RA_ERR_STATE, "out of host memory");
    c->L = layers;
    c->H = q_heads;
    c->KVH = kv_heads;
    c->G = q_heads / kv_heads;
    c->D = head_dim;
    c->page = page;
    c->page_shift = page == 16 ? 4 : page == 32 ? 5 : page == 64 ? 6 : 7;
    c->pages = pages;
    c->max_batch = max_batch;
    c->max_len = max_len;
    c->max_pages = max_pages;
    c->format = format;
    c->bounds = bounds != 0;
    const size_t heads = (size_t)pages * kv_heads;
    c->layer_rows = up256(heads * page_bytes(format, head_dim, page));
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t o = at;
        at += up256(n);
        return o;
    };
    c->off_rows = take(c->layer_rows * layers);
    if (c->bounds) {
        c->layer_lohi = up256(heads * 2 * head_dim) * 2;  // half of it for the 8-bit form, a multiple of 256 too
        c->layer_exp = up256(heads);
        c->off_lohi = take(c->layer_lohi * layers);
        c->off_lohi8 = take(c->layer_lohi / 2 * layers);
        c->off_exp = take(c->layer_exp * layers);
        c->off_keys = take((size_t)max_batch * kv_heads * max_pages * 4);
    }
    c->off_partial = take(format == RA_PAGED_FP8 ? paged_partial_bytes_fp8(c->G, head_dim, kPagedMaxSMs)
                                                 : paged_partial_bytes_bf16(c->G, head_dim, kPagedMaxSMs));
    c->off_err = take(4);
    c->bytes = at;
    *out = c;
    return RA_OK;
}

size_t ra_paged_device_bytes(const ra_paged* c) { return c ? c->bytes : 0; }

int ra_paged_bind(ra_paged* c, void* device_arena, size_t bytes, void* stream)
{
    if (!c) return fail(nullptr, RA_ERR_INVALID_ARG, "ctx is NULL");
    if (!device_arena || (reinterpret_cast<uintptr_t>(device_arena) & 255u))
        return fail(c, RA_ERR_INVALID_ARG, "arena must be a non-NULL 256-byte aligned device pointer");
    if (bytes < c->bytes) return fail(c, RA_ERR_INVALID_ARG, "arena has %zu bytes, need %zu", bytes, c->bytes);
    cudaError_t e;
    cudaPointerAttributes attr{};
    if ((e = cudaPointerGetAttributes(&attr, device_arena)) != cudaSuccess) return cuda_fail(c, e, "arena attributes");
    if (attr.type != cudaMemoryTypeDevice) return fail(c, RA_ERR_INVALID_ARG, "arena is not device memory");
    int dev = -1, sms = 0;
    if ((e = cudaGetDevice(&dev)) != cudaSuccess) return cuda_fail(c, e, "cudaGetDevice");
    if (attr.device != dev) return fail(c, RA_ERR_INVALID_ARG, "arena lives on device %d, current is %d", attr.device, dev);
    if ((e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) return cuda_fail(c, e, "SM count");
    if (sms > kPagedMaxSMs) return fail(c, RA_ERR_UNSUPPORTED, "more than %d SMs", kPagedMaxSMs);
    e = c->format == RA_PAGED_FP8 ? paged_attn_prepare_fp8(c->D, c->page, c->G) : paged_attn_prepare_bf16(c->D, c->page, c->G);
    if (e != cudaSuccess) return cuda_fail(c, e, "attention kernel attributes");
    uint8_t* a = (uint8_t*)device_arena;
    // the error word; rows and bounds are written before they are read
    if ((e = cudaMemsetAsync(a + c->off_err, 0, 4, (cudaStream_t)stream)) != cudaSuccess)
        return cuda_fail(c, e, "arena initialisation");
    c->arena = a;
    c->device = dev;
    c->sms = sms;
    c->bound = true;
    return RA_OK;
}

int ra_paged_write(ra_paged* c, int layer, const uint16_t* k, const uint16_t* v, int64_t row_stride, int64_t head_stride, int batch,
                   const int32_t* rows, int n_rows, const int32_t* lens, const int32_t* table, int table_stride, void* stream)
{
    return rows_call(c, layer, k, v, row_stride, head_stride, batch, rows, n_rows, lens, table, table_stride, true, stream);
}

int ra_paged_read(ra_paged* c, int layer, uint16_t* k, uint16_t* v, int64_t row_stride, int64_t head_stride, int batch,
                  const int32_t* rows, int n_rows, const int32_t* lens, const int32_t* table, int table_stride, void* stream)
{
    return rows_call(c, layer, k, v, row_stride, head_stride, batch, rows, n_rows, lens, table, table_stride, false, stream);
}

int ra_paged_attn(ra_paged* c, int layer, const uint16_t* q, int64_t q_row_stride, int64_t q_head_stride, uint16_t* out, float* lse,
                  int batch, const int32_t* lens, const int32_t* table, int table_stride, float scale, void* stream)
{
    return attn_call(c, layer, q, q_row_stride, q_head_stride, out, lse, batch, lens, table, table_stride, nullptr, 0, scale, stream);
}

int ra_paged_select(ra_paged* c, int layer, const uint16_t* q, int64_t q_row_stride, int64_t q_head_stride, int batch,
                    const int32_t* lens, const int32_t* table, int table_stride, int top, int first, int last, int32_t* sel,
                    void* stream)
{
    PagedSelectParams p{};
    int rc = view(c, layer, batch, lens, table, table_stride, p.c);
    if (rc != RA_OK) return rc;
    if (!c->bounds) return fail(c, RA_ERR_STATE, "the cache was created without bounds");
    if (!q || !aligned16(q)) return fail(c, RA_ERR_INVALID_ARG, "q must be non-NULL and 16-byte aligned");
    if ((rc = check_strides(c, "q", q_row_stride, q_head_stride)) != RA_OK) return rc;
    if (top < 1 || top > RA_PAGED_MAX_TOP) return fail(c, RA_ERR_INVALID_ARG, "top %d out of [1, %d]", top, RA_PAGED_MAX_TOP);
    if (first < 0 || last < 0 || (long long)first + last > top)
        return fail(c, RA_ERR_INVALID_ARG, "first %d and last %d must be non-negative and at most top %d together", first, last, top);
    if (!sel || (reinterpret_cast<uintptr_t>(sel) & 3u)) return fail(c, RA_ERR_INVALID_ARG, "sel must be non-NULL and 4-byte aligned");
    p.q = q;
    p.q_row_stride = q_row_stride;
    p.q_head_stride = q_head_stride;
    p.top = top;
    p.first = first;
    p.last = last;
    p.sel = sel;
    p.keys = (uint32_t*)(c->arena + c->off_keys);
    p.max_pages = c->max_pages;
    const cudaError_t e = launch_paged_select(c->D, p, c->sms, (cudaStream_t)stream);
    return e == cudaSuccess ? RA_OK : cuda_fail(c, e, "paged select launch");
}

int ra_paged_sparse_attn(ra_paged* c, int layer, const uint16_t* q, int64_t q_row_stride, int64_t q_head_stride, uint16_t* out,
                         float* lse, int batch, const int32_t* lens, const int32_t* table, int table_stride, const int32_t* sel,
                         int top, float scale, void* stream)
{
    if (!c) return fail(nullptr, RA_ERR_INVALID_ARG, "ctx is NULL");
    if (!sel || (reinterpret_cast<uintptr_t>(sel) & 3u)) return fail(c, RA_ERR_INVALID_ARG, "sel must be non-NULL and 4-byte aligned");
    if (top < 1 || top > RA_PAGED_MAX_TOP) return fail(c, RA_ERR_INVALID_ARG, "top %d out of [1, %d]", top, RA_PAGED_MAX_TOP);
    return attn_call(c, layer, q, q_row_stride, q_head_stride, out, lse, batch, lens, table, table_stride, sel, top, scale, stream);
}

int ra_paged_debug_timeout_probe(ra_paged* c, int layer, const uint16_t* q, int64_t q_row_stride, int64_t q_head_stride, uint16_t* out,
                                 float* lse, int batch, const int32_t* lens, const int32_t* table, int table_stride, int share, int tile,
                                 uint64_t limit_ns, void* stream)
{
    if (!c) return fail(nullptr, RA_ERR_INVALID_ARG, "ctx is NULL");
    if (c->D != 64 || c->page != 16 || c->G > 8)
        return fail(c, RA_ERR_UNSUPPORTED, "the probe is built for heads of 64 channels, pages of 16 and at most 8 query heads per KV head");
    if (limit_ns < 1000ull || limit_ns > 100000000ull)
        return fail(c, RA_ERR_INVALID_ARG, "limit_ns %llu outside [1e3, 1e8]", (unsigned long long)limit_ns);
    if (share < 0 || tile < 0) return fail(c, RA_ERR_INVALID_ARG, "share %d and tile %d must not be negative", share, tile);
    return attn_call(c, layer, q, q_row_stride, q_head_stride, out, lse, batch, lens, table, table_stride, nullptr, 0, 0.f, stream, limit_ns,
                     share, tile);
}

int ra_paged_check(ra_paged* c, void* stream)
{
    int rc;
    if ((rc = check_bound(c)) != RA_OK) return rc;
    const cudaStream_t s = (cudaStream_t)stream;
    int32_t* word = (int32_t*)(c->arena + c->off_err);
    cudaError_t e;
    if ((e = cudaStreamSynchronize(s)) != cudaSuccess) return cuda_fail(c, e, "stream sync");
    int32_t w = 0;
    if ((e = cudaMemcpy(&w, word, 4, cudaMemcpyDeviceToHost)) != cudaSuccess) return cuda_fail(c, e, "err read");
    if (w != 0 && ((e = cudaMemsetAsync(word, 0, 4, s)) != cudaSuccess || (e = cudaStreamSynchronize(s)) != cudaSuccess))  // reported once
        return cuda_fail(c, e, "err clear");
    if (w & kDeviceErrTimeout) return fail(c, RA_ERR_DEVICE_TIMEOUT, "a kernel gave up a bounded wait");
    if (w & kPagedErrInput) return fail(c, RA_ERR_INVALID_ARG, "a length, row count, page or page index on the device was out of range");
    if (w != 0) return fail(c, RA_ERR_STATE, "device error word %d", w);
    return RA_OK;
}

void ra_paged_destroy(ra_paged* c) { delete c; }

}  // extern "C"
