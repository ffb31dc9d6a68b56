// ra_paged_attn.cu -- attention of one new token per sequence over a paged cache (built once per format, see RA_PAGED_FMT).
//
// The rows of every (sequence, KV head) are cut into tiles, all tiles of the launch are laid end to end, and every warp
// takes an equal share of them.  It makes one pass over its K and V rows with a running maximum and sum per query head, and
// crosses from head to head as it goes.  What bounds it is memory: 2 D bytes (8 bits) or 4 D bytes per row are read once for
// all G query heads.  So each warp keeps a ring of tiles in flight (one bulk copy per unit of a page, issued by the
// lane that looked the page up) and works on the oldest, on mma.sync, transposed (S^T = K Q^T, O^T += V^T P^T: 16 rows of the
// cache by 8 query heads, so that a group of up to 8 leaves little of the operands unused): a few hundred instructions a
// tile, where its bytes take an SM several hundred clocks to fetch.
//   bf16:  weights in two bf16 parts (nearest, and what that left out), in products of their own.
//   8 bits: codes become f16 (exactly) in registers, queries f16 at a power of two of their row (exactly, but for
//          channels below 2^-31 of the largest, which keep steps of 2^-38 of it), weights in two f16 parts (22 bits; with one,
//          11 bits, values that cancel showed it).  A row's power-of-two scales go to its logit (K) and its
//          weight (V); the unit of the sums of values follows logit + log2 of the V scale, so that a weight fits f16
//          whatever the scale.  (8-bit operands, queries in three parts, took more instructions than the kernel then
//          had, 808 per tile of 32 rows against 603; it has 488 now.)
// A head that lies in one share is written by its warp; the parts of the others go to records that a second kernel
// joins, which is on the SMs by then and starts as the first one ends.
// Measured, the join included: 1.19 GB of 48 ragged sequences in 8 bits (4 query heads per KV head) 183 us, 6.5 TB/s, 0.96
// of a copy's rate; 1.22 GB of 32 sequences in bf16 (8 heads) 179 us, 6.8 TB/s, 1.00; 0.27 GB of one sequence of 131k rows
// 51.5 us, 5.2 TB/s; one of 577 rows 7.3 us, of which 1.5 us pass before the first copy and 2.8 us in the join.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "ra_internal.h"
#include "ra_paged.h"
#include "ra_ptx.cuh"

#ifndef RA_PAGED_FMT
#error "build with -DRA_PAGED_FMT=0 (bf16) or 1 (8 bits)"
#endif

namespace ra {
namespace {

constexpr unsigned kAll = 0xffffffffu;
constexpr uint64_t kWaitLimitNs = 2000000000ull;  // bounded mbarrier waits: 2 s
// 16 KB (bf16 rows of 128 channels) or 8 KB tiles, two per warp: 128 KB under way on an SM.  With three per warp 48 ragged
// sequences in 8 bits take 195 us (182 with two), 131k rows of one user 54 (51.6), 32 sequences of 9280 rows in bf16 185 (180).  Warps, by
// time: the 48 sequences 256 us with 4, 197 with 6, 182 with 8, 196 with 10 and 191 with 12; the one user 55, 51.5, 51.6, 55 and 60; the 32 in bf16
// 180 with 3, 180 with 4, 179 with 5 and 181 with 6, 16 of 2000 rows 27.5, 26.7, 28.1 and 28.2.
constexpr int kStages = 2;
template <int D>
constexpr int kWarps = PagedGeo<RA_PAGED_FMT, D>::kRow == 256 ? 4 : 8;
constexpr size_t kSmemMost = 224 * 1024;

__device__ __forceinline__ void ldsm_x4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
__device__ __forceinline__ void ldsm_x4_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr));
}
// C[16x8] += A[16x16] B[16x8], 32-bit accumulators
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
#if RA_PAGED_FMT == 1
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
#else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
#endif
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&r);
}
[[maybe_unused]] __device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 r = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&r);
}
// two e4m3 codes -> two f16 (exact)
[[maybe_unused]] __device__ __forceinline__ uint32_t codes_f16(uint32_t two)
{
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
    return r;
}
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// over the 8 lanes that share a pair of heads
__device__ __forceinline__ float rows_max(float x)
{
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) x = fmaxf(x, __shfl_xor_sync(kAll, x, o));
    return x;
}
__device__ __forceinline__ float rows_sum(float x)
{
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) x += __shfl_xor_sync(kAll, x, o);
    return x;
}
// Transpose of an 8x8 matrix of 16-bit values (lane l: row l / 4, columns 2 (l % 4) + {0, 1}).
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// The reference m of a head's weights is set kAbove over the largest logit so far (log2 units) and moves (what is summed
// being rescaled) only when one passes it: weights stay at or below 1, as V rows of up to 2^128 would take larger ones out
// of 32 bits.  8 bits: the second product takes a weight times its row's V scale, in f16; the unit of its sums is 2^u, u set
// kBelow under the largest logit + log2 of the V scale so far, moved when one could pass it by kHigh.  The sum of the
// softmax keeps to m: with one reference for both, the rows beside a V row of 2^100 and more fell below 32 bits.
constexpr float kAbove = 8.f, kHigh = 14.f, kBelow = 6.f;

// A record: o [G][D] (not divided), m [G], l [G], whether any row counted, 8 bits: u [G]; floats, a multiple of 4.
__host__ __device__ constexpr int record_floats(int G, int D)
{
    return G * D + ((RA_PAGED_FMT == RA_PAGED_FP8 ? 3 : 2) * G + 1 + 3) / 4 * 4;
}

struct Work {  // the launch's tiles in a CTA's shared memory
    int32_t pre[RA_MAX_BATCH + 1];  // tiles before sequence b
    int32_t n[RA_MAX_BATCH];        // tiles of one KV head
    int32_t len[RA_MAX_BATCH];
    int32_t sum[32];
};

// The launch's tiles in equal shares, one per warp (fewer where there are fewer tiles), numbered in the order of the tiles.
// (Shares of which the last quarter was cut again, to be claimed by warps that were done, gained 20 us of 200 while three
// tiles per warp were in flight; with two, SMs keep pace: 48 ragged sequences 185 us equal and 186 claimed, 16 sequences of
// 16 query heads per KV head 161 and 188, their records being five times as many.)
struct Split {
    int W, share, longer;  // the first `longer` shares have a tile more
    __device__ __forceinline__ Split(int tiles, int warps)
    {
        W = min(warps, tiles);
        share = tiles / max(W, 1);
        longer = tiles - share * W;
    }
    __device__ __forceinline__ int begin(int w) const { return w * share + min(w, longer); }
    __device__ __forceinline__ int of(int tile) const
    {
        const int head = longer * (share + 1);
        return tile < head ? tile / (share + 1) : longer + (tile - head) / share;
    }
};

struct Smem {  // offsets into dynamic shared memory
    int bars, meta, work, total;
};
__host__ __device__ constexpr Smem smem_of(int stage_bytes, int warps)
{
    Smem s{};
    s.bars = warps * kStages * stage_bytes;
    s.meta = s.bars + warps * kStages * 8;
    s.work = s.meta + warps * kStages * 4;
    s.total = s.work + (int)sizeof(Work);
    return s;
}

// Tiles per sequence and their prefix sums, by NT threads (up to 32 sequences: by the first warp).
template <int NT>
__device__ __forceinline__ void count_tiles(const PagedAttnParams& p, int T, Work& work)
{
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, page = 1 << p.c.page_shift;
    auto tiles_of = [&](int b) {
        const int len = paged_len(p.c, b);
        work.len[b] = len;
        int rows = len;
        if (p.sel) rows = min(p.top, (len + page - 1) >> p.c.page_shift) << p.c.page_shift;
        work.n[b] = (rows + T - 1) / T;
        return work.n[b] * p.c.KVH;
    };
    auto scan = [&](int x) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(kAll, x, o);
            if (lane >= o) x += y;
        }
        return x;
    };
    if (p.c.batch <= 32) {
        if (warp == 0) {
            const int mine = lane < p.c.batch ? tiles_of(lane) : 0, inc = scan(mine);
            if (lane < p.c.batch) work.pre[lane] = inc - mine;
            if (lane == 31) work.pre[p.c.batch] = inc;
        }
        __syncthreads();
        return;
    }
    constexpr int per = (RA_MAX_BATCH + NT - 1) / NT;
    int tiles[per], mine = 0;
#pragma unroll
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        tiles[i] = b < p.c.batch ? tiles_of(b) : 0;
        mine += tiles[i];
    }
    const int inc = scan(mine);
    if (lane == 31) work.sum[warp] = inc;
    __syncthreads();
    int at = inc - mine;
    for (int w = 0; w < warp; ++w) at += work.sum[w];
#pragma unroll
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        if (b < p.c.batch) work.pre[b] = at;
        at += tiles[i];
    }
    if (tid == NT - 1) work.pre[p.c.batch] = at;  // (the last thread's sum is the total)
    __syncthreads();
}

// Which tile of which head a position in the launch's tiles is.
struct Cursor {
    int b, h, t, n;  // sequence, KV head, tile of the head, tiles per head
    __device__ __forceinline__ void seek(const Work& w, int batch, int at)
    {
        int lo = 0, hi = batch;  // largest b with pre[b] <= at
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (w.pre[mid] <= at) lo = mid;
            else hi = mid;
        }
        b = lo;
        n = w.n[b];
        const int rem = at - w.pre[b];
        h = rem / n;
        t = rem - h * n;
    }
    __device__ __forceinline__ void next(const Work& w, int KVH, int batch)
    {
        if (++t < n) return;
        t = 0;
        if (++h < KVH) return;
        h = 0;
        do ++b;
        while (b < batch && w.pre[b + 1] == w.pre[b]);
        if (b < batch) n = w.n[b];
    }
};

// What a head (all of it, or its part in record `rec`) reads as when its rows did not arrive: NaN, not an earlier call's values.
__device__ __noinline__ void lost(const PagedAttnParams& p, int lane, int D, const Cursor& head, bool whole, float* rec)
{
    const int G = p.c.G;
    const long long row0 = ((long long)head.b * p.c.KVH + head.h) * G;
    for (int i = lane; i < G * D; i += 32) {
        if (whole) p.out[row0 * D + i] = 0x7fffu;
        else rec[i] = NAN;
    }
    for (int i = lane; i < G; i += 32) {
        if (whole && p.lse) p.lse[row0 + i] = NAN;
        if (whole) continue;
        rec[G * D + i] = 0.f;
        rec[G * D + G + i] = NAN;
        if (RA_PAGED_FMT == RA_PAGED_FP8) rec[G * D + 2 * G + 1 + i] = 0.f;
    }
    if (!whole && lane == 0) rec[G * D + 2 * G] = 1.f;
}

// The running state of a head's rows: NH sets of 8 query heads.  This lane (gq = lane / 4, t = lane % 4): heads 2 t and
// 2 t + 1 of a set; of O^T's 16 channels i the rows gq and gq + 8.
template <int D, int NH>
struct Piece {
    static constexpr bool kSplit = RA_PAGED_FMT == RA_PAGED_BF16;  // R: the weights' second parts
    float O[NH][D / 16][4];
    float R[kSplit ? NH : 1][kSplit ? D / 16 : 1][4];
    float m[NH][2], l[NH][2];
    float u[kSplit ? 1 : NH][2], down[kSplit ? 1 : NH][2];  // down: 2^(m - u), a power of two
    int any;
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int s = 0; s < NH; ++s) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    O[s][i][e] = 0.f;
                    if constexpr (kSplit) R[s][i][e] = 0.f;
                }
            m[s][0] = m[s][1] = -INFINITY;
            l[s][0] = l[s][1] = 0.f;
            if constexpr (!kSplit) {
                u[s][0] = u[s][1] = -INFINITY;
                down[s][0] = down[s][1] = 1.f;
            }
        }
        any = 0;
    }
    __device__ __forceinline__ float value(int s, int i, int e) const
    {
        if constexpr (kSplit) return isinf(O[s][i][e]) ? O[s][i][e] : O[s][i][e] + R[s][i][e];  // (infinity times a part of zero: NaN)
        else return O[s][i][e];
    }
    __device__ __forceinline__ void rescale(int s, int hd, float f)
    {
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int e = hd; e < 4; e += 2) {
                O[s][i][e] *= f;
                if constexpr (kSplit) R[s][i][e] *= f;
            }
    }
    // f(set, 0 or 1, head, channel, value) over this lane's part of the output
    template <typename F>
    __device__ __forceinline__ void each(int lane, int G, F f) const
    {
        const int gq = lane >> 2, t = lane & 3;
#pragma unroll
        for (int s = 0; s < NH; ++s)
#pragma unroll
            for (int hd = 0; hd < 2; ++hd) {
                const int head = 8 * s + 2 * t + hd;
                if (head >= G) continue;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {  // 8 bits: rows gq, gq + 8 are channels 2 gq, 2 gq + 1 (as the codes lie)
                    f(s, hd, head, 16 * i + (kSplit ? gq : 2 * gq), value(s, i, hd));
                    f(s, hd, head, 16 * i + (kSplit ? gq + 8 : 2 * gq + 1), value(s, i, 2 + hd));
                }
            }
    }
};

// PROBE: a test's launch, in which one tile of a share expects more bytes than are copied, so that its wait runs out.
template <int D, int U, int NH, bool PROBE>
__global__ void __launch_bounds__(32 * kWarps<D>, 1) paged_attn_kernel(const PagedAttnParams p)
{
    using Geo = PagedGeo<RA_PAGED_FMT, D>;
    constexpr bool FP8 = RA_PAGED_FMT == RA_PAGED_FP8;
    constexpr int T = Geo::kTile, NU = T / U, UB = Geo::unit_stride(U), STAGE = NU * UB, ROW = Geo::kRow;
    constexpr int KS = D / 16;  // k-steps of K Q^T
    constexpr int W = kWarps<D>;
    extern __shared__ __align__(128) uint8_t smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, G = p.c.G, KVH = p.c.KVH;
    const Smem lay = smem_of(STAGE, W);
    Work& work = *reinterpret_cast<Work*>(smem + lay.work);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem + lay.bars) + warp * kStages;
    uint32_t* meta = reinterpret_cast<uint32_t*>(smem + lay.meta) + warp * kStages;  // rows of a tile that count, a byte per unit
    uint8_t* ring = smem + warp * kStages * STAGE;
    const int page = 1 << p.c.page_shift;

    if (lane == 0)
        for (int s = 0; s < kStages; ++s) mbar_init(&bars[s], 1);
    fence_mbar_init();
    {
        const int i = blockIdx.x * blockDim.x + threadIdx.x, n = gridDim.x * blockDim.x;
        prefetch_sequences(p.c, i, n);
        prefetch_heads(p.q, p.q_row_stride, p.q_head_stride, KVH * G, D, p.c.batch, i, n);
        if (p.sel) prefetch_lines(p.sel, 4ll * p.c.batch * KVH * p.top, i, n);
    }
    pdl_wait();
    count_tiles<32 * W>(p, T, work);
    const int H = KVH * G;
    const Split split(work.pre[p.c.batch], gridDim.x * W);
    const int mine = warp * gridDim.x + blockIdx.x;  // (few shares: over as many SMs as there are)
    pdl_launch_dependents();  // the join may come onto the SMs (with a warp's last fetch instead: no difference)
    if (mine >= split.W) return;

    {
        const int end = split.begin(mine + 1);
        int at = split.begin(mine);  // the next tile to be fetched
        const int tiles = end - at;
        // ---- units: 32 looked up at a time, one per lane; the next 32 are under way while these are copied (their
        // page is not touched until then, so that nothing waits for the table)
        struct Unit {
            int page, sub, rows;  // pool page, unit of the page's units of all heads, rows that count
        };
        auto look_up = [&](int first) {  // of the share's tiles from `first` on
            Unit u{-1, 0, 0};
            const int tile = first + lane / NU;
            if (tile >= end) return u;
            Cursor c;
            c.seek(work, p.c.batch, tile);
            const int row = c.t * T + lane % NU * U, len = work.len[c.b];
            int i = row >> p.c.page_shift;
            const int pages = (len + page - 1) >> p.c.page_shift;
            if (p.sel) {
                if (i >= min(p.top, pages)) return u;
                i = p.sel[((long long)c.b * KVH + c.h) * p.top + i];
                if (i < -1 || i >= pages) atomicOr(p.c.err, kPagedErrInput);
                if (i < 0) return u;
            }
            if (i >= pages) return u;
            const int in_page = row & (page - 1), left = len - (i << p.c.page_shift) - in_page;
            if (left <= 0) return u;
            u.page = p.c.table[(long long)c.b * p.c.table_stride + i];
            u.sub = (c.h << p.c.page_shift) / U + in_page / U;
            u.rows = min(left, U);
            return u;
        };
        const uint8_t* src = nullptr;
        int rows = 0;
        auto resolve = [&](const Unit& u) {
            rows = u.rows;
            if (rows > 0 && (u.page < 0 || u.page >= p.c.pages)) {
                atomicOr(p.c.err, kPagedErrInput);
                rows = 0;
            }
            src = rows > 0 ? p.c.rows + ((long long)u.page * KVH * (page / U) + u.sub) * UB : nullptr;
        };
        resolve(look_up(at));
        Unit ahead{-1, 0, 0};  // (of the first batch: after its first copies)
        int in_batch = 0, issued = 0, next_stage = 0;
        auto issue = [&]() {  // the next tile's copies into its stage
            if (in_batch == 32) {
                resolve(ahead);
                ahead = look_up(at + 32 / NU);
                in_batch = 0;
            }
            const int st = next_stage;
            if (++next_stage == kStages) next_stage = 0;
            const int j = lane - in_batch;
            const bool live = j >= 0 && j < NU && rows > 0;
            const unsigned mask = __ballot_sync(kAll, live);
            if (lane == 0) {
                meta[st] = 0;
                const int never = PROBE && mine == p.probe_share && issued == p.probe_tile ? 16 : 0;
                mbar_arrive_expect_tx(&bars[st], __popc(mask) * Geo::unit_bytes(U) + never);
            }
            __syncwarp();
            if (live) {
                reinterpret_cast<uint8_t*>(&meta[st])[j] = (uint8_t)rows;
                bulk_load(ring + st * STAGE + j * UB, src, Geo::unit_bytes(U), &bars[st]);
            }
            in_batch += NU;
            ++at;
            ++issued;
        };
        while (issued < kStages && issued < tiles) issue();
        ahead = look_up(at - issued + 32 / NU);

        // ---- the warp's tiles
        Cursor cur;
        const int gq = lane >> 2, t = lane & 3, mi = lane >> 3, ri = lane & 7;
        uint32_t qb[NH][KS][2];
        float qs[NH][2];  // logit = accumulator * qs, this lane's heads
        Piece<D, NH> st;
        cur.seek(work, p.c.batch, end - tiles);
        bool from_start = cur.t == 0, fresh = true;
        int stage = -1;
        uint32_t parity = 1;
        for (int it = 0; it < tiles; ++it) {
            if (++stage == kStages) stage = 0;
            if (stage == 0) parity ^= 1;
            if (fresh) {
                fresh = false;
                st.clear();
                const uint16_t* q = p.q + cur.b * p.q_row_stride + (long long)cur.h * G * p.q_head_stride;
#pragma unroll
                for (int o = 0; o < NH; ++o) {  // lane: query head 8 o + gq
                    const bool live = 8 * o + gq < G;
                    const uint16_t* row = q + (8 * o + gq) * p.q_head_stride;
                    if constexpr (FP8) {  // k-step kk: channels 16 kk + 4 t .. + 3, as the codes lie
                        uint2 x[KS];
                        uint32_t amax = 0;
#pragma unroll
                        for (int kk = 0; kk < KS; ++kk) {
                            x[kk] = live ? *reinterpret_cast<const uint2*>(row + 16 * kk + 4 * t) : make_uint2(0, 0);
                            const uint32_t a = __vmaxu2(x[kk].x & 0x7fff7fffu, x[kk].y & 0x7fff7fffu);
                            amax = max(amax, max(a & 0xffffu, a >> 16));
                        }
                        amax = max(amax, __shfl_xor_sync(kAll, amax, 1));
                        amax = max(amax, __shfl_xor_sync(kAll, amax, 2));
                        const int e = max((int)(amax >> 7) - 127, -110);
                        const float up = exp2i(14 - e);
                        const float f = amax < 0x7f80u ? p.scale_log2 * exp2i(e - 14) : NAN;
                        qs[o][0] = __shfl_sync(kAll, f, 8 * t);
                        qs[o][1] = __shfl_sync(kAll, f, 8 * t + 4);
#pragma unroll
                        for (int kk = 0; kk < KS; ++kk) {
                            qb[o][kk][0] = pack_f16(bf16lo(x[kk].x) * up, bf16hi(x[kk].x) * up);
                            qb[o][kk][1] = pack_f16(bf16lo(x[kk].y) * up, bf16hi(x[kk].y) * up);
                        }
                    } else {
                        qs[o][0] = qs[o][1] = p.scale_log2;
#pragma unroll
                        for (int kk = 0; kk < KS; ++kk) {
                            qb[o][kk][0] = live ? *reinterpret_cast<const uint32_t*>(row + 16 * kk + 2 * t) : 0u;
                            qb[o][kk][1] = live ? *reinterpret_cast<const uint32_t*>(row + 16 * kk + 8 + 2 * t) : 0u;
                        }
                    }
                }
            }
            const uint64_t limit_ns = PROBE ? p.probe_ns : kWaitLimitNs;
            if (!__all_sync(kAll, mbar_wait_bounded(&bars[stage], parity, limit_ns))) {  // (the lanes leave together or not at all)
                // Give up: flag it, let the copies already issued land (bounded), leave NaN for the rest of the share.
                if (lane == 0) atomicOr(p.c.err, kDeviceErrTimeout);
                for (int u = it + 1; u < issued; ++u)
                    (void)mbar_wait_bounded(&bars[u % kStages], (uint32_t)((u / kStages) & 1), limit_ns);
                for (int left = tiles - it, n; left > 0; left -= n) {
                    n = min(cur.n - cur.t, left);
                    lost(p, lane, D, cur, from_start && cur.t + n == cur.n,
                         p.partial + ((long long)mine * 2 + (from_start ? 1 : 0)) * record_floats(G, D));
                    from_start = true;
                    cur.t += n - 1;
                    cur.next(work, KVH, p.c.batch);
                }
                return;
            }
            __syncwarp();
            uint8_t* tile = ring + stage * STAGE;
            const uint32_t base = smem_u32(tile);
            const uint32_t valid = meta[stage];
            constexpr uint32_t kFull = NU == 1 ? U : NU == 2 ? U * 0x101u : U * 0x1010101u;
            const bool full = valid == kFull;
            st.any |= valid != 0;
            // rows of the tile: unit r / U, row r % U of it
            auto counts = [&](int r) { return full || (r % U) < (int)((valid >> (8 * (r / U))) & 255u); };
            if (!full) {  // weights of rows that do not count are 0: their V (and its scale) must be finite
#pragma unroll 4
                for (int i = lane; i < T * (ROW / 16); i += 32) {
                    const int r = i / (ROW / 16), c = i % (ROW / 16);
                    if (!counts(r)) *reinterpret_cast<uint4*>(tile + r / U * UB + U * ROW + (r % U) * ROW + 16 * c) = make_uint4(0, 0, 0, 0);
                }
                if constexpr (FP8)
                    for (int r = lane; r < T; r += 32)
                        if (!counts(r)) tile[r / U * UB + 2 * U * ROW + U + r % U] = 0;
                fence_proxy_async_smem();
                __syncwarp();
            }
            // ---- S^T = K Q^T, 16 rows at a time: this lane's rows 16 i + gq and + 8, heads 2 t and 2 t + 1
            float s[T / 16][NH][4];
#pragma unroll
            for (int i = 0; i < T / 16; ++i) {
                const uint32_t krow = base + (i * 16) / U * UB;
                const int r = (i * 16) % U + (mi & 1) * 8 + ri;
                float y[NH][4];  // a second chain
#pragma unroll
                for (int o = 0; o < NH; ++o)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[i][o][e] = y[o][e] = 0.f;
#pragma unroll
                for (int c = 0; c < ROW / 16; c += 2) {
                    uint32_t k[4];  // rows 0-7 and 8-15 at chunk c, then at chunk c + 1
                    ldsm_x4(k, krow + Geo::chunk(r, c + (mi >> 1)));
                    if constexpr (FP8) {
                        const uint32_t a[4] = {codes_f16(k[0] & 0xffffu), codes_f16(k[1] & 0xffffu), codes_f16(k[0] >> 16), codes_f16(k[1] >> 16)};
                        const uint32_t b[4] = {codes_f16(k[2] & 0xffffu), codes_f16(k[3] & 0xffffu), codes_f16(k[2] >> 16), codes_f16(k[3] >> 16)};
#pragma unroll
                        for (int o = 0; o < NH; ++o) {
                            mma(s[i][o], a, qb[o][c][0], qb[o][c][1]);
                            mma(y[o], b, qb[o][c + 1][0], qb[o][c + 1][1]);
                        }
                    } else {
#pragma unroll
                        for (int o = 0; o < NH; ++o) mma(c & 2 ? y[o] : s[i][o], k, qb[o][c / 2][0], qb[o][c / 2][1]);
                    }
                }
#pragma unroll
                for (int o = 0; o < NH; ++o)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[i][o][e] += y[o][e];
            }
            // ---- logits (log2 units)
            float vs[FP8 ? T / 16 : 1][2];  // scales of this lane's V rows
            float top[NH][2];
#pragma unroll
            for (int o = 0; o < NH; ++o) top[o][0] = top[o][1] = -INFINITY;
#pragma unroll
            for (int i = 0; i < T / 16; ++i) {
                if constexpr (FP8) {
                    const uint8_t* sc = tile + (i * 16) / U * UB + 2 * U * ROW + (i * 16) % U + gq;
                    const float k0 = __uint_as_float((uint32_t)sc[0] << 23), k1 = __uint_as_float((uint32_t)sc[8] << 23);
                    vs[i][0] = __uint_as_float((uint32_t)sc[U] << 23);
                    vs[i][1] = __uint_as_float((uint32_t)sc[U + 8] << 23);
#pragma unroll
                    for (int o = 0; o < NH; ++o)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[i][o][e] *= (e < 2 ? k0 : k1) * qs[o][e & 1];  // (the scales first: neither may overflow alone)
                } else {
#pragma unroll
                    for (int o = 0; o < NH; ++o)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[i][o][e] *= qs[o][e & 1];
                }
                if (!full) {
                    const bool ok0 = counts(i * 16 + gq), ok1 = counts(i * 16 + gq + 8);
#pragma unroll
                    for (int o = 0; o < NH; ++o)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[i][o][e] = (e < 2 ? ok0 : ok1) ? s[i][o][e] : -INFINITY;
                }
#pragma unroll
                for (int o = 0; o < NH; ++o) {
                    top[o][0] = fmaxf(top[o][0], fmaxf(s[i][o][0], s[i][o][2]));
                    top[o][1] = fmaxf(top[o][1], fmaxf(s[i][o][1], s[i][o][3]));
                }
            }
            // The references move only when they have to.  8 bits: this lane's largest V scale bounds its rows' weights, and only
            // where that is too much is each row's own looked at.
            float room = 0.f;
            if constexpr (FP8) {
                int e = 0;
#pragma unroll
                for (int i = 0; i < T / 16; ++i) e = max(e, max(__float_as_int(vs[i][0]), __float_as_int(vs[i][1])));
                room = (float)((e >> 23) - 127);
            }
            bool raise = false;
#pragma unroll
            for (int o = 0; o < NH; ++o)
#pragma unroll
                for (int hd = 0; hd < 2; ++hd) {
                    raise = raise || top[o][hd] > st.m[o][hd];
                    if constexpr (FP8) raise = raise || top[o][hd] + room > st.u[o][hd] + kHigh;
                }
            if (__any_sync(kAll, raise)) {
#pragma unroll
                for (int o = 0; o < NH; ++o)
#pragma unroll
                    for (int hd = 0; hd < 2; ++hd) {
                        const float x = rows_max(top[o][hd]), m = st.m[o][hd];
                        const float mn = x > m ? x + kAbove : m;
                        if (mn != m) {
                            st.l[o][hd] *= ex2(m - mn);
                            st.m[o][hd] = mn;
                        }
                        if constexpr (FP8) {
                            float y = -INFINITY;
#pragma unroll
                            for (int i = 0; i < T / 16; ++i)
#pragma unroll
                                for (int e = 0; e < 2; ++e)
                                    y = fmaxf(y, s[i][o][2 * e + hd] + (float)((__float_as_int(vs[i][e]) >> 23) - 127));
                            y = rows_max(y);
                            const float u = st.u[o][hd];
                            if (mn != m || y > u + kBelow) {
                                float c = rintf((y > u + kBelow ? y - kBelow : u) - mn);
                                if (!(fabsf(c) < 126.f)) c = 0.f;  // (no finite logit; else within -75 to 115: a V scale, kBelow, kAbove)
                                st.u[o][hd] = mn + c;
                                st.down[o][hd] = exp2i(-(int)c);
                                st.rescale(o, hd, ex2(u - (mn + c)));
                            }
                        } else if (mn != m) {
                            st.rescale(o, hd, ex2(m - mn));
                        }
                    }
            }
            float ref[NH][2];  // (no finite logit yet: every weight is 0)
#pragma unroll
            for (int o = 0; o < NH; ++o)
#pragma unroll
                for (int hd = 0; hd < 2; ++hd) ref[o][hd] = st.m[o][hd] == -INFINITY ? 0.f : st.m[o][hd];
            // ---- weights and O^T += V^T P^T, 16 rows at a time
#pragma unroll
            for (int i = 0; i < T / 16; ++i) {
                uint32_t w[NH][2], left[NH][2];
#pragma unroll
                for (int o = 0; o < NH; ++o)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const float x = ex2(s[i][o][2 * half] - ref[o][0]);
                        const float y = ex2(s[i][o][2 * half + 1] - ref[o][1]);
                        st.l[o][0] += x;
                        st.l[o][1] += y;
                        if constexpr (FP8) {
                            const float xv = x * vs[i][half] * st.down[o][0], yv = y * vs[i][half] * st.down[o][1];
                            const __half2 v = __floats2half2_rn(xv, yv);
                            w[o][half] = transpose8(*reinterpret_cast<const uint32_t*>(&v));
                            left[o][half] = transpose8(pack_f16(xv - __low2float(v), yv - __high2float(v)));
                        } else {
                            const uint32_t v = pack_bf16(x, y);
                            w[o][half] = transpose8(v);
                            left[o][half] = transpose8(pack_bf16(x - bf16lo(v), y - bf16hi(v)));
                        }
                    }
                const uint32_t vrow = base + (i * 16) / U * UB + U * ROW;
                // matrices of a load -- 8 bits: rows 0-7 and 8-15 at chunk c, then at chunk c + 1; bf16: chunks c, c + 1 of rows 0-7, then 8-15
                const int r = (i * 16) % U + (FP8 ? mi & 1 : mi >> 1) * 8 + ri;
#pragma unroll
                for (int c = 0; c < ROW / 16; c += 2) {
                    uint32_t v[4];
                    ldsm_x4_t(v, vrow + Geo::chunk(r, c + (FP8 ? mi >> 1 : mi & 1)));
                    if constexpr (FP8) {  // byte pairs of rows 2 t, 2 t + 1: even channels, odd channels
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const uint32_t x = __byte_perm(v[2 * j], 0, 0x3120), y = __byte_perm(v[2 * j + 1], 0, 0x3120);
                            const uint32_t a[4] = {codes_f16(x & 0xffffu), codes_f16(x >> 16), codes_f16(y & 0xffffu), codes_f16(y >> 16)};
#pragma unroll
                            for (int o = 0; o < NH; ++o) {
                                mma(st.O[o][c + j], a, w[o][0], w[o][1]);
                                mma(st.O[o][c + j], a, left[o][0], left[o][1]);
                            }
                        }
                    } else {
#pragma unroll
                        for (int o = 0; o < NH; ++o) {
                            mma(st.O[o][c / 2], v, w[o][0], w[o][1]);
                            mma(st.R[o][c / 2], v, left[o][0], left[o][1]);
                        }
                    }
                }
            }
            __syncwarp();
            if (issued < tiles) issue();

            // ---- the head's end, or the share's
            const bool head_end = cur.t == cur.n - 1;
            if (head_end || it == tiles - 1) {
                float l[NH][2];
#pragma unroll
                for (int o = 0; o < NH; ++o)
#pragma unroll
                    for (int hd = 0; hd < 2; ++hd) l[o][hd] = rows_sum(st.l[o][hd]);
                if (from_start && head_end) {  // all of it
                    const long long row0 = (long long)cur.b * H + cur.h * G;
                    float inv[NH][2];
                    [[maybe_unused]] float up[NH][2];
#pragma unroll
                    for (int o = 0; o < NH; ++o)
#pragma unroll
                        for (int hd = 0; hd < 2; ++hd) {
                            inv[o][hd] = 1.f / l[o][hd];
                            if constexpr (FP8) up[o][hd] = 1.f / st.down[o][hd];
                        }
                    st.each(lane, G, [&](int o, int hd, int head, int d, float x) {
                        x *= inv[o][hd];
                        if constexpr (FP8) x *= up[o][hd];  // (last: before, it could overflow where the output does not)
                        p.out[(row0 + head) * D + d] = st.any ? __bfloat16_as_ushort(__float2bfloat16_rn(x)) : (uint16_t)0;
                    });
                    if (p.lse && gq == 0)
#pragma unroll
                        for (int o = 0; o < NH; ++o)
#pragma unroll
                            for (int hd = 0; hd < 2; ++hd)
                                if (8 * o + 2 * t + hd < G)
                                    p.lse[row0 + 8 * o + 2 * t + hd] =
                                        st.any ? (st.m[o][hd] + log2f(l[o][hd])) * 0.6931471805599453f : -INFINITY;
                } else {
                    float* rec = p.partial + ((long long)mine * 2 + (from_start ? 1 : 0)) * record_floats(G, D);
                    st.each(lane, G, [&](int, int, int head, int d, float x) { rec[head * D + d] = x; });
                    if (gq == 0)
#pragma unroll
                        for (int o = 0; o < NH; ++o)
#pragma unroll
                            for (int hd = 0; hd < 2; ++hd)
                                if (8 * o + 2 * t + hd < G) {
                                    rec[G * D + 8 * o + 2 * t + hd] = st.m[o][hd];
                                    rec[G * D + G + 8 * o + 2 * t + hd] = l[o][hd];
                                    if constexpr (FP8) rec[G * D + 2 * G + 1 + 8 * o + 2 * t + hd] = st.u[o][hd];
                                }
                    if (lane == 0) rec[G * D + 2 * G] = st.any ? 1.f : 0.f;
                }
                from_start = true;
                fresh = true;
            }
            cur.next(work, KVH, p.c.batch);
        }
    }
}

// The heads that several shares hold.  A CTA per sequence and `hg` query heads of a KV head: all of them (8 at most) where
// there are many KV heads, with a handful of records each; one, and a part of its channels (gridDim.z parts), where there
// are few, with hundreds.  It finds its records (slot 1 of the share where the KV head starts, slot 0 of the others)
// while the attention still runs, then sums them, each thread 4 channels of every parts-th record.  Its registers and
// shared memory fit beside the attention's.  Also the zeros of empty slots.  What bounds it is latency, two rounds of
// loads: done 2.8 us after the last warp of one user's 577 rows (19 records a head), 5 us after that of 131k rows (152).  (By the
// last CTA of a head to arrive instead, each of those steps waited for the one before: 3.7 and 8 us.)
constexpr int kJoinThreads = 256;
template <int D, bool GROUP>
__global__ void __launch_bounds__(kJoinThreads, 4) paged_join_kernel(const PagedAttnParams p, const int T, const int warps, const int group)
{
    const int hg = GROUP ? group : 1;
    constexpr int kW = kJoinThreads / 32, kAtOnce = GROUP ? 4 : 8;  // loads under way per thread
    constexpr int kBlock = 512;                         // records * heads whose maxima and sums are in shared memory at a time
    __shared__ __align__(16) uint8_t shared[sizeof(Work)];
    constexpr bool FP8 = RA_PAGED_FMT == RA_PAGED_FP8;
    __shared__ float s_m[kBlock], s_l[kBlock], s_top[kW], s_sum[kJoinThreads];
    [[maybe_unused]] __shared__ float s_u[FP8 ? kBlock : 1], s_top_u[kW];  // (8 bits: the unit of o is 2^u)
    __shared__ float4 s_later[GROUP ? kJoinThreads : 1];
    static_assert(sizeof(Work) >= kJoinThreads * sizeof(float4), "the sums of a CTA's only head take the place of the tiles");
    Work& work = *reinterpret_cast<Work*>(shared);
    float4* s_o = GROUP ? s_later : reinterpret_cast<float4*>(shared);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, G = p.c.G, KVH = p.c.KVH;
    const int groups = (G + hg - 1) / hg, items = GROUP ? KVH * groups * p.c.batch : 0;
    const int lpr = D / 4 / gridDim.z, cols = hg * lpr, parts = kJoinThreads / cols;
    const int part = tid / cols, j = tid % cols / lpr, c = blockIdx.z * lpr + tid % lpr;  // this thread's records, head and 4 channels
    count_tiles<kJoinThreads>(p, T, work);
    const Split split(work.pre[p.c.batch], warps);
    pdl_wait();
    pdl_launch_dependents();
    int item = blockIdx.x;  // groups: of all sequences' heads, as many CTAs as fit; else the CTA's own head
    do {
        const int b = GROUP ? item / (KVH * groups) : blockIdx.y, at = GROUP ? item % (KVH * groups) : blockIdx.x;
        const int h = at / groups, g0 = at % groups * hg;
        const bool live = part < parts && g0 + j < G;
        const long long row = ((long long)b * KVH + h) * G + g0 + j;
        const int n = work.n[b], first = work.pre[b] + h * n;
        int from = 0, count = 0;
        if (n > 0) {
            from = split.of(first);
            count = split.of(first + n - 1) - from + 1;
        }
        const bool lead = live && part == 0 && c == 0;
        if (count == 1) continue;
        if (count == 0) {
            if (live && part == 0) reinterpret_cast<uint2*>(p.out + row * D)[c] = make_uint2(0u, 0u);
            if (p.lse && lead) p.lse[row] = -INFINITY;
            continue;
        }
        const int stride = record_floats(G, D), most = kBlock / hg;
        auto rec = [&](int i) { return p.partial + ((long long)(from + i) * 2 + (i == 0 ? 1 : 0)) * stride; };
        float m = -INFINITY, l = 0.f, u = -INFINITY;
        bool any = false;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int base = 0; base < count; base += most) {
            const int here = min(most, count - base);
            float4 x[kAtOnce];
            auto load = [&](int i0) {
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const int i = i0 + k * parts;
                    x[k] = live && i < here ? reinterpret_cast<const float4*>(rec(base + i) + (g0 + j) * D)[c] : make_float4(0.f, 0.f, 0.f, 0.f);
                }
            };
            load(part);  // (before the factors they wait for)
            bool some = false;
            float top = -INFINITY, top_u = -INFINITY;
            for (int i = tid; i < here * hg; i += kJoinThreads) {
                const int g = g0 + i % hg;
                const float* r = rec(base + i / hg) + G * D;
                const float mi = g < G ? r[g] : -INFINITY;
                s_m[i] = mi;
                s_l[i] = g < G ? r[G + g] : 0.f;
                some = some || r[2 * G] != 0.f;
                top = fmaxf(top, mi);
                if constexpr (FP8) {
                    const float ui = g < G ? r[2 * G + 1 + g] : -INFINITY;
                    s_u[i] = ui;
                    top_u = fmaxf(top_u, ui);
                }
            }
            if constexpr (!GROUP) {
#pragma unroll
                for (int y = 16; y; y >>= 1) {
                    top = fmaxf(top, __shfl_xor_sync(kAll, top, y));
                    if constexpr (FP8) top_u = fmaxf(top_u, __shfl_xor_sync(kAll, top_u, y));
                }
                if (lane == 0) {
                    s_top[warp] = top;
                    s_top_u[warp] = top_u;
                }
            }
            any = __syncthreads_or(some) || any;
            top = m;
            top_u = u;
            if constexpr (!GROUP) {
#pragma unroll
                for (int w = 0; w < kW; ++w) {
                    top = fmaxf(top, s_top[w]);
                    if constexpr (FP8) top_u = fmaxf(top_u, s_top_u[w]);
                }
            } else {
#pragma unroll 4
                for (int i = 0; i < here; ++i) {
                    top = fmaxf(top, s_m[i * hg + j]);
                    if constexpr (FP8) top_u = fmaxf(top_u, s_u[i * hg + j]);
                }
            }
            auto factor = [](float from, float to) { return from == -INFINITY ? 0.f : ex2(from - to); };
            const float keep_l = factor(m, top), keep = FP8 ? factor(u, top_u) : keep_l;
            m = top;
            u = top_u;
            l *= keep_l;
            if (base) {  // (a piece whose weights are all zero still carries the NaN that an infinity times them is)
                o.x *= keep;
                o.y *= keep;
                o.z *= keep;
                o.w *= keep;
            }
            for (int i0 = part; i0 < here; i0 += parts * kAtOnce) {
                if (i0 != part) load(i0);
#pragma unroll
                for (int k = 0; k < kAtOnce; ++k) {
                    const int i = i0 + k * parts;
                    if (i >= here) break;
                    const float of_l = factor(s_m[i * hg + j], m), f = FP8 ? factor(s_u[i * hg + j], u) : of_l;
                    l += of_l * s_l[i * hg + j];
                    o.x += f * x[k].x;
                    o.y += f * x[k].y;
                    o.z += f * x[k].z;
                    o.w += f * x[k].w;
                }
            }
            __syncthreads();
        }
        if constexpr (!GROUP) {  // (lpr is a power of two, a column's threads lie lpr apart: first over the warp)
            for (int y = lpr; y < 32; y <<= 1) {
                o.x += __shfl_xor_sync(kAll, o.x, y);
                o.y += __shfl_xor_sync(kAll, o.y, y);
                o.z += __shfl_xor_sync(kAll, o.z, y);
                o.w += __shfl_xor_sync(kAll, o.w, y);
                l += __shfl_xor_sync(kAll, l, y);
            }
        }
        const int step = GROUP ? cols : 32, sets = GROUP ? parts : kW;
        if (sets > 1) {  // then the rest: thread `tid` of the first set sums its column's
            s_o[tid] = o;
            s_sum[tid] = l;
            __syncthreads();
            if (part == 0)
#pragma unroll 7
                for (int i = 1; i < sets; ++i) {
                    const float4 y = s_o[tid + i * step];
                    o.x += y.x;
                    o.y += y.y;
                    o.z += y.z;
                    o.w += y.w;
                    l += s_sum[tid + i * step];
                }
            if (GROUP) __syncthreads();  // (the next head's sums come here)
        }
        if (part == 0 && live) {
            const float up = FP8 ? ex2(u - m) : 1.f;  // (last, as in the attention)
            reinterpret_cast<uint2*>(p.out + row * D)[c] =
                any ? make_uint2(pack_bf16(o.x / l * up, o.y / l * up), pack_bf16(o.z / l * up, o.w / l * up)) : make_uint2(0u, 0u);
            if (p.lse && lead) p.lse[row] = any ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
        }
    } while (GROUP && (item += gridDim.x) < items);
}

template <int D, int U, int NH, bool PROBE = false>
cudaError_t launch(const PagedAttnParams& p, int sms, cudaStream_t s)
{
    using Geo = PagedGeo<RA_PAGED_FMT, D>;
    constexpr int stage = Geo::kTile / U * Geo::unit_stride(U);
    static_assert(smem_of(stage, kWarps<D>).total <= (int)kSmemMost, "the ring fits");
    cudaError_t e = launch_pdl(paged_attn_kernel<D, U, NH, PROBE>, dim3(sms), dim3(32 * kWarps<D>), smem_of(stage, kWarps<D>).total, s, p);
    if (e != cudaSuccess) return e;
    // Up to a head per SM each has its CTAs, up to 4 for parts of its channels; above, groups of heads share one.  Single heads and
    // groups: 64 heads of one sequence of 131k rows in 8 bits 50.4 and 82.3 us, 128 of four of 3000 rows 11.2 and 15.0, 160 of five of 1500
    // 11.2 and 13.5, 256 of 16 of up to 2500 15.2 and 14.7, 512 of 16 of 2000 16.0 and 15.8.  Parts, 1, 2 and 4: 32 heads of one of 4000
    // rows 9.1, 8.1 and 8.2 us (of 577 rows 6.5, 6.6 and 6.9), 64 of one of 131k 51.3, 50.4 and 50.9, 128 of four 11.3, 12.3 and 12.2.
    const int heads = p.c.KVH * p.c.G * p.c.batch;
    if (heads > sms) {
        const int hg = p.c.G < 8 ? p.c.G : 8;
        const int items = p.c.KVH * ((p.c.G + hg - 1) / hg) * p.c.batch;
        return launch_pdl(paged_join_kernel<D, true>, dim3(items < 4 * sms ? items : 4 * sms), dim3(kJoinThreads), 0, s, p,
                          (int)Geo::kTile, sms * kWarps<D>, hg);
    }
    return launch_pdl(paged_join_kernel<D, false>, dim3(p.c.KVH * p.c.G, p.c.batch, heads * 4 <= sms ? 4 : heads * 2 <= sms ? 2 : 1),
                      dim3(kJoinThreads), 0, s, p, (int)Geo::kTile, sms * kWarps<D>, 1);
}

template <int D, int U, int NH>
cudaError_t prepare()
{
    if (D == 64 && U == 16 && NH == 1) {
        const cudaError_t e = cudaFuncSetAttribute(paged_attn_kernel<64, 16, 1, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost);
        if (e != cudaSuccess) return e;
    }
    return cudaFuncSetAttribute(paged_attn_kernel<D, U, NH, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost);
}

// f(integral constants D, unit rows, sets of 8 heads) for a cache
template <int... N>
struct Ints {};
template <int D, int U, typename F>
cudaError_t pick(int G, F f)
{
    return G > 8 ? f(Ints<D, U, 2>()) : f(Ints<D, U, 1>());
}
template <int D, typename F>
cudaError_t pick(int page, int G, F f)
{
    using Geo = PagedGeo<RA_PAGED_FMT, D>;
    const int U = Geo::unit_rows(page);
    if (U == 16) return pick<D, 16>(G, f);
    if (U == 32) return pick<D, 32>(G, f);
    return pick<D, Geo::kTile>(G, f);
}
template <typename F>
cudaError_t pick(int D, int page, int G, F f)
{
    return D == 128 ? pick<128>(page, G, f) : pick<64>(page, G, f);
}
template <int D, int U, int NH>
cudaError_t launch_of(Ints<D, U, NH>, const PagedAttnParams& p, int sms, cudaStream_t s)
{
    return launch<D, U, NH>(p, sms, s);
}
template <int D, int U, int NH>
cudaError_t prepare_of(Ints<D, U, NH>)
{
    return prepare<D, U, NH>();
}

}  // namespace

#if RA_PAGED_FMT == 1
#define RA_PAGED_NAME(x) x##_fp8
#else
#define RA_PAGED_NAME(x) x##_bf16
#endif
size_t RA_PAGED_NAME(paged_partial_bytes)(int G, int D, int sms)
{
    return (size_t)sms * (D == 128 ? kWarps<128> : kWarps<64>) * 2 * record_floats(G, D) * 4;
}
cudaError_t RA_PAGED_NAME(paged_attn_prepare)(int D, int page, int G)
{
    return pick(D, page, G, [](auto n) { return prepare_of(n); });
}
cudaError_t RA_PAGED_NAME(launch_paged_attn)(int D, const PagedAttnParams& p, int sms, cudaStream_t s)
{
    if (p.probe_ns) return launch<64, 16, 1, true>(p, sms, s);  // (the caller has seen to the shape)
    return pick(D, 1 << p.c.page_shift, p.c.G, [&](auto n) { return launch_of(n, p, sms, s); });
}

}  // namespace ra
