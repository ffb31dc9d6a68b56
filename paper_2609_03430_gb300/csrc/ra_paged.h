// ra_paged.h -- layout, launch parameters and launchers of the paged cache (host API and the kernels that write,
// read back and choose in ra_paged.cu, attention in ra_paged_attn.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "ra.h"

namespace ra {

constexpr int kPagedErrInput = 4;  // value of the device error word: a length, row count or page outside its range
constexpr int kPagedPrefetchTable = 128 << 10;  // bytes of tables that are brought into L2 ahead of their use
constexpr int kPagedPrefetchCtas = 512;         // CTAs of a launch that bring them (a CTA per row of the largest batch)
constexpr int kPagedMaxG = 16;     // query heads per KV head (two sets of 8, the columns of an mma.sync operand)

// Exponents of the power-of-two scales, stored as e + 127.  8-bit rows: the smallest 2^e with max |x| <= 448 * 2^e;
// not below 2^-60, so that the attention's sums, which carry 2^-e, stay far inside 32 bits (rows that small keep
// an absolute error of 2^-70).  Whole-number scales (bounds, queries): max |x| <= 127 * 2^e.
constexpr int kFp8MinExp = -60;
constexpr int kInt8MinExp = -120;
constexpr int kScaleNaN = 255;  // the scale byte of a page that holds an infinite key or a NaN (a row in 8 bits: all codes NaN)

// A page's rows of one KV head are stored in units of `U` = min(page, tile) rows, each contiguous, so that one bulk
// copy brings a unit: U K rows, U V rows, and in 8 bits their U + U scale bytes.  16-byte chunks of a row are
// permuted by the row's index, the way the shared-memory reads of the tensor-core operands want them (8 rows at one chunk index hit
// 8 different bank groups); the copy then needs no layout of its own.
template <int FMT, int D>
struct PagedGeo {
    static constexpr int kES = FMT == RA_PAGED_FP8 ? 1 : 2;     // bytes per element
    static constexpr int kRow = D * kES;                        // bytes per row: 64, 128 or 256
    static constexpr int kTile = kRow == 64 ? 64 : 32;          // rows of K and V that attention takes at a time
    static constexpr int kScales = FMT == RA_PAGED_FP8 ? 1 : 0;  // scale bytes per row
    __host__ __device__ static constexpr int unit_rows(int page) { return page < kTile ? page : kTile; }
    __host__ __device__ static constexpr int unit_bytes(int U) { return 2 * U * (kRow + kScales); }
    // from one unit to the next: a bulk copy whose source lies across 128-byte lines as its target does not is slower
    __host__ __device__ static constexpr int unit_stride(int U) { return (unit_bytes(U) + 127) / 128 * 128; }
    // byte of 16-byte chunk c of row r within the K (or V) rows of a unit
    __host__ __device__ static constexpr int chunk(int r, int c)
    {
        return r * kRow + ((c ^ (kRow == 64 ? (r >> 1) & 3 : r & 7)) << 4);
    }
};

// One layer's cache and the caller's sequences.
struct PagedView {
    uint8_t* rows;        // [pages][KVH][page / U] units
    uint16_t* lohi;       // [pages][KVH][2][D] bf16: lowest and highest key per channel (null without bounds)
    int8_t* lohi8;        // [pages][KVH][2][D] the same rounded outwards at the page's scale
    uint8_t* lohi_exp;    // [pages][KVH] its exponent + 127
    int32_t* err;         // device error word
    const int32_t* lens;  // [batch]
    const int32_t* table; // [batch][table_stride]
    int KVH, G, page_shift, pages, max_len, batch, table_stride;
};

struct PagedRowsParams {  // write / read back
    PagedView c;
    const uint16_t* k_in;
    const uint16_t* v_in;
    uint16_t* k_out;
    uint16_t* v_out;
    long long row_stride, head_stride;
    const int32_t* rows;  // [batch + 1] first row of each sequence; null: row b is sequence b's
    int n_rows;
};

struct PagedAttnParams {
    PagedView c;
    const uint16_t* q;
    long long q_row_stride, q_head_stride;
    uint16_t* out;       // [batch][H][D]
    float* lse;          // [batch][H] or null
    const int32_t* sel;  // [batch][KVH][top] page indices (-1: none); null: every row
    int top;
    float scale_log2;    // scale * log2 e
    float* partial;      // records of heads that several warps hold
    uint64_t probe_ns;   // a test's launch: its waits' limit, and the tile of a share whose wait runs out (0: none)
    int probe_share, probe_tile;
};

struct PagedSelectParams {
    PagedView c;
    const uint16_t* q;
    long long q_row_stride, q_head_stride;
    int top, first, last;
    int32_t* sel;     // [batch][KVH][top]
    uint32_t* keys;   // [batch][KVH][max_pages]
    int max_pages;
    int cluster;      // CTAs per head (set by the launcher)
};

cudaError_t launch_paged_write(int fmt, int D, const PagedRowsParams& p, int sms, cudaStream_t s);
cudaError_t launch_paged_read(int fmt, int D, const PagedRowsParams& p, int sms, cudaStream_t s);
cudaError_t launch_paged_select(int D, PagedSelectParams p, int sms, cudaStream_t s);
cudaError_t launch_paged_attn_bf16(int D, const PagedAttnParams& p, int sms, cudaStream_t s);
// Launch attributes on the current device (called where a cache is bound).
cudaError_t paged_attn_prepare_bf16(int D, int page, int G);
cudaError_t paged_attn_prepare_fp8(int D, int page, int G);
// Scratch for the records on a device of `sms` SMs.
size_t paged_partial_bytes_bf16(int G, int D, int sms);
size_t paged_partial_bytes_fp8(int G, int D, int sms);
cudaError_t launch_paged_attn_fp8(int D, const PagedAttnParams& p, int sms, cudaStream_t s);

// Which lines thread `thread` of CTA (x, y) brings into L2 ahead: those of thread i of n, none where i < 0.  Only a launch's
// first CTAs take part: a grid sized by a caller's upper bound on rows may hold more threads than 32 bits count, and
// the CTAs behind the first find the lines in L2 anyway.
struct PrefetchShare {
    int i, n;
};
__host__ __device__ inline PrefetchShare prefetch_share(unsigned grid_x, unsigned grid_y, unsigned x, unsigned y, int threads, int thread)
{
    const unsigned long long ctas = (unsigned long long)grid_x * grid_y, cta = (unsigned long long)y * grid_x + x;
    const int most = ctas < (unsigned long long)kPagedPrefetchCtas ? (int)ctas : kPagedPrefetchCtas;
    return PrefetchShare{cta < (unsigned long long)most ? (int)cta * threads + thread : -1, most * threads};
}

// Whether any two of n_rows x heads rows of D elements, row r of head h at r * row + h * head (neither negative), share an
// element: row r' of head h' meets it where (h' - h) * head is within D of (r - r') * row.
inline bool rows_overlap(long long row, long long head, int n_rows, int heads, int D)
{
    if ((n_rows > 1 && row < D) || (heads > 1 && head < D)) return true;
    if (n_rows < 2 || heads < 2 || (row - D) / head >= heads - 1 || (head - D) / row >= n_rows - 1) return false;  // (whole rows or heads apart)
    for (int dh = 1; dh < heads; ++dh) {
        const __int128 at = (__int128)dh * head;
        const __int128 dr = at / row, below = at - dr * row;
        if ((dr >= 1 && dr < n_rows && below < D) || (dr + 1 < n_rows && row - below < D)) return true;
    }
    return false;
}

#ifdef __CUDACC__
// Brings lines into L2 ahead of their first use (thread i of n, before the kernel waits for its predecessor: L2 is
// where a predecessor's writes arrive, so a line fetched early is not a stale one).
__device__ __forceinline__ void prefetch_lines(const void* base, long long bytes, int i, int n)
{
    const char* from = static_cast<const char*>(base);
    for (long long at = (long long)i * 128; at < bytes; at += (long long)n * 128)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(from + at));
}
__device__ __forceinline__ void prefetch_heads(const uint16_t* base, long long row_stride, long long head_stride, int heads, int D,
                                               int batch, int i, int n)
{
    const int lines = D / 64;  // of a head
    for (int at = i; at < batch * heads * lines; at += n) {
        const int head = at / lines;
        asm volatile("prefetch.global.L2 [%0];" ::"l"(base + head / heads * row_stride + head % heads * head_stride + at % lines * 64));
    }
}
__device__ __forceinline__ void prefetch_sequences(const PagedView& c, int i, int n)
{
    const long long table = 4ll * c.batch * c.table_stride;
    prefetch_lines(c.lens, 4ll * c.batch, i, n);
    if (table <= kPagedPrefetchTable) prefetch_lines(c.table, table, i, n);  // (a wide one is mostly columns no length covers)
}

// The sequence's length as the kernels use it: 0 and a flagged error where it is outside [0, max_len] or the table.
__device__ __forceinline__ int paged_len(const PagedView& c, int b)
{
    const int n = c.lens[b];
    const int most = min((long long)c.max_len, (long long)c.table_stride << c.page_shift);
    if (n < 0 || n > most) {
        atomicOr(c.err, kPagedErrInput);
        return 0;
    }
    return n;
}
// The sequence's i-th page (i within its length), -1 and a flagged error where the table holds none of the pool's.
__device__ __forceinline__ int paged_page(const PagedView& c, int b, int i)
{
    const int page = c.table[(long long)b * c.table_stride + i];
    if (page < 0 || page >= c.pages) {
        atomicOr(c.err, kPagedErrInput);
        return -1;
    }
    return page;
}
#endif

}  // namespace ra
