// What fills a paged key-value cache, for gfx950.
//
// K and V are [P, Hkv, page, D] (any strides, rows of D contiguous elements);
// row r's position pos is slot pos % page of page table[r, pos / page].  A
// position whose table entry names no page of the cache is not written.
#include <stdint.h>

#include "div.h"
#include "grid.h"
#include "launch.h"

namespace fs {
namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// The last of the rows lo .. R - 1 whose tokens begin at or before token n (lo if none).
__device__ __forceinline__ int row_of(const int32_t *offsets, int lo, int R, int n) {
    int hi = R;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (offsets[mid] <= n ? lo : hi) = mid;
    }
    return lo;
}

// A workgroup moves the key and value rows of one token after another, kAhead of them
// at a time: which row a token is of, and where that has it, is the same for all its
// lanes.  Lane i moves 16 bytes of every token: chunk i of its Hkv * chunks.  Bound by
// HBM: 48000 tokens of 4 KB, 393 MB in and out, 81 us, 4.9 TB/s (97 with a lane per 16
// bytes that finds its own row).
constexpr int kThreads = 256;
template <int kAhead>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(PagedCache c, const unsigned char *k, const unsigned char *v,
                                                                long long token_bytes, long long khead_bytes, int N,
                                                                const int32_t *start, const int32_t *offsets, int R,
                                                                int per, Div by_chunks, int chunks, Div by_page)
{
    const unsigned first = wide_index() * kAhead;
    if (first >= (unsigned)N) return;
    const int n0 = (int)first;
    long long at[kAhead];   // of each token's slot, or -1
    int lo = offsets ? row_of(offsets, 0, R, n0) : 0;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
        const int n = n0 + e;
        at[e] = -1;
        if (n >= N) continue;
        long long pos;
        if (offsets) {
            // the next one: by steps over many rows without tokens it took 758 us where these are 100000
            if (lo + 1 < R && offsets[lo + 1] <= n) lo = row_of(offsets, lo + 1, R, n);
            if (n < offsets[lo] || n >= offsets[lo + 1]) continue;
            pos = (long long)start[lo] + (n - offsets[lo]);
        } else {
            lo = n;
            pos = start[n];
        }
        if (pos < 0 || pos > 0x7fffffff) continue;
        const int j = (int)by_page((unsigned)pos);
        if (j >= c.cols) continue;
        const int pg = c.table[(size_t)lo * c.ld_table + j];
        if (pg >= 0 && pg < c.pages) at[e] = pg * c.page_bytes + ((int)pos - j * c.page) * c.slot_bytes;
    }
    for (int i = threadIdx.x; i < per; i += kThreads) {
        const int h = (int)by_chunks((unsigned)i), ch = i - h * chunks;
        const size_t from = (size_t)n0 * token_bytes + (size_t)h * khead_bytes + (size_t)ch * 16;
        const size_t to = (size_t)h * c.head_bytes + (size_t)ch * 16;
        u32x4_t x[kAhead], y[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            // a token that goes nowhere reads the first one's row
            const size_t f = from + (at[e] >= 0 ? (size_t)e * token_bytes : 0);
            x[e] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(k + f));
            y[e] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(v + f));
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            if (at[e] < 0) continue;
            *reinterpret_cast<u32x4_t *>(c.K + at[e] + to) = x[e];
            *reinterpret_cast<u32x4_t *>(c.V + at[e] + to) = y[e];
        }
    }
}

}  // namespace

hipError_t launch_paged_append(const PagedCache &cache, const void *k, const void *v, long long token_bytes,
                               long long khead_bytes, int N, const int32_t *start, const int32_t *offsets, int R, int Hkv,
                               int row_bytes, hipStream_t stream)
{
    const int chunks = row_bytes / 16;
    // a token a workgroup until they fill the chip; then four, whose loads are on their way together
    auto launch = [&](auto kernel, int ahead) {
        hipLaunchKernelGGL(kernel, wide_grid((N + (long long)ahead - 1) / ahead), dim3(kThreads), 0, stream, cache,
                           static_cast<const unsigned char *>(k), static_cast<const unsigned char *>(v), token_bytes,
                           khead_bytes, N, start, offsets, R, Hkv * chunks, make_div(chunks), chunks, make_div(cache.page));
    };
    if (N <= 2048) launch(paged_append_kernel<1>, 1);
    else launch(paged_append_kernel<4>, 4);
    return hipGetLastError();
}

}  // namespace fs
