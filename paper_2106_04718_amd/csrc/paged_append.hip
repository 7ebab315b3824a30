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

// A workgroup moves the key and value rows of kAhead tokens, whose loads are on their way
// together.  Lane i moves 16 bytes of each: chunk i of its Hkv * chunks, `per` in all.
//   SIDE    (tokens of up to kThreads / 4 chunks)  `side` tokens stand side by side, and a
//           lane finds the places of its own.
//   !SIDE   which row a token is of, and where that has it, is the same for all lanes.
// Bound by HBM where tokens are many: 48000 of 4 KB, 393 MB in and out, 81 us, 4.9 TB/s
// (97 with a lane per 16 bytes that finds its own row).  A workgroup takes some 3 ns to
// start, so tokens of few bytes would wait for that: a million of 512 bytes 211 us side by
// side and 773 one behind another, 65536 of 512 bytes 16 and 54.
constexpr int kThreads = 256;
template <int kAhead, bool SIDE>
__global__ __launch_bounds__(kThreads) void paged_append_kernel(PagedCache c, const unsigned char *k, const unsigned char *v,
                                                                long long token_bytes, long long khead_bytes, int N,
                                                                const int32_t *start, const int32_t *offsets, int R,
                                                                int per, int side, Div by_per, Div by_chunks, int chunks,
                                                                Div by_page)
{
    const int s = SIDE ? (int)by_per(threadIdx.x) : 0, step = SIDE ? side : 1;   // tokens s, s + step, ..
    const unsigned first = wide_index() * (unsigned)(kAhead * step) + s;
    if (s >= step || first >= (unsigned)N) return;
    const int n0 = (int)first;
    auto token = [&](int e) { return N - n0 > e * step ? n0 + e * step : n0; };   // past the last: looked up, not moved
    long long at[kAhead];   // of each token's slot, or -1
    int row[kAhead];
    if (SIDE && offsets) {   // all at once: as many loads on their way
#pragma unroll
        for (int e = 0; e < kAhead; ++e) row[e] = 0;
        for (int half = R > 1 ? 1 << (31 - __builtin_clz(R - 1)) : 0; half > 0; half /= 2) {
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const int r = R - row[e] > half ? row[e] + half : 0;
                if (offsets[r] <= token(e)) row[e] = r > row[e] ? r : row[e];
            }
        }
    } else if (offsets) {    // mostly one row's: the next one's is searched for where that ends
        row[0] = row_of(offsets, 0, R, n0);
#pragma unroll
        for (int e = 1; e < kAhead; ++e) {
            const int lo = row[e - 1];
            row[e] = lo + 1 < R && offsets[lo + 1] <= token(e) ? row_of(offsets, lo + 1, R, token(e)) : lo;
        }
    } else {
#pragma unroll
        for (int e = 0; e < kAhead; ++e) row[e] = token(e);
    }
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
        const int n = token(e), lo = row[e];
        at[e] = -1;
        if (e > 0 && n == n0) continue;
        long long pos = start[lo];
        if (offsets) {
            const int begin = offsets[lo];
            if (n < begin || n >= offsets[lo + 1]) continue;
            pos += n - begin;
        }
        if (pos < 0 || pos > 0x7fffffff) continue;
        const int j = (int)by_page((unsigned)pos);
        if (j >= c.cols) continue;
        const int pg = c.table[(size_t)lo * c.ld_table + j];
        if (pg >= 0 && pg < c.pages) at[e] = pg * c.page_bytes + ((int)pos - j * c.page) * c.slot_bytes;
    }
    for (int i = SIDE ? (int)threadIdx.x - s * per : (int)threadIdx.x; i < per; i += kThreads) {
        const int h = (int)by_chunks((unsigned)i), ch = i - h * chunks;
        const size_t from = (size_t)n0 * token_bytes + (size_t)h * khead_bytes + (size_t)ch * 16;
        const size_t to = (size_t)h * c.head_bytes + (size_t)ch * 16;
        u32x4_t x[kAhead], y[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            // a token that goes nowhere reads the first one's row
            const size_t f = from + (at[e] >= 0 ? (size_t)e * step * token_bytes : 0);
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
    const int chunks = row_bytes / 16, per = Hkv * chunks, side = per <= kThreads / 4 ? kThreads / per : 1;
    // a token a workgroup (and place side by side) until they fill the chip; then four,
    // whose loads are on their way together
    auto launch = [&](auto kernel, int ahead) {
        const long long tokens = (long long)ahead * side;
        hipLaunchKernelGGL(kernel, wide_grid((N + tokens - 1) / tokens), dim3(kThreads), 0, stream, cache,
                           static_cast<const unsigned char *>(k), static_cast<const unsigned char *>(v), token_bytes,
                           khead_bytes, N, start, offsets, R, per, side, make_div(per), make_div(chunks), chunks,
                           make_div(cache.page));
    };
    const bool few = N <= 2048ll * side;
    if (side > 1) few ? launch(paged_append_kernel<1, true>, 1) : launch(paged_append_kernel<4, true>, 4);
    else few ? launch(paged_append_kernel<1, false>, 1) : launch(paged_append_kernel<4, false>, 4);
    return hipGetLastError();
}

}  // namespace fs
