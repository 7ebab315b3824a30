// What fills a paged key-value cache, for gfx950.
//
// K and V are [P, Hkv, page, D] (any strides, rows of D contiguous elements);
// row r's position pos is slot pos % page of page table[r, pos / page].  A
// position whose table entry names no page of the cache is not written.
#include <stdint.h>

#include "launch.h"

namespace fs {
namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// The slot of position pos of row r, in bytes from the cache's base, or -1.
__device__ __forceinline__ long long slot_of(const PagedCache &c, int r, int pos) {
    const int j = pos / c.page;
    if (pos < 0 || j >= c.cols) return -1;
    const int pg = c.table[(size_t)r * c.ld_table + j];
    if (pg < 0 || pg >= c.pages) return -1;
    return pg * c.page_bytes + (pos - j * c.page) * c.slot_bytes;
}

// One lane moves 16 bytes of one token's key and value row.
__global__ __launch_bounds__(256) void paged_append_kernel(PagedCache c, const unsigned char *k, const unsigned char *v,
                                                           long long token_bytes, long long khead_bytes, int N,
                                                           const int32_t *start, const int32_t *offsets, int R, int Hkv,
                                                           int chunks)
{
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int per = Hkv * chunks;
    const int n = (int)(id / per);
    if (n >= N) return;
    const int h = (int)(id % per) / chunks, ch = (int)(id % per) % chunks;
    int r = n, i = 0;
    if (offsets) {   // the last row whose tokens begin at or before n
        int lo = 0, hi = R;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            (offsets[mid] <= n ? lo : hi) = mid;
        }
        if (n < offsets[lo] || n >= offsets[lo + 1]) return;
        r = lo;
        i = n - offsets[lo];
    }
    const long long pos = (long long)start[r] + i;
    const long long at = pos > 0x7fffffff ? -1 : slot_of(c, r, (int)pos);
    if (at < 0) return;
    const size_t from = (size_t)n * token_bytes + (size_t)h * khead_bytes + ch * 16;
    const size_t to = (size_t)at + (size_t)h * c.head_bytes + ch * 16;
    *reinterpret_cast<u32x4_t *>(c.K + to) = *reinterpret_cast<const u32x4_t *>(k + from);
    *reinterpret_cast<u32x4_t *>(c.V + to) = *reinterpret_cast<const u32x4_t *>(v + from);
}

}  // namespace

hipError_t launch_paged_append(const PagedCache &cache, const void *k, const void *v, long long token_bytes,
                               long long khead_bytes, int N, const int32_t *start, const int32_t *offsets, int R, int Hkv,
                               int row_bytes, hipStream_t stream)
{
    const int chunks = row_bytes / 16;
    const long long n = (long long)N * Hkv * chunks;
    hipLaunchKernelGGL(paged_append_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, stream, cache,
                       static_cast<const unsigned char *>(k), static_cast<const unsigned char *>(v), token_bytes,
                       khead_bytes, N, start, offsets, R, Hkv, chunks);
    return hipGetLastError();
}

}  // namespace fs
