// Paged key-value cache for gfx950: what fills it and the attention that reads
// it, for rows that grow independently of each other.
//
// K and V are [P, Hkv, page, D] (any strides, rows of D contiguous elements);
// row r's position pos is slot pos % page of page table[r, pos / page].  A
// position whose table entry names no page of the cache holds nothing: it is
// not attended and not written.
#include <math.h>
#include <stdint.h>

#include "launch.h"

namespace fs {
namespace {

constexpr int kWave = 64;
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
// fp32 -> T, to nearest even
template <typename T>
__device__ __forceinline__ T narrow(float x);
template <>
__device__ __forceinline__ float narrow<float>(float x) { return x; }
template <>
__device__ __forceinline__ uint16_t narrow<uint16_t>(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

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

__device__ __forceinline__ float wave_sum(float x) {
    for (int m = 1; m < kWave; m *= 2) x += __shfl_xor(x, m);
    return x;
}

// One wave per (row, query head): the keys one after another, a running
// maximum and sum of the softmax, lanes over the elements of a row.
template <typename T, int D>
__global__ __launch_bounds__(kWave) void paged_attn_kernel(PagedAttn a)
{
    const int r = blockIdx.x / a.Hq, hq = blockIdx.x % a.Hq, G = a.Hq / a.Hkv, h = hq / G, lane = threadIdx.x;
    constexpr int E = (D + kWave - 1) / kWave;
    const PagedCache &c = a.cache;
    const int cap = c.cols * c.page;
    int L = a.kv_len[r];
    L = L < 0 ? 0 : L > cap ? cap : L;
    const T *q = reinterpret_cast<const T *>(a.q + (size_t)r * a.q_row_bytes + (size_t)hq * a.q_head_bytes);
    float qv[E], o[E];
    for (int e = 0; e < E; ++e) {
        qv[e] = lane + e * kWave < D ? widen(q[lane + e * kWave]) * a.scale : 0.f;
        o[e] = 0.f;
    }
    float m = -INFINITY, l = 0.f;
    bool any = false;
    const size_t knew = (size_t)r * a.new_row_bytes + (size_t)h * a.new_head_bytes;
    for (int j = 0; j < L; ++j) {
        const long long at = slot_of(c, r, j);
        const bool fresh = a.k && j == L - 1;
        if (at < 0) continue;
        const size_t off = (size_t)at + (size_t)h * c.head_bytes;
        const T *kr = reinterpret_cast<const T *>(fresh ? a.k + knew : c.K + off);
        const T *vr = reinterpret_cast<const T *>(fresh ? a.v + knew : c.V + off);
        float s = 0.f;
        for (int e = 0; e < E; ++e)
            if (lane + e * kWave < D) s = fmaf(qv[e], widen(kr[lane + e * kWave]), s);
        s = wave_sum(s);
        any = true;
        const float mn = fmaxf(m, s);
        // a score of -inf has no weight, whatever the maximum; NaN and +inf make the row NaN
        const float w = s == -INFINITY ? 0.f : __expf(s - mn), f = m == -INFINITY ? 1.f : __expf(m - mn);
        l = l * f + w;
        for (int e = 0; e < E; ++e)
            if (lane + e * kWave < D) {
                o[e] = o[e] * f + w * widen(vr[lane + e * kWave]);
                if (fresh && hq % G == 0) {   // the new token's own row
                    reinterpret_cast<T *>(c.K + off)[lane + e * kWave] = kr[lane + e * kWave];
                    reinterpret_cast<T *>(c.V + off)[lane + e * kWave] = vr[lane + e * kWave];
                }
            }
        m = mn;
    }
    T *out = reinterpret_cast<T *>(a.out) + ((size_t)r * a.Hq + hq) * D;
    for (int e = 0; e < E; ++e)
        if (lane + e * kWave < D) out[lane + e * kWave] = narrow<T>(any ? o[e] / l : 0.f);
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

size_t paged_attn_workspace_bytes(int, int, int, int, int, int) { return 16; }

hipError_t launch_paged_attn(const PagedAttn &a, int D, bool bf16, hipStream_t stream)
{
    const dim3 gd((unsigned)(a.R * a.Hq)), bd(kWave);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, gd, bd, 0, stream, a); };
    switch (D) {
    case 16: bf16 ? launch(paged_attn_kernel<uint16_t, 16>) : launch(paged_attn_kernel<float, 16>); break;
    case 32: bf16 ? launch(paged_attn_kernel<uint16_t, 32>) : launch(paged_attn_kernel<float, 32>); break;
    case 64: bf16 ? launch(paged_attn_kernel<uint16_t, 64>) : launch(paged_attn_kernel<float, 64>); break;
    default: bf16 ? launch(paged_attn_kernel<uint16_t, 128>) : launch(paged_attn_kernel<float, 128>); break;
    }
    return hipGetLastError();
}

}  // namespace fs
