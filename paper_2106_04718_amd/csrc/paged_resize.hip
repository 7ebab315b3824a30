// Rows of a paged cache that grow and shrink, for gfx950: pages taken from a stack of free
// ones and given back, and the position and slot of every new token.
//
// Which pages a row gets follows from sums over the rows before it: of the pages returned,
// of the pages wanted (a row is granted while their sum is within what is free) and of the
// new tokens.  One workgroup makes these sums, a row a lane and 1024 rows at a time, and
// takes the returned pages, 8192 at a time.  What is then one independent step per page taken
// and per token is done by the same workgroup where these are few, from LDS, or by a second
// kernel over the chip.
//
// Bound by latency: the first kernel is a chain of trips (lengths, returned pages, sums, taken
// pages) on one CU, and the launches cost more than the bytes.  256 rows that take up to
// 8 positions or give them back: 6 to 8 us; 1500 rows and some 280000 tokens: sums 21 to 25 us, pages and
// slots 6.9.
#include <limits.h>
#include <stdint.h>

#include "div.h"
#include "grid.h"
#include "launch.h"
#include "paged_tile.h"

namespace fs {
namespace {

constexpr int kRows = 1024;   // rows at a time, one a lane
constexpr int kParts = kRows / kWave;

// A row before and after: positions and pages.
struct Change {
    int held, want, has, need;
    __device__ __forceinline__ int added() const { return want > held ? want - held : 0; }
};

// Pages of n positions.
__device__ __forceinline__ int pages_of(const Div &by_page, int page, int n) {
    const int j = (int)by_page((unsigned)n);
    return j + (n - j * page > 0 ? 1 : 0);
}

__device__ __forceinline__ Change change_of(const PagedResize &a, const Div &by_page, int held, int want) {
    const int cap = a.cols * a.page;   // at most 2^30
    Change c;
    c.held = held < 0 ? 0 : held > cap ? cap : held;
    c.want = want < 0 ? 0 : want;
    c.has = pages_of(by_page, a.page, c.held), c.need = pages_of(by_page, a.page, c.want);
    return c;
}

// Sums of whole numbers up to INT_MAX, and no more than that.
__device__ __forceinline__ unsigned add_up(unsigned a, unsigned b) { return min(a + b, (unsigned)INT_MAX); }

template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ unsigned add_from(unsigned x) {
    return add_up(x, (unsigned)dpp<CTRL, ROWS>((int)x));   // lanes that get nothing add 0
}
// Inclusive sums over the rows of 16 lanes, and over the wave.
__device__ __forceinline__ unsigned row_scan(unsigned x) {
    x = add_from<0x111>(x);
    x = add_from<0x112>(x);
    x = add_from<0x114>(x);
    return add_from<0x118>(x);
}
__device__ __forceinline__ unsigned scan(unsigned x) {
    x = row_scan(x);
    x = add_from<0x142, 0xA>(x);
    return add_from<0x143, 0xC>(x);
}
__device__ __forceinline__ unsigned lane_of(unsigned x, int lane) {
    return (unsigned)__builtin_amdgcn_readlane((int)x, __builtin_amdgcn_readfirstlane(lane));
}

// Sum over the lanes before this one, and over all, of the workgroup.
struct Scan {
    unsigned before, all;
};
__device__ __forceinline__ Scan block_scan(unsigned x, unsigned *part) {
    const int lane = (int)threadIdx.x & 63, w = (int)threadIdx.x / kWave;
    const unsigned run = scan(x);
    if (lane == 63) part[w] = run;
    __syncthreads();
    const unsigned sums = row_scan(part[lane & 15]);
    Scan r;
    const unsigned waves = w ? lane_of(sums, w - 1) : 0;
    // run - x would not undo a sum that has reached INT_MAX
    unsigned left = (unsigned)__shfl_up((int)run, 1);
    r.before = add_up(waves, lane ? left : 0);
    r.all = lane_of(sums, 15);
    return r;
}

// The rows' sums.  held: the positions a row held, with the upper bit set if it was refused;
// wanted: pages wanted by the rows before it, and offsets: tokens (R + 1 of them).
struct Sums {
    int *held, *wanted, *offsets;
    int *taken, *top;   // pages taken, and pages on the stack before
};

// The last of the entries lo .. hi - 1 that is at most x (the first is).
__device__ __forceinline__ int last_at_most(const int *sums, int lo, int hi, int x) {
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (sums[mid] <= x ? lo : hi) = mid;
    }
    return lo;
}

// The same of all R entries for a wave's lanes, x rising from lane to lane.  Bisection is a chain of
// some ten trips: the first and the last lane's are found with 64 entries looked at at a time,
// and mostly few rows lie between.
__device__ __forceinline__ int last_of_wave(const int *sums, int R, int x) {
    const int lane = (int)threadIdx.x & 63;
    int lo[2] = {0, 0}, n = R;
    const int ends[2] = {__builtin_amdgcn_readlane(x, 0), __builtin_amdgcn_readlane(x, 63)};
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        int v[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) v[e] = sums[at < n && lo[e] + at < R ? lo[e] + at : 0];
#pragma unroll
        for (int e = 0; e < 2; ++e)
            lo[e] += step * (63 - __clzll((long long)__ballot(at == 0 || (at < n && lo[e] + at < R && v[e] <= ends[e]))));
        n = step;
    }
    return last_at_most(sums, lo[0], lo[1] + 1, x);
}

// The pages taken and the tokens, from those numbered `first` on in steps of `step`, a wave's
// lanes side by side.
__device__ __forceinline__ void fill(const PagedResize &a, const Div &by_page, const int *held, const int *wanted, const int *offsets,
                                     int taken, int top, long long first, long long step)
{
    const int lane = (int)threadIdx.x & 63;
    for (long long i = first; i - lane < taken; i += step) {   // those wanted first, as far as they were there
        const int r = last_of_wave(wanted, a.R, i < taken ? (int)i : taken - 1);
        if (i >= taken) break;
        const int has = pages_of(by_page, a.page, held[r] & INT_MAX);
        a.table[(size_t)r * a.ld_table + has + ((int)i - wanted[r])] = a.free_pages[top - 1 - (int)i];
    }
    if (!a.positions && !a.slots) return;
    const int tokens = offsets[a.R];
    for (long long i = first; i - lane < a.N; i += step) {
        int pos = 0;
        long long slot = -1;
        const int r = i - lane < tokens ? last_of_wave(offsets, a.R, i < tokens ? (int)i : tokens - 1) : 0;
        if (i >= a.N) break;
        if (i < tokens) {
            const int h = held[r];
            pos = (h & INT_MAX) + ((int)i - offsets[r]);
            if (a.slots && h >= 0) {   // granted: below 2^30
                const int j = (int)by_page((unsigned)pos), has = pages_of(by_page, a.page, h);
                // a page taken now may not be in the table yet
                const int pg = j < has ? a.table[(size_t)r * a.ld_table + j] : a.free_pages[top - 1 - (wanted[r] + (j - has))];
                if (pg >= 0 && pg < a.pages) slot = (long long)pg * a.page + (pos - j * a.page);
            }
        }
        if (a.positions) a.positions[i] = pos;
        if (a.slots) a.slots[i] = slot;
    }
}

constexpr int kAhead = 8;   // returned pages of a lane on their way together

// ALL: at most kRows rows, and few enough pages and tokens for one workgroup.
template <bool ALL>
__global__ __launch_bounds__(kRows) void resize_rows_kernel(PagedResize a, Div by_page, Sums s)
{
    __shared__ unsigned part[3][kParts], valid_of[kAhead * kParts];
    __shared__ int cut[kRows], keep[kRows];   // pages returned by the rows before, and pages that a row keeps
    __shared__ int held_of[ALL ? kRows : 1], wanted_of[ALL ? kRows + 1 : 1], offset_of[ALL ? kRows + 1 : 1], most;
    const int tid = (int)threadIdx.x, lane = tid & 63, w = tid / kWave;
    const int cap = a.cols * a.page, blocks = (a.R + kRows - 1) / kRows;
    int count = *a.free_count;
    unsigned pushed = (unsigned)(count < 0 ? 0 : count > a.pages ? a.pages : count);
    if (tid == 0) most = 0;

    Change c{};
    // The last row's last page goes on the stack first: rows and pages from the last to the first.
    for (int b = blocks - 1; b >= 0; --b) {
        const int r0 = b * kRows, r = r0 + tid;
        c = Change{};
        if (r < a.R) c = change_of(a, by_page, a.kv_len[r], a.want[r]);
        const int cuts = c.need < c.has ? c.has - c.need : 0;
        if (!__syncthreads_or(cuts)) continue;
        const Scan at = block_scan((unsigned)cuts, part[0]);   // the table has at most INT_MAX entries
        cut[tid] = (int)at.before, keep[tid] = c.need;
        const unsigned all = at.all;   // 2^31 - 1 at most; q0 may end behind that
        __syncthreads();
        for (unsigned q0 = 0; q0 < all; q0 += kAhead * kRows) {
            int pg[kAhead], *from[kAhead], i[kAhead], f[kAhead];
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                const unsigned q = q0 + (unsigned)(e * kRows + tid);
                pg[e] = q < all ? 0 : -1;
                f[e] = (int)(all - 1 - (q < all ? q : all - 1));
                i[e] = 0;
            }
#pragma unroll
            for (int half = kRows / 2; half > 0; half /= 2) {   // the row of each, all at once
#pragma unroll
                for (int e = 0; e < kAhead; ++e) i[e] += cut[i[e] + half] <= f[e] ? half : 0;
            }
#pragma unroll
            for (int e = 0; e < kAhead; ++e)
                from[e] = a.table + (size_t)(r0 + i[e]) * a.ld_table + keep[i[e]] + (f[e] - cut[i[e]]);
#pragma unroll
            for (int e = 0; e < kAhead; ++e) pg[e] |= *from[e];   // -1 where there is none
            unsigned long long valid[kAhead];
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                valid[e] = __ballot(pg[e] >= 0 && pg[e] < a.pages);
                if (lane == 0) valid_of[e * kParts + w] = (unsigned)__popcll(valid[e]);
            }
            __syncthreads();
            unsigned sums[kAhead * kParts / kWave], here = 0;   // of the pages before, 64 waves' at a time
#pragma unroll
            for (int x = 0; x < kAhead * kParts / kWave; ++x) {
                sums[x] = here + scan(valid_of[x * kWave + lane]);
                here = lane_of(sums[x], 63);
            }
#pragma unroll
            for (int e = 0; e < kAhead; ++e) {
                if (q0 + (unsigned)(e * kRows + tid) >= all) continue;
                *from[e] = -1;
                const int before = e * kParts + w;
                const unsigned to = pushed + (before ? lane_of(sums[(before - 1) / kWave], (before - 1) % kWave) : 0) + (unsigned)__popcll(valid[e] & ((1ull << lane) - 1));
                if ((valid[e] >> lane & 1) && to < (unsigned)a.pages) a.free_pages[to] = pg[e];   // no more than there are
            }
            pushed += here;   // below 2^32: at most 2^31 pages and entries each
            __syncthreads();
        }
    }
    const int top = pushed < (unsigned)a.pages ? (int)pushed : a.pages;

    unsigned wanted = 0, tokens = 0;   // by the rows before
    for (int b = 0; b < blocks; ++b) {
        const int r = b * kRows + tid;
        if (b > 0) {   // the first is the one that the loop above ended with
            c = Change{};
            if (r < a.R) c = change_of(a, by_page, a.kv_len[r], a.want[r]);
            __syncthreads();
        }
        const bool fits = c.want <= cap;
        const unsigned more = fits && c.need > c.has ? (unsigned)(c.need - c.has) : 0;
        const Scan x = block_scan(more, part[1]), y = block_scan((unsigned)c.added(), part[2]);
        const unsigned before = add_up(wanted, x.before), run = add_up(before, more);
        const bool ok = fits && (more == 0 || run <= (unsigned)top);
        const int off = (int)add_up(tokens, y.before), end = (int)add_up((unsigned)off, (unsigned)c.added());
        // what the last granted row that needs pages leaves
        const unsigned long long granted = __ballot(ok && more > 0);
        if (granted && lane == 63 - __clzll((long long)granted)) atomicMax(&most, (int)run);
        if (r < a.R) {
            if (ok) a.kv_len[r] = c.want;
            if (a.start) a.start[r] = c.held;
            if (a.offsets) a.offsets[r + 1] = end;
            const int h = ok ? c.held : c.held | INT_MIN;
            if constexpr (ALL) held_of[tid] = h, wanted_of[tid] = (int)before, offset_of[tid + 1] = end;
            else s.held[r] = h, s.wanted[r] = (int)before, s.offsets[r + 1] = end;
        }
        // Nothing is taken by a refused row's tokens: its table names no page where they would lie
        for (unsigned long long left = __ballot(!ok && c.need > c.has); left; left &= left - 1) {
            const int from = __ffsll((long long)left) - 1, row = b * kRows + w * kWave + from;
            const int behind = (int)lane_of((unsigned)c.has, from), need = (int)lane_of((unsigned)c.need, from);
            for (int j = behind + lane; j < need && j < a.cols; j += kWave) a.table[(size_t)row * a.ld_table + j] = -1;
        }
        wanted = add_up(wanted, x.all), tokens = add_up(tokens, y.all);
    }
    __syncthreads();
    const int taken = most;
    if (tid == 0) {
        if (a.offsets) a.offsets[0] = 0;
        *a.free_count = top - taken;
        if constexpr (ALL) offset_of[0] = 0;
        else s.offsets[0] = 0, *s.taken = taken, *s.top = top;
    }
    if constexpr (ALL) {
        __syncthreads();
        fill(a, by_page, held_of, wanted_of, offset_of, taken, top, tid, kRows);
    }
}

__global__ __launch_bounds__(256) void resize_fill_kernel(PagedResize a, Div by_page, Sums s)
{
    fill(a, by_page, s.held, s.wanted, s.offsets, *s.taken, *s.top, (long long)blockIdx.x * 256 + threadIdx.x,
         (long long)gridDim.x * 256);
}

}  // namespace

size_t paged_resize_workspace_bytes(int R) { return ((size_t)3 * R + 4) * sizeof(int); }

hipError_t launch_paged_resize(const PagedResize &a, hipStream_t stream)
{
    int *ws = reinterpret_cast<int *>(a.workspace);
    const Sums s{ws + 2, ws + 2 + a.R, ws + 2 + 2 * (size_t)a.R, ws, ws + 1};
    const Div by_page = make_div(a.page);
    // the tokens known here, and as many pages as they can take or, without them, as there are
    const long long most = (a.positions || a.slots ? a.N : 0) + (a.N > 0 ? (long long)a.N / a.page + a.R : a.pages);
    const bool all = a.R <= kRows && most <= 4 * kRows;
    hipLaunchKernelGGL(all ? resize_rows_kernel<true> : resize_rows_kernel<false>, dim3(1), dim3(kRows), 0, stream, a, by_page, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || all) return e;
    const long long groups = (most + 255) / 256;
    hipLaunchKernelGGL(resize_fill_kernel, dim3((unsigned)(groups < 2048 ? groups : 2048)), dim3(256), 0, stream, a, by_page, s);
    return hipGetLastError();
}

}  // namespace fs
