// Rows of a paged cache that grow and shrink, for gfx950: pages taken from a stack of free
// ones and given back, and the position and slot of every new token.
//
// Which pages a row gets follows from sums over the rows before it: of the pages returned,
// of the pages wanted (a row is granted while their sum is within what is free) and of the
// new tokens.  One workgroup makes these sums, a row a lane and 1024 rows at a time, and
// takes the returned pages; what is then one independent step per page taken and per token
// is done by the same workgroup where these are few, or by a second kernel over the chip.
//
// Bound by latency: the first kernel is a chain of some ten trips (lengths, sums, pages) and the
// launches cost more than the bytes.
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

typedef unsigned long long u64_t;

__device__ __forceinline__ u64_t up(u64_t x, int by) {
    const unsigned lo = __shfl_up((unsigned)x, by), hi = __shfl_up((unsigned)(x >> 32), by);
    return (u64_t)hi << 32 | lo;
}

// Inclusive sum over the workgroup's lanes; `all` is the whole.
__device__ __forceinline__ u64_t block_scan(u64_t x, u64_t *part, u64_t &all) {
    const int lane = (int)threadIdx.x & 63, w = (int)threadIdx.x / kWave;
#pragma unroll
    for (int by = 1; by < kWave; by *= 2) {
        const u64_t y = up(x, by);
        if (lane >= by) x += y;
    }
    if (lane == 63) part[w] = x;
    __syncthreads();
    u64_t before = 0;
    all = 0;
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        if (i < w) before += part[i];
        all += part[i];
    }
    __syncthreads();   // part may be used again
    return before + x;
}

// What the rows' sums leave in the workspace.  held: the positions a row held, with the
// upper bit set if it was refused; taken: pages taken by the rows before it (R + 1 of them);
// offsets: tokens before it (R + 1), no more than INT_MAX.
struct Sums {
    int *held, *taken, *offsets;
    int *top;   // pages on the stack before any was taken
};

// The last of the entries 0 .. R - 1 that is at most x (the first is 0).
__device__ __forceinline__ int last_at_most(const int *sums, int R, int x) {
    int lo = 0, hi = R;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        (sums[mid] <= x ? lo : hi) = mid;
    }
    return lo;
}

// The pages taken and the tokens, from those numbered `first` on in steps of `step`.
__device__ __forceinline__ void fill(const PagedResize &a, const Div &by_page, const Sums &s, long long first, long long step) {
    const int taken = s.taken[a.R], top = *s.top;
    for (long long i = first; i < taken; i += step) {
        const int r = last_at_most(s.taken, a.R, (int)i);
        const int has = pages_of(by_page, a.page, s.held[r] & INT_MAX);
        a.table[(size_t)r * a.ld_table + has + ((int)i - s.taken[r])] = a.free_pages[top - 1 - (int)i];
    }
    if (!a.positions && !a.slots) return;
    const int tokens = s.offsets[a.R];
    for (long long i = first; i < a.N; i += step) {
        int pos = 0;
        long long slot = -1;
        if (i < tokens) {
            const int r = last_at_most(s.offsets, a.R, (int)i), held = s.held[r];
            pos = (held & INT_MAX) + ((int)i - s.offsets[r]);
            if (a.slots && held >= 0) {   // granted: below 2^30
                const int j = (int)by_page((unsigned)pos), has = pages_of(by_page, a.page, held);
                // a page taken now may not be in the table yet
                const int pg = j < has ? a.table[(size_t)r * a.ld_table + j] : a.free_pages[top - 1 - (s.taken[r] + (j - has))];
                if (pg >= 0 && pg < a.pages) slot = (long long)pg * a.page + (pos - j * a.page);
            }
        }
        if (a.positions) a.positions[i] = pos;
        if (a.slots) a.slots[i] = slot;
    }
}

__global__ __launch_bounds__(kRows) void resize_rows_kernel(PagedResize a, Div by_page, Sums s, bool all)
{
    __shared__ u64_t part[kParts];
    const int tid = (int)threadIdx.x, lane = tid & 63;
    const int cap = a.cols * a.page;
    int count = *a.free_count;
    count = count < 0 ? 0 : count > a.pages ? a.pages : count;

    // pages of the cache among those returned by the rows before, in s.taken for now
    u64_t returned = 0;
    for (int r0 = 0; r0 < a.R; r0 += kRows) {
        const int r = r0 + tid;
        Change c{};
        if (r < a.R) c = change_of(a, by_page, a.kv_len[r], a.want[r]);
        u64_t mine = 0;
        for (u64_t left = __ballot(c.need < c.has); left; left &= left - 1) {   // a wave takes such rows one by one
            const int from = __ffsll((long long)left) - 1;
            const int j0 = __shfl(c.need, from), j1 = __shfl(c.has, from);
            const int *row = a.table + (size_t)(r0 + (tid & ~63) + from) * a.ld_table;
            int n = 0;
            for (int j = j0; j < j1; j += kWave) {
                const int pg = j + lane < j1 ? row[j + lane] : -1;
                n += __popcll(__ballot(pg >= 0 && pg < a.pages));
            }
            if (lane == from) mine = n;
        }
        u64_t whole;
        const u64_t run = block_scan(mine, part, whole);
        if (r < a.R) s.taken[r] = (int)(returned + run - mine);   // the table has at most INT_MAX entries
        returned += whole;
    }
    const long long sum = count + (long long)returned;
    const int top = sum < a.pages ? (int)sum : a.pages;

    u64_t wanted = 0, tokens = 0, taken = 0;
    for (int r0 = 0; r0 < a.R; r0 += kRows) {
        const int r = r0 + tid;
        Change c{};
        if (r < a.R) c = change_of(a, by_page, a.kv_len[r], a.want[r]);
        const int before = r < a.R ? s.taken[r] : 0;
        for (u64_t left = __ballot(c.need < c.has); left; left &= left - 1) {
            const int from = __ffsll((long long)left) - 1;
            const int j0 = __shfl(c.need, from), j1 = __shfl(c.has, from);
            // the last row's last page comes first: place sum - 1 - (pages before)
            long long to = sum - 1 - __shfl(before, from);
            int *row = a.table + (size_t)(r0 + (tid & ~63) + from) * a.ld_table;
            for (int j = j0; j < j1; j += kWave) {
                const int pg = j + lane < j1 ? row[j + lane] : -1;
                const u64_t valid = __ballot(pg >= 0 && pg < a.pages);
                const long long at = to - __popcll(valid & ((1ull << lane) - 1));
                if ((valid >> lane & 1) && at < a.pages) a.free_pages[at] = pg;   // no more than there are, whatever the table holds
                if (j + lane < j1) row[j + lane] = -1;
                to -= __popcll(valid);
            }
        }
        const bool fits = c.want <= cap;
        const u64_t more = fits && c.need > c.has ? (u64_t)(c.need - c.has) : 0;
        u64_t whole;
        const u64_t run = wanted + block_scan(more, part, whole);
        wanted += whole;
        const bool ok = fits && (more == 0 || run <= (u64_t)top);
        const u64_t run_tokens = tokens + block_scan((u64_t)c.added(), part, whole);
        tokens += whole;
        const u64_t got = ok ? more : 0, run_taken = taken + block_scan(got, part, whole);
        taken += whole;
        if (r < a.R) {
            if (ok) a.kv_len[r] = c.want;
            if (a.start) a.start[r] = c.held;
            s.held[r] = ok ? c.held : c.held | INT_MIN;
            s.taken[r] = (int)(run_taken - got);
            const u64_t off = run_tokens < INT_MAX ? run_tokens : INT_MAX;
            s.offsets[r + 1] = (int)off;
            if (a.offsets) a.offsets[r + 1] = (int)off;
        }
    }
    if (tid == 0) {
        s.offsets[0] = 0;
        if (a.offsets) a.offsets[0] = 0;
        s.taken[a.R] = (int)taken;
        *s.top = top;
        *a.free_count = top - (int)taken;
    }
    if (all) {
        __syncthreads();
        fill(a, by_page, s, tid, kRows);
    }
}

__global__ __launch_bounds__(256) void resize_fill_kernel(PagedResize a, Div by_page, Sums s)
{
    fill(a, by_page, s, (long long)blockIdx.x * 256 + threadIdx.x, (long long)gridDim.x * 256);
}

}  // namespace

size_t paged_resize_workspace_bytes(int R) { return ((size_t)3 * R + 4) * sizeof(int); }

hipError_t launch_paged_resize(const PagedResize &a, hipStream_t stream)
{
    int *ws = reinterpret_cast<int *>(a.workspace);
    const Sums s{ws + 1, ws + 1 + a.R, ws + 2 + 2 * (size_t)a.R, ws};
    const Div by_page = make_div(a.page);
    // the tokens known here, and as many pages as they can take or, without them, as there are
    const long long most = (a.positions || a.slots ? a.N : 0) + (a.N > 0 ? (long long)a.N / a.page + a.R : a.pages);
    const bool all = most <= 2 * kRows;
    hipLaunchKernelGGL(resize_rows_kernel, dim3(1), dim3(kRows), 0, stream, a, by_page, s, all);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || all) return e;
    const long long groups = (most + 255) / 256;
    hipLaunchKernelGGL(resize_fill_kernel, dim3((unsigned)(groups < 2048 ? groups : 2048)), dim3(256), 0, stream, a, by_page, s);
    return hipGetLastError();
}

}  // namespace fs
