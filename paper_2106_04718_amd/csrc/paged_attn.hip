// Attention of one new token per row over a paged key-value cache, for gfx950.
//
// For row r and query head h, reading key-value head h / G: softmax(scale q K^T) V
// over the row's first L positions, which lie in the pages that the row's table
// names.  Every byte of K and V that a row attends is needed once for its G
// query heads, about 2 G flop per 2-byte element: bound by HBM bandwidth.
//
// Tiles.  A wave attends 32 positions for up to 16 query heads at a time on the
// matrix cores, straight from global memory to the operand registers; lane
// l = 16 g + n:
//   QK^T  S^T[key][head] = K . q^T, two blocks of 16 keys.  Lane: key 16 kb + n,
//         16 bytes per step at dim 32 s + 8 g (bf16; 16 s + 4 g in fp32).  It
//         gets the scores of head n for the keys 16 kb + 4 g + i.
//   PV    O^T[dim][head] = V^T . P^T, contracting over the keys in the order in
//         which the score registers hold them, so that P^T needs no exchange
//         between lanes.  Lane: of each of its eight keys the D / 16 elements
//         that begin at n D / 16, so that 16 lanes read a whole row; a
//         transposition of 16-bit pairs inside the lane makes the operands.
//         Lane l gets 4 D / 16 elements of head n, and its softmax state needs
//         no exchange either.
// For bf16 values the weights are taken as the sum of three bf16 values, which hold
// all 24 bits of them.  The third costs nothing measurable (64 ragged rows 108 us,
// 128 of 12 heads of 64 49 us, with it and without); with two, 2 to 3 results in 1000
// were not the bf16 value next to the exact one, with three 0.2 to 0.6.
//
// Division of the work.  The positions of all rows are cut into chunks of c units
// of 128 (4 waves), c such that as many workgroups as fit the chip, or a few times as
// many, have one each: lengths are known on the device alone, so every workgroup adds them up and finds its
// own chunk (up to kScanRows rows; above, a kernel before this one does it for
// all).  Few rows are thus spread over the chip, and a long row among short ones
// is no one workgroup's.  A row that is one chunk is written at once.  The chunks
// of the others leave their softmax states in the workspace, and the last of
// them to arrive joins them, in the order of the chunks: groups of about the
// square root of their number first.
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "div.h"
#include "grid.h"
#include "launch.h"
#include "paged_tile.h"

namespace fs {
namespace {

constexpr int kHeads = 16;              // query heads of a workgroup
constexpr int kPlaces = 512;            // workgroups that fit the 256 CUs at once, two each (some kernels three)
constexpr int kTasks = 4 * kPlaces;     // chunks at most, but for one begun per row
constexpr int kJoin = 64;               // states joined at a time
constexpr int kScanRows = 256;          // rows whose lengths every workgroup looks at: four a lane

// What a launch knows beside PagedAttn.
struct Geo {
    Div by_page, by_ht, by_hkv;
    int G, heads;              // query heads of a key-value head, and of a workgroup
    int ht;                    // workgroups side by side over one chunk: Hkv * ceil(G / kHeads)
    unsigned page16, slot16;   // strides in units of 16 bytes
    int record;                // floats of a chunk's state: heads * (D + 2)
    unsigned *group_count, *row_count;   // arrivals, by the first record of the group or row
    const int4 *tasks;         // made before the launch (more than kScanRows rows), or null
    float *records;
};

// One chunk: units [first, first + c) of row r, the split-th of `splits`; the
// records of the row's chunks are slot .. slot + splits - 1 (times ht).
struct Task {
    int r, split, splits, slot, c;
};

__device__ __forceinline__ int units_of(int L) { return L <= 0 ? 1 : (L + kUnit - 1) / kUnit; }

__device__ __forceinline__ int clamp_len(const PagedAttn &a, int L) {
    const int cap = a.cache.cols * a.cache.page;
    return L < 0 ? 0 : L > cap ? cap : L;
}

// Units per chunk for a total of `units` (of all rows; each is attended by ht
// workgroups).  As many chunks as workgroups fit the CUs at once; where that makes
// them long, two or four times as many, so that they end together (64 ragged rows of
// 2000 positions: 110 us with chunks of 9 units, 121 with 17).  Where they are short,
// `spare` of the places are left to the chunks that the rows' ends add: a few of them
// would run after all others (40 rows, 16 heads a key-value head: 83 us, not 94).  That
// may make them long again (us as they are and halved: 19 units 92 and 97, 20 units 100 and
// 103; 21 and 22 units 103 and 105, 109 and 102, 98 and 94, 104 and 100).
__device__ __forceinline__ int chunk_units(unsigned long long units, int ht, int spare) {
    const unsigned long long all = units * ht;
    unsigned long long c = (all + kPlaces - 1) / kPlaces;
    if (c > 16) c = (c + 1) / 2;
    else if (spare && (c = (all + kPlaces - spare - 1) / (kPlaces - spare)) > 20) c = (c + 1) / 2;
    if (c > 24) c = (c + 1) / 2;
    return c < 1 ? 1 : c > (1 << 24) ? 1 << 24 : (int)c;
}
__device__ __forceinline__ int spare_places(int R, int ht) { return R * ht / 2 < kPlaces / 4 ? R * ht / 2 : kPlaces / 4; }

// The t-th chunk of up to kScanRows rows; false: there are fewer.
__device__ __forceinline__ bool find_task(const PagedAttn &a, int ht, int t, Task &out) {
    const int lane = (int)threadIdx.x & 63;
    int u[4], s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = a.kv_len[4 * lane + i < a.R ? 4 * lane + i : a.R - 1];   // all in flight at once
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = 4 * lane + i < a.R ? units_of(clamp_len(a, u[i])) : 0;
    // the sum may pass 32 bits: the upper and lower halves of the units apart
    int lo = 0, hi = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) lo += u[i] & 0xffff, hi += u[i] >> 16;
    lo = wave_sum(lo);
    hi = wave_sum(hi);
    const unsigned long long units = ((unsigned long long)hi << 16) + (unsigned)lo;
    int c = chunk_units(units, ht, 0), count = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) count += (u[i] + c - 1) / c;
    if ((long long)wave_sum(count) * ht > kPlaces) c = chunk_units(units, ht, spare_places(a.R, ht));
    int chunks = 0, split_chunks = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] = (u[i] + c - 1) / c;
        chunks += s[i];
        split_chunks += s[i] > 1 ? s[i] : 0;
    }
    const int all = wave_scan(chunks), slots = wave_scan(split_chunks);
    const unsigned long long past = __ballot(all > t);
    if (past == 0) return false;
    int at = all - chunks, slot = slots - split_chunks, row = 4 * lane, n = 1, first = at;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (at <= t && s[i] > 0) row = 4 * lane + i, n = s[i], first = at;
        if (at <= t && at + s[i] <= t) slot += s[i] > 1 ? s[i] : 0;
        at += s[i];
    }
    const int owner = __ffsll((long long)past) - 1;
    out.r = __builtin_amdgcn_readlane(row, owner);
    out.split = t - __builtin_amdgcn_readlane(first, owner);
    out.splits = __builtin_amdgcn_readlane(n, owner);
    out.slot = __builtin_amdgcn_readlane(slot, owner);
    out.c = c;
    return true;
}

// The chunks of any number of rows, by one workgroup: tasks[1 + t] = (row,
// split, splits, slot), tasks[0] = (number of chunks, units per chunk).  It costs 2.4 us
// where the rows are short (256 and 257 of up to 64 positions: 9.0 and 11.4), 6 where they
// are cut (of up to 1000 positions, 530 MB: 95 and 101).
__global__ __launch_bounds__(1024) void paged_plan_kernel(PagedAttn a, int ht, int4 *tasks) {
    __shared__ unsigned long long total;
    __shared__ int part[2][16], base[2];
    const int tid = (int)threadIdx.x, lane = tid & 63, w = tid / kWave;
    if (tid == 0) total = 0, base[0] = base[1] = 0;
    __syncthreads();
    unsigned long long mine = 0;
    for (int r = tid; r < a.R; r += 1024) mine += units_of(clamp_len(a, a.kv_len[r]));
    atomicAdd(&total, mine);
    __syncthreads();
    // places are left without a look at the chunks' number: rows alone make more than kScanRows of them
    const int c = chunk_units(total, ht, spare_places(a.R, ht));
    for (int r0 = 0; r0 < a.R; r0 += 1024) {
        const int r = r0 + tid;
        const int s = r < a.R ? (units_of(clamp_len(a, a.kv_len[r])) + c - 1) / c : 0, m = s > 1 ? s : 0;
        const int x = wave_scan(s), y = wave_scan(m);
        if (lane == 63) part[0][w] = x, part[1][w] = y;
        __syncthreads();
        int t = base[0] + x - s, slot = base[1] + y - m;
        for (int i = 0; i < w; ++i) t += part[0][i], slot += part[1][i];
        for (int i = 0; i < s; ++i) tasks[1 + t + i] = make_int4(r, i, s, slot);
        __syncthreads();
        if (tid == 1023) base[0] = t + s, base[1] = slot + m;
        __syncthreads();
    }
    if (tid == 0) tasks[0] = make_int4(base[0], c, 0, 0);
}

// Up to kHeads query heads on a key-value head, each byte is read once a call.  A cache
// that the last level (256 MB) does not keep until the next call is then streamed past
// it, a small one may stay there (us, streamed and not: 2 GB 342 and 364, 787 MB 128 and
// 142, 235 MB 52 and 56; 50 MB 18.2 and 16.3).  More heads are of several workgroups,
// which read the same bytes: never streamed (64 heads on one, 393 MB: 310 and 243; 32 on
// each of two, 197 MB: 93 and 77; 24 on each of eight, 787 MB: 316 and 248).
constexpr long long kStays = 128ll << 20;

// Three where the registers allow it: small caches gain (D = 64; 33 MB 11.8 us, with two
// 12.3; 50 MB 16.4 and 16.7), large ones do not (230 MB 52 to 53 with either).
template <int D, bool BF16>
constexpr int kWavesPerSimd = BF16 && D <= 64 ? 3 : 2;

template <int D, bool BF16, bool STREAM>
__global__ __launch_bounds__(kBlock, (kWavesPerSimd<D, BF16>)) void paged_attn_kernel(PagedAttn a, Geo geo)
{
    using T = Tile<D, BF16, STREAM>;
    constexpr int kEsize = BF16 ? 2 : 4, kPad = D + 4;
    constexpr bool kHalf = BF16 && D == 16;   // a row is half of what an instruction contracts
    __shared__ __align__(16) float so[kWaves][kHeads][kPad];
    __shared__ float sm[kWaves][kHeads], sl[kWaves][kHeads];
    __shared__ float sf[kJoin][kHeads], sg[kJoin][kHeads];
    __shared__ unsigned arrived;

    const int lane = (int)threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int n = lane & 15, g = lane >> 4;
    const unsigned wg = wide_index();
    const int t = (int)geo.by_ht(wg), ht = (int)wg - t * geo.ht;
    Task task;
    if (geo.tasks) {
        const int4 head = geo.tasks[0];
        if (t >= head.x) return;
        const int4 x = geo.tasks[1 + t];
        task = Task{x.x, x.y, x.z, x.w, head.y};
    } else if (!find_task(a, geo.ht, t, task)) {
        return;
    }
    const int qt = (int)geo.by_hkv(ht), h = ht - qt * a.Hkv;
    const int heads = geo.G - qt * kHeads < kHeads ? geo.G - qt * kHeads : kHeads;
    const int r = task.r, given = a.kv_len[r], L = clamp_len(a, given);
    const int begin = task.split * task.c * kUnit;   // below 2^31: a unit of the row's
    const int end = L - begin < task.c * (long long)kUnit ? L : begin + task.c * kUnit;

    // queries: column n, zero past the heads
    u32x4_t q[T::kSteps];
    {
        const unsigned char *qp = a.q + (size_t)r * a.q_row_bytes +
                                  (size_t)(h * geo.G + qt * kHeads + (n < heads ? n : 0)) * a.q_head_bytes;
#pragma unroll
        for (int s = 0; s < T::kSteps; ++s) q[s] = *reinterpret_cast<const u32x4_t *>(qp + 64 * s + 16 * (kHalf ? g & 1 : g));
#pragma unroll
        for (int s = 0; s < T::kSteps; ++s) {
            if (n >= heads || (kHalf && g >= 2)) q[s] = u32x4_t{0u, 0u, 0u, 0u};
        }
    }
    const PagedCache &c = a.cache;
    const unsigned char *Kh = c.K + (size_t)h * c.head_bytes, *Vh = c.V + (size_t)h * c.head_bytes;
    const int32_t *table = c.table + (size_t)r * c.ld_table;
    const size_t fresh_off = (size_t)r * a.new_row_bytes + (size_t)h * a.new_head_bytes;
    const int fresh = a.k && given == L ? L - 1 : -1;   // a row past its table has no place for the token

    // Pages: lane l looks up position t0 + l % 32 of a tile, two tiles ahead of
    // its use; `off` is the position's slot in units of 16 bytes and `live` the
    // tile's positions that exist.
    auto page_of = [&](int t0) {
        const int pos = t0 + (lane & 31);
        const int pg = table[geo.by_page((unsigned)(pos < end ? pos : begin))];
        return pos < end ? pg : -1;
    };
    auto slot_of = [&](int t0, int pg, unsigned &off, unsigned &live) {
        const int pos = t0 + (lane & 31);
        const bool ok = pg >= 0 && pg < c.pages;
        off = ok ? (unsigned)pg * geo.page16 + (unsigned)(pos - (int)geo.by_page((unsigned)pos) * c.page) * geo.slot16 : 0u;
        live = (unsigned)__ballot(ok);
    };
    auto row_of = [&](const unsigned char *base, const unsigned char *mine, unsigned off, int t0, int key) {
        const unsigned o = (unsigned)__builtin_amdgcn_ds_bpermute(key << 2, (int)off);
        const unsigned char *p = base + (size_t)o * 16;
        return t0 + key == fresh ? mine + fresh_off : p;
    };
    T x;
    auto load_k = [&](int t0, unsigned off) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) x.load_k(kb, row_of(Kh, a.k, off, t0, 16 * kb + n), g);
    };
    auto load_v = [&](int t0, unsigned off) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x.load_v(j, row_of(Vh, a.v, off, t0, 16 * (j / 4) + 4 * g + j % 4), n);
    };

    const float scale = a.scale * 1.44269504f;   // scores in the base-2 domain
    f32x4_t o[T::kVe];
#pragma unroll
    for (int e = 0; e < T::kVe; ++e) o[e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    bool any = false;

    // the softmax of a tile's scores, then its values
    auto attend = [&](f32x4_t (&sc)[2], unsigned live) {
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[kb][i] *= scale;
        }
        if (live != 0xffffffffu) {   // a position that is not there read anything: its weight is 0, its value too
            const unsigned mine = live >> (4 * g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool is = (mine >> (16 * (j / 4) + j % 4)) & 1u;
                sc[j / 4][j % 4] = is ? sc[j / 4][j % 4] : -INFINITY;
#pragma unroll
                for (int e = 0; e < T::kVwords; ++e) x.v[j][e] = is ? x.v[j][e] : 0u;
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) mx = fmaxf(mx, sc[j / 4][j % 4]);
        any |= live != 0u;
        mx = fmaxf(m, col_max(mx));
        if (__any(mx > m)) {
            const float f = weight(m, mx);
            l *= f;
#pragma unroll
            for (int e = 0; e < T::kVe; ++e) o[e] *= f;
            m = mx;
        }
        f32x8_t p;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            p[j] = weight(sc[j / 4][j % 4], m);
            l += p[j];
        }
        x.accumulate(p, o);
    };

    int t0 = begin + w * kTile;
    if (t0 < end) {
        // The keys of the next tile are asked for as soon as this tile's scores
        // are there, its values behind this tile's: a tile of each is always on
        // its way.  Loads stand outside of every branch, or the compiler waits
        // for all of them where the branches meet.
        unsigned off, live;
        f32x4_t sc[2];
        const int pg = page_of(t0);
        int pg_next = page_of(end - t0 > kUnit ? t0 + kUnit : t0);
        slot_of(t0, pg, off, live);
        load_k(t0, off);
        load_v(t0, off);
        while (end - t0 > kUnit) {
            const int t1 = t0 + kUnit;
            sc[0] = x.scores(0, q), sc[1] = x.scores(1, q);
            unsigned off_next, live_next;
            slot_of(t1, pg_next, off_next, live_next);
            pg_next = page_of(end - t1 > kUnit ? t1 + kUnit : t1);
            load_k(t1, off_next);
            attend(sc, live);
            load_v(t1, off_next);
            t0 = t1, off = off_next, live = live_next;
        }
        sc[0] = x.scores(0, q), sc[1] = x.scores(1, q);
        attend(sc, live);
        // the new token's own row: it is in the last tile of the wave that has it
        if (fresh >= t0 && fresh - t0 < kTile && qt == 0 && ((live >> (fresh - t0)) & 1u)) {
            const size_t to = (size_t)(unsigned)__builtin_amdgcn_readlane((int)off, fresh - t0) * 16;
            constexpr int kPer = D * kEsize / 16;
            if (lane < kPer) {
                *reinterpret_cast<u32x4_t *>(const_cast<unsigned char *>(Kh) + to + 16 * lane) =
                    *reinterpret_cast<const u32x4_t *>(a.k + fresh_off + 16 * lane);
                *reinterpret_cast<u32x4_t *>(const_cast<unsigned char *>(Vh) + to + 16 * lane) =
                    *reinterpret_cast<const u32x4_t *>(a.v + fresh_off + 16 * lane);
            }
        }
    }

    // the four waves' states, joined
    l = col_sum(l);
    if (n < heads) {
#pragma unroll
        for (int e = 0; e < T::kVe; ++e) {
#pragma unroll
            for (int i = 0; i < 4; ++i) so[w][n][T::dim_of(e, 4 * g + i)] = o[e][i];
        }
        if (g == 0) sm[w][n] = m, sl[w][n] = any ? l : -1.f;
    }
    __syncthreads();
    unsigned char *out = a.out + ((size_t)r * a.Hq + (size_t)h * geo.G + qt * kHeads) * D * kEsize;
    const bool whole = task.splits == 1;
    float *rec = geo.records + ((size_t)(task.slot + task.split) * geo.ht + ht) * geo.record;
    for (int i = (int)threadIdx.x; i < heads * D; i += kBlock) {
        const int hd = i / D, d = i % D;
        float oo, mm, ll;
        join([&](int k, int what) { return what == 0 ? so[k][hd][d] : what == 1 ? sm[k][hd] : sl[k][hd]; }, oo, mm, ll);
        if (whole) {
            store_out<BF16>(out, i, ll < 0.f ? 0.f : oo / ll);
        } else {
            put(rec + i, oo);
            if (d == 0) put(rec + geo.heads * D + 2 * hd, mm), put(rec + geo.heads * D + 2 * hd + 1, ll);
        }
    }
    if (whole) return;

    // Arrivals.  A record has arrived before its workgroup counts itself, and is
    // read by the workgroup that counts last; counters end at zero.
    int group = task.splits;   // chunks of a group: at most 64, and as many groups (a row has at most kTasks + 1)
    if (task.splits > 16) {
        group = 16;
        while (group * group < task.splits) group *= 2;
    }
    static_assert((kJoin & (kJoin - 1)) == 0 && kJoin * kJoin >= kTasks + 1, "groups and their number fit the arrays");
    const int groups = (task.splits + group - 1) / group;
    for (int level = 0; level < 2; ++level) {
        // level 0: the chunks of this one's group, into its first record; level 1: the groups
        if (level == 1 && groups == 1) break;
        const int first = level == 0 ? task.split / group * group : 0;
        const int count = level == 0 ? (task.splits - first < group ? task.splits - first : group) : groups;
        const int step = level == 0 ? 1 : group;
        unsigned *counter = (level == 0 ? geo.group_count : geo.row_count) + (size_t)(task.slot + first) * geo.ht + ht;
        __builtin_amdgcn_s_waitcnt(0);   // this thread's stores have arrived, then everybody's
        __syncthreads();
        if (threadIdx.x == 0)
            arrived = count > 1 ? __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
        __syncthreads();
        if (arrived != (unsigned)count - 1) return;
        if (threadIdx.x == 0 && count > 1) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        float *base = geo.records + ((size_t)(task.slot + first) * geo.ht + ht) * geo.record;
        const size_t stride = (size_t)step * geo.ht * geo.record;
        const bool last = level == 1 || groups == 1;
        // each state's share of the joined one: exp2 of its maximum's distance, in sf
        for (int i = (int)threadIdx.x; i < count * heads; i += kBlock) {
            const int k = i / heads, hd = i - k * heads;
            const float *state = base + k * stride + geo.heads * D + 2 * hd;
            const float mm = get(state), ll = get(state + 1);
            sf[k][hd] = ll < 0.f ? -INFINITY : mm, sg[k][hd] = ll;
        }
        __syncthreads();
        if ((int)threadIdx.x < heads) {
            const int hd = (int)threadIdx.x;
            float top = -INFINITY, sum = -1.f;
            for (int k = 0; k < count; ++k) top = fmaxf(top, sf[k][hd]);
            for (int k = 0; k < count; ++k) {
                const float f = weight(sf[k][hd], top), ll = sg[k][hd];
                sf[k][hd] = f;
                if (!(ll < 0.f)) sum = (sum < 0.f ? 0.f : sum) + ll * f;
            }
            sm[0][hd] = top, sl[0][hd] = sum;
        }
        __syncthreads();
        for (int i = (int)threadIdx.x; i < heads * D; i += kBlock) {
            const int hd = i / D;
            float oo = 0.f;
            for (int k0 = 0; k0 < count; k0 += 8) {   // eight on their way at a time
                float x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = get(base + (k0 + k < count ? k0 + k : k0) * stride + i);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k0 + k < count) oo += x[k] * sf[k0 + k][hd];
            }
            const float ll = sl[0][hd];
            if (last) store_out<BF16>(out, i, ll < 0.f ? 0.f : oo / ll);
            else put(base + i, oo);   // read by this thread alone
        }
        if (!last && (int)threadIdx.x < heads) {
            const int hd = (int)threadIdx.x;
            put(base + geo.heads * D + 2 * hd, sm[0][hd]), put(base + geo.heads * D + 2 * hd + 1, sl[0][hd]);
        }
    }
}

struct Layout {
    int G, heads, ht, record;
    long long grid, slots;             // workgroups and records at most
    size_t row_count, tasks, records, bytes;   // byte offsets in the workspace
};

Layout layout_of(int R, int Hq, int Hkv, int page, int cols, int D) {
    Layout y{};
    y.G = Hq / Hkv;
    y.heads = y.G < kHeads ? y.G : kHeads;
    y.ht = Hkv * ((y.G + kHeads - 1) / kHeads);
    y.record = y.heads * (D + 2);
    const long long units = ((long long)cols * page + kUnit - 1) / kUnit, most = units < 1 ? 1 : units;
    // a chunk of a cut row is more than half used on average: at most 2 kTasks of them
    y.slots = 2ll * kTasks < (long long)R * y.ht * most ? 2ll * kTasks : (long long)R * y.ht * most;
    y.grid = kTasks + (long long)R * y.ht;
    if (y.grid > (long long)R * y.ht * most) y.grid = (long long)R * y.ht * most;
    // the counters lie where every call has them, whatever its sizes
    y.row_count = 2 * kTasks * sizeof(unsigned);
    y.tasks = 2 * y.row_count;
    y.records = y.tasks + (R > kScanRows ? ((size_t)R + kTasks + 1) * sizeof(int4) : 0);
    y.bytes = y.records + (size_t)y.slots * y.record * sizeof(float);
    return y;
}

}  // namespace

size_t paged_attn_workspace_bytes(int R, int Hq, int Hkv, int page, int cols, int D) {
    return layout_of(R, Hq, Hkv, page, cols, D).bytes;
}

hipError_t launch_paged_attn(const PagedAttn &a, int D, bool bf16, hipStream_t stream)
{
    const Layout y = layout_of(a.R, a.Hq, a.Hkv, a.cache.page, a.cache.cols, D);
    Geo geo{};
    geo.by_page = make_div(a.cache.page), geo.by_ht = make_div(y.ht), geo.by_hkv = make_div(a.Hkv);
    geo.G = y.G, geo.heads = y.heads, geo.ht = y.ht, geo.record = y.record;
    geo.page16 = (unsigned)(a.cache.page_bytes / 16), geo.slot16 = (unsigned)(a.cache.slot_bytes / 16);
    geo.group_count = reinterpret_cast<unsigned *>(a.workspace);
    geo.row_count = reinterpret_cast<unsigned *>(a.workspace + y.row_count);
    geo.records = reinterpret_cast<float *>(a.workspace + y.records);
    if (a.R > kScanRows) {
        auto *tasks = reinterpret_cast<int4 *>(a.workspace + y.tasks);
        geo.tasks = tasks;
        hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(1024), 0, stream, a, y.ht, tasks);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 gd = wide_grid(y.grid), bd(kBlock);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, gd, bd, 0, stream, a, geo); };
    const PagedCache &c = a.cache;
    const bool stream_past = y.G <= kHeads && 2ll * c.pages * c.page * a.Hkv * D * (bf16 ? 2 : 4) > kStays;
    auto of_width = [&](auto width) {
        constexpr int W = decltype(width)::value;
        if (bf16) stream_past ? launch(paged_attn_kernel<W, true, true>) : launch(paged_attn_kernel<W, true, false>);
        else stream_past ? launch(paged_attn_kernel<W, false, true>) : launch(paged_attn_kernel<W, false, false>);
    };
    switch (D) {
    case 16: of_width(std::integral_constant<int, 16>{}); break;
    case 32: of_width(std::integral_constant<int, 32>{}); break;
    case 64: of_width(std::integral_constant<int, 64>{}); break;
    default: of_width(std::integral_constant<int, 128>{}); break;
    }
    return hipGetLastError();
}

}  // namespace fs
