// Causal attention of several new tokens per row over a paged key-value cache, for gfx950.
//
// Row r's tokens i = 0 .. n - 1 are the last n of its kv_len positions; query head h of token
// i attends the positions up to kv_len - n + i in the key-value head h / G.  A row's queries
// of one key-value head are n G columns, column m being head m % G of token m / G.
//
// Tiles.  A wave attends 32 positions for 16 NC columns at a time on the matrix cores, as
// paged_tile.h describes, its four waves the positions in turn; their softmax states are
// joined at the end.
//
// Division of the work.  The columns of a row are cut into tiles, and a tile's positions, in
// units of 128, into as many chunks as the tiles leave room on the chip for.  Lengths are
// known on the device alone, so every workgroup adds the rows' work up and finds its own
// piece (up to kScanRows rows; above, a kernel before this one does it for all).  A tile of
// one chunk is written at once; the chunks of the others leave their softmax states in the
// workspace, and the last of them to arrive joins them, in the order of the chunks.
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "div.h"
#include "grid.h"
#include "launch.h"
#include "paged_tile.h"

namespace fs {
namespace {

constexpr int kPlaces = 512;      // workgroups that fit the 256 CUs at once, two each
constexpr int kChunks = 2 * kPlaces;   // chunks that the work is cut into at most, but for one begun per tile
constexpr int kJoin = 64;         // states joined at a time
constexpr int kScanRows = 256;    // rows whose lengths every workgroup looks at: four a lane

constexpr int kWideTile = 64;     // positions that a workgroup attends at a time in a wide tile
constexpr int kWideColumns = 32 * kWaves;

template <int D, bool BF16>
constexpr int kTiles16 = BF16 || D <= 64 ? 2 : 1;   // NC: 16 columns each, as many as the registers hold
template <int D, bool BF16>
constexpr bool kHasWide = BF16 && D >= 32;

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
constexpr int kSchedValu = 0x2, kSchedMfma = 0x8, kSchedRead = 0x100;   // kinds of instructions

// What a launch knows beside PagedChunk.
struct Geo {
    Div by_page, by_hkv, by_g;
    int G;
    int narrow, wide;          // columns of a tile of a row of up to `narrow` columns, and of others
    unsigned page16, slot16;   // strides in units of 16 bytes
    int record;                // floats of a chunk's state: wide * (D + 2)
    unsigned *group_count, *tile_count;   // arrivals, by the first record of the group or tile
    const int4 *plan;          // made before the launch (more than kScanRows rows), or null
    float *records;
    long long slots;           // records that there are
};

// A row's part of the work.
struct Row {
    int first_pos;   // of its first token; may be negative, then that token attends nothing
    int begin, columns;   // first token, and columns (of one key-value head)
    int width, tiles;     // columns of a tile
    int units;            // of its last tile, the longest
};

// A piece of it: units [split * c, split * c + c) of tile `tile` of row r; the records of the
// tile's chunks begin at `slot`.
struct Task {
    int r, tile, split, splits, slot;
};

__device__ __forceinline__ int units_of(int L) { return L <= 0 ? 1 : (L + kUnit - 1) / kUnit; }

__device__ __forceinline__ Row row_of(const PagedChunk &a, const Geo &geo, int kv_len, int o0, int o1) {
    const int cap = a.cache.cols * a.cache.page;
    o0 = o0 < 0 ? 0 : o0, o1 = o1 < a.N ? o1 : a.N;   // of tokens that there are
    const int n = o1 > o0 ? o1 - o0 : 0, L = kv_len < 0 ? 0 : kv_len;
    Row w;
    w.first_pos = L - n;
    w.begin = o0;
    w.columns = n * geo.G;
    w.width = w.columns <= geo.narrow ? geo.narrow : geo.wide;   // powers of two
    w.tiles = (int)(((unsigned)w.columns + w.width - 1) >> (31 - __builtin_clz(w.width)));
    w.units = units_of(L < cap ? L : cap);
    return w;
}

// Units of a tile that begins and ends at these columns, and units per chunk for work of
// `units` (tiles of a head times their units) in all.
__device__ __forceinline__ int units_per_chunk(unsigned long long units, int heads) {
    const unsigned long long c = (units * heads + kChunks - 1) / kChunks;
    return c < 1 ? 1 : c > (1 << 24) ? 1 << 24 : (int)c;
}
__device__ __forceinline__ int splits_of(const Row &w, int c) { return (w.units + c - 1) / c; }

// Sum over the lanes of values below 2^60.
__device__ __forceinline__ unsigned long long wave_sum64(unsigned long long x) {
    const unsigned long long a = (unsigned)wave_sum((int)(x & 0xfffff)), b = (unsigned)wave_sum((int)(x >> 20 & 0xfffff)),
                             c = (unsigned)wave_sum((int)(x >> 40));
    return a + (b << 20) + (c << 40);
}

// The t-th task of up to kScanRows rows; false: there are fewer.
__device__ __forceinline__ bool find_task(const PagedChunk &a, const Geo &geo, int t, Task &out) {
    const int lane = (int)threadIdx.x & 63;
    int len[4], off[5];
#pragma unroll
    for (int i = 0; i < 4; ++i) len[i] = a.kv_len[4 * lane + i < a.R ? 4 * lane + i : a.R - 1];   // all in flight at once
#pragma unroll
    for (int i = 0; i < 5; ++i) off[i] = a.offsets[4 * lane + i < a.R ? 4 * lane + i : a.R];
    Row w[4];
    unsigned long long work = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = row_of(a, geo, len[i], off[i], off[i + 1]);   // none behind the last row: it would begin at its end
        work += (unsigned long long)w[i].tiles * (unsigned)w[i].units;
    }
    const int c = units_per_chunk(wave_sum64(work), a.Hkv);
    int s[4], tasks = 0, records = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[i] = splits_of(w[i], c);
        tasks += w[i].tiles * s[i];
        records += s[i] > 1 ? w[i].tiles * s[i] : 0;
    }
    const int all = wave_scan(tasks), slots = wave_scan(records);
    const unsigned long long past = __ballot(all > t);
    if (past == 0) return false;
    int at = all - tasks, slot = slots - records, row = 4 * lane, n = 1, m = 1, first = at, begin = slot;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int here = w[i].tiles * s[i];
        if (at <= t && here > 0) row = 4 * lane + i, n = s[i], m = w[i].tiles, first = at, begin = slot;
        at += here;
        slot += s[i] > 1 ? here : 0;
    }
    const int owner = __ffsll((long long)past) - 1;
    out.r = __builtin_amdgcn_readlane(row, owner);
    out.splits = __builtin_amdgcn_readlane(n, owner);
    const int x = t - __builtin_amdgcn_readlane(first, owner);
    out.tile = x / out.splits;
    out.split = x - out.tile * out.splits;
    out.slot = __builtin_amdgcn_readlane(begin, owner) + out.tile * out.splits;
    out.tile = __builtin_amdgcn_readlane(m, owner) - 1 - out.tile;   // the longest first
    return true;
}

// For any number of rows, by one workgroup: plan[1 + r] = (tasks and records of the rows
// before r, splits of its tiles, its tiles), plan[0] = (tasks).
__global__ __launch_bounds__(1024) void chunk_plan_kernel(PagedChunk a, Geo geo, int4 *plan) {
    __shared__ unsigned long long total;
    __shared__ int part[2][16], base[2];
    const int tid = (int)threadIdx.x, lane = tid & 63, wv = tid / kWave;
    if (tid == 0) total = 0, base[0] = base[1] = 0;
    __syncthreads();
    unsigned long long mine = 0;
    for (int r = tid; r < a.R; r += 1024) {
        const Row w = row_of(a, geo, a.kv_len[r], a.offsets[r], a.offsets[r + 1]);
        mine += (unsigned long long)w.tiles * (unsigned)w.units;
    }
    atomicAdd(&total, mine);
    __syncthreads();
    const int c = units_per_chunk(total, a.Hkv);
    for (int r0 = 0; r0 < a.R; r0 += 1024) {
        const int r = r0 + tid;
        Row w{};
        if (r < a.R) w = row_of(a, geo, a.kv_len[r], a.offsets[r], a.offsets[r + 1]);
        const int s = r < a.R ? splits_of(w, c) : 1, tasks = w.tiles * s, records = s > 1 ? tasks : 0;
        const int x = wave_scan(tasks), y = wave_scan(records);
        if (lane == 63) part[0][wv] = x, part[1][wv] = y;
        __syncthreads();
        int t = base[0] + x - tasks, slot = base[1] + y - records;
        for (int i = 0; i < wv; ++i) t += part[0][i], slot += part[1][i];
        if (r < a.R) plan[1 + r] = make_int4(t, slot, s, w.tiles);
        __syncthreads();
        if (tid == 1023) base[0] = t + tasks, base[1] = slot + records;
        __syncthreads();
    }
    if (tid == 0) plan[0] = make_int4(base[0], 0, 0, 0);
}

// The t-th task of a plan: 64 rows are looked at at a time.
__device__ __forceinline__ bool find_planned(const int4 *plan, int R, int t, Task &out) {
    if (t >= plan[0].x) return false;
    const int lane = (int)threadIdx.x & 63;
    int lo = 0, n = R;   // the last of rows lo .. lo + n - 1 that begins at or before t
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        const bool before = at < n && plan[1 + lo + at].x <= t;
        const int last = 63 - __clzll((long long)__ballot(before));   // lane 0 always is
        lo += last * step;
        n = n - last * step < step ? n - last * step : step;
    }
    const int4 x = plan[1 + lo];
    out.r = lo, out.splits = x.z;
    const int i = t - x.x;
    out.tile = i / x.z;
    out.split = i - out.tile * x.z;
    out.slot = x.y + out.tile * x.z;
    out.tile = x.w - 1 - out.tile;
    return true;
}

// What a workgroup knows of its piece of work.
struct Piece {
    int r, h, col0, cols;     // the row, the key-value head, the tile's columns
    int begin, end;           // positions of the chunk
    int seen;                 // positions that all columns attend
    int split, splits;
    Row row;
    unsigned char *out;       // of the row and head
    float *record;
    // positions that a column attends: those below its limit
    __device__ __forceinline__ int limit(const PagedChunk &a, const Geo &geo, int column) const {
        const int p = row.first_pos + (int)geo.by_g((unsigned)column), cap = a.cache.cols * a.cache.page;
        return p < 0 ? 0 : p < cap ? p + 1 : cap;
    }
    __device__ __forceinline__ const unsigned char *query(const PagedChunk &a, const Geo &geo, int column) const {
        const int token = (int)geo.by_g((unsigned)column), head = h * geo.G + column - token * geo.G;
        return a.q + (size_t)(row.begin + token) * a.q_token_bytes + (size_t)head * a.q_head_bytes;
    }
    // element d of column c of the tile
    template <int D>
    __device__ __forceinline__ size_t place(const PagedChunk &a, const Geo &geo, int c, int d) const {
        const int token = (int)geo.by_g((unsigned)(col0 + c));
        return (size_t)token * a.Hq * D + (size_t)(col0 + c - token * geo.G) * D + d;
    }
};

// Slot of position pos in units of 16 bytes, of page pg.
__device__ __forceinline__ unsigned slot16(const PagedChunk &a, const Geo &geo, int pg, int pos) {
    return (unsigned)pg * geo.page16 + (unsigned)(pos - (int)geo.by_page((unsigned)pos) * a.cache.page) * geo.slot16;
}

template <int D>
struct NarrowLds {
    float so[kWaves][16][D + 4];
    float sm[kWaves][16], sl[kWaves][16];
};

// A tile of 16 NC columns: every wave has all of them and a quarter of the positions, whose
// operands go from global memory straight to its registers.
template <int D, bool BF16>
__device__ __forceinline__ void attend_narrow(const PagedChunk &a, const Geo &geo, const Piece &w, NarrowLds<D> &lds)
{
    using T = Tile<D, BF16, false>;
    constexpr int NC = kTiles16<D, BF16>;
    constexpr bool kHalf = BF16 && D == 16;   // a row is half of what an instruction contracts
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int n = lane & 15, g = lane >> 4;
    const int begin = w.begin, end = w.end;

    // queries and limits: column 16 nc + n, zero past the last
    u32x4_t q[NC][T::kSteps];
    int lim[NC];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
        const int c = 16 * nc + n, column = w.col0 + (c < w.cols ? c : 0);
        const unsigned char *qp = w.query(a, geo, column);
        lim[nc] = w.limit(a, geo, column);
#pragma unroll
        for (int s = 0; s < T::kSteps; ++s)
            q[nc][s] = *reinterpret_cast<const u32x4_t *>(qp + 64 * s + 16 * (kHalf ? g & 1 : g));
#pragma unroll
        for (int s = 0; s < T::kSteps; ++s) {
            if (c >= w.cols || (kHalf && g >= 2)) q[nc][s] = u32x4_t{0u, 0u, 0u, 0u};
        }
    }
    const PagedCache &c = a.cache;
    const unsigned char *Kh = c.K + (size_t)w.h * c.head_bytes, *Vh = c.V + (size_t)w.h * c.head_bytes;
    const int32_t *table = c.table + (size_t)w.r * c.ld_table;

    // Pages: lane l looks up position t0 + l % 32 of a tile, two tiles ahead of its use;
    // `off` is the position's slot in units of 16 bytes and `live` the tile's positions
    // that exist.
    auto page_of = [&](int t0) {
        const int pos = t0 + (lane & 31);
        const int pg = table[geo.by_page((unsigned)(pos < end ? pos : begin))];
        return pos < end ? pg : -1;
    };
    auto slot_of = [&](int t0, int pg, unsigned &off, unsigned &live) {
        const int pos = t0 + (lane & 31);
        const bool ok = pg >= 0 && pg < c.pages;
        off = ok ? slot16(a, geo, pg, pos) : 0u;
        live = (unsigned)__ballot(ok);
    };
    auto at_key = [&](const unsigned char *base, unsigned off, int key) {
        return base + (size_t)(unsigned)__builtin_amdgcn_ds_bpermute(key << 2, (int)off) * 16;
    };
    T x;
    auto load_k = [&](unsigned off) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) x.load_k(kb, at_key(Kh, off, 16 * kb + n), g);
    };
    auto load_v = [&](unsigned off) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x.load_v(j, at_key(Vh, off, 16 * (j / 4) + 4 * g + j % 4), n);
    };

    const float scale = a.scale * 1.44269504f;   // scores in the base-2 domain
    f32x4_t o[NC][T::kVe];
    float m[NC], l[NC];
    bool any[NC];
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
#pragma unroll
        for (int e = 0; e < T::kVe; ++e) o[nc][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        m[nc] = -INFINITY, l[nc] = 0.f, any[nc] = false;
    }

    // the softmax of a tile's scores, then its values
    auto attend = [&](f32x4_t (&sc)[NC][2], int t0, unsigned live) {
        const bool partly = t0 + kTile > w.seen;   // some column does not attend all of it
        if (live != 0xffffffffu) {   // a position that is not there read anything
            const unsigned mine = live >> (4 * g);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool is = (mine >> (16 * (j / 4) + j % 4)) & 1u;
#pragma unroll
                for (int e = 0; e < T::kVwords; ++e) x.v[j][e] = is ? x.v[j][e] : 0u;
            }
        }
        if (partly) {
            // An infinity or NaN among the values would reach columns that do not attend its
            // position, as 0 times it.  Such elements are taken out and added to the columns
            // that do.
            bool bad[8], some = false;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                bad[j] = false;
#pragma unroll
                for (int e = 0; e < T::kVe; ++e) bad[j] |= !(fabsf(x.value(j, e)) < INFINITY);
                some |= bad[j];
            }
            if (__any(some)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (!__any(bad[j])) continue;
#pragma unroll 1
                    for (int g2 = 0; g2 < 4; ++g2) {
                        const int pos = t0 + 16 * (j / 4) + 4 * g2 + j % 4;
#pragma unroll
                        for (int e = 0; e < T::kVe; ++e) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float v = __uint_as_float((unsigned)__builtin_amdgcn_ds_bpermute(
                                    (16 * g2 + 4 * g + i) << 2, (int)__float_as_uint(x.value(j, e))));
                                if (!(fabsf(v) < INFINITY)) {
#pragma unroll
                                    for (int nc = 0; nc < NC; ++nc) o[nc][e][i] += pos < lim[nc] ? v : 0.f;
                                }
                            }
                        }
                    }
#pragma unroll
                    for (int e = 0; e < T::kVe; ++e) x.drop_unless_finite(j, e);
                }
            }
        }
#pragma unroll
        for (int nc = 0; nc < NC; ++nc) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sc[nc][kb][i] *= scale;
            }
            if (partly || live != 0xffffffffu) {
                const int left = lim[nc] - t0;   // positions of the tile below the column's limit
                const unsigned there = left <= 0 ? 0u : left >= kTile ? live : live & ((1u << left) - 1u);
                const unsigned mine = there >> (4 * g);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (!((mine >> (16 * (j / 4) + j % 4)) & 1u)) sc[nc][j / 4][j % 4] = -INFINITY;
                any[nc] |= there != 0u;
            } else {
                any[nc] = true;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) mx = fmaxf(mx, sc[nc][j / 4][j % 4]);
            mx = fmaxf(m[nc], col_max(mx));
            if (__any(mx > m[nc])) {
                const float f = m[nc] == -INFINITY ? 1.f : weight(m[nc], mx);   // nothing yet, but perhaps an infinity
                l[nc] *= f;
#pragma unroll
                for (int e = 0; e < T::kVe; ++e) o[nc][e] *= f;
                m[nc] = mx;
            }
            f32x8_t p;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                p[j] = weight(sc[nc][j / 4][j % 4], m[nc]);
                l[nc] += p[j];
            }
            x.accumulate(p, o[nc]);
        }
    };

    int t0 = begin + wave * kTile;
    if (t0 < end) {
        // The keys of the next tile are asked for as soon as this tile's scores are there, its
        // values behind this tile's: a tile of each is always on its way.  Loads stand
        // outside of every branch, or the compiler waits for all of them where the branches
        // meet.
        unsigned off, live;
        f32x4_t sc[NC][2];
        auto scores = [&]() {
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) sc[nc][0] = x.scores(0, q[nc]), sc[nc][1] = x.scores(1, q[nc]);
        };
        const int pg = page_of(t0);
        int pg_next = page_of(end - t0 > kUnit ? t0 + kUnit : t0);
        slot_of(t0, pg, off, live);
        load_k(off);
        load_v(off);
        while (end - t0 > kUnit) {
            const int t1 = t0 + kUnit;
            scores();
            unsigned off_next, live_next;
            slot_of(t1, pg_next, off_next, live_next);
            pg_next = page_of(end - t1 > kUnit ? t1 + kUnit : t1);
            load_k(off_next);
            attend(sc, t0, live);
            load_v(off_next);
            t0 = t1, off = off_next, live = live_next;
        }
        scores();
        attend(sc, t0, live);
    }

    // the four waves' states, joined, 16 columns at a time
    const bool whole = w.splits == 1;
#pragma unroll
    for (int nc = 0; nc < NC; ++nc) {
        l[nc] = col_sum(l[nc]);
        if (nc) __syncthreads();
#pragma unroll
        for (int e = 0; e < T::kVe; ++e) {
#pragma unroll
            for (int i = 0; i < 4; ++i) lds.so[wave][n][T::dim_of(e, 4 * g + i)] = o[nc][e][i];
        }
        if (g == 0) lds.sm[wave][n] = m[nc], lds.sl[wave][n] = any[nc] ? l[nc] : -1.f;
        __syncthreads();
        const int here = w.cols - 16 * nc < 16 ? w.cols - 16 * nc : 16;
        for (int i = (int)threadIdx.x; i < here * D; i += kBlock) {
            const int ci = i / D, d = i % D, cc = 16 * nc + ci;
            float oo, mm, ll;
            join([&](int k, int what) { return what == 0 ? lds.so[k][ci][d] : what == 1 ? lds.sm[k][ci] : lds.sl[k][ci]; }, oo, mm, ll);
            if (whole) {
                store_out<BF16>(w.out, w.place<D>(a, geo, cc, d), ll < 0.f ? 0.f : oo / ll);
            } else {
                put(w.record + cc * D + d, oo);
                if (d == 0) put(w.record + geo.wide * D + 2 * cc, mm), put(w.record + geo.wide * D + 2 * cc + 1, ll);
            }
        }
    }
}

// Rows of a wide tile in LDS.  With 16 bytes between them the same 16 bytes of 16 keys, and with
// 64 (or rows of 64) the same 64 bytes of four values, lie in different banks.
template <int D>
struct WideLds {
    static constexpr int kKeyRow = D * 2 + 16, kValueRow = D == 32 ? D * 2 : D * 2 + 64;
    unsigned char k[2][kWideTile * kKeyRow], v[2][kWideTile * kValueRow];
    unsigned bad[2];   // whether a value of the tile is infinite or NaN, where that matters
};

// A lane's elements of a column, divided by its sum (negative: none), to the column's row from
// its dim 4 h on.
template <int D>
__device__ __forceinline__ void write_wide(unsigned char *to, const f32x16_t (&o)[D / 32], float sum) {
    const float r = sum < 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
            bf16x4_t x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = (__bf16)(sum < 0.f ? 0.f : o[d][i + j] * r);
            *reinterpret_cast<bf16x4_t *>(to + (32 * d + 2 * i) * 2) = x;
        }
    }
}

// A tile of 128 columns, 32 a wave, over tiles of 64 positions that all four read from LDS.
// The next tile's rows are on their way to registers meanwhile.  Lane l = 32 h + n:
//   QK^T  S^T[key][column] = K . q^T, two blocks of 32 keys.  It gets the scores of column n
//         for the keys 32 b + 8 (i / 4) + 4 h + i % 4.
//   PV    O^T[dim][column] = V^T . P^T, contracting over 16 keys at a time in the order in which
//         the score registers hold them.  V^T comes by transposing reads of LDS, four keys of
//         16 dims a group of 16 lanes.
template <int D>
__device__ __forceinline__ void attend_wide(const PagedChunk &a, const Geo &geo, const Piece &w, WideLds<D> &lds)
{
    constexpr int kPieces = D / 8, kLoads = kWideTile * kPieces / kBlock, kSteps = D / 16, kDims = D / 32;
    constexpr int kKeyRow = WideLds<D>::kKeyRow, kValueRow = WideLds<D>::kValueRow;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int n = lane & 31, h = lane >> 5;
    const int begin = w.begin, end = w.end;
    const PagedCache &c = a.cache;
    const unsigned char *Kh = c.K + (size_t)w.h * c.head_bytes, *Vh = c.V + (size_t)w.h * c.head_bytes;
    const int32_t *table = c.table + (size_t)w.r * c.ld_table;

    // this wave's columns
    const int c0 = 32 * wave, mine = w.cols - c0 < 32 ? w.cols - c0 : 32;
    const int column = w.col0 + (c0 + n < w.cols ? c0 + n : 0);
    const int lim = w.limit(a, geo, column);
    const int first_lim = mine > 0 ? w.limit(a, geo, w.col0 + c0) : 0, last_lim = mine > 0 ? w.limit(a, geo, w.col0 + c0 + mine - 1) : 0;
    // Scores are scaled as they are taken to the base-2 exponent, which needs their largest: a
    // negative scale turns the queries' signs, and one of zero is that of zero queries.
    float scale = a.scale * 1.44269504f;
    bf16x8_t q[kSteps];
    {
        const unsigned char *qp = w.query(a, geo, column);
        const uint32_t keep = scale == 0.f || c0 + n >= w.cols ? 0u : 0xffffffffu, turn = scale < 0.f && keep ? 0x80008000u : 0u;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            u32x4_t x = *reinterpret_cast<const u32x4_t *>(qp + 32 * s + 16 * h);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (x[i] & keep) ^ turn;
            q[s] = __builtin_bit_cast(bf16x8_t, x);
        }
        scale = scale == 0.f ? 1.f : fabsf(scale);
    }

    // Lane l looks up position t0 + l of a tile, two tiles ahead of its use.
    auto page_of = [&](int t0) {
        const int pos = t0 + lane;
        const int pg = table[geo.by_page((unsigned)(pos < end ? pos : begin))];
        return pos < end ? pg : -1;
    };
    u32x4_t kx[kLoads], vx[kLoads];
    unsigned long long live_next = 0;
    auto load = [&](int t0, int pg) {
        const int pos = t0 + lane;
        const bool ok = pg >= 0 && pg < c.pages;
        const unsigned off = ok ? slot16(a, geo, pg, pos) : 0u;
        live_next = __ballot(ok);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int piece = tid + kBlock * i, key = piece / kPieces;
            const size_t at = (size_t)(unsigned)__builtin_amdgcn_ds_bpermute(key << 2, (int)off) * 16 + (piece % kPieces) * 16;
            kx[i] = *reinterpret_cast<const u32x4_t *>(Kh + at);
            vx[i] = *reinterpret_cast<const u32x4_t *>(Vh + at);
        }
    };
    auto stage = [&](int buf, int t0) {
        const bool partly = t0 + kWideTile > w.seen;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int piece = tid + kBlock * i, key = piece / kPieces, c16 = (piece % kPieces) * 16;
            if (live_next != ~0ull) {   // a position that is not there read anything
                const uint32_t is = (live_next >> key & 1) ? 0xffffffffu : 0u;
#pragma unroll
                for (int j = 0; j < 4; ++j) kx[i][j] &= is, vx[i][j] &= is;
            }
            if (partly) {
#pragma unroll
                for (int j = 0; j < 4; ++j) bad |= (vx[i][j] & 0x7f80u) == 0x7f80u || (vx[i][j] & 0x7f800000u) == 0x7f800000u;
            }
            *reinterpret_cast<u32x4_t *>(lds.k[buf] + key * kKeyRow + c16) = kx[i];
            *reinterpret_cast<u32x4_t *>(lds.v[buf] + key * kValueRow + c16) = vx[i];
        }
        if (partly && __any(bad) && lane == 0) lds.bad[buf] = 1u;
    };

    f32x16_t o[kDims];
#pragma unroll
    for (int d = 0; d < kDims; ++d) {
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    }
    float m = -INFINITY, l = 0.f;   // m: of the unscaled scores
    bool any = false;

    // operands: of K the lane's key n, of V^T its dim n of the keys 4 h + 0 .. 3, by a transposition
    // of the four keys that 16 lanes read
    const unsigned char *k_at = lds.k[0] + n * kKeyRow + 16 * h;
    const unsigned char *v_at = lds.v[0] + (4 * h + (lane & 15) / 4) * kValueRow + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
    struct Values {
        bf16x8_t x[kDims];
    };
    struct Weights {
        bf16x8_t hi, lo;   // each weight is the sum of the two
    };
    auto values = [&](const unsigned char *at, int s) {   // of 16 keys: 16 s + 4 h + 0 .. 3 and 8 behind
        Values r;
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
            s16x4_t v[2];
#pragma unroll
            for (int x = 0; x < 2; ++x)
                v[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4_t *)(at + (16 * s + 8 * x) * kValueRow + 64 * d));
            r.x[d] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
        return r;
    };
    auto attend = [&](int buf, int t0, unsigned long long live) {
        const unsigned char *kt = k_at + buf * (kWideTile * kKeyRow), *vt = v_at + buf * (kWideTile * kValueRow);
        f32x16_t sc[2];
        bf16x8_t kf[2][kSteps];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) kf[b][s] = *reinterpret_cast<const bf16x8_t *>(kt + 32 * b * kKeyRow + 32 * s);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[b][i] = 0.f;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[b][s], q[s], sc[b], 0, 0, 0);
        }
        Values v = values(vt, 0);
        // the second block's operands come while the first's are multiplied, the first values'
        // while the second's are
        __builtin_amdgcn_sched_group_barrier(kSchedRead, kSteps, 0);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedRead, 1, 0);
        }
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kSchedRead, 1, 0);
        }
        if (t0 + kWideTile > first_lim || live != ~0ull) {
            const int left = lim - t0;   // positions of the tile below the column's limit
            const unsigned long long there = left <= 0 ? 0ull : left >= kWideTile ? live : live & ((1ull << left) - 1);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const unsigned is = (unsigned)(there >> (32 * b)) >> (4 * h);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((is >> (8 * (i / 4) + i % 4)) & 1u)) sc[b][i] = -INFINITY;
            }
            any |= there != 0;
        } else {
            any = true;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[b][i]);
        }
        {
            float lo, hi;
            lane_pair<32>(mx, lo, hi);
            mx = fmaxf(lo, hi);
        }
        // Weights are taken relative to a maximum that may be left behind by up to 2^8: what has
        // been added up is scaled down seldom, and sums of 32 bits do not mind.
        if (__any((mx - m) * scale > 8.f || m == -INFINITY)) {
            const float top = fmaxf(m, mx);
            const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - top) * scale);   // nothing yet, but perhaps an infinity
            l *= f;
#pragma unroll
            for (int d = 0; d < kDims; ++d) o[d] *= f;
            m = top;
        }
        const float base = m == -INFINITY ? 0.f : m * scale;
        float sum[2] = {0.f, 0.f};
        auto weights = [&](int s) {
            Weights r;
            u32x4_t hi, lo;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f32x2_t p;
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    p[x] = __builtin_amdgcn_exp2f(fmaf(sc[s / 2][8 * (s % 2) + 2 * j + x], scale, -base));
                    sum[x] += p[x];
                }
                const uint32_t both = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2_t));
                p[0] -= __uint_as_float(both << 16), p[1] -= __uint_as_float(both & 0xffff0000u);
                hi[j] = both, lo[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2_t));
            }
            r.hi = __builtin_bit_cast(bf16x8_t, hi), r.lo = __builtin_bit_cast(bf16x8_t, lo);
            return r;
        };
        Weights p = weights(0);
#pragma unroll
        for (int s = 0; s < 4; ++s) {   // 16 keys at a time; the next ones' operands are made meanwhile
            Values v_next;
            Weights p_next;
            if (s < 3) v_next = values(vt, s + 1), p_next = weights(s + 1);
#pragma unroll
            for (int d = 0; d < kDims; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.x[d], p.hi, o[d], 0, 0, 0);
#pragma unroll
            for (int d = 0; d < kDims; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.x[d], p.lo, o[d], 0, 0, 0);
            if (s < 3) {
#pragma unroll
                for (int d = 0; d < 2 * kDims; ++d) {
                    __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kSchedRead, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kSchedValu, 48 / (2 * kDims), 0);
                }
                v = v_next, p = p_next;
            }
        }
        l += sum[0] + sum[1];
    };

    // An infinity or NaN among the values would reach columns that do not attend its position,
    // as 0 times it.  Such elements are added to the columns that do and taken out.
    auto sort_out = [&](int buf, int t0) {
        for (int key = 0; key < kWideTile; ++key) {
#pragma unroll
            for (int d = 0; d < kDims; ++d) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int dim = 32 * d + 8 * (i / 4) + 4 * h + i % 4;
                    const uint16_t bits = *reinterpret_cast<const uint16_t *>(lds.v[buf] + key * kValueRow + dim * 2);
                    const float v = __uint_as_float((uint32_t)bits << 16);
                    if (!(fabsf(v) < INFINITY) && t0 + key < lim) o[d][i] += v;
                }
            }
        }
        __syncthreads();
        for (int i = tid; i < kWideTile * D; i += kBlock) {
            uint16_t *x = reinterpret_cast<uint16_t *>(lds.v[buf] + i / D * kValueRow) + i % D;
            if ((*x & 0x7f80u) == 0x7f80u) *x = 0;
        }
        if (tid == 0) lds.bad[buf] = 0u;
        __syncthreads();
    };

    if (begin < end) {
        if (tid < 2) lds.bad[tid] = 0u;
        __syncthreads();
        int pg = page_of(begin), pg_next = page_of(end - begin > kWideTile ? begin + kWideTile : begin), buf = 0;
        load(begin, pg);
        stage(0, begin);
        unsigned long long live = live_next;
        __syncthreads();
        for (int t0 = begin;; buf ^= 1) {
            const bool more = end - t0 > kWideTile;
            if (more) {
                load(t0 + kWideTile, pg_next);
                pg_next = page_of(end - t0 > 2 * kWideTile ? t0 + 2 * kWideTile : begin);
            }
            if (t0 + kWideTile > w.seen && lds.bad[buf]) sort_out(buf, t0);
            if (t0 < last_lim) attend(buf, t0, live);
            if (!more) break;
            t0 += kWideTile;
            stage(buf ^ 1, t0);
            live = live_next;
            __syncthreads();
        }
    }

    {
        float lo, hi;
        lane_pair<32>(l, lo, hi);
        l = lo + hi;
    }
    if (n < mine) {
        const int cc = c0 + n;
        if (w.splits == 1) {
            write_wide<D>(w.out + w.place<D>(a, geo, cc, 4 * h) * 2, o, any ? l : -1.f);
        } else if (h == 0) {
            put(w.record + geo.wide * D + 2 * cc, m * scale), put(w.record + geo.wide * D + 2 * cc + 1, any ? l : -1.f);
        }
    }
    if (w.splits > 1) {   // as the registers hold them, so that a wave's stores lie side by side
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
#pragma unroll
            for (int i = 0; i < 16; ++i) put(w.record + ((wave * kDims + d) * 16 + i) * kWave + lane, o[d][i]);
        }
    }
}

struct JoinLds {
    float sf[kJoin][16], sg[kJoin][16], sm[16], sl[16];
    unsigned arrived;
};
template <int D>
union NarrowOnlyLds {
    NarrowLds<D> narrow;
    JoinLds join;
};

// Joins the records of `count` states of a tile, `stride` floats apart from `base` on, 16 columns
// at a time: into the output (last), or into the first record.
template <int D, bool BF16>
__device__ __forceinline__ void join_narrow(const PagedChunk &a, const Geo &geo, const Piece &w, float *base, size_t stride,
                                            int count, bool last, JoinLds &lds)
{
    for (int c0 = 0; c0 < w.cols; c0 += 16) {
        const int here = w.cols - c0 < 16 ? w.cols - c0 : 16;
        float *states = base + geo.wide * D + 2 * c0;
        __syncthreads();
        // each state's share of the joined one: exp2 of its maximum's distance, in sf
        for (int i = (int)threadIdx.x; i < count * here; i += kBlock) {
            const int k = i / here, ci = i - k * here;
            const float mm = get(states + k * stride + 2 * ci), ll = get(states + k * stride + 2 * ci + 1);
            lds.sf[k][ci] = ll < 0.f ? -INFINITY : mm, lds.sg[k][ci] = ll;
        }
        __syncthreads();
        if ((int)threadIdx.x < here) {
            const int ci = (int)threadIdx.x;
            float top = -INFINITY, sum = -1.f;
            for (int k = 0; k < count; ++k) top = fmaxf(top, lds.sf[k][ci]);
            for (int k = 0; k < count; ++k) {
                const float f = weight(lds.sf[k][ci], top), ll = lds.sg[k][ci];
                lds.sf[k][ci] = f;
                if (!(ll < 0.f)) sum = (sum < 0.f ? 0.f : sum) + ll * f;
            }
            lds.sm[ci] = top, lds.sl[ci] = sum;
        }
        __syncthreads();
        for (int i = (int)threadIdx.x; i < here * D; i += kBlock) {
            const int ci = i / D;
            float *from = base + c0 * D + i;
            float oo = 0.f;
            for (int k0 = 0; k0 < count; k0 += 8) {   // eight on their way at a time
                float y[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = get(from + (k0 + k < count ? k0 + k : k0) * stride);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k0 + k < count && !(lds.sg[k0 + k][ci] < 0.f)) oo += y[k] * lds.sf[k0 + k][ci];
            }
            const float ll = lds.sl[ci];
            if (last) store_out<BF16>(w.out, w.place<D>(a, geo, c0 + ci, i % D), ll < 0.f ? 0.f : oo / ll);
            else put(from, oo);   // read by this thread alone
        }
        if (!last && (int)threadIdx.x < here) {
            const int ci = (int)threadIdx.x;
            put(states + 2 * ci, lds.sm[ci]), put(states + 2 * ci + 1, lds.sl[ci]);
        }
    }
}

// The same for a wide tile: a lane has the column and the elements that it had of the sum.
template <int D>
__device__ __forceinline__ void join_wide(const PagedChunk &a, const Geo &geo, const Piece &w, float *base, size_t stride, int count,
                                          bool last)
{
    constexpr int kDims = D / 32;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid / kWave, h = lane >> 5, cc = 32 * wave + (lane & 31);
    if (32 * wave >= w.cols) return;
    float *states = base + geo.wide * D + 2 * (cc < w.cols ? cc : 0);
    float top = -INFINITY, sum = -1.f;
    for (int k = 0; k < count; ++k) {
        const float mm = get(states + k * stride), ll = get(states + k * stride + 1);
        top = fmaxf(top, ll < 0.f ? -INFINITY : mm);
    }
    f32x16_t o[kDims];
#pragma unroll
    for (int d = 0; d < kDims; ++d) {
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    }
    for (int k = 0; k < count; ++k) {
        const float mm = get(states + k * stride), ll = get(states + k * stride + 1);
        const float f = weight(ll < 0.f ? -INFINITY : mm, top);
        if (!(ll < 0.f)) sum = (sum < 0.f ? 0.f : sum) + ll * f;
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
            float y[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) y[i] = get(base + k * stride + ((wave * kDims + d) * 16 + i) * kWave + lane);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] += ll < 0.f ? 0.f : y[i] * f;
        }
    }
    if (last) {
        if (cc < w.cols) write_wide<D>(w.out + w.place<D>(a, geo, cc, 4 * h) * 2, o, sum);
        return;
    }
#pragma unroll
    for (int d = 0; d < kDims; ++d) {
#pragma unroll
        for (int i = 0; i < 16; ++i) put(base + ((wave * kDims + d) * 16 + i) * kWave + lane, o[d][i]);
    }
    if (h == 0 && cc < w.cols) put(states, top), put(states + 1, sum);
}

// The chunk's record is written; the last of the tile's chunks to arrive joins them, in the
// order of the chunks, groups of about the square root of their number first.
template <int D, bool BF16>
__device__ __forceinline__ void join_chunks(const PagedChunk &a, const Geo &geo, const Piece &w, int slot, JoinLds &lds)
{
    // A record has arrived before its workgroup counts itself, and is read by the workgroup that
    // counts last; counters end at zero.
    int group = w.splits;   // chunks of a group: at most 64, and as many groups
    if (w.splits > 16) {
        group = 16;
        while (group * group < w.splits) group *= 2;
    }
    static_assert((kJoin & (kJoin - 1)) == 0 && kJoin * kJoin >= kChunks + 1, "groups and their number fit the arrays");
    const int groups = (w.splits + group - 1) / group;
    for (int level = 0; level < 2; ++level) {
        // level 0: the chunks of this one's group, into its first record; level 1: the groups
        if (level == 1 && groups == 1) break;
        const int first = level == 0 ? w.split / group * group : 0;
        const int count = level == 0 ? (w.splits - first < group ? w.splits - first : group) : groups;
        const int step = level == 0 ? 1 : group;
        unsigned *counter = (level == 0 ? geo.group_count : geo.tile_count) + (size_t)(slot + first) * a.Hkv + w.h;
        __builtin_amdgcn_s_waitcnt(0);   // this thread's stores have arrived, then everybody's
        __syncthreads();
        if (threadIdx.x == 0)
            lds.arrived = count > 1 ? __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
        __syncthreads();
        if (lds.arrived != (unsigned)count - 1) return;
        if (threadIdx.x == 0 && count > 1) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        float *base = geo.records + ((size_t)(slot + first) * a.Hkv + w.h) * geo.record;
        const size_t stride = (size_t)step * a.Hkv * geo.record;
        const bool last = level == 1 || groups == 1;
        if constexpr (kHasWide<D, BF16>) {
            if (w.row.width > geo.narrow) {
                join_wide<D>(a, geo, w, base, stride, count, last);
                continue;
            }
        }
        join_narrow<D, BF16>(a, geo, w, base, stride, count, last, lds);
    }
}

template <int D, bool BF16>
union Lds {
    NarrowLds<D> narrow;
    WideLds<D> wide;
    JoinLds join;
};

template <int D, bool BF16>
__global__ __launch_bounds__(kBlock, 2) void paged_chunk_kernel(PagedChunk a, Geo geo)
{
    using Shared = std::conditional_t<kHasWide<D, BF16>, Lds<D, BF16>, NarrowOnlyLds<D>>;
    __shared__ __align__(16) Shared lds;

    const unsigned wg = wide_index();
    const int t = (int)geo.by_hkv(wg);
    Piece p;
    p.h = (int)wg - t * a.Hkv;
    Task task;
    if (geo.plan ? !find_planned(geo.plan, a.R, t, task) : !find_task(a, geo, t, task)) return;

    p.r = task.r;
    p.row = row_of(a, geo, a.kv_len[task.r], a.offsets[task.r], a.offsets[task.r + 1]);
    // offsets that decrease would lead past the output and the records
    if ((unsigned)task.tile >= (unsigned)p.row.tiles || (unsigned)task.split >= (unsigned)task.splits ||
        (task.splits > 1 && (task.slot < 0 || ((long long)task.slot + task.splits) * a.Hkv > geo.slots)))
        return;
    p.col0 = task.tile * p.row.width;
    p.cols = p.row.columns - p.col0 < p.row.width ? p.row.columns - p.col0 : p.row.width;
    const int L = p.limit(a, geo, p.col0 + p.cols - 1);
    p.seen = p.limit(a, geo, p.col0);
    const int units = units_of(L), per = (units + task.splits - 1) / task.splits;
    p.splits = (units + per - 1) / per;   // an early tile may have fewer chunks than the row's last
    p.split = task.split;
    if (p.split >= p.splits) return;
    p.begin = p.split * per * kUnit;
    p.end = L - p.begin < per * (long long)kUnit ? L : p.begin + per * kUnit;
    p.out = a.out + ((size_t)p.row.begin * a.Hq + (size_t)p.h * geo.G) * D * (BF16 ? 2 : 4);
    p.record = geo.records + ((size_t)(task.slot + p.split) * a.Hkv + p.h) * geo.record;
    if constexpr (kHasWide<D, BF16>) {
        if (p.row.width > geo.narrow) attend_wide<D>(a, geo, p, lds.wide);
        else attend_narrow<D, BF16>(a, geo, p, lds.narrow);
    } else {
        attend_narrow<D, BF16>(a, geo, p, lds.narrow);
    }
    if (p.splits > 1) join_chunks<D, BF16>(a, geo, p, task.slot, lds.join);
}

struct Layout {
    int narrow, wide, record;
    long long grid, slots;   // workgroups and records at most
    size_t tile_count, plan, records, bytes;   // byte offsets in the workspace
};

Layout layout_of(int N, int R, int Hq, int Hkv, int page, int cols, int D, bool bf16) {
    Layout y{};
    const long long columns = (long long)N * (Hq / Hkv);
    y.narrow = bf16 || D <= 64 ? 32 : 16;
    y.wide = bf16 && D >= 32 && columns > y.narrow ? kWideColumns : y.narrow;
    y.record = y.wide * (D + 2);
    const long long rows = R < N ? R : N;   // with tokens
    const long long tiles = (columns / y.wide + rows) * Hkv;
    const long long most = ((long long)cols * page + kUnit - 1) / kUnit, units = most < 1 ? 1 : most;
    // c units a chunk, work / kChunks at least: chunks are kChunks and one begun per tile at most,
    // and a cut tile's are more than half used on average
    y.grid = kChunks + tiles < tiles * units ? kChunks + tiles : tiles * units;
    y.slots = 2ll * kChunks < tiles * units ? 2ll * kChunks : tiles * units;
    // the counters lie where every call has them, whatever its sizes
    y.tile_count = 2 * kChunks * sizeof(unsigned);
    y.plan = 2 * y.tile_count;
    y.records = y.plan + (R > kScanRows ? ((size_t)R + 1) * sizeof(int4) : 0);
    y.bytes = y.records + (units > 1 ? (size_t)y.slots * y.record * sizeof(float) : 0);
    return y;
}

}  // namespace

size_t paged_chunk_attn_workspace_bytes(int N, int R, int Hq, int Hkv, int page, int cols, int D, bool bf16) {
    return layout_of(N, R, Hq, Hkv, page, cols, D, bf16).bytes;
}

hipError_t launch_paged_chunk_attn(const PagedChunk &a, int D, bool bf16, hipStream_t stream)
{
    const Layout y = layout_of(a.N, a.R, a.Hq, a.Hkv, a.cache.page, a.cache.cols, D, bf16);
    Geo geo{};
    geo.G = a.Hq / a.Hkv, geo.narrow = y.narrow, geo.wide = y.wide, geo.record = y.record, geo.slots = y.slots;
    geo.by_page = make_div(a.cache.page), geo.by_hkv = make_div(a.Hkv), geo.by_g = make_div(geo.G);
    geo.page16 = (unsigned)(a.cache.page_bytes / 16), geo.slot16 = (unsigned)(a.cache.slot_bytes / 16);
    geo.group_count = reinterpret_cast<unsigned *>(a.workspace);
    geo.tile_count = reinterpret_cast<unsigned *>(a.workspace + y.tile_count);
    geo.records = reinterpret_cast<float *>(a.workspace + y.records);
    if (a.R > kScanRows) {
        auto *plan = reinterpret_cast<int4 *>(a.workspace + y.plan);
        geo.plan = plan;
        hipLaunchKernelGGL(chunk_plan_kernel, dim3(1), dim3(1024), 0, stream, a, geo, plan);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 gd = wide_grid(y.grid), bd(kBlock);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, gd, bd, 0, stream, a, geo); };
    switch (D) {
    case 16: bf16 ? launch(paged_chunk_kernel<16, true>) : launch(paged_chunk_kernel<16, false>); break;
    case 32: bf16 ? launch(paged_chunk_kernel<32, true>) : launch(paged_chunk_kernel<32, false>); break;
    case 64: bf16 ? launch(paged_chunk_kernel<64, true>) : launch(paged_chunk_kernel<64, false>); break;
    default: bf16 ? launch(paged_chunk_kernel<128, true>) : launch(paged_chunk_kernel<128, false>); break;
    }
    return hipGetLastError();
}

}  // namespace fs
