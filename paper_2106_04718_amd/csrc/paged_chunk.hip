// Causal attention of several new tokens per row over a paged key-value cache, for gfx950.
//
// Row r's tokens i = 0 .. n - 1 are the last n of its kv_len positions; query head h of token
// i attends the positions up to kv_len - n + i in the key-value head h / G.  A row's queries
// of one key-value head are n G columns, column m being head m % G of token m / G.
//
// Tiles.  A workgroup takes up to 128 columns (bf16, heads of 32 elements and more: wide), or 16 or
// 32 (narrow).  In a narrow tile a wave attends 32 positions for all columns at a time, as
// paged_tile.h describes, the four waves the positions in turn; their softmax states are
// joined at the end.  In a wide one each wave has 32 columns and all positions, 64 of them at a
// time, which the four read from LDS: from global memory straight to each wave's registers the
// same keys would be asked for four times.
// fp32 keeps to narrow tiles: 16 x 16 x 4 products of 32 columns a wave and all positions, the
// caches serving four waves' loads, took 118 us where this takes 70 (8 rows of 1 to 257 tokens behind
// 400 to 1024 positions, 16 heads of 64), and gained at one of five other sizes (272 -> 214 us).
//
// Bound.  A token of n over p positions has 4 p D operations, and a row's keys and values are read
// once for all of its tokens and a key-value head's G heads: few tokens (32 rows of 5 over 200 to
// 4096 positions, 285 MB: 75 us, 3.8 TB/s) are bound by HBM, many by the
// matrix cores and what stands between their products.  2048 tokens over 32500 positions, 32 heads
// of 128: 1.76 to 1.85 ms, 573 to 601 TFLOP/s of 4 p D, which the weights' second and third parts double;
// the matrix cores are busy 57 % of the cycles.
//
// Division of the work.  The columns of a row are cut into tiles.  Either workgroups take whole
// tiles, the longest first; or all tiles of a key-value head, one behind another, are cut into
// as many equal shares as the head has of the workgroups that fit the chip.  A share may begin
// and end within a tile, at a unit of 128 positions; the tile's parts then leave their softmax
// states in the workspace, where the last of them to arrive joins them, in their order.
// Lengths are known on the device alone, so every workgroup adds the rows' work up and finds
// its own (up to kScanRows rows; above, a kernel before this one adds up, and the work is cut).
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "div.h"
#include "grid.h"
#include "launch.h"
#include "paged_tile.h"

namespace fs {
namespace {

constexpr int kMostShares = 4 * 1024;   // of all heads together
constexpr int kJoin = 64;         // states joined at a time
constexpr int kScanRows = 256;    // rows whose lengths every workgroup looks at: four a lane
constexpr int kStart = 128;       // what a tile takes beside its positions, in positions
constexpr int kLeast = 512;       // a share at least

constexpr int kWideTile = 64;     // positions that a workgroup attends at a time in a wide tile
constexpr int kWideColumns = 32 * kWaves;

template <int D, bool BF16>
constexpr int kTiles16 = BF16 || D <= 64 ? 2 : 1;   // NC: 16 columns each, as many as the registers hold
template <int D, bool BF16>
constexpr bool kHasWide = BF16 && D >= 32;

typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
constexpr int kSchedValu = 0x2, kSchedMfma = 0x8, kSchedRead = 0x100;   // kinds of instructions

typedef unsigned long long u64_t;

// What a launch knows beside PagedChunk.
struct Geo {
    Div by_page, by_hkv, by_g;
    int G;
    int width;                 // columns of a tile: a power of two
    double half;               // half of the tokens of a tile
    unsigned page16, slot16;   // strides in units of 16 bytes
    int shares;                // of a key-value head
    int record;                // floats of a part's state: width * (D + 2)
    unsigned *group_count, *tile_count;   // arrivals, by the first record of the group or tile
    const u64_t *plan;         // work before each row and of all, made before the launch (more than kScanRows rows), or null
    float *records;
};

struct Row {
    int first_pos;   // of its first token; may be negative, then that token attends nothing
    int begin, tokens;
    int columns, tiles;   // of one key-value head
};

__device__ __forceinline__ int units_of(int L) { return L <= 0 ? 1 : (L + kUnit - 1) / kUnit; }

__device__ __forceinline__ Row row_of(const PagedChunk &a, const Geo &geo, int kv_len, int o0, int o1) {
    o0 = o0 < 0 ? 0 : o0;
    const int last = o1 < a.N ? o1 : a.N;   // of tokens that there are
    const int n = last > o0 ? last - o0 : 0, L = kv_len < 0 ? 0 : kv_len;
    Row w;
    w.first_pos = L - (n ? o1 - o0 : 0);   // those behind the N have their positions too
    w.begin = o0, w.tokens = n;
    w.columns = n * geo.G;
    w.tiles = (int)(((unsigned)w.columns + geo.width - 1) >> (31 - __builtin_clz(geo.width)));
    return w;
}

// Work of a row's tiles before tile i, in positions: those that a tile's last token attends, and
// kStart.  Rising with i.  Where the tiles differ by little they count alike, so that shares
// of a tile or a whole part of one begin together, and its neighbours find their keys in the L2.
__device__ __forceinline__ u64_t work_before(const PagedChunk &a, const Geo &geo, const Row &w, int i) {
    const int cap = a.cache.cols * a.cache.page, p = w.first_pos < 0 ? 0 : w.first_pos < cap ? w.first_pos : cap;
    if (p / 2 >= w.tokens) return (u64_t)(unsigned)i * (unsigned)(p + w.tokens / 2 + kStart);
    return (u64_t)(unsigned)i * (unsigned)(p + kStart) + (u64_t)((double)i * (double)(i + 1) * geo.half);
}

__device__ __forceinline__ u64_t shfl_up64(u64_t x, int by) {
    const unsigned lo = __shfl_up((unsigned)x, by), hi = __shfl_up((unsigned)(x >> 32), by);
    return (u64_t)hi << 32 | lo;
}
__device__ __forceinline__ u64_t wave_scan64(u64_t x) {
#pragma unroll
    for (int by = 1; by < kWave; by *= 2) {
        const u64_t y = shfl_up64(x, by);
        if ((int)(threadIdx.x & 63) >= by) x += y;
    }
    return x;
}
__device__ __forceinline__ u64_t uniform64(u64_t x) {
    return (u64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)x);
}

// What a workgroup knows of up to kScanRows rows.
struct Rows {
    u64_t sums[kScanRows + 1];   // work before each of them, and of all
    int len[kScanRows], off[kScanRows + 1];
    int tiles[kScanRows + 1];    // of a head before each of them, and of all
    int longest;                 // units of the longest
    int row, tile;               // where tiles are taken whole: the one found
};

__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
    for (int by = 1; by < kWave; by *= 2) {
        const int y = __shfl_xor(x, by);
        x = x > y ? x : y;
    }
    return x;
}

// Reads and adds them up, by one wave.
__device__ __forceinline__ void add_rows(const PagedChunk &a, const Geo &geo, Rows &rows) {
    const int lane = (int)threadIdx.x & 63, cap = a.cache.cols * a.cache.page;
    int len[4], off[5];
#pragma unroll
    for (int i = 0; i < 4; ++i) len[i] = a.kv_len[4 * lane + i < a.R ? 4 * lane + i : a.R - 1];   // all in flight at once
#pragma unroll
    for (int i = 0; i < 5; ++i) off[i] = a.offsets[4 * lane + i < a.R ? 4 * lane + i : a.R];
    u64_t work[4], sum = 0;
    int longest = 0, tiles[4], all_tiles = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const Row w = row_of(a, geo, len[i], off[i], off[i + 1]);   // none behind the last row: it would begin at its end
        work[i] = work_before(a, geo, w, w.tiles), sum += work[i];
        const int seen = w.first_pos + w.tokens;   // by its last token
        const int u = w.tiles ? units_of(seen < cap ? seen : cap) : 0;
        longest = longest > u ? longest : u, tiles[i] = w.tiles, all_tiles += w.tiles;
        rows.len[4 * lane + i] = len[i], rows.off[4 * lane + i] = off[i];
    }
    u64_t at = wave_scan64(sum) - sum;
    int tile = wave_scan(all_tiles) - all_tiles;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        rows.sums[4 * lane + i] = at, rows.tiles[4 * lane + i] = tile;
        at += work[i], tile += tiles[i];
    }
    longest = wave_max(longest);
    if (lane == 63) rows.sums[kScanRows] = at, rows.off[kScanRows] = off[4], rows.tiles[kScanRows] = tile, rows.longest = longest;
}

// The first tile of a row with at least x units (its tiles if there is none).
__device__ __forceinline__ int first_of(const PagedChunk &a, const Geo &geo, const Row &w, int x) {
    if (x <= 1) return 0;   // every tile has one, if only to be written
    if ((long long)(x - 1) * kUnit >= (long long)a.cache.cols * a.cache.page) return w.tiles;
    const long long q = (long long)(x - 1) * kUnit - w.first_pos;   // a tile's last token has to be this one or behind
    if (q <= 0) return 0;
    return q * geo.G >= w.columns ? w.tiles : (int)((unsigned)(q * geo.G) >> (31 - __builtin_clz(geo.width)));
}

// The t-th tile of a head in the order of falling length, by one wave: those of at least x units
// are counted in closed form, and x found by bisection.
__device__ __forceinline__ void find_tile(const PagedChunk &a, const Geo &geo, Rows &rows, int t) {
    const int lane = (int)threadIdx.x & 63;
    Row w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = row_of(a, geo, rows.len[4 * lane + i], rows.off[4 * lane + i], rows.off[4 * lane + i + 1]);
    auto longer = [&](int x) {
        int m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m += w[i].tiles - first_of(a, geo, w[i], x);
        return wave_sum(m);
    };
    int lo = 1, hi = rows.longest + 1, behind = 0;   // tiles of at least hi units
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2, m = longer(mid);
        if (m > t) lo = mid;
        else hi = mid, behind = m;
    }
    t -= behind;
    int here[4], sum = 0;   // of just lo units
#pragma unroll
    for (int i = 0; i < 4; ++i) here[i] = first_of(a, geo, w[i], lo + 1) - first_of(a, geo, w[i], lo), sum += here[i];
    int at = wave_scan(sum) - sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (at <= t && t < at + here[i]) rows.row = 4 * lane + i, rows.tile = first_of(a, geo, w[i], lo) + t - at;
        at += here[i];
    }
}

// The work before each of any number of rows, and of all, by one workgroup.
__global__ __launch_bounds__(1024) void chunk_plan_kernel(PagedChunk a, Geo geo, u64_t *sums) {
    __shared__ u64_t part[16];
    const int tid = (int)threadIdx.x, wave = tid / kWave;
    u64_t before = 0;
    for (int r0 = 0; r0 < a.R; r0 += 1024) {
        const int r = r0 + tid;
        u64_t work = 0;
        if (r < a.R) {
            const Row w = row_of(a, geo, a.kv_len[r], a.offsets[r], a.offsets[r + 1]);
            work = work_before(a, geo, w, w.tiles);
        }
        const u64_t run = wave_scan64(work);
        if ((tid & 63) == 63) part[wave] = run;
        __syncthreads();
        u64_t at = before + run - work;
        for (int i = 0; i < 16; ++i) {
            if (i < wave) at += part[i];
            before += part[i];
        }
        if (r < a.R) sums[r] = at;
        __syncthreads();
    }
    if (tid == 0) sums[a.R] = before;
}

// The last row whose work (or tiles) begins at or before x, 64 looked at at a time.
template <typename T>
__device__ __forceinline__ int row_at(const T *sums, int R, T x) {
    const int lane = (int)threadIdx.x & 63;
    int lo = 0, n = R;
    while (n > 1) {
        const int step = (n + 63) / 64, at = lane * step;
        const bool there = at < n && lo + at < R;
        const T v = sums[there ? lo + at : 0];
        lo += step * (63 - __clzll((long long)__ballot(lane == 0 || (there && v <= x))));
        n = step;
    }
    return lo;
}

// The tile of a row in which x lies, x behind the row's beginning by less than its work.
__device__ __forceinline__ int tile_at(const PagedChunk &a, const Geo &geo, const Row &w, u64_t x) {
    const u64_t one = work_before(a, geo, w, 1);
    if (work_before(a, geo, w, w.tiles) == one * (unsigned)w.tiles) {   // all alike
        const int i = (int)((double)x / (double)one);
        return i > 0 && one * (unsigned)i > x ? i - 1 : i + 1 < w.tiles && one * (unsigned)(i + 1) <= x ? i + 1 : i;
    }
    const double lin = (double)one, h = geo.half;   // about h i^2 + (lin - h) i
    const double guess = 2.0 * (double)x / ((lin - h) + sqrt((lin - h) * (lin - h) + 4.0 * h * (double)x) + 1.0);
    int i = guess < (double)(w.tiles - 1) ? (int)guess : w.tiles - 1;
    i = i < 0 ? 0 : i;
    while (i > 0 && work_before(a, geo, w, i) > x) --i;
    while (i + 1 < w.tiles && work_before(a, geo, w, i + 1) <= x) ++i;
    return i;
}

// What a workgroup knows of its piece of work.
struct Piece {
    int r, h, tile, col0, cols;   // the row, the key-value head, the tile and its columns
    int begin, end;           // positions of the chunk
    int seen;                 // positions that all columns attend
    int share, first, parts;  // the tile lies in the shares first .. first + parts - 1
    Row row;
    unsigned char *out;       // of the row and head
    // a share has one tile that began before it, and one that began in it, which others end
    __device__ __forceinline__ size_t record_of(const PagedChunk &a, int x) const { return (size_t)(2 * x + (x == first ? 1 : 0)) * a.Hkv + h; }
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
    const bool whole = w.parts == 1;
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
                if (d == 0) put(w.record + geo.width * D + 2 * cc, mm), put(w.record + geo.width * D + 2 * cc + 1, ll);
            }
        }
    }
}

// Rows of a wide tile in LDS, as loads that go there directly leave them: 1024 bytes of a
// wave's lanes side by side, D / 8 groups of rows; key k is row k / (D / 8) of group k % (D / 8).
// With 16 bytes between the groups the same 16 bytes of 16 keys, and with 64 the same 64 bytes of
// four values, lie in different banks.
template <int D>
struct WideLds {
    static constexpr int kGroups = D / 8, kKeyGroup = 1024 + 16, kValueGroup = 1024 + 64;
    struct Rows {
        unsigned char k[kGroups * kKeyGroup], v[kGroups * kValueGroup];
    } tile[2];
    unsigned bad;   // whether a value of the tile is infinite or NaN, where that matters
    static __device__ __forceinline__ int value(int key) { return key % kGroups * kValueGroup + key / kGroups * (D * 2); }
};

// 16 bytes from each lane's address to LDS, a wave's side by side.
__device__ __forceinline__ void copy16(const unsigned char *from, unsigned char *to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

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
// The next tile's rows are on their way there meanwhile.  Lane l = 32 h + n:
//   QK^T  S^T[key][column] = K . q^T, two blocks of 32 keys.  It gets the scores of column n
//         for the keys 32 b + 8 (i / 4) + 4 h + i % 4.
//   PV    O^T[dim][column] = V^T . P^T, contracting over 16 keys at a time in the order in which
//         the score registers hold them.  V^T comes by transposing reads of LDS, four keys of
//         16 dims a group of 16 lanes.
template <int D>
__device__ __forceinline__ void attend_wide(const PagedChunk &a, const Geo &geo, const Piece &w, WideLds<D> &lds)
{
    using Lds = WideLds<D>;
    constexpr int kGroups = Lds::kGroups, kSteps = D / 16, kDims = D / 32;
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

    // Lane l looks up position t0 + l of a tile, two tiles ahead of its use.  Nothing is made of what
    // is looked up before that, or the tile on its way, asked for earlier, would be waited for too.
    auto page_of = [&](int t0) {
        const int pos = t0 + lane;
        return table[geo.by_page((unsigned)(pos < end ? pos : begin))];
    };
    using Tile64 = typename Lds::Rows;
    auto load = [&](const unsigned char *__restrict K, const unsigned char *__restrict V, Tile64 *__restrict to, int t0, int pg)
                    __attribute__((always_inline)) {   // asks for a tile; which of its positions there are
        const int pos = t0 + lane;
        const bool ok = pos < end && pg >= 0 && pg < c.pages;
        const unsigned off = ok ? slot16(a, geo, pg, pos) : 0u;
#pragma unroll
        for (int i = 0; i < kDims; ++i) {
            const int g = kDims * wave + i, key = lane / kGroups * kGroups + g;
            const size_t at = (size_t)(unsigned)__builtin_amdgcn_ds_bpermute(key << 2, (int)off) * 16 + lane % kGroups * 16;
            copy16(K + at, to->k + g * Lds::kKeyGroup);
            copy16(V + at, to->v + g * Lds::kValueGroup);
        }
        return __ballot(ok);
    };

    f32x16_t o[kDims];
#pragma unroll
    for (int d = 0; d < kDims; ++d) {
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    }
    float m = -INFINITY, l = 0.f;   // m: scaled
    bool any = false;

    // operands: of K the lane's key n, of V^T its dim n of the keys 4 h + 0 .. 3, by a transposition
    // of the four keys that 16 lanes read
    const int k_at = n % kGroups * Lds::kKeyGroup + n / kGroups * (D * 2) + 16 * h;
    const int v_at = Lds::value(4 * h + (lane & 15) / 4) + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
    struct Values {
        bf16x8_t x[kDims];
    };
    // Each weight is the sum of three bf16 values, eight bits of it and a part, cut off: all its 24
    // bits, so that the only rounding as coarse as the type's is the last.  With two parts, within 2^-17,
    // 2.2 to 2.7 results in 1000 were not the bf16 value next to the exact one, with three 0.2 to
    // 1.3 (2048 tokens over 32500 positions; elementary operations in 32 bits 1.9).  The third costs
    // 1496 -> 1765 us there, 113 -> 131 for 512 tokens behind 7680, 73 -> 81 for 32 prompts of 1 to 1164.
    struct Weights {
        bf16x8_t part[3];
    };
    auto values = [&](const unsigned char *at, int s) {   // of 16 keys: 16 s + 4 h + 0 .. 3 and 8 behind
        Values r;
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
            s16x4_t v[2];
#pragma unroll
            for (int x = 0; x < 2; ++x)
                v[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4_t *)(at + Lds::value(16 * s + 8 * x) + 64 * d));
            r.x[d] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
        return r;
    };
    auto attend = [&](const Tile64 *now, int t0, unsigned long long live) __attribute__((always_inline)) {
        const unsigned char *kt = now->k + k_at, *vt = now->v + v_at;
        f32x16_t sc[2];
        bf16x8_t kf[2][kSteps];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) kf[b][s] = *reinterpret_cast<const bf16x8_t *>(kt + 32 / kGroups * b * (D * 2) + 32 * s);
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
        if (live == ~0ull && t0 + kWideTile > first_lim) {
            const int left = lim - t0 - 4 * h;   // positions of the tile below the column's limit, from the lane's first on
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (left <= 32 * b + 8 * (i / 4) + i % 4) sc[b][i] = -INFINITY;
            }
            any |= lim > t0;
        } else if (live != ~0ull) {
            const int left = lim - t0;
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
            mx = fmaxf(lo, hi) * scale;
        }
        // Weights are taken relative to a maximum that may be left behind by up to 2^8: what has
        // been added up is scaled down seldom, and sums of 32 bits do not mind.
        if (__any(mx - m > 8.f || m == -INFINITY)) {
            const float top = fmaxf(m, mx);
            const float f = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top);   // nothing yet, but perhaps an infinity
            l *= f;
#pragma unroll
            for (int d = 0; d < kDims; ++d) o[d] *= f;
            m = top;
        }
        const float base = m == -INFINITY ? 0.f : m;
        // A score's product with the scale is not rounded before the maximum, which is, leaves it: a
        // factor of all weights, of at most 2 where the maximum is below 2^24.  Above, where it would be
        // any, these products are rounded too.
        float factor = scale;
        if (__any(fabsf(base) >= 0x1p24f)) {
            const bool far = fabsf(base) >= 0x1p24f;
            factor = far ? 1.f : scale;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[b][i] *= far ? scale : 1.f;
            }
        }
        float sum[2] = {0.f, 0.f};
        auto weights = [&](int s) {
            Weights r;
            u32x4_t part[3];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float p[2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    p[x] = __builtin_amdgcn_exp2f(fmaf(sc[s / 2][8 * (s % 2) + 2 * j + x], factor, -base));
                    sum[x] += p[x];
                }
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    part[i][j] = __builtin_amdgcn_perm(__float_as_uint(p[1]), __float_as_uint(p[0]), 0x07060302u);
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        if (i < 2) p[x] -= __uint_as_float(__float_as_uint(p[x]) & 0xffff0000u);
                }
            }
#pragma unroll
            for (int i = 0; i < 3; ++i) r.part[i] = __builtin_bit_cast(bf16x8_t, part[i]);
            return r;
        };
        Weights p = weights(0);
#pragma unroll
        for (int s = 0; s < 4; ++s) {   // 16 keys at a time; the next ones' operands are made meanwhile
            Values v_next;
            Weights p_next;
            if (s < 3) v_next = values(vt, s + 1), p_next = weights(s + 1);
#pragma unroll
            for (int i = 0; i < 3; ++i) {
#pragma unroll
                for (int d = 0; d < kDims; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.x[d], p.part[i], o[d], 0, 0, 0);
            }
            if (s < 3) {
#pragma unroll
                for (int d = 0; d < 3 * kDims; ++d) {
                    __builtin_amdgcn_sched_group_barrier(kSchedMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kSchedRead, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kSchedValu, 72 / (3 * kDims), 0);
                }
                v = v_next, p = p_next;
            }
        }
        l += sum[0] + sum[1];
    };

    // Values of positions that are not there become zeros: the loads brought anything.  And an
    // infinity or NaN would reach columns that do not attend its position, as 0 times it: such
    // elements are added to the columns that do and taken out.
    auto tidy = [&](Tile64 *now, int t0, unsigned long long live) __attribute__((always_inline)) {
        constexpr int kMine = kWideTile * D * 2 / 16 / kBlock;   // 16-byte pieces of a lane's
        bool bad = false;
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int piece = tid + kBlock * i, key = piece / kGroups;
            auto *x = reinterpret_cast<u32x4_t *>(now->v + Lds::value(key) + piece % kGroups * 16);
            if (!(live >> key & 1)) {
                *x = u32x4_t{0u, 0u, 0u, 0u};
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) bad |= ((*x)[j] & 0x7f80u) == 0x7f80u || ((*x)[j] & 0x7f800000u) == 0x7f800000u;
            }
        }
        if (__any(bad) && lane == 0) lds.bad = 1u;
        __syncthreads();
        if (!lds.bad) return;   // 0 from the beginning
        for (int key = 0; key < kWideTile; ++key) {
#pragma unroll
            for (int d = 0; d < kDims; ++d) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int dim = 32 * d + 8 * (i / 4) + 4 * h + i % 4;
                    const float v = __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t *>(now->v + Lds::value(key) + dim * 2) << 16);
                    if (!(fabsf(v) < INFINITY) && t0 + key < lim) o[d][i] += v;
                }
            }
        }
        __syncthreads();
        for (int i = tid; i < kWideTile * D; i += kBlock) {
            auto *x = reinterpret_cast<uint16_t *>(now->v + Lds::value(i / D)) + i % D;
            if ((*x & 0x7f80u) == 0x7f80u) *x = 0;
        }
        if (tid == 0) lds.bad = 0u;
        __syncthreads();
    };

    if (begin < end) {
        int pg = page_of(begin), buf = 0;
        int pg_next = page_of(end - begin > kWideTile ? begin + kWideTile : begin);
        unsigned long long live = load(Kh, Vh, lds.tile, begin, pg);
        if (tid == 0) lds.bad = 0u;
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        // Two tiles of one variable: that reads of `now` and the loads that go to `next` never meet is
        // said by __restrict, or every read of LDS waits for all of these loads (32 rows of 5 tokens
        // 78 us, 36 of 1 and 4 of 129 to 512 tokens 144; so 74 and 136; weights of two parts).  Between steps everybody
        // waits for them.
        auto step = [&](const unsigned char *__restrict K, const unsigned char *__restrict V, Tile64 *__restrict now,
                        Tile64 *__restrict next, int t0, bool more) __attribute__((always_inline)) {
            unsigned long long live_next = 0;
            if (more) {
                live_next = load(K, V, next, t0 + kWideTile, pg_next);
                pg_next = page_of(end - t0 > 2 * kWideTile ? t0 + 2 * kWideTile : begin);
            }
            if (t0 + kWideTile > w.seen || live != ~0ull) tidy(now, t0, live);
            if (t0 < last_lim) attend(now, t0, live);
            live = live_next;
        };
        for (int t0 = begin;; t0 += kWideTile, buf ^= 1) {
            const bool more = end - t0 > kWideTile;
            step(Kh, Vh, lds.tile + buf, lds.tile + (buf ^ 1), t0, more);
            if (!more) break;
            __builtin_amdgcn_s_waitcnt(0);   // the next tile's rows have arrived, then everybody's
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
        if (w.parts == 1) {
            write_wide<D>(w.out + w.place<D>(a, geo, cc, 4 * h) * 2, o, any ? l : -1.f);
        } else if (h == 0) {
            put(w.record + geo.width * D + 2 * cc, m), put(w.record + geo.width * D + 2 * cc + 1, any ? l : -1.f);
        }
    }
    if (w.parts > 1 && mine > 0) {   // as the registers hold them, so that a wave's stores lie side by side
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
// Joins the records of the `count` shares from x0 on in steps of `step`, 16 columns at a time:
// into the output (last), or into the first of them.
template <int D, bool BF16>
__device__ __forceinline__ void join_narrow(const PagedChunk &a, const Geo &geo, const Piece &w, int x0, int step,
                                            int count, bool last, JoinLds &lds)
{
    auto record = [&](int k) { return geo.records + w.record_of(a, x0 + k * step) * geo.record; };
    for (int c0 = 0; c0 < w.cols; c0 += 16) {
        const int here = w.cols - c0 < 16 ? w.cols - c0 : 16;
        const int states = geo.width * D + 2 * c0;
        __syncthreads();
        // each state's share of the joined one: exp2 of its maximum's distance, in sf
        for (int i = (int)threadIdx.x; i < count * here; i += kBlock) {
            const int k = i / here, ci = i - k * here;
            const float mm = get(record(k) + states + 2 * ci), ll = get(record(k) + states + 2 * ci + 1);
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
            float oo = 0.f;
            for (int k0 = 0; k0 < count; k0 += 8) {   // eight on their way at a time
                float y[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = get(record(k0 + k < count ? k0 + k : k0) + c0 * D + i);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k0 + k < count && !(lds.sg[k0 + k][ci] < 0.f)) oo += y[k] * lds.sf[k0 + k][ci];
            }
            const float ll = lds.sl[ci];
            if (last) store_out<BF16>(w.out, w.place<D>(a, geo, c0 + ci, i % D), ll < 0.f ? 0.f : oo / ll);
            else put(record(0) + c0 * D + i, oo);   // read by this thread alone
        }
        if (!last && (int)threadIdx.x < here) {
            const int ci = (int)threadIdx.x;
            put(record(0) + states + 2 * ci, lds.sm[ci]), put(record(0) + states + 2 * ci + 1, lds.sl[ci]);
        }
    }
}

// The same for a wide tile: a lane has the column and the elements that it had of the sum.
template <int D>
__device__ __forceinline__ void join_wide(const PagedChunk &a, const Geo &geo, const Piece &w, int x0, int step, int count, bool last)
{
    auto record = [&](int k) { return geo.records + w.record_of(a, x0 + k * step) * geo.record; };
    constexpr int kDims = D / 32;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid / kWave, h = lane >> 5, cc = 32 * wave + (lane & 31);
    if (32 * wave >= w.cols) return;
    const int states = geo.width * D + 2 * (cc < w.cols ? cc : 0);
    float top = -INFINITY, sum = -1.f;
    for (int k = 0; k < count; ++k) {
        const float mm = get(record(k) + states), ll = get(record(k) + states + 1);
        top = fmaxf(top, ll < 0.f ? -INFINITY : mm);
    }
    f32x16_t o[kDims];
#pragma unroll
    for (int d = 0; d < kDims; ++d) {
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    }
    for (int k = 0; k < count; ++k) {
        const float mm = get(record(k) + states), ll = get(record(k) + states + 1);
        const float f = weight(ll < 0.f ? -INFINITY : mm, top);
        if (!(ll < 0.f)) sum = (sum < 0.f ? 0.f : sum) + ll * f;
        f32x16_t y[kDims];   // all on their way at once
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
#pragma unroll
            for (int i = 0; i < 16; ++i) y[d][i] = get(record(k) + ((wave * kDims + d) * 16 + i) * kWave + lane);
        }
#pragma unroll
        for (int d = 0; d < kDims; ++d) {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] += ll < 0.f ? 0.f : y[d][i] * f;
        }
    }
    if (last) {
        if (cc < w.cols) write_wide<D>(w.out + w.place<D>(a, geo, cc, 4 * h) * 2, o, sum);
        return;
    }
#pragma unroll
    for (int d = 0; d < kDims; ++d) {
#pragma unroll
        for (int i = 0; i < 16; ++i) put(record(0) + ((wave * kDims + d) * 16 + i) * kWave + lane, o[d][i]);
    }
    if (h == 0 && cc < w.cols) put(record(0) + states, top), put(record(0) + states + 1, sum);
}

// The part's record is written; the last of the tile's parts to arrive joins them, in their
// order, groups of about the square root of their number first.
template <int D, bool BF16>
__device__ __forceinline__ void join_parts(const PagedChunk &a, const Geo &geo, const Piece &w, JoinLds &lds)
{
    // A record has arrived before its workgroup counts itself, and is read by the workgroup that
    // counts last; counters end at zero.
    int group = w.parts;   // parts of a group: at most 64, and as many groups
    if (w.parts > 16) {
        group = 16;
        while (group * group < w.parts) group *= 2;
    }
    static_assert((kJoin & (kJoin - 1)) == 0 && kJoin * kJoin >= kMostShares, "groups and their number fit the arrays");
    const int groups = (w.parts + group - 1) / group;
    for (int level = 0; level < 2; ++level) {
        // level 0: the parts of this one's group, into its first record; level 1: the groups
        if (level == 1 && groups == 1) break;
        const int first = level == 0 ? (w.share - w.first) / group * group : 0;
        const int count = level == 0 ? (w.parts - first < group ? w.parts - first : group) : groups;
        unsigned *counter = (level == 0 ? geo.group_count : geo.tile_count) + w.record_of(a, w.first + first);
        __builtin_amdgcn_s_waitcnt(0);   // this thread's stores have arrived, then everybody's
        __syncthreads();
        if (threadIdx.x == 0)
            lds.arrived = count > 1 ? __hip_atomic_fetch_add(counter, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0u;
        __syncthreads();
        if (lds.arrived != (unsigned)count - 1) return;
        if (threadIdx.x == 0 && count > 1) __hip_atomic_store(counter, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const bool last = level == 1 || groups == 1;
        if constexpr (kHasWide<D, BF16>) join_wide<D>(a, geo, w, w.first + first, level == 0 ? 1 : group, count, last);
        else join_narrow<D, BF16>(a, geo, w, w.first + first, level == 0 ? 1 : group, count, last, lds);
    }
}

template <int D, bool BF16>
union Lds {
    std::conditional_t<kHasWide<D, BF16>, WideLds<D>, NarrowLds<D>> attend;
    JoinLds join;
};

// Waves a SIMD, and workgroups a CU: as many as the registers and the LDS hold.  bf16 heads of 64 spill
// 6 registers, 28 bytes a lane, at 3: 32 prompts of 1 to 1164 tokens of 12 heads take 81 us, with 2 93.
constexpr int occupancy(int D, bool bf16) { return D <= (bf16 ? 64 : 32) ? 3 : 2; }

template <int D, bool BF16>
__global__ __launch_bounds__(kBlock, (occupancy(D, BF16))) void paged_chunk_kernel(PagedChunk a, Geo geo)
{
    __shared__ __align__(16) struct {
        Lds<D, BF16> lds;
        Rows rows;
    } shared;
    Lds<D, BF16> &lds = shared.lds;
    Rows &rows = shared.rows;

    const unsigned wg = wide_index();
    Piece p;
    p.share = (int)geo.by_hkv(wg);
    if (p.share >= geo.shares) return;
    p.h = (int)wg - p.share * a.Hkv;
    if (!geo.plan) {
        if (threadIdx.x < kWave) add_rows(a, geo, rows);
        __syncthreads();
    }
    const u64_t *sums = geo.plan ? geo.plan : rows.sums;
    const u64_t all = uniform64(sums[a.R]);
    u64_t share = (all + (unsigned)geo.shares - 1) / (unsigned)geo.shares;
    // Whole tiles take the longest's time or the mean of the shares.  Cut ones take that, a part's
    // record and the joining, and wide ones find less of their keys in the L2 (us, whole and cut: 2048
    // tokens over 32500 positions 1844 and 1849, 32 prompts of 1 to 1164 tokens 81 and 91, 8 of 1 to 257
    // in fp32 71 and 75; 32 rows of 5 tokens over 200 to 4096 127 and 75, 512 tokens over 8192 249 and 133).
    bool whole = false;
    if (!geo.plan) {
        const float mean = (float)share, longest = (float)(rows.longest * kUnit + kStart);
        const float least = fmaxf(mean, (float)kLeast), cut = 1.12f * least + 3 * kStart;
        whole = (rows.tiles[kScanRows] <= geo.shares ? longest : 1.05f * fmaxf(longest, mean)) <= cut;
    }
    share = share < kLeast ? kLeast : share;

    const u64_t begin = share * (unsigned)p.share, end = begin + share < all ? begin + share : all;
    const int tiles = geo.plan ? 0 : __builtin_amdgcn_readfirstlane(rows.tiles[kScanRows]);
    u64_t x = begin;                  // of its share, done so far
    int turn = 0, t = p.share;        // or its next tile
    auto known = [&](int r) {
        auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
        return row_of(a, geo, same(rows.len[r]), same(rows.off[r]), same(rows.off[r + 1]));
    };
    for (;; __syncthreads()) {   // everybody has left the tile in LDS
        if (whole) {
            if (t >= tiles) return;
            if (tiles <= geo.shares) {   // one each: in any order
                p.r = row_at(rows.tiles, a.R, t);
                p.tile = t - __builtin_amdgcn_readfirstlane(rows.tiles[p.r]);
                t = tiles;
            } else {
                if (threadIdx.x < kWave) find_tile(a, geo, rows, t);
                // there and back again: who had the longest of a turn has the shortest of the next
                ++turn;
                t = turn * geo.shares + (turn & 1 ? geo.shares - 1 - p.share : p.share);
                __syncthreads();
                p.r = __builtin_amdgcn_readfirstlane(rows.row), p.tile = __builtin_amdgcn_readfirstlane(rows.tile);
            }
            p.row = known(p.r);
        } else {
            if (x >= end) return;
            p.r = row_at(sums, a.R, x);
            p.row = geo.plan ? row_of(a, geo, a.kv_len[p.r], a.offsets[p.r], a.offsets[p.r + 1]) : known(p.r);
            p.tile = __builtin_amdgcn_readfirstlane(tile_at(a, geo, p.row, x - uniform64(sums[p.r])));
        }
        p.col0 = p.tile * geo.width;
        p.cols = p.row.columns - p.col0 < geo.width ? p.row.columns - p.col0 : geo.width;
        p.seen = p.limit(a, geo, p.col0);
        const int L = p.limit(a, geo, p.col0 + p.cols - 1);
        p.out = a.out + ((size_t)p.row.begin * a.Hq + (size_t)p.h * geo.G) * D * (BF16 ? 2 : 4);
        p.first = p.share, p.parts = 1;
        p.begin = 0, p.end = L;
        if (!whole) {
            const u64_t row_begin = uniform64(sums[p.r]);
            const u64_t t0 = row_begin + uniform64(work_before(a, geo, p.row, p.tile));
            const u64_t t1 = row_begin + uniform64(work_before(a, geo, p.row, p.tile + 1));
            x = t1;
            // The tile's units before the border of two shares, as both and the tile's others
            // reckon them.  A border within half a unit of the tile's begins or ends there.
            const int units = units_of(L);
            auto unit_at = [&](u64_t at) {
                const int u = at <= t0 ? 0 : at >= t1 ? units : (int)((double)units * ((double)(at - t0) / (double)(t1 - t0)) + 0.5);
                return __builtin_amdgcn_readfirstlane(u < units ? u : units);
            };
            p.first = (int)(t0 / share);
            int last = (int)((t1 - 1) / share);
            if (last > p.first && unit_at(share * (unsigned)(p.first + 1)) == 0) ++p.first;
            if (last > p.first && unit_at(share * (unsigned)last) == units) --last;
            if (p.share < p.first || p.share > last) continue;
            p.parts = last - p.first + 1;
            if (p.share > p.first) p.begin = unit_at(begin) * kUnit;   // below 2^31: a unit of the row's
            const long long stop = p.share == last ? L : (long long)unit_at(begin + share) * kUnit;
            p.end = stop < L ? (int)stop : L;
        }
        p.record = geo.records + p.record_of(a, p.share) * geo.record;
        if constexpr (kHasWide<D, BF16>) attend_wide<D>(a, geo, p, lds.attend);
        else attend_narrow<D, BF16>(a, geo, p, lds.attend);
        if (p.parts > 1) join_parts<D, BF16>(a, geo, p, lds.join);
    }
}

struct Layout {
    int width, record, shares;
    size_t tile_count, plan, records, bytes;   // byte offsets in the workspace
};

Layout layout_of(int N, int R, int Hq, int Hkv, int page, int cols, int D, bool bf16) {
    Layout y{};
    y.width = bf16 ? (D >= 32 ? kWideColumns : 32) : D <= 64 ? 32 : 16;
    y.record = y.width * (D + 2);
    const int places = 256 * occupancy(D, bf16);   // workgroups that fit the 256 CUs at once
    // all places to the heads alike; two rounds of them where that would leave many empty
    long long shares = Hkv <= places / 8 ? places / Hkv : 2 * places / Hkv;
    const long long columns = (long long)N * (Hq / Hkv), rows = R < N ? R : N;   // rows with tokens
    const long long tiles = columns / y.width + rows, units = ((long long)cols * page + kUnit - 1) / kUnit + 1;
    if (shares > tiles * units) shares = tiles * units;
    y.shares = shares < 1 ? 1 : (int)shares;
    // the counters lie where every call has them, whatever its sizes
    y.tile_count = 2 * kMostShares * sizeof(unsigned);
    y.plan = 2 * y.tile_count;
    y.records = y.plan + (R > kScanRows ? ((size_t)R + 2) / 2 * 2 * sizeof(u64_t) : 0);
    y.bytes = y.records + (y.shares > 1 ? 2 * (size_t)y.shares * Hkv * y.record * sizeof(float) : 0);
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
    geo.G = a.Hq / a.Hkv, geo.width = y.width, geo.half = 0.5 * y.width / geo.G, geo.record = y.record, geo.shares = y.shares;
    geo.by_page = make_div(a.cache.page), geo.by_hkv = make_div(a.Hkv), geo.by_g = make_div(geo.G);
    geo.page16 = (unsigned)(a.cache.page_bytes / 16), geo.slot16 = (unsigned)(a.cache.slot_bytes / 16);
    geo.group_count = reinterpret_cast<unsigned *>(a.workspace);
    geo.tile_count = reinterpret_cast<unsigned *>(a.workspace + y.tile_count);
    geo.records = reinterpret_cast<float *>(a.workspace + y.records);
    if (a.R > kScanRows) {
        auto *plan = reinterpret_cast<u64_t *>(a.workspace + y.plan);
        geo.plan = plan;
        hipLaunchKernelGGL(chunk_plan_kernel, dim3(1), dim3(1024), 0, stream, a, geo, plan);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const dim3 gd = wide_grid((long long)y.shares * a.Hkv), bd(kBlock);
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
