// Sampling of one token per row for gfx950: temperature, top-k, top-p and min-p,
// drawn with a given uniform number.
//
// With the row's logits x, in the order of falling x (equal logits in the order
// of their index), and w_i = exp((x_i - max x) / T):
//   K  the first k of the order;
//   P  those of K before which less than p of K's mass lies;
//   M  those with w_i >= m.
// Every one of the three is a beginning of the order, so what is left is one too:
// a threshold logit and, among the logits equal to it, a last index (Cut).  The
// draw is the first token, in the order of the indices, at which the running sum
// of the kept w exceeds u times their total.
//
// A draw next to a border of two tokens depends on the sums, and a large
// vocabulary has many borders: with weights and sums in 32 bits 7 draws in 1000 would
// be another token's, with the weights alone in 32 bits 1 in 100000 (4 million draws
// from rows of 50257 normal logits of deviation 1.5).  Weights and sums are 64-bit.
//
// No pass sorts or scans the row:
//   top-k      The k-th largest of the threads' 1024 maxima is a bound that at
//              least k logits reach, and few more do.  Those go to a list in LDS,
//              which is sorted; top-p, min-p and the draw happen in the list.
//   top-p      alone: one pass adds up all weights, and those that can matter
//              (together the others have less than half of 1 - p) by value, in
//              2048 bins.  The list has the logits down to the bin in which the
//              mass reaches p; the draw happens in it.  If they are too many, the
//              list has that bin alone, for the cut.
//   otherwise  (the list's capacity exceeded, or k above kTopK) the cut is found by
//              digits of the logits' bits.
//   The draw of what no list holds goes by sums of parts of the row, and then of
//   parts of the part that has the token.
//
// Two ways through a row.
//   sample_row     one workgroup has it and reads it two to four times (with the
//                  search by digits seven to fifteen), after the first time from the
//                  caches (held in registers, it needs unrolled passes, which run once a
//                  row: waiting for their instructions cost more than reading again).
//                  For many rows, and for the rows that the other way gives up.
//   four kernels   with a workgroup per slice of 4096 logits, for up to
//                  kSliceRows rows of more than kSliceFrom logits (and, with
//                  top-k, of small k):
//     slice_kernel   reads the logits.  Its maximum, and what goes by it alone:
//                    greedy's token, top-k's candidates of the slice, the sum of the
//                    weights (of the slice's maximum).
//     merge_kernel   joins these: greedy, top-k and unfiltered rows are done.  The
//                    others know their maximum now: top-p's bins.
//     gather_kernel  top-p: the list, and the draw by the last slice to arrive.
//                    min-p alone: the sums of what is kept, and the draw.
//     rest_kernel    nuclei that exceed the list: the sums of what is kept, and the
//                    draw.  sample_row for rows given up.
//                  One row of 131072 then is on 32 CUs, and the bins' atomic
//                  additions, which are what a CU's LDS is slowest at, with it.
//
// Measured, calls back to back: 128 rows of 50264 with top-k and top-p 17.7 us, 512 bf16
// rows of 50257 without a filter 44 (one launch by itself 48), 256 rows of 151936 with
// settings of their own 154, one row of 131072 with top-p 33.
#include <math.h>
#include <stdint.h>

#include "div.h"
#include "launch.h"

namespace fs {
namespace {

constexpr int kWave = 64;
constexpr int kBins = 2048;   // of a digit of 11 bits, and of top-p's weights
constexpr int kStep = 4 * kWave;   // logits of a wave's load

typedef float f32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// Order-preserving map of the floats to integers (both zeros to one: they are equal).
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// ---- exchange between lanes ---------------------------------------------------
// On the words of a value: DPP inside rows of 16 lanes, permlane swaps across them.
template <typename V, typename F>
__device__ __forceinline__ V by_words(V x, F f) {
    if constexpr (sizeof(V) == 4) {
        return __builtin_bit_cast(V, f(__builtin_bit_cast(uint32_t, x)));
    } else {
        const auto u = __builtin_bit_cast(unsigned long long, x);
        return __builtin_bit_cast(V, (unsigned long long)f((uint32_t)(u >> 32)) << 32 | f((uint32_t)u));
    }
}
template <int CTRL, int ROWS = 0xF, typename V>
__device__ __forceinline__ V dpp(V x) {   // 0 where the source lane does not exist or the row is masked
    return by_words(x, [](uint32_t u) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, CTRL, ROWS, 0xF, CTRL < 0x142 || CTRL > 0x143);
    });
}
template <int MASK, typename V>
__device__ __forceinline__ V other_row(V x) {   // of lane ^ MASK, MASK = 16 or 32
    return by_words(x, [](uint32_t u) {
        const bool up = (__lane_id() & MASK) != 0;
        if constexpr (MASK == 16) {
            const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
            return (uint32_t)(up ? r[0] : r[1]);
        } else {
            const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
            return (uint32_t)(up ? r[0] : r[1]);
        }
    });
}
template <int MASK, typename V>
__device__ __forceinline__ V xor_lane(V x) {   // of lane ^ MASK, a power of two
    if constexpr (MASK == 1) return dpp<0xB1>(x);
    else if constexpr (MASK == 2) return dpp<0x4E>(x);
    else if constexpr (MASK == 4)
        return by_words(x, [](uint32_t u) { return (uint32_t)__builtin_amdgcn_ds_swizzle((int)u, 0x1F | (4 << 10)); });
    else if constexpr (MASK == 8) return dpp<0x128>(x);   // eight lanes round in the row
    else return other_row<MASK>(x);
}
template <typename V, typename Op>
__device__ __forceinline__ V wave_reduce(V x, Op op) {   // the same bits in every lane: each step pairs lanes
    x = op(x, dpp<0xB1>(x));    // lane ^ 1
    x = op(x, dpp<0x4E>(x));    // lane ^ 2
    x = op(x, dpp<0x141>(x));   // the other four of eight
    x = op(x, dpp<0x140>(x));   // the other eight of sixteen
    x = op(x, other_row<16>(x));
    return op(x, other_row<32>(x));
}
template <typename V>
__device__ __forceinline__ V wave_scan(V x) {   // inclusive sums over the lanes
    x += dpp<0x111>(x);         // of the row: from 1, 2, 4 and 8 lanes before
    x += dpp<0x112>(x);
    x += dpp<0x114>(x);
    x += dpp<0x118>(x);
    x += dpp<0x142, 0xA>(x);    // the last of row 0 and 2 to row 1 and 3
    return x + dpp<0x143, 0xC>(x);   // the last of row 1 to rows 2 and 3
}

struct Add { template <typename V> __device__ V operator()(V a, V b) const { return a + b; } };
struct Max { __device__ float operator()(float a, float b) const { return fmaxf(a, b); } };
struct Min { template <typename V> __device__ V operator()(V a, V b) const { return a < b ? a : b; } };

// What is kept of a row: the logits above the threshold, and those equal to it up
// to an index.
struct Cut {
    float x;
    int last;
    __device__ __forceinline__ bool keeps(float v, int i) const { return v > x || (v == x && i <= last); }
};

// Weights exp((x - top) / T), to some 4e-14 of themselves: 2^y with y split into a
// whole number and a rest f of at most a half, 2^f = 1 + f q(f) with q the
// interpolation of (2^f - 1) / f in the nine Chebyshev nodes.  The weight of top
// is exactly 1, that of -inf 0.
struct Mass {
    double top, c;   // the largest logit; log2(e) / T
    double unit;     // of whole(): 2^-44 of the largest weight (2^-38 for 2^24 logits)
    double q[9];     // in scalar registers: as literals they would take vector registers
    __device__ __forceinline__ Mass(float top_, float temp, int V) {
        const int lg = V > 1 ? 32 - __clz(V - 1) : 0;
        top = (double)uniform(top_), c = uniform(1.4426950408889634 / (double)temp);
        unit = uniform(ldexp(1.0, lg > 18 ? 62 - lg : 44));
        q[0] = 0x1.62e42fefa39efp-1, q[1] = 0x1.ebfbdff823cedp-3, q[2] = 0x1.c6b08d7047e52p-5;
        q[3] = 0x1.3b2ab7181b755p-7, q[4] = 0x1.5d87fe86fe88ep-10, q[5] = 0x1.4308ac85aa947p-13;
        q[6] = 0x1.ffcb9515a8016p-17, q[7] = 0x1.63d136366db24p-20, q[8] = 0x1.b63880a30e9ffp-24;
#pragma unroll
        for (int i = 0; i < 9; ++i) asm("" : "+s"(q[i]));
    }
    // a value that all lanes have, in scalar registers
    template <typename V>
    static __device__ __forceinline__ V uniform(V x) {
        return by_words(x, [](uint32_t u) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)u); });
    }
    __device__ __forceinline__ double log2w(float x) const { return ((double)x - top) * c; }
    __device__ __forceinline__ double w(float x) const {
        const double y = fmax(log2w(x), -2000.0);   // 0 below; -inf and NaN (of -inf at T = inf) too
        constexpr double kRound = 6755399441055744.0;   // 1.5 * 2^52: its sum with y has y's whole part in its low bits
        const double z = y + kRound;
        const double f = y - (z - kRound);
        double p = q[8];
#pragma unroll
        for (int i = 7; i >= 0; --i) p = fma(p, f, q[i]);
        return ldexp(fma(p, f, 1.0), (int)(uint32_t)__builtin_bit_cast(unsigned long long, z));
    }
    // as whole numbers, whose sums do not depend on the order of atomic additions
    __device__ __forceinline__ unsigned long long whole_of(double w) const { return (unsigned long long)(w * unit + 0.5); }
    __device__ __forceinline__ unsigned long long whole(float x) const { return whole_of(w(x)); }
};

// Of sums, one a lane (the same in every wave: no exchange between waves), the first
// positive one at which the running sum, from `run` on, exceeds goal, or the last
// positive one: its lane, the sum before it; -1: none is positive.  passed: one did.
__device__ __forceinline__ int pick_lane(double sum, double goal, double run, double &before, bool &passed) {
    const double upto = run + wave_scan(sum);
    const unsigned long long has = __ballot(sum > 0.0), past = __ballot(sum > 0.0 && upto > goal);
    passed = past != 0;
    const int at = past ? __ffsll((long long)past) - 1 : 63 - __clzll((long long)has);   // -1 for has == 0
    before = __shfl(upto - sum, at & 63);
    return at;
}

// One step of a bitonic sort of entries in lanes: pairs J apart, falling where down.
template <int J>
__device__ __forceinline__ void sort_step(unsigned long long &x, bool down) {
    const unsigned long long y = xor_lane<J>(x);
    const bool first = ((int)threadIdx.x & J) == 0;
    x = (x < y) == (first == down) ? y : x;
}
template <int J>
__device__ __forceinline__ void merge_lanes(unsigned long long &x, bool down) {   // steps J, J / 2, .., 1
    sort_step<J>(x, down);
    if constexpr (J > 1) merge_lanes<J / 2>(x, down);
}
template <int K>
__device__ __forceinline__ void sort_lanes(unsigned long long &x, bool down) {   // the lanes, falling where down
    if constexpr (K > 2) sort_lanes<K / 2>(x, K == 64 ? ((int)threadIdx.x & 32) == 0 : ((int)threadIdx.x & (K / 2)) == 0);
    merge_lanes<K / 2>(x, down);
}

// The cut of min-p: w >= m where (x - top) c >= log2 m; the least such float, at most top.
__device__ Cut cut_of_min_p(const Mass &mass, float m, float top, int V) {
    const double least = log2(fmin((double)m, 1.0));
    float f = (float)(mass.top + least / mass.c);
    if (mass.log2w(f) < least) f = nextafterf(f, INFINITY);
    else if (f > -INFINITY && mass.log2w(nextafterf(f, -INFINITY)) >= least) f = nextafterf(f, -INFINITY);
    return Cut{f > top ? top : f, V};
}

// A row's settings.
struct Setting {
    float temp, p, mp, u;
    int k;
    __device__ __forceinline__ Setting(const TokenSample &a, int r)
        : temp(a.temperature ? a.temperature[r] : 1.f), p(a.top_p ? a.top_p[r] : 1.f), mp(a.min_p ? a.min_p[r] : 0.f),
          u(a.u[r]), k(a.top_k ? a.top_k[r] : 0) {}
    __device__ __forceinline__ bool cuts_k(int V) const { return k > 0 && k < V; }
    __device__ __forceinline__ bool cuts_p() const { return p < 1.f; }
    __device__ __forceinline__ bool cuts_m() const { return mp > 0.f; }
    __device__ __forceinline__ double share() const { return (double)fmaxf(p, 0.f); }   // of the mass
};

__device__ __forceinline__ Cut cut_of_m(const Setting &st, const Mass &mass, float top, int V) {
    return st.cuts_m() && mass.c > 0.0 ? cut_of_min_p(mass, st.mp, top, V) : Cut{-INFINITY, -1};
}

__device__ __forceinline__ void no_distribution(const TokenSample &a, int r) {
    if (threadIdx.x == 0) a.token[r] = -1, a.logprob[r] = NAN;
}

// Top-p's bins by value: in 32 bits, falling with x and the same in every pass.  The
// weights past the last bin, below 2^-deep, have less than half of 1 - p together.
struct Bins {
    float top, per;
    __device__ __forceinline__ Bins(const Setting &st, const Mass &mass, float top_, int V) : top(top_) {
        const double deep = log2((double)V / (1.0 - st.share())) + 1.0;
        per = (float)((double)kBins / deep * mass.c);
    }
    __device__ __forceinline__ float of(float x) const { return fmaxf((top - x) * per, 0.f); }
};

// ---- what a workgroup of kWaves waves does ------------------------------------

template <int kWaves>
struct Block {
static constexpr int kBlock = kWave * kWaves;
static constexpr int kList = kWaves == 16 ? 2048 : 1024;   // logits that are sorted in LDS
static constexpr int kEach = kList / kBlock;               // of these, a thread's
static constexpr int kTopK = kBlock / 4 * 3;   // the list then has some twice as many logits of a smooth distribution

struct Shared {
    static constexpr int kRoom = kList;
    unsigned long long hist[kBins];   // also the sorted list's weights
    uint32_t hits[kBins];             // logits of each bin
    unsigned long long list[kList];   // key << 32 | ~index: sorted by falling value, then index
    unsigned long long part[kWaves];
    double sum[kWaves];
    float fpart[kWaves];
    int ints[kWaves];
    unsigned long long above;
    double total;
    int bin, count, pick;
};

// Reduction over the workgroup; part: kWaves words of LDS that nothing else uses meanwhile.
template <typename V, typename Op>
static __device__ __forceinline__ V block_reduce(V x, V *part, Op op) {
    x = wave_reduce(x, op);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x / kWave] = x;
    __syncthreads();
    V y = part[0];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) y = op(y, part[w]);
    return y;
}
// Inclusive sums over the threads.
template <typename V>
static __device__ __forceinline__ V block_scan(V x, V *part) {
    const int wv = (int)threadIdx.x / kWave;
    x = wave_scan(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) part[wv] = x;
    __syncthreads();
    V base = 0;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w) {   // all read at once, no loop of dependent reads
        const V y = part[w];
        base += w < wv ? y : V(0);
    }
    return base + x;
}

// The row, wave w's part being [w * span, (w + 1) * span).
template <typename T>
struct Row {
    const T *x;
    int V, begin, end;   // of the wave

    struct __attribute__((packed, aligned(sizeof(T)))) Four { T e[4]; };   // rows begin at any element
    static __device__ __forceinline__ f32x4_t wide(const Four &f) {
        return f32x4_t{widen(f.e[0]), widen(f.e[1]), widen(f.e[2]), widen(f.e[3])};
    }
    __device__ __forceinline__ f32x4_t load(int i) const {   // logits i .. i + 3, -inf past the end
        if (i + 4 <= V) return wide(*reinterpret_cast<const Four *>(x + i));
        f32x4_t r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = i + e < V ? widen(x[i + e]) : -INFINITY;
        return r;
    }
    static __device__ __forceinline__ int span_of(int V) { return (V + kWaves * kStep - 1) / (kWaves * kStep) * kStep; }
    __device__ __forceinline__ Row(const T *p, int V_) : x(p), V(V_) {
        const int span = span_of(V), w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
        begin = w * span < V ? w * span : V;
        end = V - begin < span ? V : begin + span;
    }
    // f(four logits, index of the first), in the order of the indices; every lane of a wave takes every step
    template <int kAhead = 4, typename F>
    __device__ __forceinline__ void each4(F f) const {
        const int lane4 = 4 * ((int)threadIdx.x & 63);
        int i = begin;
        for (; end - i >= kAhead * kStep; i += kAhead * kStep) {   // whole loads, kAhead of them on their way
            Four q[kAhead];
#pragma unroll
            for (int s = 0; s < kAhead; ++s) q[s] = *reinterpret_cast<const Four *>(x + i + s * kStep + lane4);
#pragma unroll
            for (int s = 0; s < kAhead; ++s) f(wide(q[s]), i + s * kStep + lane4);
        }
        for (; i < end; i += kStep) f(load(i + lane4), i + lane4);
    }
    template <int kAhead = 4, typename F>
    __device__ __forceinline__ void each(F f) const {
        each4<kAhead>([&](const f32x4_t &q, int i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) f(q[e], i + e);
        });
    }
};

// The bin, counted from bin 0 of `bins`, in which the running sum of sh.hist first
// reaches target: sh.bin and the sum before it, sh.above; sh.bin = -1 if none does.
// DOWN: the bins are counted from the last one.
template <bool DOWN>
static __device__ __forceinline__ void find_bin(Shared &sh, int bins, unsigned long long above, unsigned long long target) {
    constexpr int kMine = kBins / kBlock;   // bins of a thread
    const int tid = (int)threadIdx.x;
    if (tid == 0) sh.bin = -1;
    unsigned long long x[kMine], sum = 0;
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
        const int b = kMine * tid + e;
        x[e] = b < bins ? sh.hist[DOWN ? bins - 1 - b : b] : 0;
        sum += x[e];
    }
    unsigned long long run = above + block_scan(sum, sh.part) - sum;
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
        const int b = kMine * tid + e;
        if (run < target && target <= run + x[e]) sh.bin = DOWN ? bins - 1 - b : b, sh.above = run;
        run += x[e];
    }
    __syncthreads();
}

static __device__ __forceinline__ void clear_bins(Shared &sh) {
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kBins; b += kBlock) sh.hist[b + threadIdx.x] = 0;
    __syncthreads();
}

// The cut at which the sum of f over the logits that `from` keeps, in the order,
// first reaches `target` (1 <= target <= the sum), by digits of the key, the
// highest first.  f: 1 (counts) or the weight (equal logits have one f).
template <typename R, typename F>
static __device__ __forceinline__ Cut find_cut(Shared &sh, const R &row, const Cut &from, unsigned long long target, F f) {
    uint32_t prefix = 0, mask = 0;
    unsigned long long above = 0;
    const int tid = (int)threadIdx.x;
    for (int level = 0; level < 3; ++level) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bins = level == 2 ? 1024 : 2048;
        clear_bins(sh);
        row.each([&](float x, int i) {
            const uint32_t k = key_of(x);
            if ((k & mask) == prefix && from.keeps(x, i)) {
                const unsigned long long v = f(x);
                if (v) atomicAdd(&sh.hist[(k >> shift) & (bins - 1)], v);
            }
        });
        __syncthreads();
        find_bin<true>(sh, bins, above, target);
        prefix |= (uint32_t)sh.bin << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        above = sh.above;
        __syncthreads();
    }
    // the logits equal to the threshold: as many as reach the target, by index
    const float xt = value_of(prefix);
    const unsigned long long one = f(xt);
    const int need = (int)((target - above + one - 1) / one);
    int mine = 0;
    row.each([&](float x, int i) { mine += x == xt && from.keeps(x, i); });
    const int upto = wave_reduce(mine, Add{});
    if ((tid & 63) == 0) sh.ints[tid / kWave] = upto;
    if (tid == 0) sh.pick = row.V;
    __syncthreads();
    int seen = 0;
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w) {
        const int y = sh.ints[w];
        seen += w < tid / kWave ? y : 0;
    }
    if (seen < need && need <= seen + upto) {   // the wave that has the last one
        row.each4([&](const f32x4_t &q, int i) {
            int m = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) m += q[e] == xt && from.keeps(q[e], i + e);
            const int after = wave_scan(m);
            int rank = seen + after - m;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (q[e] == xt && from.keeps(q[e], i + e) && ++rank == need) sh.pick = i + e;
            seen += __shfl(after, 63);
        });
    }
    __syncthreads();
    return Cut{xt, sh.pick};
}

// Collects the logits for which is(x, i) into sh.list; their number (above its room:
// the list is not complete).
template <typename SH, typename R, typename F>
static __device__ __forceinline__ int collect(SH &sh, const R &row, F is) {
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    row.each4([&](const f32x4_t &q, int i) {
        bool hit[4];
        unsigned long long all[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) hit[e] = is(q[e], i + e), all[e] = __ballot(hit[e]);
        if ((all[0] | all[1] | all[2] | all[3]) == 0) return;
        // one addition for the wave: additions to one address wait for each other
        int base = 0;
        const int lane = (int)threadIdx.x & 63;
        if (lane == 0) base = atomicAdd(&sh.count, __popcll(all[0]) + __popcll(all[1]) + __popcll(all[2]) + __popcll(all[3]));
        base = __builtin_amdgcn_readfirstlane(base);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int at = base + __popcll(all[e] & ((1ull << lane) - 1));
            if (hit[e] && at < SH::kRoom) sh.list[at] = (unsigned long long)key_of(q[e]) << 32 | (uint32_t)~(i + e);
            base += __popcll(all[e]);
        }
    });
    __syncthreads();
    return sh.count;
}

// Sorts the first n entries of sh.list, falling: bitonic, thread t with the entries t,
// t + kBlock, .. in registers; only pairs of different waves meet in LDS.
static __device__ __forceinline__ void sort_list(Shared &sh, int n) {
    const int t = (int)threadIdx.x;
    int size = kWave;
    while (size < n) size *= 2;
    unsigned long long x[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int at = t + e * kBlock;
        x[e] = at < n ? sh.list[at] : 0;   // 0: below every entry
        if (at < size) sort_lanes<64>(x[e], (at & 64) == 0 || size == 64);
    }
    for (int k = 128; k <= size; k *= 2) {
#pragma unroll 1
        for (int j = k / 2; j >= kWave; j /= 2) {
            if (j >= kBlock) {   // the thread's own
#pragma unroll
                for (int e = 0; e < kEach; ++e)
#pragma unroll
                    for (int d = 1; d < kEach; d *= 2)
                        if (d * kBlock == j && !(e & d)) {
                            const bool down = ((t + e * kBlock) & k) == 0;
                            const unsigned long long lo = x[e], hi = x[e | d];
                            if ((lo < hi) == down) x[e] = hi, x[e | d] = lo;
                        }
                continue;
            }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kEach; ++e)
                if (t + e * kBlock < size) sh.list[t + e * kBlock] = x[e];
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kEach; ++e) {
                const int at = t + e * kBlock;
                if (at < size) {
                    const unsigned long long y = sh.list[at ^ j];
                    x[e] = (x[e] < y) == (((at & j) == 0) == ((at & k) == 0)) ? y : x[e];
                }
            }
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (t + e * kBlock < size) merge_lanes<32>(x[e], ((t + e * kBlock) & k) == 0);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kEach; ++e)
        if (t + e * kBlock < size) sh.list[t + e * kBlock] = x[e];
    __syncthreads();
}
static __device__ __forceinline__ float list_value(const Shared &sh, int i) { return value_of((uint32_t)(sh.list[i] >> 32)); }

// A bound that at least k of the threads' maxima reach (k <= kBlock), and not many
// more: the least of those down to the bin, of kBlock between the largest and the
// least finite one, in which the k-th is.  Where outliers crowd the others into
// one bin, again between that bin's ends.  -inf: fewer than k are finite.
template <typename SH>
static __device__ __forceinline__ float bound_of(SH &sh, float own, float top, int k) {
    uint32_t *count = reinterpret_cast<uint32_t *>(sh.hist), *least = count + kBlock;
    const int tid = (int)threadIdx.x;
    float hi = top, lo = block_reduce(own > -INFINITY ? own : top, sh.fpart, Min{}), bound = -INFINITY;
    int before = 0;
    for (int level = 0; level < 4; ++level) {
        count[tid] = 0, least[tid] = 0xffffffffu;
        if (tid == 0) sh.bin = -1;
        __syncthreads();
        const float per = (float)kBlock / (hi - lo);   // infinite: all in the first bin, or NaN, which is no bin
        const float b = (hi - own) * per;
        const int bin = own == hi ? 0 : b < (float)kBlock ? (int)b : kBlock - 1;
        const bool in = own >= lo && own <= hi;
        if (in) atomicAdd(&count[bin], 1u), atomicMin(&least[bin], key_of(own));
        __syncthreads();
        const int c = (int)count[tid], upto = before + block_scan(c, sh.ints);
        if (upto - c < k && k <= upto) sh.bin = tid, sh.above = (unsigned long long)(upto - c) << 32 | (unsigned)c;
        __syncthreads();
        if (sh.bin < 0) return -INFINITY;
        bound = value_of(least[sh.bin]);
        before = (int)(sh.above >> 32);
        const int here = (int)(uint32_t)sh.above;
        if (before + here <= k + k / 4 + 32) break;
        // the ends of that bin, by its members
        const float high = block_reduce(in && bin == sh.bin ? own : -INFINITY, sh.fpart, Max{});
        if (high == bound) break;
        hi = high, lo = bound;
        __syncthreads();
    }
    return bound;
}

// The draw among the first n entries of the sorted list: in the order of the indices.
static __device__ __forceinline__ void draw_from_list(Shared &sh, const TokenSample &a, const Mass &mass, int r, float u, int n) {
    const int tid = (int)threadIdx.x;
    __syncthreads();
    if (n <= kWave) {   // by one wave
        if (tid >= kWave) return;
        unsigned long long x = tid < n ? sh.list[tid] : 0;
        x = x << 32 | x >> 32;   // ~index, key
        sort_lanes<64>(x, true);
        const double w = tid < n ? mass.w(value_of((uint32_t)x)) : 0.0;
        const double total = wave_reduce(w, Add{});
        double before;
        bool passed;
        const int at = pick_lane(w, (double)u * total, 0.0, before, passed);
        if (tid == at) a.token[r] = (int)~(uint32_t)(x >> 32), a.logprob[r] = (float)log(w / total);
        return;
    }
#pragma unroll
    for (int e = 0; e < kList; e += kBlock) {
        const unsigned long long x = sh.list[e + tid];
        if (e + tid < n) sh.list[e + tid] = x << 32 | x >> 32;
    }
    __syncthreads();
    sort_list(sh, n);
    double w[kEach], sum = 0.0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int i = kEach * tid + e;
        w[e] = i < n ? mass.w(value_of((uint32_t)sh.list[i])) : 0.0;
        sum += w[e];
    }
    const double upto = block_scan(sum, sh.sum);
    if (tid == kBlock - 1) sh.total = upto;
    if (tid == 0) sh.pick = kList, sh.count = 0;
    __syncthreads();
    const double total = sh.total, goal = (double)u * total;
    int hit = kList, last = 0;
    double run = upto - sum;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        run += w[e];
        if (w[e] > 0.0) {
            last = kEach * tid + e;
            if (hit == kList && run > goal) hit = last;
        }
    }
    // one lane of a wave speaks for it
    const int first = wave_reduce(hit, Min{}), end = -wave_reduce(-last, Min{});
    if ((tid & 63) == 0) atomicMin(&sh.pick, first), atomicMax(&sh.count, end);
    __syncthreads();
    const int at = sh.pick < kList ? sh.pick : sh.count;   // the last one where no sum exceeds u's share
    if (tid == 0) {
        const unsigned long long x = sh.list[at];
        a.token[r] = (int)~(uint32_t)(x >> 32);
        a.logprob[r] = (float)log(mass.w(value_of((uint32_t)x)) / total);
    }
}

// Top-k (k <= kTopK), from a list of n <= kList logits, not sorted yet, that has the
// k largest of the row: the rest of the filters, and the draw.
static __device__ __forceinline__ void draw_top_k(Shared &sh, const TokenSample &a, const Setting &st, const Mass &mass,
                                           const Cut &cut_m, int r, int n) {
    const int tid = (int)threadIdx.x;
    sort_list(sh, n);
    const int kept = n < st.k ? n : st.k;   // fewer than k logits are finite
    int left = 0;
    if (st.cuts_p()) {
        double w[kEach], before[kEach], sum = 0.0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int i = kEach * tid + e;
            w[e] = i < kept ? mass.w(list_value(sh, i)) : 0.0;
            before[e] = sum;
            sum += w[e];
        }
        const double upto = block_scan(sum, sh.sum);
        if (tid == kBlock - 1) sh.total = upto;
        __syncthreads();
        const double goal = st.share() * sh.total;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int i = kEach * tid + e;
            left += i < kept && (i == 0 || upto - sum + before[e] < goal) && list_value(sh, i) >= cut_m.x;
        }
        left = block_reduce(left, sh.ints, Add{});
    } else if (cut_m.x > -INFINITY) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) left += kEach * tid + e < kept && list_value(sh, kEach * tid + e) >= cut_m.x;
        left = block_reduce(left, sh.ints, Add{});
    } else {
        left = kept;
    }
    draw_from_list(sh, a, mass, r, st.u, left);
}

// Adds the weights of what `cut` keeps of `row` to the bins; this thread's sum of all.
template <typename R>
static __device__ __forceinline__ double fill_bins(Shared &sh, const R &row, const Cut &cut, const Mass &mass, const Bins &bins) {
    clear_bins(sh);
    for (int b = (int)threadIdx.x; b < kBins; b += kBlock) sh.hits[b] = 0;
    __syncthreads();
    double all = 0.0;
    row.each4([&](const f32x4_t &q, int i) {
        double w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = cut.keeps(q[e], i + e) ? mass.w(q[e]) : 0.0;   // no branch: four at once
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            all += w[e];
            const float b = bins.of(q[e]);
            if (b < kBins && w[e] > 0.0) {
                atomicAdd(&sh.hist[(int)b], mass.whole_of(w[e]));
                atomicAdd(&sh.hits[(int)b], 1u);
            }
        }
    });
    __syncthreads();
    return all;
}

// Where the mass of filled bins reaches p: the bin (-1: in none), the mass before it,
// and which logits go to the list: all down to the bin, or, if these are too many,
// the bin's (collects: those of bins [from, bin]).
struct Nucleus {
    unsigned long long target, above;
    int bin;
    bool whole, fits;   // the list has all of it; the list has room
    float from;
    __device__ __forceinline__ Nucleus(Shared &sh, const Setting &st, const Mass &mass, double all) {
        const int tid = (int)threadIdx.x;
        const double t = ceil(st.share() * all * mass.unit);
        target = t < 1.0 ? 1ull : (unsigned long long)t;
        find_bin<false>(sh, kBins, 0, target);
        bin = sh.bin;
        above = sh.above;
        int upto = 0;
#pragma unroll
        for (int b = 0; b < kBins; b += kBlock) upto += b + tid <= bin ? (int)sh.hits[b + tid] : 0;
        upto = block_reduce(upto, sh.ints, Add{});
        whole = upto <= kList;
        fits = bin >= 0 && (whole || sh.hits[bin < 0 ? 0 : bin] <= kList);
        from = whole ? 0.f : (float)bin;
    }
    __device__ __forceinline__ bool collects(const Bins &bins, float x) const {
        const float b = bins.of(x);
        return b >= from && b < (float)(bin + 1);
    }
};

// Top-p from the list of n logits that the nucleus collects: the draw (true), or the cut.
static __device__ __forceinline__ bool draw_top_p(Shared &sh, const TokenSample &a, const Setting &st, const Mass &mass,
                                           const Cut &cut_m, const Nucleus &nu, int r, int n, Cut &cut) {
    const int tid = (int)threadIdx.x;
    sort_list(sh, n);
    unsigned long long w[kEach], sum = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        w[e] = kEach * tid + e < n ? mass.whole(list_value(sh, kEach * tid + e)) : 0;
        sum += w[e];
    }
    unsigned long long run = (nu.whole ? 0 : nu.above) + block_scan(sum, sh.part) - sum;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (run < nu.target && nu.target <= run + w[e]) sh.pick = kEach * tid + e;
        run += w[e];
    }
    __syncthreads();
    if (nu.whole) {
        const int upto = sh.pick + 1;
        int left = upto;
        if (cut_m.x > -INFINITY) {
            left = 0;
#pragma unroll
            for (int e = 0; e < kEach; ++e) left += kEach * tid + e < upto && list_value(sh, kEach * tid + e) >= cut_m.x;
            left = block_reduce(left, sh.ints, Add{});
        }
        draw_from_list(sh, a, mass, r, st.u, left);
        return true;
    }
    const unsigned long long at = sh.list[sh.pick];
    cut = Cut{value_of((uint32_t)(at >> 32)), (int)~(uint32_t)at};
    return false;
}

// The sum of the weights of what `cut` keeps: this thread's part.
template <typename R>
static __device__ __forceinline__ double kept_mass(const R &row, const Cut &cut, const Mass &mass) {
    double mine = 0.0;
    row.each4([&](const f32x4_t &q, int i) {
        bool kept[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) kept[e] = cut.keeps(q[e], i + e);
        if (!__any(kept[0] || kept[1] || kept[2] || kept[3])) return;
        double w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = mass.w(q[e]);
#pragma unroll
        for (int e = 0; e < 4; ++e) mine += kept[e] ? w[e] : 0.0;
    });
    return mine;
}

// The draw in the part [begin, end) of the row: kept weights before it `before`, of
// all `total`.  A sum per wave and load, all of which every wave has in its lanes.
template <typename R>
static __device__ __forceinline__ void draw_from_part(Shared &sh, const TokenSample &a, const R &row, const Cut &cut,
                                               const Mass &mass, int r, float u, int begin, int end, double before,
                                               double total) {
    constexpr int kLoads = 4;
    static_assert(kLoads * kWaves <= kWave, "a sum a lane");
    const int tid = (int)threadIdx.x, lane = tid & 63, wv = tid / kWave;
    const double goal = (double)u * total;
    double *sums = reinterpret_cast<double *>(sh.hist);
    int at = -1;          // the last kept token so far
    double w_at = 0.0;
    for (int i0 = begin; i0 < end; i0 += kLoads * 4 * kBlock) {
        f32x4_t q[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int i = i0 + 4 * (j * kBlock + tid);
            q[j] = row.load(i < end ? i : row.V);
        }
        double w[kLoads][4], mine[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int i = i0 + 4 * (j * kBlock + tid);
#pragma unroll
            for (int e = 0; e < 4; ++e) w[j][e] = i + e < end && cut.keeps(q[j][e], i + e) ? mass.w(q[j][e]) : 0.0;
            mine[j] = (w[j][0] + w[j][1]) + (w[j][2] + w[j][3]);
            const double sum = wave_reduce(mine[j], Add{});
            if (lane == 0) sums[j * kWaves + wv] = sum;
        }
        __syncthreads();
        double base, from;
        bool passed, in_lane;
        const double sum = lane < kLoads * kWaves ? sums[lane] : 0.0;   // in the order of the indices: by load, then wave
        const int part = pick_lane(sum, goal, before, base, passed);
        before += __shfl(wave_scan(sum), 63);
        __syncthreads();
        if (part >= 0 && part % kWaves == wv) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
                if (part / kWaves == j) {
                    const int l = pick_lane(mine[j], goal, base, from, in_lane);
                    // the lane's four: the first whose sum exceeds goal, or its last
                    double x = from;
                    int hit = -1, last = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x += w[j][e];
                        if (w[j][e] > 0.0) {
                            last = e;
                            if (hit < 0 && x > goal) hit = e;
                        }
                    }
                    const int e = hit < 0 ? last : hit;
                    at = __shfl(i0 + 4 * (j * kBlock + tid) + e, l & 63);
                    w_at = __shfl(e == 0 ? w[j][0] : e == 1 ? w[j][1] : e == 2 ? w[j][2] : w[j][3], l & 63);
                }
            if (lane == 0) sh.pick = at, sh.total = w_at;
        }
        __syncthreads();
        if (part >= 0) at = sh.pick, w_at = sh.total;
        if (passed) break;
    }
    if (tid == 0) a.token[r] = at, a.logprob[r] = (float)log(w_at / total);
}

template <typename T>
static __device__ __forceinline__ void sample_row(Shared &sh, const TokenSample &a, int r) {
    const int tid = (int)threadIdx.x, V = a.V;
    const Setting st(a, r);
    const Row<T> row(static_cast<const T *>(a.logits) + (size_t)r * a.ld, V);

    float own = -INFINITY;
    bool bad = false;
    row.template each<8>([&](float x, int) {
        own = fmaxf(own, x);
        bad |= !(x < INFINITY);
    });
    // a NaN or +inf logit goes through the maximum as +inf
    const float top = block_reduce(bad ? INFINITY : own, sh.fpart, Max{});
    if (!(fabsf(top) < INFINITY) || !(st.temp >= 0.f)) return no_distribution(a, r);
    if (st.temp == 0.f) {
        int at = V;
        if (own == top) row.each([&](float x, int i) { at = x == top && i < at ? i : at; });
        at = block_reduce(at, sh.ints, Min{});
        if (tid == 0) a.token[r] = at, a.logprob[r] = 0.f;
        return;
    }
    const Mass mass(top, st.temp, V);
    const Cut cut_m = cut_of_m(st, mass, top, V);

    Cut cut{-INFINITY, -1};   // every finite logit
    if (st.cuts_k(V)) {
        if (st.k <= kTopK) {
            const float bound = bound_of(sh, own, top, st.k);
            const int n = collect(sh, row, [&](float x, int) { return x > -INFINITY && x >= bound; });
            if (n <= kList) return draw_top_k(sh, a, st, mass, cut_m, r, n);
        }
        int live = 0;
        row.each([&](float x, int) { live += x > -INFINITY; });
        live = block_reduce(live, sh.ints, Add{});
        if (st.k < live) cut = find_cut(sh, row, cut, (unsigned long long)st.k, [](float) { return 1ull; });
    }
    if (st.cuts_p()) {
        const Bins bins(st, mass, top, V);
        const double all = block_reduce(fill_bins(sh, row, cut, mass, bins), sh.sum, Add{});
        const Nucleus nu(sh, st, mass, all);
        int n = kList + 1;
        if (nu.fits) n = collect(sh, row, [&](float x, int i) { return cut.keeps(x, i) && nu.collects(bins, x); });
        if (n <= kList) {
            if (draw_top_p(sh, a, st, mass, cut_m, nu, r, n, cut)) return;
        } else {   // more of one value, or nearly, than the list takes
            unsigned long long whole = 0;
            row.each([&](float x, int i) { whole += cut.keeps(x, i) ? mass.whole(x) : 0ull; });
            whole = block_reduce(whole, sh.part, Add{});
            cut = find_cut(sh, row, cut, nu.target < whole ? nu.target : whole, [&](float x) { return mass.whole(x); });
        }
    }
    if (cut_m.x > cut.x) cut = cut_m;
    // the wave that has the token, then the part of its part
    const double sum = wave_reduce(kept_mass(row, cut, mass), Add{});
    __syncthreads();
    if ((tid & 63) == 0) sh.sum[tid / kWave] = sum;
    __syncthreads();
    const double part = (tid & 63) < kWaves ? sh.sum[tid & 63] : 0.0, total = wave_reduce(part, Add{});
    double before;
    bool passed;
    const int wave = pick_lane(part, (double)st.u * total, 0.0, before, passed);
    const int span = Row<T>::span_of(V), begin = wave * span;
    draw_from_part(sh, a, row, cut, mass, r, st.u, begin, V - begin < span ? V : begin + span, before, total);
}

};   // Block

template <typename T>
__global__ __launch_bounds__(Block<16>::kBlock, 4) void token_sample_kernel(TokenSample a)
{
    __shared__ Block<16>::Shared sh;
    Block<16>::sample_row<T>(sh, a, blockIdx.x);
}

// ---- rows in slices -------------------------------------------------------------

using B = Block<4>;
constexpr int kCus = 256;
// Slices pay for four more launches and for what they hand each other.  Rows of
// 131072, one / 32 / 128 of them, in slices and by one workgroup each (us): top-p 33,
// 64, 173 and 101, 102, 113; no filter 18, 19, 30 and 34, 36, 45.  Rows of 10000: 32, 51,
// 55 and 22, 29, 30 with top-p.
constexpr int kSliceRows = 32;
constexpr int kSliceFrom = 32768;
// Top-k: the slices' candidates grow with k, and a workgroup's time for a row does not.
// One row of 131072 with k = 8, 48, 64, 192 in slices 15, 23, 27, 77 us; left to a workgroup
// behind the slices' launches 20, 21, 23, 29; by one at once 16, 17, 18, 25.  (50264: 14, 17, 19,
// 43; 17, 17, 17, 24; 12, 13, 13, 20.  2^20: 27, 94, 124, 516; 96, 98, 99, 105; 93, 93, 95, 102.)
// The settings are on the device: there, rows of k above kSliceTopK are left out of the
// slices.  The host knows which are not given: with top-k and no top-p, rows of up to
// kSliceFromTopK logits go by a workgroup at once.
constexpr int kSliceTopK = 48;
constexpr int kSliceFromTopK = 131072;
constexpr int kLoads = 4;                              // loads of four logits a thread
constexpr int kSlice = 4 * kLoads * B::kBlock;         // logits of a slice: 4096
constexpr int kSlices = 1024;                          // of a row at most
// Of a slice, for top-k: kSliceTopK and the equal or nearly equal logits that come with
// them; more give the row up.  (Room for 1024 took 4 times the workspace, 268 MB for 32 rows of
// 2^22 logits, and the same time.)
constexpr int kCandidates = 256;

struct SliceRecord {
    float top;      // largest logit; +inf: there is a NaN or +inf
    int at;         // greedy: its index
    int count;      // top-k: candidates
    int unused;
    double mass;    // sum of the weights (what is said where it is written)
};
enum RowKind { kDone = 0, kTopP, kCutKnown, kCutLate, kGivenUp };
struct RowState {
    int kind, late;    // by merge_kernel for gather_kernel, and by that for rest_kernel
    int count;         // entries of the list
    float cut_x;
    int cut_last;
};

struct Slices {
    Div by_r;   // workgroup s * R + r: where one slice of a row works on, the rows' are on all XCDs
    int S;                          // slices of a row
    unsigned *arrived;              // [kSliceRows], zero between calls
    RowState *state;                // [R]
    SliceRecord *record;            // [R, S]
    unsigned long long *hist;       // [R, kBins] top-p's bins
    uint32_t *hits;
    unsigned long long *list;       // [R, B::kList]
    unsigned long long *candidate;  // [R, S, kCandidates]
};

// The LDS of a workgroup that sorts nothing: more of them fit a CU.
struct SmallShared {
    static constexpr int kRoom = kCandidates;
    unsigned long long hist[B::kBlock], list[kRoom];
    unsigned long long above;
    double sum[4];
    float fpart[4];
    int ints[4];
    int bin, count;
};
struct RowShared : B::Shared {
    unsigned short rows[kSliceRows];
};

// Over a row's records, 64 at a time, by every wave for itself (no exchange between
// waves): the largest logit; the sum of the masses.
__device__ __forceinline__ float top_of(const SliceRecord *rec, int S) {
    float top = -INFINITY;
    for (int s = (int)threadIdx.x & 63; s < S; s += kWave) top = fmaxf(top, rec[s].top);
    return wave_reduce(top, Max{});
}
template <typename F>
__device__ __forceinline__ double sum_of(int S, F mass_of_slice) {
    double sum = 0.0;
    for (int s = (int)threadIdx.x & 63; s < S; s += kWave) sum += mass_of_slice(s);
    return wave_reduce(sum, Add{});
}
// The slice that has the draw, and the sum before it.
template <typename F>
__device__ __forceinline__ int pick_slice(int S, double goal, F mass_of_slice, double &before) {
    int at = 0;
    double run = 0.0;
    for (int s0 = 0; s0 < S; s0 += kWave) {
        const int s = s0 + ((int)threadIdx.x & 63);
        const double sum = s < S ? mass_of_slice(s) : 0.0;
        double b;
        bool passed;
        const int l = pick_lane(sum, goal, run, b, passed);
        if (l >= 0) at = s0 + l, before = b;
        if (passed) break;
        run += __shfl(wave_scan(sum), 63);
    }
    return at;
}

// A slice in registers: load j of thread t has logits begin + 4 (j * kBlock + t) on.
template <typename T>
struct Slice {
    const T *x;
    int V, begin;
    f32x4_t v[kLoads];
    __device__ __forceinline__ f32x4_t load(int i) const {   // logits i .. i + 3, -inf past the end
        using Four = typename B::Row<T>::Four;
        if (i + 4 <= V) return B::Row<T>::wide(*reinterpret_cast<const Four *>(x + i));
        f32x4_t r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = i + e < V ? widen(x[i + e]) : -INFINITY;
        return r;
    }
    __device__ __forceinline__ Slice(const T *p, int V_, int s) : x(p), V(V_), begin(s * kSlice) {
        using Four = typename B::Row<T>::Four;
        const int at = begin + 4 * (int)threadIdx.x;
        if (V - begin >= kSlice) {   // all of it: loads outside of branches
            Four f[kLoads];
#pragma unroll
            for (int j = 0; j < kLoads; ++j) f[j] = *reinterpret_cast<const Four *>(x + at + j * 4 * B::kBlock);
#pragma unroll
            for (int j = 0; j < kLoads; ++j) v[j] = B::Row<T>::wide(f[j]);
        } else {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) v[j] = load(at + j * 4 * B::kBlock);
        }
    }
    template <typename F>
    __device__ __forceinline__ void each4(F f) const {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) f(v[j], begin + 4 * (j * B::kBlock + (int)threadIdx.x));
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        each4([&](const f32x4_t &q, int i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) f(q[e], i + e);
        });
    }
};
template <typename T>
__device__ __forceinline__ const T *logits_of(const TokenSample &a, int r) {
    return static_cast<const T *>(a.logits) + (size_t)r * a.ld;
}

// What the slices of a row leave for its last one goes past the caches (the eight
// L2s do not keep each other's lines).
template <typename V>
__device__ __forceinline__ void put(V *p, V x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename V>
__device__ __forceinline__ V get(const V *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Whether this is the last of the row's slices to arrive, with what all of them have
// put before.
__device__ __forceinline__ bool last_slice(RowShared &sh, const Slices &z, int r) {
    __builtin_amdgcn_s_waitcnt(0);   // this thread's stores have arrived, then everybody's
    __syncthreads();
    if (threadIdx.x == 0) {
        const unsigned n = __hip_atomic_fetch_add(z.arrived + r, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sh.pick = n == (unsigned)z.S - 1;
        if (sh.pick) put(z.arrived + r, 0u);
    }
    __syncthreads();
    const bool last = sh.pick != 0;
    __syncthreads();
    return last;
}

template <typename T>
__global__ __launch_bounds__(B::kBlock, 8) void slice_kernel(TokenSample a, Slices z)
{
    __shared__ SmallShared sh;
    const int s = (int)z.by_r(blockIdx.x), r = (int)blockIdx.x - s * a.R, tid = (int)threadIdx.x, V = a.V;
    const Setting st(a, r);
    if (st.cuts_k(V) && st.k > kSliceTopK && st.temp != 0.f) {   // sample_row's
        if (tid == 0 && s == 0) z.state[r] = RowState{kGivenUp, kDone, 0, 0.f, 0};
        return;
    }
    const Slice<T> row(logits_of<T>(a, r), V, s);
    float own = -INFINITY;
    bool bad = false;
    row.each([&](float x, int) {
        own = fmaxf(own, x);
        bad |= !(x < INFINITY);
    });
    SliceRecord rec{-INFINITY, V, 0, 0, 0.0};
    if (st.temp > 0.f && !st.cuts_k(V) && !st.cuts_p() && !st.cuts_m()) {
        // no filter: the sum of the weights, by every wave of its largest logit's
        const float wave_top = wave_reduce(bad ? INFINITY : own, Max{});
        double sum = 0.0;
        if (fabsf(wave_top) < INFINITY) {
            const Mass mass(wave_top, st.temp, V);
            row.each4([&](const f32x4_t &q, int) {
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += mass.w(q[e]);
            });
            sum = wave_reduce(sum, Add{});
        }
        if ((tid & 63) == 0) sh.fpart[tid / kWave] = wave_top, sh.sum[tid / kWave] = sum;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < B::kBlock / kWave; ++w) rec.top = fmaxf(rec.top, sh.fpart[w]);
        if (tid == 0 && fabsf(rec.top) < INFINITY) {
            const Mass mass(rec.top, st.temp, V);
#pragma unroll
            for (int w = 0; w < B::kBlock / kWave; ++w) rec.mass += sh.sum[w] > 0.0 ? sh.sum[w] * mass.w(sh.fpart[w]) : 0.0;
        }
    } else {
        rec.top = B::block_reduce(bad ? INFINITY : own, sh.fpart, Max{});
        if (!(fabsf(rec.top) < INFINITY)) {
            // nothing of it is drawn, or nothing of the row
        } else if (st.temp == 0.f) {
            int at = V;
            row.each([&](float x, int i) { at = x == rec.top && i < at ? i : at; });
            rec.at = B::block_reduce(at, sh.ints, Min{});
        } else if (st.cuts_k(V)) {
            const float bound = B::bound_of(sh, own, rec.top, st.k);
            rec.count = B::collect(sh, row, [&](float x, int) { return x > -INFINITY && x >= bound; });
            unsigned long long *to = z.candidate + ((size_t)r * z.S + s) * kCandidates;
            for (int i = tid; i < rec.count && i < kCandidates; i += B::kBlock) to[i] = sh.list[i];
        }
        if (st.cuts_p() && !st.cuts_k(V))   // for the next kernel
            for (int b = s * B::kBlock + tid; b < kBins; b += z.S * B::kBlock)
                z.hist[(size_t)r * kBins + b] = 0, z.hits[(size_t)r * kBins + b] = 0;
    }
    if (tid == 0) {
        z.record[(size_t)r * z.S + s] = rec;
        if (s == 0) z.state[r] = RowState{kDone, kDone, 0, 0.f, 0};
    }
}

// The rows for which is(r), in sh.rows; their number.  What is left to do is a matter
// of the settings, which are on the device alone: a workgroup for each slice that may
// have something to do would take longer to start than most have to do.
template <typename F>
__device__ __forceinline__ int rows_where(RowShared &sh, int R, F is) {
    const int tid = (int)threadIdx.x, wv = tid / kWave;
    int n = 0;
    for (int r0 = 0; r0 < R; r0 += B::kBlock) {
        const bool in = r0 + tid < R && is(r0 + tid);
        const unsigned long long all = __ballot(in);
        __syncthreads();
        if ((tid & 63) == 0) sh.ints[wv] = __popcll(all);
        __syncthreads();
        int before = n;
#pragma unroll
        for (int w = 0; w < B::kBlock / kWave; ++w) {
            const int y = sh.ints[w];
            before += w < wv ? y : 0;
            n += y;
        }
        if (in) sh.rows[before + __popcll(all & ((1ull << (tid & 63)) - 1))] = (unsigned short)(r0 + tid);
    }
    __syncthreads();
    return n;
}

// Top-p's bins of one slice, into the row's.
template <typename T>
__device__ __forceinline__ void bins_of_slice(RowShared &sh, const TokenSample &a, const Slices &z, int r, int s) {
    const int tid = (int)threadIdx.x, V = a.V;
    const Slice<T> row(logits_of<T>(a, r), V, s);
    const Setting st(a, r);
    const float top = top_of(z.record + (size_t)r * z.S, z.S);
    if (!(fabsf(top) < INFINITY)) return;
    const Mass mass(top, st.temp, V);
    const Bins bins(st, mass, top, V);
    const double sum = B::block_reduce(B::fill_bins(sh, row, Cut{-INFINITY, -1}, mass, bins), sh.sum, Add{});
    for (int b = tid; b < kBins; b += B::kBlock) {
        const uint32_t n = sh.hits[b];
        if (n) {
            atomicAdd(z.hist + (size_t)r * kBins + b, sh.hist[b]);
            atomicAdd(z.hits + (size_t)r * kBins + b, n);
        }
    }
    if (tid == 0) {
        z.record[(size_t)r * z.S + s].mass = sum;
        if (s == 0) z.state[r] = RowState{kTopP, kDone, 0, 0.f, 0};
    }
}

// Top-k from the slices' candidates, which have the row's k largest logits.
__device__ __forceinline__ void merge_top_k(RowShared &sh, const TokenSample &a, const Slices &z, const Setting &st,
                                            const Mass &mass, float top, int r) {
    constexpr int kMine = kSlices / B::kBlock;
    const int tid = (int)threadIdx.x;
    int *start = reinterpret_cast<int *>(sh.hits);   // of the slices, among all candidates
    int count[kMine], sum = 0;
    bool given_up = false;
#pragma unroll
    for (int e = 0; e < kMine; ++e) {
        const int s = kMine * tid + e;
        count[e] = s < z.S ? z.record[(size_t)r * z.S + s].count : 0;
        given_up |= count[e] > kCandidates;
        sum += count[e];
    }
    int at = B::block_scan(sum, sh.ints) - sum;
#pragma unroll
    for (int e = 0; e < kMine; ++e) start[kMine * tid + e] = at, at += count[e];
    if (tid == B::kBlock - 1) sh.count = at;
    given_up = __syncthreads_or(given_up);
    const int total = sh.count;
    auto candidate = [&](int i) {   // its slice is the last that starts at or before it
        int at = 0;
        for (int step = kSlices / 2; step > 0; step /= 2)
            if (at + step < z.S && start[at + step] <= i) at += step;
        return z.candidate[((size_t)r * z.S + at) * kCandidates + (i - start[at])];
    };
    auto value = [](unsigned long long c) { return value_of((uint32_t)(c >> 32)); };
    int n = given_up ? B::kList + 1 : total;
    // the k-th largest of the threads' maxima bounds them once more: a shorter list to sort
    if (!given_up && total > 2 * kWave && total > 2 * st.k) {
        float own = -INFINITY;
        for (int i = tid; i < total; i += B::kBlock) own = fmaxf(own, value(candidate(i)));
        const float bound = B::bound_of(sh, own, top, st.k);
        __syncthreads();
        if (tid == 0) sh.count = 0;
        __syncthreads();
        for (int i = tid; i < total; i += B::kBlock) {
            const unsigned long long c = candidate(i);
            if (value(c) < bound) continue;
            const int at = atomicAdd(&sh.count, 1);
            if (at < B::kList) sh.list[at] = c;
        }
        __syncthreads();
        n = sh.count;
    } else if (!given_up) {
        for (int i = tid; i < total; i += B::kBlock) sh.list[i] = candidate(i);
    }
    if (n > B::kList) {
        if (tid == 0) z.state[r].kind = kGivenUp;
        return;
    }
    __syncthreads();
    B::draw_top_k(sh, a, st, mass, cut_of_m(st, mass, top, a.V), r, n);
}

// The draw of a row whose slices' kept weights are known.
template <typename T, typename F>
__device__ __forceinline__ void draw_by_masses(RowShared &sh, const TokenSample &a, const Slices &z, const Setting &st,
                                               const Mass &mass, const Cut &cut, int r, F mass_of_slice) {
    const double total = sum_of(z.S, mass_of_slice);
    double before = 0.0;
    const int begin = pick_slice(z.S, (double)st.u * total, mass_of_slice, before) * kSlice;
    B::draw_from_part(sh, a, B::Row<T>(logits_of<T>(a, r), a.V), cut, mass, r, st.u, begin,
                      a.V - begin < kSlice ? a.V : begin + kSlice, before, total);
}

// Workgroup r < R: row r; those behind: slices of the rows that need bins.
template <typename T>
__global__ __launch_bounds__(B::kBlock, 4) void merge_kernel(TokenSample a, Slices z)
{
    __shared__ RowShared sh;
    const int tid = (int)threadIdx.x, V = a.V;
    if ((int)blockIdx.x >= a.R) {
        const int n = rows_where(sh, a.R, [&](int i) {
            const Setting st(a, i);
            return st.cuts_p() && !st.cuts_k(V) && st.temp > 0.f;
        });
        for (int t = (int)blockIdx.x - a.R; t < n * z.S; t += (int)gridDim.x - a.R) {
            bins_of_slice<T>(sh, a, z, sh.rows[t % n], t / n);
            __syncthreads();
        }
        return;
    }
    const int r = (int)blockIdx.x;
    const Setting st(a, r);
    if (z.state[r].kind == kGivenUp) return;
    const SliceRecord *rec = z.record + (size_t)r * z.S;
    const float top = top_of(rec, z.S);
    if (!(fabsf(top) < INFINITY) || !(st.temp >= 0.f)) return no_distribution(a, r);
    if (st.temp == 0.f) {
        int at = V;
        for (int i = tid & 63; i < z.S; i += kWave) at = rec[i].top == top && rec[i].at < at ? rec[i].at : at;
        at = wave_reduce(at, Min{});
        if (tid == 0) a.token[r] = at, a.logprob[r] = 0.f;
        return;
    }
    const Mass mass(top, st.temp, V);
    if (st.cuts_k(V)) return merge_top_k(sh, a, z, st, mass, top, r);
    if (st.cuts_p()) return;   // the workgroups behind
    if (st.cuts_m()) {         // min-p alone
        const Cut cut = cut_of_m(st, mass, top, V);
        if (tid == 0) z.state[r] = RowState{kCutKnown, kDone, 0, cut.x, cut.last};
        return;
    }
    draw_by_masses<T>(sh, a, z, st, mass, Cut{-INFINITY, -1}, r,
                      [&](int i) { return rec[i].top > -INFINITY ? rec[i].mass * mass.w(rec[i].top) : 0.0; });
}

// The sums of what `cut` keeps of each slice, and the draw by the last slice.
template <typename T>
__device__ __forceinline__ void draw_by_slices(RowShared &sh, const TokenSample &a, const Slices &z, const Setting &st,
                                               const Mass &mass, const Cut &cut, int r, int s) {
    const Slice<T> row(logits_of<T>(a, r), a.V, s);
    const double sum = B::block_reduce(B::kept_mass(row, cut, mass), sh.sum, Add{});
    SliceRecord *rec = z.record + (size_t)r * z.S;
    if (threadIdx.x == 0)
        put(reinterpret_cast<unsigned long long *>(&rec[s].mass), __builtin_bit_cast(unsigned long long, sum));
    if (!last_slice(sh, z, r)) return;
    draw_by_masses<T>(sh, a, z, st, mass, cut, r, [&](int i) {
        return __builtin_bit_cast(double, get(reinterpret_cast<unsigned long long *>(&rec[i].mass)));
    });
}

template <typename T>
__device__ __forceinline__ void gather_slice(RowShared &sh, const TokenSample &a, const Slices &z, int r, int s) {
    const int tid = (int)threadIdx.x, V = a.V;
    const Setting st(a, r);
    const SliceRecord *rec = z.record + (size_t)r * z.S;
    const float top = top_of(rec, z.S);
    const Mass mass(top, st.temp, V);
    if (z.state[r].kind == kCutKnown)
        return draw_by_slices<T>(sh, a, z, st, mass, Cut{z.state[r].cut_x, z.state[r].cut_last}, r, s);

    const Slice<T> row(logits_of<T>(a, r), V, s);
    const double all = sum_of(z.S, [&](int i) { return rec[i].mass; });
#pragma unroll
    for (int b = 0; b < kBins; b += B::kBlock) {
        sh.hist[b + tid] = z.hist[(size_t)r * kBins + b + tid];
        sh.hits[b + tid] = z.hits[(size_t)r * kBins + b + tid];
    }
    __syncthreads();
    const B::Nucleus nu(sh, st, mass, all);
    if (!nu.fits) {
        if (s == 0 && tid == 0) z.state[r].late = kGivenUp;
        return;
    }
    const Bins bins(st, mass, top, V);
    const int mine = B::collect(sh, row, [&](float x, int) { return x > -INFINITY && nu.collects(bins, x); });
    if (tid == 0) sh.bin = mine ? __hip_atomic_fetch_add(&z.state[r].count, mine, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
    __syncthreads();
    const int base = sh.bin;
    unsigned long long *list = z.list + (size_t)r * B::kList;
    for (int i = tid; i < mine && base + i < B::kList; i += B::kBlock) put(list + base + i, sh.list[i]);
    if (!last_slice(sh, z, r)) return;
    const int n = min(get(&z.state[r].count), B::kList);
    for (int i = tid; i < n; i += B::kBlock) sh.list[i] = get(list + i);
    __syncthreads();
    Cut cut{-INFINITY, -1};
    const Cut cut_m = cut_of_m(st, mass, top, V);
    const bool done = B::draw_top_p(sh, a, st, mass, cut_m, nu, r, n, cut);
    if (tid == 0 && !done) {
        if (cut_m.x > cut.x) cut = cut_m;
        z.state[r].late = kCutLate, z.state[r].cut_x = cut.x, z.state[r].cut_last = cut.last;
    }
}

template <typename T>
__global__ __launch_bounds__(B::kBlock, 4) void gather_kernel(TokenSample a, Slices z)
{
    __shared__ RowShared sh;
    const int n = rows_where(sh, a.R, [&](int i) { return z.state[i].kind == kTopP || z.state[i].kind == kCutKnown; });
    for (int t = (int)blockIdx.x; t < n * z.S; t += (int)gridDim.x) {
        gather_slice<T>(sh, a, z, sh.rows[t % n], t / n);
        __syncthreads();
    }
}

// The slices of rows whose cut came late.
template <typename T>
__global__ __launch_bounds__(B::kBlock, 4) void rest_kernel(TokenSample a, Slices z)
{
    __shared__ RowShared sh;
    const int n = rows_where(sh, a.R, [&](int i) { return z.state[i].late == kCutLate; });
    for (int t = (int)blockIdx.x; t < n * z.S; t += (int)gridDim.x) {
        const int r = sh.rows[t % n];
        const Setting st(a, r);
        const float top = top_of(z.record + (size_t)r * z.S, z.S);
        draw_by_slices<T>(sh, a, z, st, Mass(top, st.temp, a.V), Cut{z.state[r].cut_x, z.state[r].cut_last}, r, t / n);
        __syncthreads();
    }
}
template <typename T>
__global__ __launch_bounds__(Block<16>::kBlock, 4) void given_up_kernel(TokenSample a, Slices z)
{
    __shared__ Block<16>::Shared sh;
    const RowState state = z.state[blockIdx.x];
    if (state.kind == kGivenUp || state.late == kGivenUp) Block<16>::sample_row<T>(sh, a, blockIdx.x);
}

// Sizes and places of the slices' workspace; S == 0: sample_row.
struct Layout {
    int S;
    size_t state, record, hist, hits, list, candidate, bytes;
};
Layout layout_of(int R, int V) {
    Layout y{};
    y.bytes = 16;
    if (R > kSliceRows || V <= kSliceFrom || V > kSlice * kSlices) return y;
    y.S = (V + kSlice - 1) / kSlice;
    size_t at = kSliceRows * sizeof(unsigned);   // arrivals: where every call has them
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += (bytes + 15) / 16 * 16;
        return p;
    };
    y.state = take((size_t)R * sizeof(RowState));
    y.record = take((size_t)R * y.S * sizeof(SliceRecord));
    y.hist = take((size_t)R * kBins * 8);
    y.hits = take((size_t)R * kBins * 4);
    y.list = take((size_t)R * B::kList * 8);
    y.candidate = take((size_t)R * y.S * kCandidates * 8);
    y.bytes = at;
    return y;
}

template <typename T>
hipError_t launch_slices(const TokenSample &a, const Layout &y, hipStream_t stream) {
    Slices z{};
    z.by_r = make_div(a.R);
    z.S = y.S;
    z.arrived = reinterpret_cast<unsigned *>(a.workspace);
    z.state = reinterpret_cast<RowState *>(a.workspace + y.state);
    z.record = reinterpret_cast<SliceRecord *>(a.workspace + y.record);
    z.hist = reinterpret_cast<unsigned long long *>(a.workspace + y.hist);
    z.hits = reinterpret_cast<uint32_t *>(a.workspace + y.hits);
    z.list = reinterpret_cast<unsigned long long *>(a.workspace + y.list);
    z.candidate = reinterpret_cast<unsigned long long *>(a.workspace + y.candidate);
    const unsigned all = (unsigned)(a.R * y.S), some = all < 4 * kCus ? all : 4 * kCus;   // as many as fit the CUs at once
    const dim3 bd(B::kBlock);
    hipLaunchKernelGGL(slice_kernel<T>, dim3(all), bd, 0, stream, a, z);
    hipLaunchKernelGGL(merge_kernel<T>, dim3((unsigned)a.R + (a.top_p ? some : 0)), bd, 0, stream, a, z);
    if (a.top_p || a.min_p) hipLaunchKernelGGL(gather_kernel<T>, dim3(some), bd, 0, stream, a, z);
    if (a.top_p) hipLaunchKernelGGL(rest_kernel<T>, dim3(some), bd, 0, stream, a, z);
    if (a.top_p || a.top_k)
        hipLaunchKernelGGL(given_up_kernel<T>, dim3((unsigned)a.R), dim3(Block<16>::kBlock), 0, stream, a, z);
    return hipGetLastError();
}

}  // namespace

size_t token_sample_workspace_bytes(int R, int V, int) { return layout_of(R, V).bytes; }

hipError_t launch_token_sample(const TokenSample &a, bool bf16, hipStream_t stream)
{
    const Layout y = layout_of(a.R, a.V);
    const bool top_k = a.top_k && !a.top_p && a.V <= kSliceFromTopK;
    if (y.S && !top_k) return bf16 ? launch_slices<uint16_t>(a, y, stream) : launch_slices<float>(a, y, stream);
    const dim3 gd((unsigned)a.R), bd(Block<16>::kBlock);
    if (bf16) hipLaunchKernelGGL(token_sample_kernel<uint16_t>, gd, bd, 0, stream, a);
    else hipLaunchKernelGGL(token_sample_kernel<float>, gd, bd, 0, stream, a);
    return hipGetLastError();
}

}  // namespace fs
