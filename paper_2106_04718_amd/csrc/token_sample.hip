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
// vocabulary has many borders: with the weights in 32 bits one draw in some ten
// thousand would be another token's.  Weights and sums are 64-bit.
//
// One workgroup has a row and reads it two or three times, after the first time
// from the caches (held in registers, it needs unrolled passes, which run once a
// row: waiting for their instructions cost more than reading again).  No pass
// sorts or scans the row:
//   top-k      The k-th largest of the threads' 1024 maxima is a bound that at
//              least k logits reach, and few more do.  Those go to a list in LDS,
//              which is sorted; top-p, min-p and the draw happen in the list.
//   top-p      alone: one pass adds up all weights, and those that can matter
//              (together the others have less than half of 1 - p) by value, in
//              2048 bins.  The list has the logits down to the bin in which the
//              mass reaches p; the draw happens in it.  If they are too many, the
//              list has that bin alone, for the cut.
//   otherwise  (no cut, or the list's capacity exceeded, or k above kTopK) the cut
//              is found by digits of the logits' bits, and the draw by the waves'
//              sums and the part of the row of the wave that holds it.
#include <math.h>
#include <stdint.h>

#include "launch.h"

namespace fs {
namespace {

constexpr int kWave = 64;
constexpr int kWaves = 16;
constexpr int kBlock = kWave * kWaves;
constexpr int kBins = 2048;   // of a digit of 11 bits, and of top-p's weights
constexpr int kList = 2048;   // logits that are sorted in LDS
constexpr int kTopK = 768;    // the list then has some 1500 logits of a smooth distribution
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

// Reduction over the workgroup; part: kWaves words of LDS that nothing else uses meanwhile.
template <typename V, typename Op>
__device__ __forceinline__ V block_reduce(V x, V *part, Op op) {
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
__device__ __forceinline__ V block_scan(V x, V *part) {
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
    __device__ __forceinline__ double log2w(float x) const { return ((double)x - top) * c; }
    static __device__ __forceinline__ double exp2_of(double y) {
        y = fmax(y, -2000.0);   // 0 below; -inf and NaN (of -inf at T = inf) too
        constexpr double kRound = 6755399441055744.0;   // 1.5 * 2^52: its sum with y has y's whole part in its low bits
        const double z = y + kRound;
        const double f = y - (z - kRound);
        double q = 0x1.b63880a30e9ffp-24;
        q = fma(q, f, 0x1.63d136366db24p-20);
        q = fma(q, f, 0x1.ffcb9515a8016p-17);
        q = fma(q, f, 0x1.4308ac85aa947p-13);
        q = fma(q, f, 0x1.5d87fe86fe88ep-10);
        q = fma(q, f, 0x1.3b2ab7181b755p-7);
        q = fma(q, f, 0x1.c6b08d7047e52p-5);
        q = fma(q, f, 0x1.ebfbdff823cedp-3);
        q = fma(q, f, 0x1.62e42fefa39efp-1);
        return ldexp(fma(q, f, 1.0), (int)(uint32_t)__builtin_bit_cast(unsigned long long, z));
    }
    __device__ __forceinline__ double w(float x) const { return exp2_of(log2w(x)); }
    // as whole numbers, whose sums do not depend on the order of atomic additions
    __device__ __forceinline__ unsigned long long whole_of(double w) const { return (unsigned long long)(w * unit + 0.5); }
    __device__ __forceinline__ unsigned long long whole(float x) const { return whole_of(w(x)); }
};

struct Shared {
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
__device__ void find_bin(Shared &sh, int bins, unsigned long long above, unsigned long long target) {
    const int tid = (int)threadIdx.x;
    if (tid == 0) sh.bin = -1;
    const int b0 = 2 * tid, at0 = DOWN ? bins - 1 - b0 : b0, at1 = DOWN ? at0 - 1 : at0 + 1;
    const unsigned long long a = b0 < bins ? sh.hist[at0] : 0, b = b0 + 1 < bins ? sh.hist[at1] : 0;
    const unsigned long long p2 = above + block_scan(a + b, sh.part), p1 = p2 - b, p0 = p1 - a;
    if (p0 < target && target <= p1) sh.bin = at0, sh.above = p0;
    if (p1 < target && target <= p2) sh.bin = at1, sh.above = p1;
    __syncthreads();
}

__device__ __forceinline__ void clear_bins(Shared &sh) {
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kBins; b += kBlock) sh.hist[b + threadIdx.x] = 0;
    __syncthreads();
}

// The cut at which the sum of f over the logits that `from` keeps, in the order,
// first reaches `target` (1 <= target <= the sum), by digits of the key, the
// highest first.  f: 1 (counts) or the weight (equal logits have one f).
template <typename R, typename F>
__device__ __forceinline__ Cut find_cut(Shared &sh, const R &row, const Cut &from, unsigned long long target, F f) {
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

// Collects the logits for which is(x, i) into sh.list; their number (above kList:
// the list is not complete).
template <typename R, typename F>
__device__ __forceinline__ int collect(Shared &sh, const R &row, F is) {
    __syncthreads();
    if (threadIdx.x == 0) sh.count = 0;
    __syncthreads();
    row.each4([&](const f32x4_t &q, int i) {
        bool hit[4], any = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) hit[e] = is(q[e], i + e), any |= hit[e];
        if (__any(any)) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (hit[e]) {
                    const int at = atomicAdd(&sh.count, 1);
                    if (at < kList) sh.list[at] = (unsigned long long)key_of(q[e]) << 32 | (uint32_t)~(i + e);
                }
        }
    });
    __syncthreads();
    return sh.count;
}

// Sorts the first n entries of sh.list, falling (bitonic; thread t has one pair).
// Pairs less than 128 apart stay inside the 128 entries of the thread's wave, whose
// LDS accesses are in order.
__device__ __forceinline__ void sort_list(Shared &sh, int n) {
    const int t = (int)threadIdx.x;
    int size = 2;
    while (size < n) size *= 2;
    for (int i = n + t; i < size; i += kBlock) sh.list[i] = 0;   // below every entry
    __syncthreads();
    for (int k = 2; k <= size; k *= 2) {
        for (int j = k / 2; j > 0; j /= 2) {
            const int a = 2 * t - (t & (j - 1)), b = a + j;
            if (b < size) {
                const unsigned long long x = sh.list[a], y = sh.list[b];
                if ((x < y) == ((a & k) == 0)) sh.list[a] = y, sh.list[b] = x;
            }
            if (j >= 128 || (j == 1 && k >= 128)) __syncthreads();
            else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"), __builtin_amdgcn_wave_barrier();
        }
    }
    __syncthreads();
}
__device__ __forceinline__ float list_value(const Shared &sh, int i) { return value_of((uint32_t)(sh.list[i] >> 32)); }

// A bound that at least k of the threads' maxima reach (k <= kBlock), and not many
// more: the least of those down to the bin, of 1024 between the largest and the
// least finite one, in which the k-th is.  Where outliers crowd the others into
// one bin, again between that bin's ends.
__device__ __forceinline__ float bound_of(Shared &sh, float own, float top, int k) {
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
        if (sh.bin < 0) return -INFINITY;   // fewer than k finite maxima
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

// The cut of min-p: w >= m where (x - top) c >= log2 m; the least such float, at most top.
__device__ Cut cut_of_min_p(const Mass &mass, float m, float top, int V) {
    const double least = log2(fmin((double)m, 1.0));
    float f = (float)(mass.top + least / mass.c);
    if (mass.log2w(f) < least) f = nextafterf(f, INFINITY);
    else if (f > -INFINITY && mass.log2w(nextafterf(f, -INFINITY)) >= least) f = nextafterf(f, -INFINITY);
    return Cut{f > top ? top : f, V};
}

// The draw among the first n entries of the sorted list: in the order of the indices.
__device__ __forceinline__ void draw_from_list(Shared &sh, const TokenSample &a, const Mass &mass, int r, float u, int n) {
    const int tid = (int)threadIdx.x;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kList; e += kBlock) {
        const unsigned long long x = sh.list[e + tid];
        if (e + tid < n) sh.list[e + tid] = x << 32 | x >> 32;   // ~index, key
    }
    __syncthreads();
    sort_list(sh, n);
    double w[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) w[e] = 2 * tid + e < n ? mass.w(value_of((uint32_t)sh.list[2 * tid + e])) : 0.0;
    const double p2 = block_scan(w[0] + w[1], sh.sum), p1 = p2 - w[1];
    if (tid == kBlock - 1) sh.total = p2;
    if (tid == 0) sh.pick = kList;
    __syncthreads();
    const double total = sh.total, goal = (double)u * total;
    const int hit = w[0] > 0.0 && p1 > goal ? 2 * tid : w[1] > 0.0 && p2 > goal ? 2 * tid + 1 : kList;
    if (hit < kList) atomicMin(&sh.pick, hit);
    __syncthreads();
    int at = sh.pick;
    if (at == kList) {   // no sum exceeds u's share: the last one
        const int last = w[1] > 0.0 ? 2 * tid + 1 : w[0] > 0.0 ? 2 * tid : 0;
        at = -block_reduce(-last, sh.ints, Min{});
    }
    if (tid == at / 2) {
        a.token[r] = (int)~(uint32_t)(sh.list[at] >> 32);
        a.logprob[r] = (float)log((at & 1 ? w[1] : w[0]) / total);
    }
}

template <typename T>
__global__ __launch_bounds__(kBlock, 4) void token_sample_kernel(TokenSample a)
{
    __shared__ Shared sh;
    const int r = blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63, wv = tid / kWave, V = a.V;
    const float temp = a.temperature ? a.temperature[r] : 1.f;
    const int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.f, mp = a.min_p ? a.min_p[r] : 0.f, u = a.u[r];
    const Row<T> row(static_cast<const T *>(a.logits) + (size_t)r * a.ld, V);

    float own = -INFINITY;
    bool bad = false;
    row.template each<8>([&](float x, int) {
        own = fmaxf(own, x);
        bad |= !(x < INFINITY);
    });
    // a NaN or +inf logit goes through the maximum as +inf
    const float top = block_reduce(bad ? INFINITY : own, sh.fpart, Max{});
    if (!(fabsf(top) < INFINITY) || !(temp >= 0.f)) {   // no distribution
        if (tid == 0) a.token[r] = -1, a.logprob[r] = NAN;
        return;
    }
    if (temp == 0.f) {
        int at = V;
        if (own == top) row.each([&](float x, int i) { at = x == top && i < at ? i : at; });
        at = block_reduce(at, sh.ints, Min{});
        if (tid == 0) a.token[r] = at, a.logprob[r] = 0.f;
        return;
    }
    int lg = 0;
    while (lg < 31 && (1ll << lg) < V) ++lg;
    const Mass mass{(double)top, 1.4426950408889634 / (double)temp, ldexp(1.0, lg > 18 ? 62 - lg : 44)};
    const Cut cut_m = mp > 0.f && mass.c > 0.0 ? cut_of_min_p(mass, mp, top, V) : Cut{-INFINITY, -1};

    Cut cut{-INFINITY, -1};   // every finite logit
    bool cut_k = k > 0 && k < V, cut_p = p < 1.f;
    if (cut_k && k <= kTopK) {
        const float bound = bound_of(sh, own, top, k);
        const int n = collect(sh, row, [&](float x, int) { return x > -INFINITY && x >= bound; });
        if (n <= kList) {
            // n >= k unless fewer logits are finite.  Two entries a thread: weights and running sums.
            sort_list(sh, n);
            const int kept = n < k ? n : k;
            double *run = reinterpret_cast<double *>(sh.hist);
            float x[2];
            double w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                x[e] = 2 * tid + e < kept ? list_value(sh, 2 * tid + e) : -INFINITY;
                w[e] = mass.w(x[e]);
            }
            const double after = block_scan(w[0] + w[1], sh.sum);
            run[2 * tid] = after - w[1], run[2 * tid + 1] = after;
            __syncthreads();
            const double goal = (double)fmaxf(p, 0.f) * run[kept - 1];
            int left = 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int i = 2 * tid + e;
                left += i < kept && (i == 0 || !cut_p || run[i - 1] < goal) && x[e] >= cut_m.x;
            }
            left = block_reduce(left, sh.ints, Add{});
            draw_from_list(sh, a, mass, r, u, left);
            return;
        }
    }
    if (cut_k) {
        int live = 0;
        row.each([&](float x, int) { live += x > -INFINITY; });
        live = block_reduce(live, sh.ints, Add{});
        if (k < live) cut = find_cut(sh, row, cut, (unsigned long long)k, [](float) { return 1ull; });
    }
    if (cut_p) {
        // the weights below 2^-deep, all together, have less than half of 1 - p
        const float deep = (float)(log2((double)V / (1.0 - (double)fmaxf(p, 0.f))) + 1.0);
        const float per = (float)((double)kBins / (double)deep * mass.c);
        // 32 bits are enough for the bins: falling with x, and the same in every pass
        auto bin_of = [&](float x) { return fmaxf((top - x) * per, 0.f); };
        clear_bins(sh);
        for (int b = tid; b < kBins; b += kBlock) sh.hits[b] = 0;
        __syncthreads();
        double all = 0.0;
        row.each4([&](const f32x4_t &q, int i) {
            double w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = cut.keeps(q[e], i + e) ? mass.w(q[e]) : 0.0;   // no branch: four at once
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                all += w[e];
                const float b = bin_of(q[e]);
                if (b < kBins && w[e] > 0.0) {
                    atomicAdd(&sh.hist[(int)b], mass.whole_of(w[e]));
                    atomicAdd(&sh.hits[(int)b], 1u);
                }
            }
        });
        all = block_reduce(all, sh.sum, Add{});
        const double t = ceil((double)fmaxf(p, 0.f) * all * mass.unit);
        const unsigned long long target = t < 1.0 ? 1ull : (unsigned long long)t;
        find_bin<false>(sh, kBins, 0, target);
        const int bin = sh.bin;
        const unsigned long long above = sh.above;
        int upto = 0;   // logits of the bins 0 .. bin
#pragma unroll
        for (int b = 0; b < kBins; b += kBlock) upto += b + tid <= bin ? (int)sh.hits[b + tid] : 0;
        upto = block_reduce(upto, sh.ints, Add{});
        const bool whole_nucleus = upto <= kList;
        const float from = whole_nucleus ? 0.f : (float)bin;
        int n = kList + 1;
        if (bin >= 0 && (whole_nucleus || sh.hits[bin] <= kList))
            n = collect(sh, row, [&](float x, int i) {
                const float b = bin_of(x);
                return cut.keeps(x, i) && b >= from && b < (float)(bin + 1);
            });
        if (n <= kList) {
            sort_list(sh, n);
            unsigned long long w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) w[e] = 2 * tid + e < n ? mass.whole(list_value(sh, 2 * tid + e)) : 0;
            const unsigned long long p2 = (whole_nucleus ? 0 : above) + block_scan(w[0] + w[1], sh.part);
            const unsigned long long p1 = p2 - w[1], p0 = p1 - w[0];
            const int hit = p0 < target && target <= p1 ? 2 * tid : p1 < target && target <= p2 ? 2 * tid + 1 : -1;
            if (hit >= 0) sh.pick = hit;
            __syncthreads();
            if (whole_nucleus) {
                const int upto = sh.pick + 1;
                int left = 0;
#pragma unroll
                for (int e = 0; e < 2; ++e) left += 2 * tid + e < upto && list_value(sh, 2 * tid + e) >= cut_m.x;
                left = block_reduce(left, sh.ints, Add{});
                draw_from_list(sh, a, mass, r, u, left);
                return;
            }
            const unsigned long long at = sh.list[sh.pick];
            cut = Cut{value_of((uint32_t)(at >> 32)), (int)~(uint32_t)at};
        } else {   // more of one value, or nearly, than the list takes
            unsigned long long whole = 0;
            row.each([&](float x, int i) { whole += cut.keeps(x, i) ? mass.whole(x) : 0ull; });
            whole = block_reduce(whole, sh.part, Add{});
            cut = find_cut(sh, row, cut, target < whole ? target : whole, [&](float x) { return mass.whole(x); });
        }
    }
    if (cut_m.x > cut.x) cut = cut_m;

    // the draw: the waves' sums, the wave that has the token, the sums of parts of its part
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
    mine = wave_reduce(mine, Add{});
    __syncthreads();
    if (lane == 0) sh.sum[wv] = mine;
    __syncthreads();
    double total = 0.0;
    for (int w = 0; w < kWaves; ++w) total += sh.sum[w];
    const double goal = (double)u * total;
    int holder = 0;
    double before = 0.0, run = 0.0;
    for (int w = 0; w < kWaves; ++w) {
        if (sh.sum[w] > 0.0) {
            holder = w, before = run;
            if (run + sh.sum[w] > goal) break;
        }
        run += sh.sum[w];
    }
    __syncthreads();
    // its part in kWaves parts of whole loads
    const int span = Row<T>::span_of(V);
    const int steps = (span / kStep + kWaves - 1) / kWaves;
    const int first = holder * span + wv * steps * kStep, stop = (holder + 1) * span;
    auto weights = [&](int s, double (&w)[4], int &i) {
        i = first + s * kStep + 4 * lane;
        const bool in = first + s * kStep < stop && i < V;
        const f32x4_t q = in ? row.load(i) : f32x4_t{-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = cut.keeps(q[e], i + e) ? mass.w(q[e]) : 0.0;
    };
    mine = 0.0;
    for (int s = 0; s < steps; ++s) {
        double w[4];
        int i;
        weights(s, w, i);
        mine += (w[0] + w[1]) + (w[2] + w[3]);
    }
    mine = wave_reduce(mine, Add{});
    if (lane == 0) sh.sum[wv] = mine;
    __syncthreads();
    int sub = 0;
    run = before;
    for (int w = 0; w < kWaves; ++w) {
        if (sh.sum[w] > 0.0) {
            sub = w, before = run;
            if (run + sh.sum[w] > goal) break;
        }
        run += sh.sum[w];
    }
    if (wv != sub) return;
    int at = -1;
    double w_at = 0.0, seen = before;
    bool done = false;
    for (int s = 0; s < steps && !done; ++s) {
        double w[4];
        int i;
        weights(s, w, i);
        const double sum = (w[0] + w[1]) + (w[2] + w[3]), after = wave_scan(sum);
        double x = seen + (after - sum);
        int hit = -1, last = -1;
        double w_hit = 0.0, w_last = 0.0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x += w[e];
            if (w[e] > 0.0) {
                last = e, w_last = w[e];
                if (hit < 0 && x > goal) hit = e, w_hit = w[e];
            }
        }
        const unsigned long long past = __ballot(hit >= 0), has = __ballot(last >= 0);
        if (past) {
            const int l = __ffsll((long long)past) - 1;
            at = __shfl(i + hit, l), w_at = __shfl(w_hit, l), done = true;
        } else if (has) {   // the last one, if no later sum passes
            const int l = 63 - __clzll((long long)has);
            at = __shfl(i + last, l), w_at = __shfl(w_last, l);
        }
        seen += __shfl(after, 63);
    }
    if (lane == 0) a.token[r] = at, a.logprob[r] = (float)log(w_at / total);
}

}  // namespace

size_t token_sample_workspace_bytes(int, int, int) { return 16; }

hipError_t launch_token_sample(const TokenSample &a, bool bf16, hipStream_t stream)
{
    const dim3 gd((unsigned)a.R), bd(kBlock);
    if (bf16) hipLaunchKernelGGL(token_sample_kernel<uint16_t>, gd, bd, 0, stream, a);
    else hipLaunchKernelGGL(token_sample_kernel<float>, gd, bd, 0, stream, a);
    return hipGetLastError();
}

}  // namespace fs
