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
// vocabulary has many borders: the weights and sums are 64-bit.
#include <math.h>
#include <stdint.h>

#include "launch.h"

namespace fs {
namespace {

constexpr int kWave = 64;
constexpr int kWaves = 16;
constexpr int kBlock = kWave * kWaves;
constexpr int kBins = 2048;   // of one digit of 11, 11 and 10 bits

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// Order-preserving map of the finite and infinite floats to integers (both zeros
// to one, as they are equal).
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

template <typename V, typename Op>
__device__ __forceinline__ V wave_reduce(V x, Op op) {
    for (int m = 1; m < kWave; m *= 2) x = op(x, __shfl_xor(x, m));
    return x;
}

// What is kept of a row: logits above the threshold, and those equal to it up to
// an index.
struct Cut {
    uint32_t key;
    int last;
    __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

struct Shared {
    unsigned long long hist[kBins];
    unsigned long long part[kWaves];
    double sum[kWaves];
    float fmax[kWaves];
    int ints[kWaves];
    unsigned long long above, in_bin;
    int bin, pick;
    double before;
};

template <typename V, typename Op>
__device__ V block_reduce(V x, V *part, Op op) {
    x = wave_reduce(x, op);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x / kWave] = x;
    __syncthreads();
    V y = part[0];
    for (int w = 1; w < kWaves; ++w) y = op(y, part[w]);
    return y;
}

// The row as the workgroup walks it: wave w has the logits [w * span, (w+1) * span).
template <typename T>
struct Row {
    const T *x;
    int V, span, begin, end;
    __device__ Row(const T *p, int V_) : x(p), V(V_) {
        span = (V + kWaves * kWave - 1) / (kWaves * kWave) * kWave;
        const long long b = (long long)(threadIdx.x / kWave) * span;
        begin = b < V ? (int)b : V;
        end = V - begin < span ? V : begin + span;
    }
    template <typename F>
    __device__ __forceinline__ void each(F f) const {   // f(logit, index); every lane of a wave takes every step
        for (int i = begin; i < end; i += kWave) {
            const int j = i + (int)(threadIdx.x & 63);
            f(j < end ? widen(x[j]) : -INFINITY, j < end ? j : V);
        }
    }
};

// Weights as whole numbers of 2^-bits of the largest: their sums do not depend
// on the order of the atomic additions.
struct Mass {
    double top, c;      // the largest logit; log2(e) / T
    double unit;        // 2^bits
    __device__ __forceinline__ double w(float x) const { return exp2(((double)x - top) * c); }
    __device__ __forceinline__ unsigned long long whole(float x) const { return (unsigned long long)(w(x) * unit + 0.5); }
};

// The cut at which the sum of f over the kept logits, in the order, first reaches
// `target` (1 <= target <= the sum over `from`), by digits of the key, the
// highest first.  f: 1 (counts) or the weight (f is the same for equal logits).
template <typename T, typename F>
__device__ Cut find_cut(Shared &sh, const Row<T> &row, const Cut &from, unsigned long long target, F f) {
    uint32_t prefix = 0, mask = 0;
    unsigned long long above = 0;
    const int tid = (int)threadIdx.x;
    for (int level = 0; level < 3; ++level) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, bins = level == 2 ? 1024 : 2048;
        __syncthreads();
        for (int b = tid; b < kBins; b += kBlock) sh.hist[b] = 0;
        __syncthreads();
        row.each([&](float x, int i) {
            const uint32_t k = key_of(x);
            if (i < row.V && (k & mask) == prefix && from.keeps(k, i)) {
                const unsigned long long v = f(x);
                if (v) atomicAdd(&sh.hist[(k >> shift) & (bins - 1)], v);
            }
        });
        __syncthreads();
        // bins from the highest: thread t has bins bins-1-2t and bins-2-2t
        const int hi = bins - 1 - 2 * tid;
        const unsigned long long a = hi >= 0 ? sh.hist[hi] : 0, b = hi >= 1 ? sh.hist[hi - 1] : 0;
        unsigned long long inc = a + b;
        for (int m = 1; m < kWave; m *= 2) {
            const unsigned long long o = __shfl_up(inc, m);
            if ((tid & 63) >= m) inc += o;
        }
        if ((tid & 63) == 63) sh.part[tid / kWave] = inc;
        __syncthreads();
        unsigned long long base = above;
        for (int w = 0; w < tid / kWave; ++w) base += sh.part[w];
        const unsigned long long p1 = base + inc - b, p0 = p1 - a, p2 = base + inc;   // before a, after a, after b
        if (p0 < target && target <= p1) sh.bin = hi, sh.above = p0, sh.in_bin = a;
        if (p1 < target && target <= p2) sh.bin = hi - 1, sh.above = p1, sh.in_bin = b;
        __syncthreads();
        prefix |= (uint32_t)sh.bin << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        above = sh.above;
    }
    // the logits equal to the threshold: as many as reach the target, by index
    const unsigned long long each = f(value_of(prefix));
    const int need = (int)((target - above + each - 1) / each);
    int mine = 0;
    row.each([&](float x, int i) { mine += i < row.V && key_of(x) == prefix && from.keeps(prefix, i); });
    mine = wave_reduce(mine, [](int p, int q) { return p + q; });
    __syncthreads();
    if ((tid & 63) == 0) sh.ints[tid / kWave] = mine;
    if (tid == 0) sh.pick = row.V;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < tid / kWave; ++w) before += sh.ints[w];
    if (before < need && need <= before + mine) {   // the wave that holds the last one
        int seen = before;
        row.each([&](float x, int i) {
            const bool eq = i < row.V && key_of(x) == prefix && from.keeps(prefix, i);
            const unsigned long long all = __ballot(eq);
            const int rank = seen + __popcll(all & ((1ull << (tid & 63)) - 1));
            if (eq && rank == need - 1) sh.pick = i;
            seen += __popcll(all);
        });
    }
    __syncthreads();
    return Cut{prefix, sh.pick};
}

template <typename T>
__global__ __launch_bounds__(kBlock) void token_sample_kernel(TokenSample a)
{
    __shared__ Shared sh;
    const int r = blockIdx.x, tid = (int)threadIdx.x;
    const Row<T> row(static_cast<const T *>(a.logits) + (size_t)r * a.ld, a.V);
    const float temp = a.temperature ? a.temperature[r] : 1.f;
    const int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.f, mp = a.min_p ? a.min_p[r] : 0.f, u = a.u[r];

    float top = -INFINITY;
    int bad = 0;
    row.each([&](float x, int) {
        top = fmaxf(top, x);
        bad |= !(x < INFINITY);
    });
    top = block_reduce(top, sh.fmax, [](float p, float q) { return fmaxf(p, q); });
    bad = block_reduce(bad, sh.ints, [](int p, int q) { return p | q; });
    if (bad || top == -INFINITY || !(temp >= 0.f)) {   // no distribution
        if (tid == 0) a.token[r] = -1, a.logprob[r] = NAN;
        return;
    }
    if (temp == 0.f) {
        int at = a.V;
        row.each([&](float x, int i) { at = x == top && i < at ? i : at; });
        at = block_reduce(at, sh.ints, [](int p, int q) { return p < q ? p : q; });
        if (tid == 0) a.token[r] = at, a.logprob[r] = 0.f;
        return;
    }
    int lg = 0;
    while (lg < 31 && (1ll << lg) < a.V) ++lg;
    const Mass mass{(double)top, 1.4426950408889634 / (double)temp, ldexp(1.0, lg > 18 ? 62 - lg : 44)};

    Cut cut{key_of(-INFINITY) + 1, a.V};   // every finite logit
    if (k > 0 && k < a.V) {
        int live = 0;
        row.each([&](float x, int) { live += x > -INFINITY; });
        live = block_reduce(live, sh.ints, [](int p, int q) { return p + q; });
        if (k < live) cut = find_cut(sh, row, cut, (unsigned long long)k, [](float) { return 1ull; });
    }
    if (p < 1.f) {
        unsigned long long all = 0;
        row.each([&](float x, int i) { all += cut.keeps(key_of(x), i) ? mass.whole(x) : 0ull; });
        all = block_reduce(all, sh.part, [](unsigned long long p, unsigned long long q) { return p + q; });
        const double t = ceil((double)fmaxf(p, 0.f) * (double)all);
        unsigned long long target = t < 1.0 ? 1ull : (unsigned long long)t;
        if (target > all) target = all;
        cut = find_cut(sh, row, cut, target, [&](float x) { return mass.whole(x); });
    }
    if (mp > 0.f && mass.c > 0.0) {   // w >= m where (x - top) * c >= log2 m
        const double least = log2(fmin((double)mp, 1.0));
        // the least logit that passes: the threshold as a float, rounded up
        double xt = mass.top + least / mass.c;
        float f = (float)xt;
        if (((double)f - mass.top) * mass.c < least) f = nextafterf(f, INFINITY);
        else if (f > -INFINITY && ((double)nextafterf(f, -INFINITY) - mass.top) * mass.c >= least) f = nextafterf(f, -INFINITY);
        if (f > top) f = top;
        if (key_of(f) > cut.key) cut = Cut{key_of(f), a.V};
    }

    // the draw: the waves' sums, then the one wave that holds the token
    double mine = 0.0;
    row.each([&](float x, int i) { mine += i < a.V && cut.keeps(key_of(x), i) ? mass.w(x) : 0.0; });
    mine = wave_reduce(mine, [](double p, double q) { return p + q; });
    __syncthreads();
    if ((tid & 63) == 0) sh.sum[tid / kWave] = mine;
    __syncthreads();
    double total = 0.0;
    for (int w = 0; w < kWaves; ++w) total += sh.sum[w];
    const double goal = (double)u * total;
    int holder = -1;
    double before = 0.0, run = 0.0;
    for (int w = 0; w < kWaves; ++w) {
        if (sh.sum[w] > 0.0) {
            holder = w, before = run;
            if (run + sh.sum[w] > goal) break;
        }
        run += sh.sum[w];
    }
    if (tid / kWave != holder) return;
    int at = -1;
    double w_at = 0.0, seen = before;
    bool done = false;
    row.each([&](float x, int i) {
        const double w = i < a.V && cut.keeps(key_of(x), i) ? mass.w(x) : 0.0;
        double inc = w;
        for (int m = 1; m < kWave; m *= 2) {
            const double o = __shfl_up(inc, m);
            if ((tid & 63) >= m) inc += o;
        }
        const unsigned long long has = __ballot(w > 0.0), past = __ballot(w > 0.0 && seen + inc > goal);
        if (!done && has) {
            const int lane = past ? __ffsll((long long)past) - 1 : 63 - __clzll((long long)has);
            at = __shfl(i, lane), w_at = __shfl(w, lane);
            done = past != 0;
        }
        seen += __shfl(inc, 63);
    });
    if ((tid & 63) == 0) a.token[r] = at, a.logprob[r] = (float)log(w_at / total);
}

}  // namespace

size_t token_sample_workspace_bytes(int, int, int) { return 16; }

hipError_t launch_token_sample(const TokenSample &a, bool bf16, hipStream_t stream)
{
    if (bf16) hipLaunchKernelGGL(token_sample_kernel<uint16_t>, dim3((unsigned)a.R), dim3(kBlock), 0, stream, a);
    else hipLaunchKernelGGL(token_sample_kernel<float>, dim3((unsigned)a.R), dim3(kBlock), 0, stream, a);
    return hipGetLastError();
}

}  // namespace fs
