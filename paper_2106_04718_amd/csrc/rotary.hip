// Rotary positions of queries and keys, for gfx950.
//
// Pair i of a head at position p is turned by the angle p * freq[i]:
//   a' = m (a cos - b sin),  b' = m (b cos + a sin)
// (a, b) being elements (i, i + rot / 2) of the head or (2i, 2i + 1); elements from rot on
// stay as they are.  Every element is read and written once, for some ten operations:
// bound by HBM bandwidth (16384 tokens of 40 bf16 heads of 128, 336 MB: 58 us, 5.7 TB/s; 5001 of 32 fp32
// heads of 64, 82 MB: 18.7 us, 4.4 TB/s; a 1 GiB copy 5.1).
//
// The angle is taken in 64 bits, for far positions turn the first pairs through a million
// radians (in 32 bits the angle of 2^20 is off by up to 0.03), and left by whole quarter
// turns before it is rounded to 32.  A workgroup makes the cosines and sines of its tokens
// once, in LDS, for all heads.
#include <stdint.h>

#include <type_traits>

#include "div.h"
#include "grid.h"
#include "launch.h"

namespace fs {
namespace {

constexpr int kThreads = 256;
constexpr int kMany = 2;   // units of a lane on their way together

// Cosine and sine of p * f, f in radians.  What is left of the angle behind the nearest
// quarter turn is at most pi / 4; the series end where a term is below 2^-28.
__device__ __forceinline__ float2 turn(int p, double f) {
    const double quarters = (double)p * f * 0.63661977236758134308;   // 2 / pi
    const double q = rint(quarters);
    const float y = (float)((quarters - q) * 1.57079632679489661923), z = y * y;
    float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);   // 1 / 9!, 1 / 7!, ..
    s = fmaf(z, s, 8.3333333e-3f);
    s = fmaf(z, s, -1.6666667e-1f);
    s = fmaf(y * z, s, y);
    float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);   // 1 / 10!, 1 / 8!, ..
    c = fmaf(z, c, -1.3888889e-3f);
    c = fmaf(z, c, 4.1666667e-2f);
    c = fmaf(z, c, -0.5f);
    c = fmaf(z, c, 1.0f);
    const int quadrant = (int)(q - 4.0 * floor(q * 0.25));
    const float a = quadrant & 1 ? s : c, b = quadrant & 1 ? c : s;
    return make_float2(quadrant == 1 || quadrant == 2 ? -a : a, quadrant >= 2 ? -b : b);
}

// 16 bytes of a row.
template <bool BF16>
struct Piece {
    typedef uint32_t words_t __attribute__((ext_vector_type(4)));
    words_t w;

    __device__ __forceinline__ void load(const unsigned char *p) {
        w = __builtin_nontemporal_load(reinterpret_cast<const words_t *>(p));
    }
    __device__ __forceinline__ void store(unsigned char *p) const { *reinterpret_cast<words_t *>(p) = w; }
    // its first n elements, an even number
    __device__ __forceinline__ void store(unsigned char *p, int n) const {
        constexpr int kOfWord = BF16 ? 2 : 1;
        if (n >= 4 * kOfWord) return store(p);
        if (n >= 2 * kOfWord) *reinterpret_cast<uint64_t *>(p) = (uint64_t)w[1] << 32 | w[0];
        if (n >= 3 * kOfWord) reinterpret_cast<uint32_t *>(p)[2] = w[2];
        else if (n >= kOfWord && n < 2 * kOfWord) reinterpret_cast<uint32_t *>(p)[0] = w[0];
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (!BF16) return __uint_as_float(w[e]);
        else return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    }
    __device__ __forceinline__ void set(int e, float x) {
        if constexpr (!BF16) {
            w[e] = __float_as_uint(x);
        } else {
            const uint32_t b = __builtin_bit_cast(uint16_t, (__bf16)x);
            w[e / 2] = e & 1 ? (w[e / 2] & 0xffffu) | b << 16 : (w[e / 2] & 0xffff0000u) | b;
        }
    }
};

// How a lane's elements meet their partners:
//   kInter   a unit is 32 bytes of a head, pairs side by side
//   kHalves  16 bytes of the first half of rot and 16 of the second
//   kAnyHalf 16 bytes of a head, whose partners lie anywhere in rot: they come from LDS
// Units below `turned` hold elements to be turned (kInter, kAnyHalf: the last of them perhaps
// elements behind rot too); the others are copied.  Units are numbered along all tokens and heads,
// and a workgroup has `batch` of them, AHEAD a lane, whose loads are on their way together: with
// whole tokens a workgroup instead, some lanes would go round more often than others (9000
// tokens of 72 heads of 128, 332 MB, 73 us; 16384 of 40 64).  In place nothing from element rot
// on is stored, for another stream may write there meanwhile (9000 tokens of 72 bf16 heads of 128, 20
// elements interleaved: 44 us, where whole units take 32).
enum class Pairs { kInter, kHalves, kAnyHalf };
template <bool BF16, Pairs PAIRS, int AHEAD, bool PARTLY>   // PARTLY: in place, and a unit goes past rot or may
__global__ __launch_bounds__(kThreads) void rotary_kernel(Rotary a, int batch, int turned, int stored, Div by_token, int token_units,
                                                          Div by_units, int units, Div by_pairs)
{
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int kVec = BF16 ? 8 : 4, kEsize = BF16 ? 2 : 4;
    constexpr bool kInter = PAIRS == Pairs::kInter, kTwo = PAIRS != Pairs::kAnyHalf;
    using P = Piece<BF16>;
    const int pairs = a.rot / 2;
    const unsigned long long begin = (unsigned long long)wide_index() * (unsigned)batch, end = (unsigned long long)a.N * (unsigned)token_units;
    if (begin >= end) return;
    const int all = end - begin < (unsigned)batch ? (int)(end - begin) : batch;
    const int n0 = begin < 0x7fffffffu ? (int)by_token((unsigned)begin) : (int)(begin / (unsigned)token_units);
    const int behind = (int)(begin - (unsigned long long)(unsigned)n0 * (unsigned)token_units);   // units of token n0 before the first
    const int tokens = (int)by_token((unsigned)(behind + all - 1)) + 1;
    float2 *turns = reinterpret_cast<float2 *>(lds + (kTwo ? 0 : AHEAD * kThreads * 16));   // [tokens][pairs], behind what the lanes hold

    P x[AHEAD], y[AHEAD];
    unsigned char *to[AHEAD], *to2[AHEAD];
    int at[AHEAD], unit[AHEAD], left[AHEAD];   // left: elements that are stored, from the unit's first on
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
        const int mine = e * kThreads + (int)threadIdx.x, i = behind + (mine < all ? mine : all - 1);   // past the last: not stored
        const int t = (int)by_token((unsigned)i), in = i - t * token_units, h = (int)by_units((unsigned)in);
        unit[e] = in - h * units;
        const bool half = PAIRS == Pairs::kHalves && unit[e] < turned;
        const int d = (half || !kTwo ? unit[e] : 2 * unit[e]) * kVec;   // behind rot halves go on in twos
        const size_t next = (size_t)(half ? pairs : kVec) * kEsize;
        const bool key = h >= a.Hq;
        const RotaryRows &r = key ? a.k : a.q;
        const long long n = (long long)n0 + t, hh = key ? h - a.Hq : h;
        const unsigned char *from = r.from + n * r.from_token + hh * r.from_head + (size_t)d * kEsize;
        to[e] = r.to + n * r.to_token + hh * r.to_head + (size_t)d * kEsize, to2[e] = to[e] + next;
        at[e] = mine < all ? t * pairs : -1;
        left[e] = PARTLY && r.from == r.to && !half ? a.rot - d : 2 * kVec;
        x[e].load(from);
        if (kTwo) y[e].load(from + next);
    }
    for (int i = (int)threadIdx.x; i < tokens * pairs; i += kThreads) {
        const int t = (int)by_pairs((unsigned)i), p = i - t * pairs;
        const float2 cs = turn(a.positions[(long long)n0 + t], a.freq[p]);
        turns[i] = make_float2(cs.x * a.magnitude, cs.y * a.magnitude);
    }
    if constexpr (!kTwo) {   // whole heads: their units are a power of two, at most 32, and divide a batch
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) x[e].store(lds + (e * kThreads + threadIdx.x) * 16);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < AHEAD; ++e) {
        if (at[e] < 0 || unit[e] >= stored) continue;
        if (unit[e] < turned) {
            if constexpr (kTwo) {
#pragma unroll
                for (int v = 0; v < kVec; ++v) {
                    const int p = unit[e] * kVec + v;
                    if (kInter && p >= pairs) continue;
                    const float2 cs = turns[at[e] + p];
                    // elements 2v and 2v + 1 of the two pieces, or v of each
                    P &first_of = kInter && 2 * v >= kVec ? y[e] : x[e], &second_of = !kInter || 2 * v + 1 >= kVec ? y[e] : x[e];
                    const int ea = kInter ? (2 * v) % kVec : v, eb = kInter ? (2 * v + 1) % kVec : v;
                    const float u = first_of.get(ea), w = second_of.get(eb);
                    first_of.set(ea, fmaf(u, cs.x, -(w * cs.y)));
                    second_of.set(eb, fmaf(w, cs.x, u * cs.y));
                }
            } else {
                const unsigned char *head = lds + (e * kThreads + threadIdx.x - unit[e]) * 16;
#pragma unroll
                for (int v = 0; v < kVec; ++v) {
                    const int d = unit[e] * kVec + v;
                    if (d >= a.rot) continue;
                    const bool low = d < pairs;
                    const int other = low ? d + pairs : d - pairs;
                    const float2 cs = turns[at[e] + (low ? d : other)];
                    const float u = x[e].get(v);
                    const float w = BF16 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(head)[other] << 16)
                                         : reinterpret_cast<const float *>(head)[other];
                    x[e].set(v, low ? fmaf(u, cs.x, -(w * cs.y)) : fmaf(u, cs.x, w * cs.y));
                }
            }
        }
        x[e].store(to[e], left[e]);
        if (kTwo) y[e].store(to2[e], left[e] - kVec);
    }
}

}  // namespace

hipError_t launch_rotary(const Rotary &a, int D, bool bf16, bool interleaved, hipStream_t stream)
{
    const int pairs = a.rot / 2, vec = bf16 ? 8 : 4;
    const Pairs how = interleaved ? Pairs::kInter : pairs % vec == 0 ? Pairs::kHalves : Pairs::kAnyHalf;
    const int turned = how == Pairs::kAnyHalf ? (a.rot + vec - 1) / vec : (pairs + vec - 1) / vec;
    // in place nothing behind rot is touched
    const bool in_place = (a.Hq == 0 || a.q.from == a.q.to) && (a.Hkv == 0 || a.k.from == a.k.to);
    const bool either = (a.Hq > 0 && a.q.from == a.q.to) || (a.Hkv > 0 && a.k.from == a.k.to);
    const bool partly = in_place ? a.rot % (how == Pairs::kInter ? 2 * vec : how == Pairs::kAnyHalf ? vec : 2) != 0 : either;
    const int whole = how == Pairs::kAnyHalf ? D / vec : D / (2 * vec), stored = in_place ? turned : whole;
    const int units = how == Pairs::kAnyHalf ? whole : stored, token_units = (a.Hq + a.Hkv) * units;
    if (stored == 0) return hipSuccess;
    const long long total = (long long)a.N * token_units;
    // a unit a lane until they fill the chip, then more; cosines and sines of at most 32 KB
    const bool few = total <= 1024ll * kThreads;
    const int most = 4096 / (pairs ? pairs : 1) - 2;   // tokens
    int batch = (few ? 1 : kMany) * kThreads;
    if (token_units * (long long)most < batch) batch = token_units * most;
    const int tokens = batch / token_units + 2;
    auto launch = [&](auto kernel, int ahead) {
        const size_t lds = (size_t)tokens * pairs * sizeof(float2) + (how == Pairs::kAnyHalf ? ahead * kThreads * 16 : 0);
        hipLaunchKernelGGL(kernel, wide_grid((total + batch - 1) / batch), dim3(kThreads), lds, stream, a, batch, turned, stored,
                           make_div(token_units), token_units, make_div(units), units, make_div(pairs ? pairs : 1));
    };
    auto of_type = [&](auto pairs_how) {
        constexpr Pairs P = decltype(pairs_how)::value;
        auto of_place = [&](auto some) {
            constexpr bool PARTLY = decltype(some)::value;
            if (bf16) few ? launch(rotary_kernel<true, P, 1, PARTLY>, 1) : launch(rotary_kernel<true, P, kMany, PARTLY>, kMany);
            else few ? launch(rotary_kernel<false, P, 1, PARTLY>, 1) : launch(rotary_kernel<false, P, kMany, PARTLY>, kMany);
        };
        partly ? of_place(std::true_type{}) : of_place(std::false_type{});
    };
    switch (how) {
    case Pairs::kInter: of_type(std::integral_constant<Pairs, Pairs::kInter>{}); break;
    case Pairs::kHalves: of_type(std::integral_constant<Pairs, Pairs::kHalves>{}); break;
    default: of_type(std::integral_constant<Pairs, Pairs::kAnyHalf>{}); break;
    }
    return hipGetLastError();
}

}  // namespace fs
