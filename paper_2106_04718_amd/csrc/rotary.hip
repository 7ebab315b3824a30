// Rotary positions of queries and keys, for gfx950.
//
// Pair i of a head at position p is turned by the angle p * freq[i]:
//   a' = m (a cos - b sin),  b' = m (b cos + a sin)
// (a, b) being elements (i, i + rot / 2) of the head or (2i, 2i + 1); elements from rot on
// stay as they are.  Every element is read and written once, for some ten operations:
// bound by HBM bandwidth.
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

// VEC elements of a row.
template <bool BF16, int VEC>
struct Piece {
    static constexpr int kBytes = VEC * (BF16 ? 2 : 4);
    using Word = std::conditional_t<kBytes == 2, uint16_t, uint32_t>;
    static constexpr int kWords = kBytes < 4 ? 1 : kBytes / 4;
    typedef Word words_t __attribute__((ext_vector_type(kWords)));
    words_t w;

    __device__ __forceinline__ void load(const unsigned char *p) {
        w = __builtin_nontemporal_load(reinterpret_cast<const words_t *>(p));
    }
    __device__ __forceinline__ void store(unsigned char *p) const { *reinterpret_cast<words_t *>(p) = w; }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (!BF16) return __uint_as_float(w[e]);
        else if constexpr (VEC == 1) return __uint_as_float((uint32_t)w[0] << 16);
        else return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    }
    __device__ __forceinline__ void set(int e, float x) {
        if constexpr (!BF16) {
            w[e] = __float_as_uint(x);
        } else {
            const uint32_t b = __builtin_bit_cast(uint16_t, (__bf16)x);
            if constexpr (VEC == 1) w[0] = (uint16_t)b;
            else w[e / 2] = e & 1 ? (w[e / 2] & 0xffffu) | b << 16 : (w[e / 2] & 0xffff0000u) | b;
        }
    }
};

// A unit is VEC pairs of a head, two pieces: units below `turned` hold pairs to be turned
// (interleaved: the last of them perhaps elements behind rot too), the others elements that
// are copied.  A workgroup has the units of `tokens` tokens, kAhead of a lane's on their way
// together.
constexpr int kAhead = 4;
template <bool BF16, int VEC, bool INTER>
__global__ __launch_bounds__(kThreads) void rotary_kernel(Rotary a, int tokens, int turned, Div by_units, int units, Div by_heads,
                                                          Div by_pairs)
{
    extern __shared__ float2 turns[];   // [tokens][pairs]
    using P = Piece<BF16, VEC>;
    constexpr int kEsize = BF16 ? 2 : 4;
    const int pairs = a.rot / 2, heads = a.Hq + a.Hkv;
    const long long n0 = (long long)wide_index() * tokens;
    if (n0 >= a.N) return;
    const int here = a.N - n0 < tokens ? (int)(a.N - n0) : tokens;
    const int all = here * heads * units;

    for (int i0 = 0, first = 1; i0 < all; i0 += kAhead * kThreads, first = 0) {
        P x[kAhead], y[kAhead];
        unsigned char *to[kAhead], *to2[kAhead];
        int at[kAhead], unit[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int mine = i0 + e * kThreads + (int)threadIdx.x, i = mine < all ? mine : all - 1;   // past the last: not stored
            const int th = (int)by_units((unsigned)i), t = (int)by_heads((unsigned)th), h = th - t * heads;
            unit[e] = i - th * units;
            const bool half = !INTER && unit[e] < turned;
            const int d = half ? unit[e] * VEC : 2 * unit[e] * VEC;   // behind rot both layouts go on in twos
            const size_t next = (size_t)(half ? pairs : VEC) * kEsize;
            const bool key = h >= a.Hq;
            const RotaryRows &r = key ? a.k : a.q;
            const long long n = n0 + t, hh = key ? h - a.Hq : h;
            const unsigned char *from = r.from + n * r.from_token + hh * r.from_head + (size_t)d * kEsize;
            to[e] = r.to + n * r.to_token + hh * r.to_head + (size_t)d * kEsize, to2[e] = to[e] + next;
            at[e] = mine < all ? t * pairs : -1;
            x[e].load(from), y[e].load(from + next);
        }
        if (first) {
            for (int i = (int)threadIdx.x; i < here * pairs; i += kThreads) {
                const int t = (int)by_pairs((unsigned)i), p = i - t * pairs;
                const float2 cs = turn(a.positions[n0 + t], a.freq[p]);
                turns[i] = make_float2(cs.x * a.magnitude, cs.y * a.magnitude);
            }
            __syncthreads();
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            if (at[e] < 0) continue;
            if (unit[e] < turned) {
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    const int p = unit[e] * VEC + v;
                    if (INTER && p >= pairs) continue;
                    const float2 cs = turns[at[e] + p];
                    // elements 2v and 2v + 1 of the two pieces, or v of each
                    P &first_of = INTER && 2 * v >= VEC ? y[e] : x[e], &second_of = !INTER || 2 * v + 1 >= VEC ? y[e] : x[e];
                    const int ea = INTER ? (2 * v) % VEC : v, eb = INTER ? (2 * v + 1) % VEC : v;
                    const float u = first_of.get(ea), w = second_of.get(eb);
                    first_of.set(ea, fmaf(u, cs.x, -(w * cs.y)));
                    second_of.set(eb, fmaf(w, cs.x, u * cs.y));
                }
            }
            x[e].store(to[e]), y[e].store(to2[e]);
        }
    }
}

}  // namespace

hipError_t launch_rotary(const Rotary &a, int D, bool bf16, bool interleaved, hipStream_t stream)
{
    const int pairs = a.rot / 2;
    // whole 16 bytes: a head's halves are apart by pairs elements, whose largest power of two
    // that divides them a piece can have
    int vec = bf16 ? 8 : 4;
    while (!interleaved && pairs % vec) vec /= 2;
    const int turned = (pairs + vec - 1) / vec;
    // in place nothing behind rot is touched
    const bool in_place = (a.Hq == 0 || a.q.from == a.q.to) && (a.Hkv == 0 || a.k.from == a.k.to);
    const int units = in_place ? turned : D / (2 * vec), heads = a.Hq + a.Hkv;
    if (units == 0) return hipSuccess;
    const int tokens = a.N <= 2048 ? 1 : 4;
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, wide_grid(((long long)a.N + tokens - 1) / tokens), dim3(kThreads),
                           (size_t)tokens * (pairs ? pairs : 1) * sizeof(float2), stream, a, tokens, turned, make_div(units), units,
                           make_div(heads), make_div(pairs ? pairs : 1));
    };
    if (interleaved) {
        bf16 ? launch(rotary_kernel<true, 8, true>) : launch(rotary_kernel<false, 4, true>);
    } else if (bf16) {
        if (vec == 8) launch(rotary_kernel<true, 8, false>);
        else if (vec == 4) launch(rotary_kernel<true, 4, false>);
        else if (vec == 2) launch(rotary_kernel<true, 2, false>);
        else launch(rotary_kernel<true, 1, false>);
    } else {
        if (vec == 4) launch(rotary_kernel<false, 4, false>);
        else if (vec == 2) launch(rotary_kernel<false, 2, false>);
        else launch(rotary_kernel<false, 1, false>);
    }
    return hipGetLastError();
}

}  // namespace fs
