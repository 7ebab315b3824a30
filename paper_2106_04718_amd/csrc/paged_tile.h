// What the kernels that attend a paged cache share: a wave's tile of 32 positions and
// 16 query columns on the matrix cores, sums over lanes, and softmax states that several
// workgroups exchange.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

namespace fs {
namespace {

constexpr int kWave = 64;
constexpr int kWaves = 4;
constexpr int kBlock = kWave * kWaves;
constexpr int kTile = 32;               // positions a wave attends at a time
constexpr int kUnit = kTile * kWaves;   // positions a workgroup attends at a time

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

// Inclusive sums over the lanes: of the row of 16 from 1, 2, 4 and 8 lanes before,
// then the last of a row to the rows behind it.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ int dpp(int x) {
    return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, ROWS == 0xF);
}
__device__ __forceinline__ int wave_scan(int x) {
    x += dpp<0x111>(x);
    x += dpp<0x112>(x);
    x += dpp<0x114>(x);
    x += dpp<0x118>(x);
    x += dpp<0x142, 0xA>(x);
    return x + dpp<0x143, 0xC>(x);
}
__device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }

// Maximum and sum over the four lanes n, n + 16, n + 32, n + 48 of a column.
template <int MASK>
__device__ __forceinline__ void lane_pair(float x, float &lo, float &hi) {
    const unsigned u = __float_as_uint(x);
    if constexpr (MASK == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        lo = __uint_as_float(r[0]), hi = __uint_as_float(r[1]);
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        lo = __uint_as_float(r[0]), hi = __uint_as_float(r[1]);
    }
}
__device__ __forceinline__ float col_max(float x) {
    float a, b;
    lane_pair<16>(x, a, b);
    x = fmaxf(a, b);
    lane_pair<32>(x, a, b);
    return fmaxf(a, b);
}
__device__ __forceinline__ float col_sum(float x) {
    float a, b;
    lane_pair<16>(x, a, b);
    x = a + b;
    lane_pair<32>(x, a, b);
    return a + b;
}

template <bool STREAM, typename V>
__device__ __forceinline__ V load(const V *p) {
    return STREAM ? __builtin_nontemporal_load(p) : *p;
}

// Operands of one tile.  kVe elements of a value row per lane.
template <int D, bool BF16, bool STREAM>
struct Tile {
    static constexpr int kVe = D / 16;
    static constexpr int kSteps = BF16 ? (D + 31) / 32 : D / 16;   // 16-byte loads of a key row per lane
    static constexpr int kVw = kVe * (BF16 ? 2 : 4) / 4;            // 4-byte words of a value row per lane (0: 2 bytes)
    static constexpr int kVwords = kVw ? kVw : 1;
    u32x4_t k[2][kSteps];
    uint32_t v[8][kVwords];

    // element e of the values of lane row x (0..15) is dim dim_of(e, x)
    static __device__ __forceinline__ int dim_of(int e, int x) {
        return !BF16 && D >= 64 ? (e / 4) * 64 + x * 4 + e % 4 : x * kVe + e;
    }
    // row: the lane's key row
    __device__ __forceinline__ void load_k(int kb, const unsigned char *row, int g) {
        if constexpr (BF16 && D == 16) {   // the upper half meets zeros of the queries: it has to be finite
            k[kb][0] = load<STREAM>(reinterpret_cast<const u32x4_t *>(row) + (g & 1));
            if (g >= 2) k[kb][0] = u32x4_t{0u, 0u, 0u, 0u};
        } else {
#pragma unroll
            for (int s = 0; s < kSteps; ++s) k[kb][s] = load<STREAM>(reinterpret_cast<const u32x4_t *>(row) + 4 * s + g);
        }
    }
    __device__ __forceinline__ void load_v(int j, const unsigned char *row, int n) {
        if constexpr (kVw == 0) {
            v[j][0] = load<STREAM>(reinterpret_cast<const uint16_t *>(row) + n);
        } else if constexpr (kVw == 1) {
            v[j][0] = load<STREAM>(reinterpret_cast<const uint32_t *>(row) + n);
        } else if constexpr (kVw == 2) {
            const auto x = load<STREAM>(reinterpret_cast<const unsigned long long *>(row) + n);
            v[j][0] = (uint32_t)x, v[j][1] = (uint32_t)(x >> 32);
        } else {
#pragma unroll
            for (int c = 0; c < kVw / 4; ++c) {
                const u32x4_t x = load<STREAM>(reinterpret_cast<const u32x4_t *>(row) + 16 * c + n);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j][4 * c + i] = x[i];
            }
        }
    }
    // element e of the lane's j-th key's values
    __device__ __forceinline__ float value(int j, int e) const {
        if constexpr (!BF16) return __uint_as_float(v[j][e]);
        else return __uint_as_float(e % 2 ? v[j][e / 2] & 0xffff0000u : v[j][e / 2] << 16);
    }
    __device__ __forceinline__ void drop_unless_finite(int j, int e) {
        if (fabsf(value(j, e)) < INFINITY) return;
        if constexpr (!BF16) v[j][e] = 0u;
        else v[j][e / 2] &= e % 2 ? 0xffffu : 0xffff0000u;
    }
    // scores of head n for the keys 16 kb + 4 g + i
    __device__ __forceinline__ f32x4_t scores(int kb, const u32x4_t *q) const {
        f32x4_t sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            if constexpr (BF16) {
                sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k[kb][s]),
                                                             __builtin_bit_cast(bf16x8_t, q[s]), sc, 0, 0, 0);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    sc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[kb][s][i]), __uint_as_float(q[s][i]), sc,
                                                              0, 0, 0);
            }
        }
        return sc;
    }
    // o += V^T P^T, p[j] the weight of head n and the lane's j-th key
    __device__ __forceinline__ void accumulate(const f32x8_t &p, f32x4_t *o) const {
        if constexpr (BF16) {
            u32x4_t part[3];   // of the eight weights: eight bits of each and a part, cut off
            f32x8_t left = p;
#pragma unroll
            for (int s = 0; s < 3; ++s) {
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    part[s][x] = __builtin_amdgcn_perm(__float_as_uint(left[2 * x + 1]), __float_as_uint(left[2 * x]), 0x07060302u);
                if (s < 2) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) left[j] -= __uint_as_float(__float_as_uint(left[j]) & 0xffff0000u);
                }
            }
#pragma unroll
            for (int e = 0; e < kVe; ++e) {
                u32x4_t a;   // element e of the eight keys
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    a[x] = __builtin_amdgcn_perm(v[2 * x + 1][e / 2], v[2 * x][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int s = 0; s < 3; ++s)
                    o[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                                   __builtin_bit_cast(bf16x8_t, part[s]), o[e], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
#pragma unroll
                for (int e = 0; e < kVe; ++e)
                    o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[j][e]), p[j], o[e], 0, 0, 0);
            }
        }
    }
};

// The states of cut rows go past the caches, which the chip's eight L2s do not
// keep coherent for ordinary accesses: these are, one by one.  (Ordinary ones
// between release and acquire fences write back and invalidate a whole L2 per
// chunk: 64 ragged rows of some 2000 positions took 314 us in place of 115.)
__device__ __forceinline__ void put(float *p, float x) {
    __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float get(const float *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// exp2 of m - top, where m == -inf has no weight whatever top is.
__device__ __forceinline__ float weight(float m, float top) {
    return __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
}

template <bool BF16>
__device__ __forceinline__ void store_out(unsigned char *out, size_t i, float x) {
    if constexpr (BF16) reinterpret_cast<uint16_t *>(out)[i] = __builtin_bit_cast(uint16_t, (__bf16)x);
    else reinterpret_cast<float *>(out)[i] = x;
}

// Joins the waves' states of one head: element d of the output, the maximum and
// the sum (negative: no position at all).
template <typename Load>
__device__ __forceinline__ void join(Load load, float &o, float &m, float &l) {
    m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) m = fmaxf(m, load(i, 1));
    o = 0.f, l = -1.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        const float li = load(i, 2), w = weight(load(i, 1), m);
        if (!(li < 0.f)) l = (l < 0.f ? 0.f : l) + li * w, o += load(i, 0) * w;
    }
}

}  // namespace
}  // namespace fs
