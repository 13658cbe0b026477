// Rows of one head of one token (16 to 512 elements of 16 bits) on lanes: what the norm and the rotation share
// between their own kernels and the cache's.
//
// A row lies on LPR lanes, a lane holds two 16-byte chunks A and B of it (a unit).  For the rotated pairs (j, j + rotary/2)
// these are the two chunks that belong together, so a rotation needs no exchange between lanes:
//     unit u < rotary/16:  A = u, B = u + rotary/16           (chunks of eight elements)
//     the units behind:    A = rotary/8 + 2 (u - rotary/16), B = A + 1
// Pairs (2j, 2j + 1) lie within a chunk and go by the same units.  A load of the lanes of a row reads 16 LPR contiguous bytes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mcf_internal.h"

namespace mcf {
namespace heads {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <typename T> union Chunk { // 16 bytes
    u32x4 bits;
    T e[8];
};

// floor(n / d) by division_magic's constants, n < 2^31
__device__ __forceinline__ uint32_t quotient(uint32_t n, uint32_t magic, int shift) { return magic ? __umulhi(n, magic) >> shift : n; }

template <int CTRL> __device__ __forceinline__ float dpp(float x) {
    return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ double dpp(double x) {
    const uint64_t b = __double_as_longlong(x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (uint32_t)b, CTRL, 0xf, 0xf, true);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (uint32_t)(b >> 32), CTRL, 0xf, 0xf, true);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}
// Sum (or maximum) over the LPR lanes of a row, in every one of them: exchanges within four lanes, mirrors of eight and
// sixteen (whose other half holds one value by then), and a shuffle across sixteen.
template <int LPR, typename F, typename Op> __device__ __forceinline__ F over_row(F x, Op op) {
    static_assert(LPR == 4 || LPR == 8 || LPR == 16 || LPR == 32, "");
    x = op(x, dpp<0xB1>(x));
    x = op(x, dpp<0x4E>(x));
    if constexpr (LPR >= 8) x = op(x, dpp<0x141>(x));
    if constexpr (LPR >= 16) x = op(x, dpp<0x140>(x));
    if constexpr (LPR >= 32) x = op(x, __shfl_xor(x, 16));
    return x;
}
template <int LPR, typename F> __device__ __forceinline__ F row_sum(F x) {
    return over_row<LPR>(x, [](F a, F b) { return a + b; });
}

// Where a lane's unit lies in its row.
struct Unit {
    int a, b;     // element offsets of the chunks
    bool there;   // the row has this unit (sizes that are no power of two leave lanes idle)
    bool turns;   // the unit is rotated
    __device__ __forceinline__ Unit(int u, int size, int rotary) {
        const int r = rotary >> 4;
        there = u < size >> 4;
        turns = u < r;
        a = 8 * (turns ? u : 2 * r + 2 * (u - r));
        b = turns ? a + 8 * r : a + 8;
        if (!there) a = b = 0;
    }
};

// Cosines and sines of a lane's eight pairs (pair e of the unit); NaN where the position is outside of the tables.
struct Turn {
    float c[8], s[8];
    __device__ __forceinline__ void load(const float *cos, const float *sin, int64_t position, int64_t table_rows, int rotary, const Unit &u, bool interleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = s[e] = __builtin_nanf("");
        if (!u.turns || position < 0 || position >= table_rows) return;
        const int64_t row = position * (rotary >> 1);
        const int first = interleaved ? u.a >> 1 : u.a, second = interleaved ? u.b >> 1 : u.a + 4;
        const f32x4 c0 = *(const f32x4 *)(cos + row + first), c1 = *(const f32x4 *)(cos + row + second);
        const f32x4 s0 = *(const f32x4 *)(sin + row + first), s1 = *(const f32x4 *)(sin + row + second);
#pragma unroll
        for (int e = 0; e < 4; ++e) { c[e] = c0[e]; c[4 + e] = c1[e]; s[e] = s0[e]; s[4 + e] = s1[e]; }
    }
    // (a, b) of every pair by the angle, or (BACK) by its negative
    template <bool BACK, typename F> __device__ __forceinline__ void turn(F a[8], F b[8], bool interleaved) const {
        F x[8], y[8];
        if (interleaved) {
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[j] = a[2 * j]; y[j] = a[2 * j + 1]; x[4 + j] = b[2 * j]; y[4 + j] = b[2 * j + 1]; }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) { x[e] = a[e]; y[e] = b[e]; }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            // (the rounding of each is written out: whoever turns a row gets the same bits)
            const F sn = BACK ? -(F)s[e] : (F)s[e], cs = (F)c[e], t = x[e];
            x[e] = __builtin_elementwise_fma(t, cs, -(y[e] * sn));
            y[e] = __builtin_elementwise_fma(y[e], cs, t * sn);
        }
        if (interleaved) {
#pragma unroll
            for (int j = 0; j < 4; ++j) { a[2 * j] = x[j]; a[2 * j + 1] = y[j]; b[2 * j] = x[4 + j]; b[2 * j + 1] = y[4 + j]; }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) { a[e] = x[e]; b[e] = y[e]; }
        }
    }
};

// A lane's sixteen weights.
template <typename T> __device__ __forceinline__ void load_weight(const void *w, bool f32, const Unit &u, float wa[8], float wb[8]) {
    if (f32) {
#pragma unroll
        for (int e = 0; e < 8; ++e) { wa[e] = ((const float *)w)[u.a + e]; wb[e] = ((const float *)w)[u.b + e]; }
    } else {
        Chunk<T> a, b;
        a.bits = *(const u32x4 *)((const T *)w + u.a);
        b.bits = *(const u32x4 *)((const T *)w + u.b);
#pragma unroll
        for (int e = 0; e < 8; ++e) { wa[e] = (float)a.e[e]; wb[e] = (float)b.e[e]; }
    }
}

// A row's norm: its elements times 1 / sqrt(mean of squares + eps) and the weights.
template <int LPR> __device__ __forceinline__ void norm_row(float a[8], float b[8], const float wa[8], const float wb[8], float inv_size, float eps) {
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(b[e], b[e], __builtin_fmaf(a[e], a[e], sum));
    const float r = 1.0f / sqrtf(__builtin_fmaf(row_sum<LPR>(sum), inv_size, eps));
#pragma unroll
    for (int e = 0; e < 8; ++e) { a[e] = a[e] * r * wa[e]; b[e] = b[e] * r * wb[e]; }
}

// Lanes that a row lies on.
inline int row_lanes(int64_t size) { return size <= 64 ? 4 : size <= 128 ? 8 : size <= 256 ? 16 : 32; }

// An mcf_rows argument: null pointers, alignment, strides that the kernels' 64-bit offsets hold; `written`: rows must not
// lie on top of one another.
inline int check_rows(const mcf_rows &r, int64_t batch, int64_t tokens, int64_t n_heads, int64_t size, bool written) {
    if (batch == 0 || tokens == 0 || n_heads == 0) return MCF_OK;
    if (!r.data) return MCF_EINVAL;
    if ((uintptr_t)r.data % 16 != 0) return MCF_EALIGN;
    int64_t extent[3] = {batch, tokens, n_heads}, stride[3] = {r.stride[0], r.stride[1], r.stride[2]};
    for (int d = 0; d < 3; ++d) {
        if (extent[d] == 1) { stride[d] = 0; continue; }
        if (stride[d] < 0) return MCF_EINVAL;
        if (stride[d] % 8 != 0) return MCF_EALIGN;
        if (stride[d] >= (1ll << 60) / extent[d]) return MCF_EUNSUPPORTED;
    }
    if (!written) return MCF_OK;
    for (int i = 0; i < 3; ++i) // ascending strides: each dimension steps over what the ones below it cover
        for (int j = i + 1; j < 3; ++j)
            if (extent[j] > 1 && (extent[i] == 1 || stride[j] < stride[i])) {
                int64_t t = stride[i]; stride[i] = stride[j]; stride[j] = t;
                t = extent[i]; extent[i] = extent[j]; extent[j] = t;
            }
    int64_t covered = size;
    for (int d = 0; d < 3; ++d) {
        if (extent[d] == 1) continue;
        if (stride[d] < covered) return MCF_EINVAL;
        covered = stride[d] * (extent[d] - 1) + covered;
    }
    return MCF_OK;
}

inline int check_tables(int64_t rotary, int64_t size, int64_t table_rows, const void *cos, const void *sin) {
    if (rotary < 0 || rotary > size || rotary % 16 != 0 || table_rows < 0) return MCF_EINVAL;
    if (rotary > 0 && table_rows > 0 && (!cos || !sin)) return MCF_EINVAL;
    if ((uintptr_t)cos % 16 != 0 || (uintptr_t)sin % 16 != 0) return MCF_EALIGN;
    if (table_rows > (1ll << 50)) return MCF_EUNSUPPORTED;
    return MCF_OK;
}

} // namespace heads
} // namespace mcf
