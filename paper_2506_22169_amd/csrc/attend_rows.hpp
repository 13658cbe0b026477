// Attention of few rows over the paged cache of 8 bits: single tokens and a few at once (attend.hpp says how the work is laid out).
//
// A block of four waves takes a tile of 16 NB rows and a chunk of tokens, each wave 32 tokens at a time:
//     S^T = K Q^T   v_mfma 16x16x32, K as its first operand: lane (i, g) = (lane % 16, lane / 16) holds 8 elements of token i
//     O^T += V^T P^T   the same instruction, contracting 32 tokens: lane (i, g) holds 8 tokens of column i
// Bound by the cache's bytes: 2 size bytes a token against 4 size flops a row and token, so that up to some 100 rows the
// matrix instructions wait.  Hence everything goes from memory to registers once, with no LDS between:
//  - the scores of S^T's result layout (lane: row i, tokens 4g .. 4g + 3 of each 16) are P^T's operand as they are, if the
//    contraction counts tokens in that order; V is read for the same tokens.
//  - V's operand wants 8 tokens of one column in a lane, memory has columns side by side: a lane reads size / 16 neighbouring
//    columns of each of its 8 tokens (whole rows over the 16 lanes) and turns bytes in registers (v_perm); column i of
//    product j is then column (size / 16) i + j of V, which leaves a lane with neighbouring columns of the result.
//  - e4m3 -> 16 bit is exact; the scale of K multiplies the scores in fp32.
// Measured: 64 sequences of up to 8192 tokens, 32 heads on 8 of 128, bf16 (529 MB), 104 us, 5.1 TB/s (a large copy: 5.15), of which the
// joining kernel is 5; with 5 rows of 8 heads each against 130000 tokens of 64 (33 MB, tiles of 48 rows) 25 us, of which 14 are what 1000 tokens take (two
// launches, their chains of loads, 256 parts a tile to join) and another 130000 tokens are 7, 4.6 TB/s; vector instructions take 53 % of the SIMDs' cycles
// and waves wait for 42 % of theirs.  4 sequences of 1000 tokens: 11.5 us, of which 5 are the call; the rest are
// dependent loads (sequence, table, values) and the second launch.
//
// Weights.  The power of two of V's scale is in V, where the widening instruction takes it; what is left of the scale (its mantissa; fp16: also what is
// beyond the powers that its range holds) is an exponent like the score's: w = 2^(s + log2 rest - m), m the running reference of these sums,
// and the sum of the softmax adds w / rest.  So the largest weight stands near 1, and pages under scales far apart have weights of all bits beside one another.
// Each weight is rounded once.  The reference moves only when a score outgrows it by 2^8.  Scales of K are not negative.
//
// Rows see prefixes of the tokens.  What no row of the tile sees is read as zero; where only some see a token whose value is NaN
// (0 NaN would be NaN for the others), its column's NaN are counted by a matrix product with who sees them.
// A query that is not finite is computed as zeros, whose sum says whether it sees any token (its scores would be NaN, or all of them -inf,
// where there is none): the check costs 0.1 us of 11.4 with 4 single tokens of 128, 0.4 of 8.2 with 7 of 256.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "attend.hpp"

namespace mcf {
namespace attend {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Mma;
template <> struct Mma<_Float16> {
    typedef f16x8 v8;
    static __device__ __forceinline__ f32x4 run(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ uint32_t lo(uint32_t x, float s) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, s, false)); }
    static __device__ __forceinline__ uint32_t hi(uint32_t x, float s) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, s, true)); }
};
template <> struct Mma<__bf16> {
    typedef bf16x8 v8;
    static __device__ __forceinline__ f32x4 run(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ uint32_t lo(uint32_t x, float s) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, false)); }
    static __device__ __forceinline__ uint32_t hi(uint32_t x, float s) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, true)); }
};
// Eight e4m3 values (in the order of their bytes) as an operand, four times the power of two of sa, four that of sb.
template <typename T> __device__ __forceinline__ typename Mma<T>::v8 widen(uint32_t a, uint32_t b, float sa = 1.f, float sb = 1.f) {
    const u32x4 w = {Mma<T>::lo(a, sa), Mma<T>::hi(a, sa), Mma<T>::lo(b, sb), Mma<T>::hi(b, sb)};
    return __builtin_bit_cast(typename Mma<T>::v8, w);
}

// The largest over the four lanes that hold one row.
__device__ __forceinline__ float over_groups(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Byte i of four words as one word, for i = 0 .. 3.
__device__ __forceinline__ void turn_bytes(uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3, uint32_t y[4]) {
    const uint32_t a = __builtin_amdgcn_perm(x1, x0, 0x05010400), b = __builtin_amdgcn_perm(x1, x0, 0x07030602);
    const uint32_t c = __builtin_amdgcn_perm(x3, x2, 0x05010400), d = __builtin_amdgcn_perm(x3, x2, 0x07030602);
    y[0] = __builtin_amdgcn_perm(c, a, 0x05040100);
    y[1] = __builtin_amdgcn_perm(c, a, 0x07060302);
    y[2] = __builtin_amdgcn_perm(d, b, 0x05040100);
    y[3] = __builtin_amdgcn_perm(d, b, 0x07060302);
}

// Columns of V in a lane: 4 (size / 64) of the first 64 (size / 64), and (size % 64) / 16 of the rest.
template <int D> struct Cols {
    static constexpr int words = D / 64, rest = D % 64 / 16; // rest: 0, 1 or 2 bytes, in a word of their own
    static constexpr int regs = words + (rest ? 1 : 0), tiles = 4 * words + rest;
    // column of product j of lane i
    static __device__ __forceinline__ int of(int i, int j) { return j < 4 * words ? 4 * words * i + j : 64 * words + rest * i + (j - 4 * words); }
};

template <int D> struct Step { // 32 tokens of K and V in registers
    static constexpr bool wide = D % 64 == 0;         // K in 16-byte pieces (two contraction steps each), else 8
    static constexpr int steps = (D + 31) / 32;
    uint32_t k[2][2 * steps];
    uint32_t v[8][Cols<D>::regs];
    float sk[2], sv[2];
    float hide[2]; // -inf: these 16 tokens are not there (K, V and K's scale are zeros then)
};

template <typename T, int D, int NB> struct Rows {
    typedef typename Mma<T>::v8 v8;
    typedef Cols<D> C;
    static constexpr int R = 16 * NB, steps = Step<D>::steps;
    static constexpr bool f16 = std::is_same<T, _Float16>::value;

    // element of the contraction that lane group g holds first in step s (8 of them; both operands alike)
    static __device__ __forceinline__ int part(int s, int g) { return Step<D>::wide ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g; }

    // The table's entries for the 32 tokens from t, as they stand there: asked for a step before they are looked at.
    static __device__ __forceinline__ void look_up(const Params &p, const int32_t *table, int t, int seen, int id[2]) {
#pragma unroll
        for (int j = 0; j < 2; ++j) id[j] = table[(t + 16 * j < seen ? t + 16 * j : seen - 1) >> p.page_log];
    }
    static __device__ __forceinline__ void load(const Params &p, int h, int t, int seen, const int ids[2], Step<D> &x) {
        const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int at = t + 16 * j, id = __builtin_amdgcn_readfirstlane(ids[j]);
            const bool there = at < seen && id >= 0 && id < p.pages;
            x.hide[j] = there ? 0.f : -INFINITY;
            if (!there) {
                x.sk[j] = 0.f;
                x.sv[j] = 1.f;
#pragma unroll
                for (int e = 0; e < 2 * steps; ++e) x.k[j][e] = 0;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < C::regs; ++e) x.v[4 * j + r][e] = 0;
                continue;
            }
            x.sk[j] = p.k_scale[id * p.ks_page + h];
            x.sv[j] = p.v_scale[id * p.vs_page + h];
            const int place = at & ((1 << p.page_log) - 1);
            const uint8_t *k = p.k + id * p.k_page + h * p.k_head + (place + i) * D;
            if constexpr (Step<D>::wide) {
#pragma unroll
                for (int s = 0; s < steps; s += 2) {
                    const u32x4 w = *(const u32x4 *)(k + part(s, g));
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.k[j][2 * s + e] = w[e];
                }
            } else {
#pragma unroll
                for (int s = 0; s < steps; ++s) {
                    const bool in = D % 32 == 0 || part(s, g) < D;
                    const u32x2 w = *(const u32x2 *)(k + (in ? part(s, g) : 0));
                    x.k[j][2 * s] = in ? w[0] : 0;
                    x.k[j][2 * s + 1] = in ? w[1] : 0;
                }
            }
            const uint8_t *v = p.v + id * p.v_page + h * p.v_head + (place + 4 * g) * D;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const uint32_t *w = (const uint32_t *)(v + r * D) + C::words * i;
#pragma unroll
                for (int e = 0; e < C::words; ++e) x.v[4 * j + r][e] = w[e];
                if constexpr (C::rest == 1) x.v[4 * j + r][C::words] = v[r * D + 64 * C::words + i];
                if constexpr (C::rest == 2) x.v[4 * j + r][C::words] = *(const uint16_t *)(v + r * D + 64 * C::words + 2 * i);
            }
        }
    }

    // f(first operand, j) for every product j: 8 tokens of column Cols::of(lane, j)
    template <typename F> static __device__ __forceinline__ void each_product(const uint32_t v[8][C::regs], float s0, float s1, F f) {
#pragma unroll
        for (int w = 0; w < C::regs; ++w) {
            uint32_t lo[4], hi[4];
            turn_bytes(v[0][w], v[1][w], v[2][w], v[3][w], lo);
            turn_bytes(v[4][w], v[5][w], v[6][w], v[7][w], hi);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (4 * w + e < C::tiles) f(widen<T>(lo[e], hi[e], s0, s1), 4 * w + e);
        }
    }

    struct State {
        v8 q[NB][steps];
        f32x4 o[NB][C::tiles];
        float m[NB], l[NB]; // reference (-inf: nothing seen) and this lane's part of the sum
        int limit[NB];
        float c; // |scale| log2(e): a negative scale turns the queries' signs
    };

    // 32 tokens from t; HIDE: some of them some row does not see (none sees those from `end` on, all see those below `all`)
    template <bool HIDE> static __device__ __forceinline__ void step(const Params &p, Step<D> &x, int t, int end, int all, State &st) {
        const int lane = threadIdx.x & 63, g = lane >> 4;
        v8 pw[NB];
        // factor and addend of the scores, V's factor, and the reciprocal of what V's scale has in the weights
        float f[2], add[2], inv[2], sv[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t bits = __builtin_amdgcn_readfirstlane(__float_as_uint(x.sv[j])), rest = scale_in_weights<f16>(bits);
            sv[j] = __uint_as_float(scale_in_v<f16>(bits));
            f[j] = st.c * x.sk[j];
            if (f[j] < 0x1p-126f) f[j] = 0x1p-126f; // (zero would make NaN of the -inf that hides a token)
            add[j] = x.hide[j] + ((x.sk[j] - x.sk[j]) + (x.sv[j] - x.sv[j])); // (NaN for whoever sees a page whose scale is not finite)
            inv[j] = 1.f;
            if ((rest & 0x7fffff) != 0) { // no power of two
                add[j] += __builtin_amdgcn_logf(__uint_as_float(rest));
                inv[j] = __builtin_amdgcn_rcpf(__uint_as_float(rest));
            } else if (f16) {
                add[j] += (float)((int)(rest >> 23) - 127);
                inv[j] = __uint_as_float((254 - (rest >> 23)) << 23);
            }
        }
        f32x4 sc[NB][2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int n = 0; n < NB; ++n) sc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < steps; ++c) {
                const v8 a = widen<T>(x.k[j][2 * c], x.k[j][2 * c + 1]);
#pragma unroll
                for (int n = 0; n < NB; ++n) sc[n][j] = Mma<T>::run(a, st.q[n][c], sc[n][j]);
            }
            if (HIDE && __any(add[j] != add[j])) { // NaN in the scores, so that rows that do not see them can be told apart
                f[j] = sv[j] = inv[j] = 1.f;
                add[j] = 0.f;
#pragma unroll
                for (int n = 0; n < NB; ++n) sc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f} + __builtin_nanf("");
            }
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            f32x4 (&s)[2] = sc[n];
            float most = -INFINITY;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                if (HIDE) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[j][r] = t + 16 * j + 4 * g + r >= st.limit[n] ? -INFINITY : s[j][r];
                }
                most = fmaxf(most, __builtin_fmaf(fmaxf(fmaxf(s[j][0], s[j][1]), fmaxf(s[j][2], s[j][3])), f[j], add[j]));
            }
            most = over_groups(most);
            if (__any(most > st.m[n] + 8.f)) {
                const float m = fmaxf(most, st.m[n]);
                const float by = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.m[n] - m);
                st.m[n] = m;
                st.l[n] *= by;
#pragma unroll
                for (int c = 0; c < C::tiles; ++c) st.o[n][c] *= by;
            }
            const float m = st.m[n] == -INFINITY ? 0.f : st.m[n];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j][r], f[j], add[j] - m));
                    st.l[n] = __builtin_fmaf(w, inv[j], st.l[n]);
                    pw[n][4 * j + r] = (T)w;
                }
        }
        if constexpr (HIDE) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool seen = t + 16 * (e >> 2) + 4 * g + (e & 3) < end;
#pragma unroll
                for (int w = 0; w < C::regs; ++w) x.v[e][w] = seen ? x.v[e][w] : 0;
            }
            if (end > all) {
                bool nan = false;
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int w = 0; w < C::regs; ++w) nan |= (((x.v[e][w] & 0x7f7f7f7f) + 0x01010101) & 0x80808080) != 0;
                if (__any(nan)) count_nans(x, t, st);
            }
        }
        each_product(x.v, sv[0], sv[1], [&](const v8 &a, int j) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < NB; ++n) st.o[n][j] = Mma<T>::run(a, pw[n], st.o[n][j]);
        });
    }

    // Takes the NaN out of V and gives them to the rows that see them.
    static __device__ __forceinline__ void count_nans(Step<D> &x, int t, State &st) {
        const int g = (threadIdx.x & 63) >> 4;
        uint32_t ones[8][C::regs];
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int w = 0; w < C::regs; ++w) {
                const uint32_t at = (((x.v[e][w] & 0x7f7f7f7f) + 0x01010101) & 0x80808080) >> 7;
                ones[e][w] = at * 0x38; // 1 in e4m3
                x.v[e][w] &= ~(at * 0xff);
            }
        v8 sees[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 8; ++e) sees[b][e] = t + 16 * (e >> 2) + 4 * g + (e & 3) < st.limit[b] ? (T)1.f : (T)0.f;
        each_product(ones, 1.f, 1.f, [&](const v8 &a, int j) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const f32x4 n = Mma<T>::run(a, sees[b], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int r = 0; r < 4; ++r) st.o[b][j][r] = n[r] > 0.f ? __builtin_nanf("") : st.o[b][j][r];
            }
        });
    }
};

// The rows of one tile over its tokens from .. to - 1 (as far as it sees any); part < 0: all of them, the result is written; else what
// they give goes to that place of the workspace.
template <typename T, int D, int NB, int WAVES> __device__ __forceinline__ void tile_part(const Params &p, const Sequence &s, int b, int h, uint32_t tile, int from, int to, int part_at) {
    typedef Rows<T, D, NB> K;
    typedef Cols<D> C;
    constexpr int R = K::R, pitch = D + 4, stride = 32 * WAVES;
    const int rows = s.rows * p.group - (int)tile * R; // of this tile, of R
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    const auto token_of = [&](int r) __attribute__((always_inline)) { return (int)quotient(tile * R + r, p.group_magic, p.group_shift); };
    const int last = limit_of(p, s, token_of(rows < R ? rows - 1 : R - 1)), all = limit_of(p, s, token_of(0));
    const int end = to < last ? to : last;

    // The first entries of the table, the queries and the first keys and values, each asked for before anything waits.
    const int32_t *const table = p.seq.table + b * p.seq.table_stride;
    int t = (from < end ? from : end) + 32 * wave, id[2];
    const int plain = all < end ? all : end; // every row sees the tokens below
    if (t < end) K::look_up(p, table, t, s.seen, id);
    typename K::State st;
    u32x4 q[NB][K::steps];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const int r = 16 * n + i < rows ? 16 * n + i : 0, tk = token_of(r), head = tile * R + r - tk * p.group;
        st.limit[n] = 16 * n + i < rows ? limit_of(p, s, tk) : s.seen; // (rows that pad the tile hide nothing)
        const T *at = (const T *)p.q + (int64_t)(s.first + tk) * p.qt + (int64_t)(h * p.group + head) * p.qh;
#pragma unroll
        for (int c = 0; c < K::steps; ++c) q[n][c] = *(const u32x4 *)(at + (D % 32 == 0 || K::part(c, g) < D ? K::part(c, g) : 0));
    }
    Step<D> x;
    const bool many = t + 32 <= plain;
    if (many) {
        K::load(p, h, t, s.seen, id, x);
        K::look_up(p, table, t + stride, s.seen, id);
    }
    st.c = fabsf(p.c);
    const uint32_t sign = p.c < 0.f ? 0x80008000u : 0u;
    // A query that is not finite counts as zeros until its sum is known: NaN if it sees any token.
    bool lost[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        st.m[n] = -INFINITY;
        st.l[n] = 0.f;
        u16x2 most = {0, 0};
#pragma unroll
        for (int c = 0; c < K::steps; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) most = larger_halves(most, q[n][c][e]);
        uint64_t rows_lost = __ballot(not_finite<K::f16>(most));
        rows_lost |= rows_lost >> 32;
        rows_lost |= rows_lost >> 16;
        lost[n] = rows_lost >> i & 1;
#pragma unroll
        for (int c = 0; c < K::steps; ++c) {
            const bool in = 16 * n + i < rows && !lost[n] && (D % 32 == 0 || K::part(c, g) < D);
            st.q[n][c] = __builtin_bit_cast(typename K::v8, in ? q[n][c] ^ sign : u32x4{0, 0, 0, 0});
        }
#pragma unroll
        for (int c = 0; c < C::tiles; ++c) st.o[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    if (many) {
        Step<D> next;
        for (;;) {
            const int u = t + stride;
            const bool more = u + 32 <= plain;
            if (more) {
                K::load(p, h, u, s.seen, id, next);
                K::look_up(p, table, u + stride, s.seen, id);
            }
            K::template step<false>(p, x, t, end, all, st);
            t = u;
            if (!more) break;
            x = next;
        }
    }
    for (; t < end; t += stride) {
        K::load(p, h, t, s.seen, id, x);
        K::look_up(p, table, t + stride, s.seen, id);
        K::template step<true>(p, x, t, end, all, st);
    }

    // The waves' parts: each scaled to the largest reference, then summed in the waves' order (of eight, the last four to the first four before).
    __shared__ float ref[WAVES][R], sum[WAVES][R];
    __shared__ float part[4][16 * pitch];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        st.l[n] += __shfl_xor(st.l[n], 16);
        st.l[n] += __shfl_xor(st.l[n], 32);
        if (lost[n] && st.l[n] != 0.f) st.l[n] = __builtin_nanf("");
        if (g == 0) { ref[wave][16 * n + i] = st.m[n]; sum[wave][16 * n + i] = st.l[n]; }
    }
    const auto top_of = [&](int r) __attribute__((always_inline)) {
        float m = ref[0][r];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m = fmaxf(m, ref[w][r]);
        return m;
    };
    const int64_t place = ((int64_t)part_at * p.heads + h) * p.part_rows;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        __syncthreads();
        const float by = st.m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st.m[n] - top_of(16 * n + i));
        const auto put = [&](float *to) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < C::tiles; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) to[i * pitch + C::of(4 * g + e, c)] = st.o[n][c][e];
        };
#pragma unroll
        for (int c = 0; c < C::tiles; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) st.o[n][c][e] = st.m[n] == -INFINITY ? 0.f : st.o[n][c][e] * by;
        if constexpr (WAVES == 8) {
            if (wave >= 4) put(part[wave - 4]);
            __syncthreads();
            if (wave < 4) {
#pragma unroll
                for (int c = 0; c < C::tiles; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) st.o[n][c][e] += part[wave][i * pitch + C::of(4 * g + e, c)];
            }
            __syncthreads();
        }
        if (wave < 4) put(part[wave]);
        __syncthreads();
        for (int at = threadIdx.x * 4; at < 16 * D; at += 256 * WAVES) {
            const int q = at / D, d = at - q * D, row = 16 * n + q;
            if (row >= rows) continue;
            f32x4 o = *(const f32x4 *)&part[0][q * pitch + d];
#pragma unroll
            for (int w = 1; w < 4; ++w) o += *(const f32x4 *)&part[w][q * pitch + d];
            const float top = top_of(row);
            float l = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) l += ref[w][row] == -INFINITY ? sum[w][row] : sum[w][row] * __builtin_amdgcn_exp2f(ref[w][row] - top); // (nothing seen: 0, or NaN by NaN scores)
            if (part_at >= 0) {
                *(f32x4 *)(p.part + (place + row) * D + d) = o;
                if (d == 0) { p.part_ml[2 * (place + row)] = top; p.part_ml[2 * (place + row) + 1] = l; }
            } else {
                const float inv = l == 0.f ? 0.f : 1.0f / l; // (0: a row that sees nothing)
                const int tk = token_of(row), head = tile * R + row - tk * p.group;
                typedef T T4 __attribute__((ext_vector_type(4)));
                T4 y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = (T)(o[e] * inv);
                *(T4 *)((T *)p.out + (int64_t)(s.first + tk) * p.ot + (int64_t)(h * p.group + head) * p.oh + d) = y;
            }
        }
    }
    __syncthreads(); // (the shared parts are free again)
}

// Eight waves: calls that are not split (a tile a block), of sequences short enough.
template <typename T, int D, int NB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(WAVES == 8 ? 2 : waves_per_simd(D, NB), WAVES == 8 ? 2 : waves_per_simd(D, NB)))) void rows_kernel(const Params p) {
    typedef Rows<T, D, NB> K;
    constexpr int R = K::R;
    const uint32_t j = blockIdx.x / (uint32_t)p.heads;
    const int h = (int)(blockIdx.x - j * p.heads);
    int b;
    uint32_t rest, at = 0, end = 1, piece = 1, tiles_before = 0, all_tiles = 0;
    Sequence s;
    Split split = {0, 0, 0, 0, 0, 0, 0, 0};
    if (p.split) {
        if (!find_piece<R>(p, j, &piece, &at, &end, &b, &rest, &s, &tiles_before, &all_tiles)) at = end = 0;
        if (p.by_tile && blockIdx.x == 0 && threadIdx.x == 0) *p.tiles = (int)all_tiles;
    } else { // tile j, as the one unit of a piece
        if (!locate(j, p.seq.batch, [&](int i) __attribute__((always_inline)) -> uint32_t { return tiles_of<R>(p, sequence(p.seq, i)); }, &b, &rest)) return;
        b = __builtin_amdgcn_readfirstlane(b);
        rest = __builtin_amdgcn_readfirstlane(rest);
        s = sequence(p.seq, b);
    }
    while (at < end) {
        const uint32_t units = p.split ? units_of(s) : 1, all = units * tiles_of<R>(p, s);
        while (rest < all && at < end) {
            const uint32_t tile = rest / units, x = rest - tile * units, n = units - x < end - at ? units - x : end - at;
            const int from = first_token(x), to = x + n == units ? 0x7fffffff : first_token(x + n);
            const bool whole = from == 0 && x + n == units;
            if (from < to) tile_part<T, D, NB, WAVES>(p, s, b, h, tile, from, to, whole ? -1 : (int)(2 * j + (from == 0)));
            if (from == 0 && to > 0) { // the first of one or more parts
                const int rows = s.rows * p.group - (int)tile * R;
                const Split first = {whole ? 0 : 1 + (int)((units - x - n + piece - 1) / piece), (int)(2 * j + 1), (int)(2 * j + 2), 2, s.first, (int)tile * R, rows < R ? rows : R, 0};
                if (!whole) split = first;
                // (starts that are not ascending can give more tiles than there is room for)
                if (p.by_tile && threadIdx.x == 0 && tiles_before + tile < p.slots) p.splits[(tiles_before + tile) * p.heads + h] = first;
            }
            rest += n;
            at += n;
        }
        if (at >= end) break;
        rest = 0;
        tiles_before += all / units;
        if (++b >= p.seq.batch) break;
        s = sequence(p.seq, b);
    }
    if (p.split && !p.by_tile && threadIdx.x == 0) p.splits[blockIdx.x] = split;
}

template <typename T> int launch_rows(const Params &p, int size, int row_blocks, int waves, unsigned blocks, void *stream) {
    const auto go = [&](auto d) {
        constexpr int D = decltype(d)::value;
        const dim3 grid(blocks), block(64 * waves);
        hipStream_t st = (hipStream_t)stream;
        if (waves == 8) hipLaunchKernelGGL((rows_kernel<T, D, 1, 8>), grid, block, 0, st, p);
        else if (row_blocks == 1) hipLaunchKernelGGL((rows_kernel<T, D, 1, 4>), grid, block, 0, st, p);
        else if (row_blocks == 2) hipLaunchKernelGGL((rows_kernel<T, D, 2, 4>), grid, block, 0, st, p);
        else if constexpr (D <= 128) {
            if (row_blocks == 3) hipLaunchKernelGGL((rows_kernel<T, D, 3, 4>), grid, block, 0, st, p);
            else if constexpr (D <= 64) hipLaunchKernelGGL((rows_kernel<T, D, 4, 4>), grid, block, 0, st, p);
        }
    };
    switch (size) {
    case 64: go(std::integral_constant<int, 64>()); break;
    case 80: go(std::integral_constant<int, 80>()); break;
    case 96: go(std::integral_constant<int, 96>()); break;
    case 128: go(std::integral_constant<int, 128>()); break;
    case 192: go(std::integral_constant<int, 192>()); break;
    default: go(std::integral_constant<int, 256>()); break;
    }
    return (int)hipGetLastError();
}

} // namespace
} // namespace attend
} // namespace mcf
