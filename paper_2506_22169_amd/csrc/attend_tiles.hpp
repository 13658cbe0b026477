// Attention of many rows over the paged cache of 8 bits: prompts and pieces of prompts (attend.hpp says how the work is laid out).
//
// A block of W waves takes a tile of 32 W rows, each wave 32 of them, and goes over the tokens TN at a time:
//     S^T = K Q^T, O^T += V^T P^T   v_mfma 32x32x16; a lane holds one row, so that its softmax needs one exchange (with lane ^ 32),
//     and S^T's result layout is P^T's operand as it is, with the tokens counted in that order.
// Bound by the matrix instructions and, next to them, by the vector instructions of the softmax and the LDS reads of their
// operands.  Therefore
//  - K and V are widened from e4m3 once for a block (exactly; V with the power of two of its scale on the way) while they go
//    from registers to LDS, K as rows, V transposed, so that every operand is one 128-bit read; two tiles of LDS in turn, one
//    barrier a tile, the loads of the tile after next in flight meanwhile.
//  - V is transposed by bytes before it is widened: a lane has 4 tokens of 4 neighbouring columns.  Which column is which row of
//    an operand is free; the order taken (Columns) spreads the writes over the banks and leaves a lane with up to 16
//    neighbouring columns of the result.
//  - Padding of 16 bytes a row puts the rows of both on different banks.
// Measured: 4096 tokens of 32 heads on 8 of 128 behind 12288 (9.6e11 flop over the visible pairs), bf16, 885 to 960 us by the card, up to 1.09 PFLOP/s (a large matrix product:
// 1.34 to 1.40).  With parts left out, each alone: without staging 130 us less, without the LDS reads of operands 130 to 170, without the exponentials
// 75; the matrix instructions alone are some 550.  7 ragged prompts of up to 1500 tokens behind up to 100, 20 heads of 80, fp16: 67 us, 0.33 PFLOP/s:
// 580 blocks of 1 to 13 steps, one at a time on each of 256 units, whose begin and end nothing covers: waves wait for 46 % of their time.
//
// Weights and what rows do not see: as in attend_rows.hpp.  A NaN in V that only some
// rows of the tile see is taken out and its first token noted for its column; rows that see that token get NaN.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>
#include <type_traits>

#include "attend.hpp"

namespace mcf {
namespace attend {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Wide;
template <> struct Wide<_Float16> {
    typedef f16x8 v8;
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f32x16 run(v8 a, v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    template <bool HI> static __device__ __forceinline__ uint32_t two(uint32_t x, float s) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, s, HI));
    }
};
template <> struct Wide<__bf16> {
    typedef bf16x8 v8;
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f32x16 run(v8 a, v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    template <bool HI> static __device__ __forceinline__ uint32_t two(uint32_t x, float s) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, HI));
    }
};

// Four columns 4c .. 4c + 3 of V (a word of a row) as rows of its operand: 128 columns at a time are four operands, 64 two, then 32
// and 16 in the last.
template <int D> struct Columns {
    static constexpr int operands = (D + 31) / 32;
    static __device__ __forceinline__ int row(int c, int e) { // of column 4c + e
        const int part = c >> 5; // 128 columns
        if (D % 128 == 0 || 128 * part + 128 <= D) return 128 * part + 32 * e + (c & 31);
        const int base = D / 128 * 128, k = c - base / 4;
        if (D % 128 >= 64 && k < 16) return base + 32 * (e >> 1) + 2 * k + (e & 1);
        return base + (D % 128 >= 64 ? 64 : 0) + 4 * (k - (D % 128 >= 64 ? 16 : 0)) + e;
    }
};

// The larger of a lane's value and that of lane ^ 32.
__device__ __forceinline__ float over_halves(float x) {
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}

// A barrier for what is in LDS: global loads stay in flight over it (__syncthreads() waits for them).
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <typename T, int D, int WAVES> struct Tiles {
    typedef typename Wide<T>::v8 v8;
    static constexpr bool f16 = std::is_same<T, _Float16>::value;
    static constexpr int TN = D <= 96 && WAVES == 8 ? 128 : D <= 128 ? 64 : 32, R = 32 * WAVES, threads = 64 * WAVES;
    static constexpr int blocks = TN / 32, groups = TN / 16, steps = D / 16, operands = Columns<D>::operands;
    static constexpr int k_pitch = 2 * D + 16, v_pitch = 2 * TN + 16; // bytes
    static constexpr int k_bytes = TN * k_pitch, v_bytes = 32 * operands * v_pitch;
    static constexpr int buffer = k_bytes + v_bytes + groups * 16; // and per 16 tokens: factor, addend, 1 / what V's scale has in the exponent
    static constexpr int k_units = TN * D / 16, v_units = TN * D / 16;
    static constexpr int per_thread = (k_units + threads - 1) / threads;
    static constexpr int lds = 2 * buffer + D * 4;
};

template <typename T, int D, int WAVES> __global__ __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, 2))) void tiles_kernel(const Params p) {
    typedef Tiles<T, D, WAVES> K;
    typedef typename K::v8 v8;
    constexpr int TN = K::TN, R = K::R, N = K::per_thread;
    extern __shared__ __align__(16) uint8_t lds[];
    int *const first_nan = (int *)(lds + 2 * K::buffer); // [D]: the first token whose value is NaN, of those that not all rows see
    const uint32_t slot = blockIdx.x / (uint32_t)p.heads;
    const int h = (int)(blockIdx.x - slot * p.heads);
    const int chunk = __builtin_amdgcn_readfirstlane(chunk_of<R>(p));
    int b;
    uint32_t tile, ch = 0, chunks = 1;
    Sequence s;
    if (!p.split && p.seq.batch <= 64) {
        if (!locate_longest<R>(p, slot, &b, &tile, &s)) return;
    } else {
        uint32_t rest;
        if (!locate_sequence(p.seq, slot, [&](const Sequence &q) __attribute__((always_inline)) -> uint32_t { return tiles_of<R>(p, q) * chunks_of(q, chunk); }, &b, &rest, &s)) {
            if (p.split && threadIdx.x == 0) p.splits[blockIdx.x].parts = 0;
            return;
        }
        rest = __builtin_amdgcn_readfirstlane(rest);
        chunks = chunks_of(s, chunk);
        tile = rest / chunks;
        ch = rest - tile * chunks;
        tile = tiles_of<R>(p, s) - 1 - tile; // the last rows, which see most, first
    }
    b = __builtin_amdgcn_readfirstlane(b);
    tile = __builtin_amdgcn_readfirstlane(tile);
    const int rows = s.rows * p.group - (int)tile * R < R ? s.rows * p.group - (int)tile * R : R;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i = lane & 31, g = lane >> 5;
    const auto token_of = [&](int r) __attribute__((always_inline)) { return (int)quotient(tile * R + r, p.group_magic, p.group_shift); };
    const int all = limit_of(p, s, token_of(0)), last = limit_of(p, s, token_of(rows - 1));
    const int64_t from64 = (int64_t)ch * chunk;
    const int end = from64 + chunk < last ? (int)from64 + chunk : last, from = from64 < end ? (int)from64 : end;
    const int plain = all < end ? all : end; // all rows see the tokens below
    if (p.split && tid == 0)
        p.splits[blockIdx.x] = {chunks > 1 && ch == 0 ? (int)chunks : 0, (int)slot, (int)slot + 1, 1, s.first, (int)tile * R, rows, 0};
    // this wave's and this lane's rows
    const int w0 = 32 * wave, row = w0 + i;
    const bool works = w0 < rows;
    const int wave_all = works ? limit_of(p, s, token_of(w0)) : 0, wave_last = works ? limit_of(p, s, token_of(w0 + 31 < rows ? w0 + 31 : rows - 1)) : 0;
    const bool real = row < rows;
    const int tok = token_of(real ? row : 0), head = (int)(tile * R) + (real ? row : 0) - tok * p.group;
    const int limit = real ? limit_of(p, s, tok) : s.seen;
    v8 q[K::steps];
    bool lost; // a query that is not finite: it counts as zeros until its sum is known, and gives NaN if it sees any token
    const float c_abs = fabsf(p.c); // (a negative scale turns the queries' signs)
    const uint32_t sign = p.c < 0.f ? 0x80008000u : 0u;
    {
        const T *src = (const T *)p.q + (int64_t)(s.first + tok) * p.qt + (int64_t)(h * p.group + head) * p.qh + 8 * g;
        u16x2 most = {0, 0};
        u32x4 w[K::steps];
#pragma unroll
        for (int c = 0; c < K::steps; ++c) {
            w[c] = *(const u32x4 *)(src + 16 * c);
#pragma unroll
            for (int e = 0; e < 4; ++e) most = larger_halves(most, w[c][e]);
        }
        uint64_t rows_lost = __ballot(not_finite<K::f16>(most));
        rows_lost |= rows_lost >> 32;
        lost = rows_lost >> i & 1;
#pragma unroll
        for (int c = 0; c < K::steps; ++c) q[c] = __builtin_bit_cast(v8, real && !lost ? w[c] ^ sign : u32x4{0, 0, 0, 0});
    }
    for (int d = tid; d < D; d += K::threads) first_nan[d] = 0x7fffffff;

    // ---- memory to registers to LDS ----
    const int32_t *const table = p.seq.table + b * p.seq.table_stride;
    const int in_page = (1 << p.page_log) - 1;
    int k_id[N], v_id[N], g_id = 0; // table entries for the tile to load next
    bool k_there[N], v_there[N], there = false;
    u32x4 kw[N];                    // 16 elements of a token
    uint32_t vw[N][4];              // 4 columns of 4 tokens
    float ks = 0.f, vs = 1.f, v_scale[N];
    int k_token[N], v_token[N], k_at[N], v_at[N]; // this lane's: tokens of a tile, offsets in a token
    const uint8_t *const k_head = p.k + h * p.k_head, *const v_head = p.v + h * p.v_head;
    const auto page = [&](const uint8_t *head, int id, int64_t stride) __attribute__((always_inline)) { return head + (uint64_t)(uint32_t)id * (uint32_t)stride; };
#pragma unroll
    for (int u = 0; u < N; ++u) { // (lanes beyond the last unit load that one again and store nothing)
        const int unit = K::k_units % K::threads != 0 && tid + u * K::threads >= K::k_units ? K::k_units - 1 : tid + u * K::threads;
        k_token[u] = unit / (D / 16);
        k_at[u] = unit % (D / 16) * 16;
        v_token[u] = unit / (D / 4) * 4;
        v_at[u] = unit % (D / 4) * 4;
    }
    // Nothing here waits for a load: entries are looked at when the loads of their tile are issued, a tile later, and what is not there
    // is read from the first page and dropped when it is stored.
    const auto entry = [&](int t) __attribute__((always_inline)) { return table[(t < s.seen ? t : s.seen - 1) >> p.page_log]; };
    const auto valid = [&](int t, int id) __attribute__((always_inline)) { return t < s.seen && (uint32_t)id < (uint32_t)p.pages; };
    const auto scale = [&](const float *scales, int id, int64_t stride) __attribute__((always_inline)) { return scales + h + (uint64_t)(uint32_t)id * (uint32_t)stride; };
    const auto look_up = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            k_id[u] = entry(t0 + k_token[u]);
            v_id[u] = entry(t0 + v_token[u]);
        }
        if (tid < K::groups) g_id = entry(t0 + 16 * tid);
    };
    const auto load = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < N; ++u) {
            k_there[u] = valid(t0 + k_token[u], k_id[u]);
            const int ki = k_there[u] ? k_id[u] : 0;
            kw[u] = *(const u32x4 *)(page(k_head, ki, p.k_page) + (((t0 + k_token[u]) & in_page) * D + k_at[u]));
            v_there[u] = valid(t0 + v_token[u], v_id[u]);
            const int vi = v_there[u] ? v_id[u] : 0;
            const uint8_t *v = page(v_head, vi, p.v_page) + (((t0 + v_token[u]) & in_page) * D + v_at[u]);
#pragma unroll
            for (int r = 0; r < 4; ++r) vw[u][r] = *(const uint32_t *)(v + r * D);
            v_scale[u] = *scale(p.v_scale, vi, p.vs_page);
        }
        if (tid < K::groups) {
            there = valid(t0 + 16 * tid, g_id);
            const int id = there ? g_id : 0;
            ks = *scale(p.k_scale, id, p.ks_page);
            vs = *scale(p.v_scale, id, p.vs_page);
        }
    };
    const auto scale_lost = [](float x) __attribute__((always_inline)) { return (__float_as_uint(x) & 0x7f800000) == 0x7f800000; };
    const auto store = [&](uint8_t *buf, int t0) __attribute__((always_inline)) {
        const bool hides = t0 + TN > plain;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (K::k_units % K::threads != 0 && tid + u * K::threads >= K::k_units) continue;
            if (__any(!k_there[u] || !v_there[u])) {
                if (!k_there[u]) kw[u] = u32x4{0, 0, 0, 0};
                if (!v_there[u]) {
                    v_scale[u] = 1.f;
#pragma unroll
                    for (int r = 0; r < 4; ++r) vw[u][r] = 0;
                }
            }
            {
                u32x4 lo, hi;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint32_t x = kw[u][e], y = kw[u][2 + e];
                    lo[2 * e] = Wide<T>::template two<false>(x, 1.f);
                    lo[2 * e + 1] = Wide<T>::template two<true>(x, 1.f);
                    hi[2 * e] = Wide<T>::template two<false>(y, 1.f);
                    hi[2 * e + 1] = Wide<T>::template two<true>(y, 1.f);
                }
                *(u32x4 *)(buf + k_token[u] * K::k_pitch + 2 * k_at[u]) = lo;
                *(u32x4 *)(buf + k_token[u] * K::k_pitch + 2 * k_at[u] + 16) = hi;
            }
            const int token = v_token[u], c = v_at[u] / 4;
            if (hides) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    uint32_t &x = vw[u][r];
                    if (t0 + token + r >= end) x = 0;
                    if (end <= all) continue; // (what is left all rows see)
                    const uint32_t nan = (((x & 0x7f7f7f7f) + 0x01010101) & 0x80808080) >> 7;
                    if (nan) {
                        x &= ~(nan * 0xff);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (nan >> (8 * e) & 1) atomicMin(first_nan + 4 * c + e, t0 + token + r);
                    }
                }
            }
            // bytes of a column together
            uint32_t y[4];
            const uint32_t a0 = __builtin_amdgcn_perm(vw[u][1], vw[u][0], 0x05010400), a1 = __builtin_amdgcn_perm(vw[u][1], vw[u][0], 0x07030602);
            const uint32_t a2 = __builtin_amdgcn_perm(vw[u][3], vw[u][2], 0x05010400), a3 = __builtin_amdgcn_perm(vw[u][3], vw[u][2], 0x07030602);
            y[0] = __builtin_amdgcn_perm(a2, a0, 0x05040100);
            y[1] = __builtin_amdgcn_perm(a2, a0, 0x07060302);
            y[2] = __builtin_amdgcn_perm(a3, a1, 0x05040100);
            y[3] = __builtin_amdgcn_perm(a3, a1, 0x07060302);
            // tokens 4t of 16 stand at 8 (t % 2) + 4 (t / 2), the order of S^T's result
            const int t = token >> 2, place = (token & ~15) + 8 * (t & 1) + 4 * ((t >> 1) & 1);
            uint8_t *const to = buf + K::k_bytes + 2 * place;
            const float sv = !K::f16 && scale_lost(v_scale[u]) ? 1.f : __uint_as_float(scale_in_v<K::f16>(__float_as_uint(v_scale[u])));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *(u32x2 *)(to + Columns<D>::row(c, e) * K::v_pitch) = u32x2{Wide<T>::template two<false>(y[e], sv), Wide<T>::template two<true>(y[e], sv)};
        }
        if (tid < K::groups) {
            const float v = !there ? 1.f : __uint_as_float(scale_in_weights<K::f16>(__float_as_uint(vs)));
            // (a factor of zero would make NaN of the -inf that hides a token; NaN for whoever sees a page whose scale is not finite)
            const bool bad = there && (scale_lost(ks) || scale_lost(vs));
            const f32x4 x = {!there || bad ? 1.f : ks * c_abs < 0x1p-126f ? 0x1p-126f : ks * c_abs, bad ? __builtin_nanf("") : there ? __builtin_amdgcn_logf(v) : -INFINITY,
                             __builtin_amdgcn_rcpf(v), 0.f};
            *(f32x4 *)(buf + K::k_bytes + K::v_bytes + 16 * tid) = x;
        }
    };

    // ---- a tile ----
    f32x16 o[K::operands];
#pragma unroll
    for (int c = 0; c < K::operands; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[c][r] = 0.f;
    float m = -INFINITY, l = 0.f;
    const auto compute = [&](const uint8_t *buf, int t0) __attribute__((always_inline)) {
        f32x16 sc[K::blocks];
        const uint8_t *kp = buf + i * K::k_pitch + 16 * g;
#pragma unroll
        for (int j = 0; j < K::blocks; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[j][r] = 0.f;
#pragma unroll
        for (int c = 0; c < K::steps; ++c)
#pragma unroll
            for (int j = 0; j < K::blocks; ++j) sc[j] = Wide<T>::run(*(const v8 *)(kp + 32 * j * K::k_pitch + 32 * c), q[c], sc[j]);
        // six operands on their way before the first product, then one more behind each
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
        for (int z = 0; z < K::blocks * K::steps - 6; ++z) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, 6, 0);
        f32x4 par[K::groups];
#pragma unroll
        for (int k = 0; k < K::groups; ++k) par[k] = *(const f32x4 *)(buf + K::k_bytes + K::v_bytes + 16 * k);
        if (t0 + TN > wave_all) { // (what is hidden is below everything under either sign of the scale)
            const int room = limit - t0 - 4 * g;
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < K::groups; ++k) sum += par[k][1];
            if (__builtin_expect(__any(sum != sum), 0)) { // NaN goes to the scores, so that rows that do not see them can be told apart
#pragma unroll
                for (int k = 0; k < K::groups; ++k) {
                    const bool nan = par[k][1] != par[k][1];
#pragma unroll
                    for (int r = 0; r < 8; ++r) sc[k / 2][8 * (k & 1) + r] = nan ? par[k][1] : sc[k / 2][8 * (k & 1) + r];
                    par[k][1] = nan ? 0.f : par[k][1];
                }
            }
#pragma unroll
            for (int j = 0; j < K::blocks; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) sc[j][r] = 32 * j + 8 * (r >> 2) + (r & 3) < room ? sc[j][r] : -INFINITY;
        }
        // the largest of each 16 tokens, which have one factor, then of all of them
        float most = -INFINITY;
#pragma unroll
        for (int k = 0; k < K::groups; ++k) {
            float x = fmaxf(sc[k / 2][8 * (k & 1)], sc[k / 2][8 * (k & 1) + 1]);
#pragma unroll
            for (int r = 2; r < 8; r += 2) x = fmaxf(fmaxf(sc[k / 2][8 * (k & 1) + r], sc[k / 2][8 * (k & 1) + r + 1]), x);
            most = fmaxf(most, __builtin_fmaf(x, par[k][0], par[k][1]));
        }
        most = over_halves(most);
        if (__any(most > m + 8.f)) {
            const float top = fmaxf(most, m), by = top == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - top);
            m = top;
            l *= by;
#pragma unroll
            for (int c = 0; c < K::operands; ++c)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[c][r] *= by;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        const uint8_t *vp = buf + K::k_bytes + i * K::v_pitch + 16 * g;
#pragma unroll
        for (int k = 0; k < K::groups; ++k) {
            v8 pw;
            const float add = par[k][1] - ref;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[k / 2][8 * (k & 1) + r], par[k][0], add));
                l = __builtin_fmaf(w, par[k][2], l);
                pw[r] = (T)w;
            }
#pragma unroll
            for (int c = 0; c < K::operands; ++c) o[c] = Wide<T>::run(*(const v8 *)(vp + 32 * c * K::v_pitch + 32 * k), pw, o[c]);
        }
    };

    if (from < end) {
        look_up(from);
        load(from);
        look_up(from + TN);
        lds_barrier(); // (first_nan)
        store(lds, from);
        load(from + TN);
        look_up(from + 2 * TN);
        lds_barrier();
        int turn = 0;
        for (int t0 = from; t0 < end; t0 += TN) {
            const auto stage = [&]() __attribute__((always_inline)) {
                if (t0 + TN < end) {
                    store(lds + (turn ^ 1) * K::buffer, t0 + TN);
                    load(t0 + 2 * TN);
                    look_up(t0 + 3 * TN);
                }
            };
            const bool early = wave & (WAVES / 2);
            if (early) stage();
            if (t0 < wave_last) compute(lds + turn * K::buffer, t0);
            if (!early) stage();
            turn ^= 1;
            lds_barrier();
        }
    } else {
        lds_barrier();
    }

    // ---- the result ----
    l += __shfl_xor(l, 32);
    if (!real) return;
    if (lost && l != 0.f) l = __builtin_nanf("");
    const bool whole = chunks == 1;
    const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.0f / l;
    const int64_t place = ((int64_t)slot * p.heads + h) * p.part_rows + row;
    if (!whole && g == 0) { p.part_ml[2 * place] = m; p.part_ml[2 * place + 1] = l; }
    T *const out = (T *)p.out + (int64_t)(s.first + tok) * p.ot + (int64_t)(h * p.group + head) * p.oh;
    // n neighbouring columns from d, their products o[c0 + x / per] at register r0 + x % per
    const auto put = [&](int d, auto count, auto value) __attribute__((always_inline)) {
        constexpr int n = decltype(count)::value;
        typedef T Tn __attribute__((ext_vector_type(n)));
        float x[n];
#pragma unroll
        for (int e = 0; e < n; ++e) {
            x[e] = value(e) * inv;
            if (end > all && first_nan[d + e] < limit) x[e] = __builtin_nanf("");
        }
        if (whole) {
            Tn y;
#pragma unroll
            for (int e = 0; e < n; ++e) y[e] = (T)x[e];
            *(Tn *)(out + d) = y;
        } else {
#pragma unroll
            for (int e = 0; e < n; e += 4) *(f32x4 *)(p.part + place * D + d + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
        }
    };
#pragma unroll
    for (int a = 0; a < 4; ++a) { // rows 8a + 4g + 0 .. 3 of the operands
#pragma unroll
        for (int c = 0; c < D / 128; ++c)
#pragma unroll
            for (int half = 0; half < 2; ++half)
                put(128 * c + 32 * a + 16 * g + 8 * half, std::integral_constant<int, 8>(), [&](int e) __attribute__((always_inline)) { return o[4 * c + (e & 3)][4 * a + 2 * half + (e >> 2)]; });
        constexpr int c64 = D / 128 * 4, d64 = D / 128 * 128;
        if constexpr (D % 128 >= 64)
            put(d64 + 16 * a + 8 * g, std::integral_constant<int, 8>(), [&](int e) __attribute__((always_inline)) { return o[c64 + ((e & 3) >> 1)][4 * a + 2 * (e >> 2) + (e & 1)]; });
        constexpr int c32 = c64 + (D % 128 >= 64 ? 2 : 0), d32 = d64 + (D % 128 >= 64 ? 64 : 0);
        if constexpr (D % 64 >= 16)
            if (8 * a + 4 * g < (D % 64) / 4 * 4 && 8 * a + 4 * g < D % 64)
                put(d32 + 8 * a + 4 * g, std::integral_constant<int, 4>(), [&](int e) __attribute__((always_inline)) { return o[c32][4 * a + e]; });
    }
}

template <typename T, int D, int WAVES> int launch_tile(const Params &p, unsigned blocks, void *stream) {
    typedef Tiles<T, D, WAVES> K;
    static std::atomic<uint64_t> set{0}; // devices that have been told
    int device = 0;
    hipError_t err = hipGetDevice(&device);
    if (err != hipSuccess) return (int)err;
    if (device >= 64 || !(set.load(std::memory_order_relaxed) >> device & 1)) {
        err = hipFuncSetAttribute((const void *)tiles_kernel<T, D, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, K::lds);
        if (err != hipSuccess) return (int)err;
        if (device < 64) set.fetch_or(1ull << device, std::memory_order_relaxed);
    }
    hipLaunchKernelGGL((tiles_kernel<T, D, WAVES>), dim3(blocks), dim3(K::threads), K::lds, (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

template <typename T> int launch_tiles(const Params &p, int size, int waves, unsigned blocks, void *stream) {
    const auto go = [&](auto d) {
        constexpr int D = decltype(d)::value;
        return waves == 4 ? launch_tile<T, D, 4>(p, blocks, stream) : launch_tile<T, D, 8>(p, blocks, stream);
    };
    switch (size) {
    case 64: return go(std::integral_constant<int, 64>());
    case 80: return go(std::integral_constant<int, 80>());
    case 96: return go(std::integral_constant<int, 96>());
    case 128: return go(std::integral_constant<int, 128>());
    case 192: return go(std::integral_constant<int, 192>());
    default: return go(std::integral_constant<int, 256>());
    }
}

} // namespace
} // namespace attend
} // namespace mcf
