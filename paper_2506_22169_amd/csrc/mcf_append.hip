// New keys and values into the paged cache of 8 bits (include/mcf_cache.h): norm and rotation of the keys, the scale of every
// page and head that tokens go into, rounding to e4m3; and, by further blocks of the same launch, norm and rotation of the
// queries.
//
// A block takes one page and head of K and V: what it needs to know of them (the largest values, the scales so far, the tokens that
// are held) concerns nobody else, so there are no atomics and the result does not depend on any order.  Its lanes keep
// the page's new values in registers between the search for the largest and the rounding, so that the inputs are read
// once, and K and V together keep twice the loads in flight for one search for the sequence.
// With prompts the bytes (2 in, 1 out an element) and the vector instructions (keys, the largest value, rounding) take about as long, behind a chain of
// loads (the sequence, then values and page together, then the scale so far): 8192 tokens of 32 + 2 x 8 heads of 128, bf16 (189 MB), 42 us, with
// a norm 44, 4.3 TB/s; 7 ragged prompts of 20 + 2 x 20 heads of 96 (153 MB, two of eight lanes idle) 47 us, with a norm 53, vector instructions in
// 82 % of the SIMDs' cycles.  64 single tokens: 5.6 us, a launch and the chain.
//
// Keys are computed in 64 bits: the rounding to e4m3 is a step of 1/16 to 1/8 of a value, and a key that lies next to a border
// between two steps would in 32 bits go to either side by a rounding of its norm, a whole step from the nearest to the definition's value.  (The order of a
// row's sums is its size's alone: a token appended alone and within a prompt gives the same bits either way.)  A row takes about 150 double
// operations a lane.  In 32 bits the calls above would take 41.8 (42.0 in 64), 42.4 (44.4), 44.4 (46.9) and 47.4 us (52.7).
#include <hip/hip_runtime.h>

#include <initializer_list>
#include <type_traits>

#include "../../include/mcf_cache.h"
#include "head_rows.hpp"
#include "sequences.hpp"

namespace mcf {
namespace heads {
namespace {

constexpr float kSmallestScale = 0x1p-100f;

struct Params {
    Sequences seq;
    const void *x[2]; // k, v
    uint8_t *page[2];
    float *scale[2];
    int64_t xt[2], xh[2], page_stride[2], head_stride[2], scale_stride[2];
    const void *q, *q_weight, *k_weight;
    void *q_out;
    int64_t qt, qh, ot, oh;
    const float *cos, *sin;
    int64_t table_rows;
    double eps;
    float inv_size;
    int32_t weight_f32, interleaved, size, rotary;
    int32_t pages, k_heads, page_log;
    uint32_t first_blocks;      // these are the cache's; of those behind, block i is the cache's where i * cache_share / 2^32 passes a whole number
    uint64_t cache_share;
    uint32_t q_items, q_heads, q_groups;
    uint32_t heads_magic, q_magic;
    int32_t heads_shift, q_shift;
};

// The least power of two that brings x (finite, not negative) to 448 = 1.75 2^8 at most, 2^-100 at least.
__device__ __forceinline__ float scale_of(float x) {
    const uint32_t b = __float_as_uint(x);
    const int e = (int)(b >> 23) - 8 + ((b & 0x7fffff) > 0x600000 ? 1 : 0); // biased
    return e < 27 ? kSmallestScale : __uint_as_float((uint32_t)e << 23);
}

__device__ __forceinline__ float wave_max(float x) {
    x = over_row<32>(x, [](float a, float b) { return fmaxf(a, b); });
    return fmaxf(x, __shfl_xor(x, 32));
}

__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Eight held values at another scale.
__device__ __forceinline__ void rescale(uint8_t *at, float by) {
    u32x2 w = *(const u32x2 *)at;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
        w[i] = pack4(lo[0] * by, lo[1] * by, hi[0] * by, hi[1] * by);
    }
    *(u32x2 *)at = w;
}

// The norm and rotation of a key in 64 bits.
template <typename T, int LPR>
__device__ __forceinline__ void key_row(const Params &p, const Unit &u, const float wa[8], const float wb[8], const Turn &turn, const Chunk<T> &a, const Chunk<T> &b,
                                        float va[8], float vb[8]) {
    double xa[8], xb[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { xa[e] = (double)(float)a.e[e]; xb[e] = (double)(float)b.e[e]; }
    if (p.k_weight) {
        double sum = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += xa[e] * xa[e] + xb[e] * xb[e];
        const double r = 1.0 / sqrt(row_sum<LPR>(sum) / p.size + p.eps);
#pragma unroll
        for (int e = 0; e < 8; ++e) { xa[e] = xa[e] * r * (double)wa[e]; xb[e] = xb[e] * r * (double)wb[e]; }
    }
    if (u.turns) turn.turn<false>(xa, xb, p.interleaved);
#pragma unroll
    for (int e = 0; e < 8; ++e) { va[e] = (float)xa[e]; vb[e] = (float)xb[e]; }
}

// Up to HPG heads of one query (head, head + groups, ...).  What a query reads of its own is asked for before its sequence is known.
template <typename T, int LPR, int HPG> __device__ __forceinline__ void query_rows(const Params &p, uint32_t item) {
    if (item >= p.q_items) return;
    const uint32_t t = quotient(item, p.q_magic, p.q_shift), first = item - t * p.q_groups;
    const Unit u(threadIdx.x % LPR, p.size, p.rotary);
    const T *x = (const T *)p.q + t * p.qt;
    T *out = (T *)p.q_out + t * p.ot;
    Chunk<T> a[HPG], c[HPG];
#pragma unroll
    for (int j = 0; j < HPG; ++j) {
        const uint32_t h = first + j * p.q_groups;
        a[j].bits = c[j].bits = u32x4{0, 0, 0, 0};
        if (u.there && h < p.q_heads) { a[j].bits = *(const u32x4 *)(x + h * p.qh + u.a); c[j].bits = *(const u32x4 *)(x + h * p.qh + u.b); }
    }
    float wa[8], wb[8];
    if (p.q_weight) load_weight<T>(p.q_weight, p.weight_f32, u, wa, wb);
    const int b = sequence_of_row(p.seq, (int)t);
    if (b < 0) return;
    const Sequence s = sequence(p.seq, b);
    Turn turn;
    turn.load(p.cos, p.sin, (int64_t)s.length - s.rows + ((int)t - s.first), p.table_rows, p.rotary, u, p.interleaved);
#pragma unroll
    for (int j = 0; j < HPG; ++j) {
        const uint32_t h = first + j * p.q_groups;
        float xa[8], xb[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { xa[e] = (float)a[j].e[e]; xb[e] = (float)c[j].e[e]; }
        if (p.q_weight) norm_row<LPR>(xa, xb, wa, wb, p.inv_size, (float)p.eps);
        if (u.turns) turn.turn<false>(xa, xb, p.interleaved);
#pragma unroll
        for (int e = 0; e < 8; ++e) { a[j].e[e] = (T)xa[e]; c[j].e[e] = (T)xb[e]; }
        if (u.there && h < p.q_heads) { *(u32x4 *)(out + h * p.oh + u.a) = a[j].bits; *(u32x4 *)(out + h * p.oh + u.b) = c[j].bits; }
    }
}

// PASSES: places of a page that a group of lanes looks after; HPG: heads of a query that go together.
template <typename T, int LPR, int PASSES, int HPG> __global__ __launch_bounds__(1024) void append_kernel(const Params p) {
    uint32_t block = blockIdx.x;
    if (block >= p.first_blocks) {
        const uint32_t i = block - p.first_blocks, among = (uint32_t)((i * p.cache_share) >> 32);
        if ((uint32_t)(((i + 1) * p.cache_share) >> 32) == among) {
            query_rows<T, LPR, HPG>(p, (i - among) * (blockDim.x / LPR) + threadIdx.x / LPR);
            return;
        }
        block = p.first_blocks + among;
    }
    const int page_size = 1 << p.page_log;
    const uint32_t slot = quotient(block, p.heads_magic, p.heads_shift), h = block - slot * p.k_heads;
    const auto range = [&](const Sequence &s, int &lo, int &hi) __attribute__((always_inline)) { // places that the new tokens have
        lo = s.length > s.rows ? s.length - s.rows : 0;
        hi = s.rows > 0 ? s.seen : 0;
    };
    int b = (int)slot;
    uint32_t nth = 0;
    Sequence s;
    if (p.seq.starts) {
        if (!locate_sequence(p.seq, slot, [&](const Sequence &q) __attribute__((always_inline)) -> uint32_t {
                int lo, hi;
                range(q, lo, hi);
                return hi > lo ? ((hi - 1) >> p.page_log) - (lo >> p.page_log) + 1 : 0;
            }, &b, &nth, &s)) return;
    } else {
        s = sequence(p.seq, b);
    }
    int lo, hi;
    range(s, lo, hi);
    if (hi <= lo) return;
    const int column = (lo >> p.page_log) + (int)nth;
    const int id = p.seq.table[b * p.seq.table_stride + column]; // (looked at when the values are on their way)
    const int base = column << p.page_log;
    const int s0 = lo > base ? lo - base : 0, s1 = hi - base < page_size ? hi - base : page_size; // new places of the page
    const Unit u(threadIdx.x % LPR, p.size, p.rotary);
    const int at_once = blockDim.x / LPR, group = threadIdx.x / LPR;
    Chunk<T> a[2][PASSES], c[2][PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int place = s0 + group + i * at_once;
        const int64_t t = s.first + (base + place - (s.length - s.rows)); // its row
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            a[v][i].bits = c[v][i].bits = u32x4{0, 0, 0, 0};
            if (place < s1 && u.there) {
                const T *const x = (const T *)p.x[v] + t * p.xt[v] + h * p.xh[v];
                a[v][i].bits = *(const u32x4 *)(x + u.a);
                c[v][i].bits = *(const u32x4 *)(x + u.b);
            }
        }
    }
    if (id < 0 || id >= p.pages) return;
    float old[2];
#pragma unroll
    for (int v = 0; v < 2; ++v) old[v] = p.scale[v][id * p.scale_stride[v] + h];
    float va[2][PASSES][8], vb[2][PASSES][8], wa[8], wb[8], most[2] = {0.f, 0.f};
    if (p.k_weight) load_weight<T>(p.k_weight, p.weight_f32, u, wa, wb);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int place = s0 + group + i * at_once;
        if (p.k_weight || p.rotary) {
            Turn turn;
            turn.load(p.cos, p.sin, base + place, p.table_rows, p.rotary, u, p.interleaved);
            key_row<T, LPR>(p, u, wa, wb, turn, a[0][i], c[0][i], va[0][i], vb[0][i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) { va[0][i][e] = (float)a[0][i].e[e]; vb[0][i][e] = (float)c[0][i].e[e]; }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) { va[1][i][e] = (float)a[1][i].e[e]; vb[1][i][e] = (float)c[1][i].e[e]; }
        // (places that are not new have values too where a position is beyond the tables)
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float *const both[2] = {&va[v][i][e], &vb[v][i][e]};
                for (float *y : both) {
                    const bool finite = fabsf(*y) < INFINITY;
                    if (!finite) *y = __builtin_nanf("");
                    most[v] = fmaxf(most[v], finite && place < s1 ? fabsf(*y) : 0.f);
                }
            }
    }
    most[0] = wave_max(most[0]);
    most[1] = wave_max(most[1]);
    if (blockDim.x > 64) {
        __shared__ float part[2][16];
        if ((threadIdx.x & 63) < 2) part[threadIdx.x & 1][threadIdx.x >> 6] = threadIdx.x & 1 ? most[1] : most[0];
        __syncthreads();
        for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
            most[0] = fmaxf(most[0], part[0][w]);
            most[1] = fmaxf(most[1], part[1][w]);
        }
    }
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        uint8_t *const page = p.page[v] + id * p.page_stride[v] + h * p.head_stride[v];
        float now = scale_of(most[v]);
        if (s0 > 0) now = fmaxf(now, old[v]);
        const float inv = 1.0f / now;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int place = s0 + group + i * at_once;
            if (place >= s1 || !u.there) continue;
            uint8_t *const to = page + place * p.size;
            u32x2 x, y;
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                x[d] = pack4(va[v][i][4 * d] * inv, va[v][i][4 * d + 1] * inv, va[v][i][4 * d + 2] * inv, va[v][i][4 * d + 3] * inv);
                y[d] = pack4(vb[v][i][4 * d] * inv, vb[v][i][4 * d + 1] * inv, vb[v][i][4 * d + 2] * inv, vb[v][i][4 * d + 3] * inv);
            }
            *(u32x2 *)(to + u.a) = x;
            *(u32x2 *)(to + u.b) = y;
        }
        if (s0 > 0 && now != old[v] && u.there) {
            for (int place = group; place < s0; place += at_once) {
                rescale(page + place * p.size + u.a, old[v] * inv);
                rescale(page + place * p.size + u.b, old[v] * inv);
            }
        }
        if (threadIdx.x == 0) p.scale[v][id * p.scale_stride[v] + h] = now;
    }
}

} // namespace
} // namespace heads

// Checks a call and lays it out; *blocks = 0: nothing to do.  MCF_OK or an error status.
static int plan_append(const mcf_append_call *c, heads::Params *p, unsigned *blocks, unsigned *threads, int *passes, int *hpg) {
    set_last_error("");
    if (!c) return MCF_EINVAL;
    if (c->dtype != MCF_F16 && c->dtype != MCF_BF16) return MCF_EUNSUPPORTED;
    if (c->q_heads < 0 || !(c->eps >= 0.0)) return MCF_EINVAL;
    const mcf_kv_cache &m = c->cache;
    int st = check_cache(m);
    if (st == MCF_OK) st = check_sequences(c->seq);
    if (st == MCF_OK) st = heads::check_tables(c->rotary, m.size, c->table_rows, c->cos, c->sin);
    if (st != MCF_OK) return st;
    for (const void *w : {c->q_weight, c->k_weight})
        if ((uintptr_t)w % 16 != 0) return MCF_EALIGN;
    const int64_t tokens = c->seq.tokens;
    if ((st = heads::check_rows(c->k, 1, tokens, m.heads, m.size, false)) != MCF_OK) return st;
    if ((st = heads::check_rows(c->v, 1, tokens, m.heads, m.size, false)) != MCF_OK) return st;
    if ((st = heads::check_rows(c->q, 1, tokens, c->q_heads, m.size, false)) != MCF_OK) return st;
    if ((st = heads::check_rows(c->q_out, 1, tokens, c->q_heads, m.size, true)) != MCF_OK) return st;
    if (c->q_heads >= 1 << 20) return MCF_EUNSUPPORTED;
    // pages that the new tokens of a sequence reach: two more than they fill at most, and no more than there are tokens
    int64_t slots = tokens / m.page_size + 2 * c->seq.batch;
    if (slots > tokens) slots = tokens;
    if (m.pages == 0) slots = 0;
    const int lanes = heads::row_lanes(m.size);
    // the new places of a page side by side in a block (one without starts), two of them a lane where they are more than it holds
    const int64_t most_places = c->seq.starts ? m.page_size : 1;
    *passes = most_places * lanes > 1024 ? 2 : 1;
    const int64_t page_lanes = most_places * lanes / *passes;
    *threads = page_lanes < 64 ? 64u : (unsigned)page_lanes;
    // heads of a query share its cosines and sines: four of them together where that leaves eight waves a compute unit (8192 tokens, as
    // above: 46.3 us by fours, 54.4 by ones; 512 tokens 6.9 and 6.5)
    *hpg = tokens * c->q_heads * lanes / 64 >= 4 * 8 * kComputeUnits ? 4 : 1;
    const int64_t q_groups = (c->q_heads + *hpg - 1) / *hpg, per_block = *threads / lanes;
    const int64_t cache_blocks = slots * m.heads, q_items = tokens * q_groups, q_blocks = (q_items + per_block - 1) / per_block;
    if (slots * m.heads >= 1ll << 30 || q_items >= 1ll << 31 || (cache_blocks + q_blocks) * *threads >= (1ll << 32) - 65536) {
        set_last_error("too many rows for one call");
        return MCF_EUNSUPPORTED;
    }
    *blocks = (unsigned)(cache_blocks + q_blocks);
    // The cache's blocks take longest (chains of loads).  Up to two rounds of them (1024 lanes a unit) begin: of 512 tokens 6.5 us, among the queries'
    // blocks 7.4.  More of them go among the queries' blocks, whose traffic fills what the chains leave: 8192 tokens of 32 heads on 8 of 128
    // 43.4 us, ahead of them 46.4.
    const int64_t resident = (int64_t)kComputeUnits * (1024 / *threads), first = cache_blocks <= 2 * resident ? cache_blocks : 0;
    const uint64_t rest = (uint64_t)(cache_blocks - first) << 32, among = (uint64_t)(cache_blocks - first + q_blocks);
    p->first_blocks = (uint32_t)first;
    p->cache_share = among ? (rest + among - 1) / among : 0; // (rounded up: all of them are reached, cache_blocks < 2^30)
    p->seq = device_sequences(c->seq, m.page_size);
    p->x[0] = c->k.data; p->x[1] = c->v.data;
    p->xt[0] = c->k.stride[1]; p->xt[1] = c->v.stride[1];
    p->xh[0] = c->k.stride[2]; p->xh[1] = c->v.stride[2];
    p->page[0] = (uint8_t *)m.k; p->page[1] = (uint8_t *)m.v;
    p->scale[0] = m.k_scale; p->scale[1] = m.v_scale;
    p->page_stride[0] = m.k_stride[0]; p->page_stride[1] = m.v_stride[0];
    p->head_stride[0] = m.k_stride[1]; p->head_stride[1] = m.v_stride[1];
    p->scale_stride[0] = m.k_scale_stride; p->scale_stride[1] = m.v_scale_stride;
    p->q = c->q.data; p->q_out = c->q_out.data; p->q_weight = c->q_weight; p->k_weight = c->k_weight;
    p->qt = c->q.stride[1]; p->qh = c->q.stride[2]; p->ot = c->q_out.stride[1]; p->oh = c->q_out.stride[2];
    p->cos = c->cos; p->sin = c->sin; p->table_rows = c->table_rows;
    p->eps = c->eps; p->inv_size = 1.0f / (float)m.size;
    p->weight_f32 = c->weight_f32 != 0; p->interleaved = c->interleaved != 0;
    p->size = (int32_t)m.size; p->rotary = (int32_t)c->rotary;
    p->pages = (int32_t)m.pages; p->k_heads = (int32_t)m.heads;
    p->page_log = m.page_size == 16 ? 4 : m.page_size == 32 ? 5 : m.page_size == 64 ? 6 : 7;
    p->q_items = (uint32_t)q_items; p->q_heads = (uint32_t)c->q_heads; p->q_groups = (uint32_t)q_groups;
    division_magic((uint32_t)m.heads, &p->heads_magic, &p->heads_shift);
    division_magic((uint32_t)q_groups, &p->q_magic, &p->q_shift);
    return MCF_OK;
}

int check_append(const mcf_append_call *c) {
    heads::Params p;
    unsigned blocks, threads;
    int passes, hpg;
    return plan_append(c, &p, &blocks, &threads, &passes, &hpg);
}

} // namespace mcf

using namespace mcf;

extern "C" int mcf_cache_append(const mcf_append_call *c, void *stream) {
    heads::Params p;
    unsigned blocks, threads;
    int passes, hpg;
    const int st = plan_append(c, &p, &blocks, &threads, &passes, &hpg);
    if (st != MCF_OK || blocks == 0) return st;
    const auto run = [&](auto t, auto lanes) {
        typedef decltype(t) T;
        constexpr int L = decltype(lanes)::value;
        const auto go = [&](auto n, auto g) {
            hipLaunchKernelGGL((heads::append_kernel<T, L, decltype(n)::value, decltype(g)::value>), dim3(blocks), dim3(threads), 0, (hipStream_t)stream, p);
        };
        const std::integral_constant<int, 1> one;
        const std::integral_constant<int, 2> two;
        const std::integral_constant<int, 4> four;
        if constexpr (L == 16) { // (rows of fewer lanes fit a block)
            if (passes == 2) { hpg == 4 ? go(two, four) : go(two, one); return; }
        }
        hpg == 4 ? go(one, four) : go(one, one);
    };
    const auto with = [&](auto t) {
        const int lanes = heads::row_lanes(p.size);
        if (lanes == 4) run(t, std::integral_constant<int, 4>());
        else if (lanes == 8) run(t, std::integral_constant<int, 8>());
        else run(t, std::integral_constant<int, 16>());
    };
    if (c->dtype == MCF_F16) with((_Float16)0);
    else with((__bf16)0);
    const hipError_t err = hipGetLastError();
    if (err == hipSuccess) return MCF_OK;
    set_last_error(hipGetErrorString(err));
    return MCF_ELAUNCH;
}
