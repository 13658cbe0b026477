// RMS norm of queries and keys for each head with the position rotation, and its gradients (include/mcf_cache.h).
//
//     y = R(p) (x r w),  r = (mean x^2 + eps)^-1/2
//     g = R(-p) dy,  dw = sum over rows of g x r,  u = g w,  dx = r (u - x r^2 mean(u x))
//
// Bound by memory: 2 bytes in and 2 out an element (4 in with gradients) against about ten operations.  So every element is
// loaded and stored once, 16 bytes a lane, a row lies on as few lanes as that allows (head_rows.hpp) and everything between is
// in registers; r is formed again in the backward pass from the x that it reads anyway.  Measured: 8192 tokens of 40 heads of 128,
// bf16 (172 MB), 38 us, 4.5 TB/s; the gradients for 4 x 4096 tokens of 32 heads of 64 (204 MB) 45 us, 4.5 TB/s, 5 of them the sum of
// the blocks' parts of the weights' (a large copy: 5.15 TB/s).  32 tokens: 6 us, a launch and what a call costs its caller.  (Inputs from memory; the
// figures beside the rules below have inputs that stay in the memory-side cache, 32 and 41 us for the same calls.)  Gradients of 100 to 700 tokens of
// 40 heads of 80 take 11.4 to 11.7 us, two launches with their chains of loads and sums; another 2714 tokens are 10 us, the copy's rate.
#include <hip/hip_runtime.h>

#include <initializer_list>
#include <type_traits>

#include "../../include/mcf_cache.h"
#include "head_rows.hpp"

namespace mcf {
namespace heads {
namespace {

struct Rows { // of q or of k
    const void *x, *dy, *w;
    void *out;
    int64_t xb, xt, xh, yb, yt, yh, ob, ot, oh;
    int32_t heads;
    int32_t groups; // of heads that go together: heads g, g + groups, g + 2 groups, ...
};

struct Params {
    Rows q, k;
    const float *cos, *sin;
    const void *positions;
    int64_t position_batch, table_rows;
    float *partial; // backward: [blocks_q + blocks_k][size]
    float eps, inv_size;
    int32_t position_bytes, weight_f32, interleaved, size, rotary;
    uint32_t tokens, items, row_items; // items of all rows, and of one: q.groups + k.groups
    uint32_t items_q, items_k;         // backward: rows times groups
    uint32_t blocks_q;
    uint32_t tokens_magic, row_magic, q_magic, k_magic;
    int32_t tokens_shift, row_shift, q_shift, k_shift;
};

__device__ __forceinline__ int64_t position_of(const Params &p, uint32_t batch, uint32_t token) {
    if (!p.positions) return token;
    const int64_t at = batch * p.position_batch + token;
    return p.position_bytes == 8 ? ((const int64_t *)p.positions)[at] : ((const int32_t *)p.positions)[at];
}

// One item: up to HPG heads of one token, in one tensor, by a group of LPR lanes.
template <typename T, int LPR, int HPG> __global__ __launch_bounds__(256) void rotate_kernel(const Params p) {
    const uint32_t item = blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    if (item >= p.items) return;
    const uint32_t row = quotient(item, p.row_magic, p.row_shift);
    const uint32_t g = item - row * p.row_items;
    const uint32_t b = quotient(row, p.tokens_magic, p.tokens_shift), t = row - b * p.tokens;
    const bool is_k = g >= (uint32_t)p.q.groups;
    const int first = is_k ? g - p.q.groups : g, step = is_k ? p.k.groups : p.q.groups, n = is_k ? p.k.heads : p.q.heads;
    const T *x = (const T *)(is_k ? p.k.x : p.q.x) + b * (is_k ? p.k.xb : p.q.xb) + t * (is_k ? p.k.xt : p.q.xt);
    T *out = (T *)(is_k ? p.k.out : p.q.out) + b * (is_k ? p.k.ob : p.q.ob) + t * (is_k ? p.k.ot : p.q.ot);
    const int64_t xh = is_k ? p.k.xh : p.q.xh, oh = is_k ? p.k.oh : p.q.oh;
    const void *w = is_k ? p.k.w : p.q.w;
    const Unit u(threadIdx.x % LPR, p.size, p.rotary);
    Chunk<T> a[HPG], c[HPG];
#pragma unroll
    for (int j = 0; j < HPG; ++j) {
        a[j].bits = c[j].bits = u32x4{0, 0, 0, 0};
        const int h = first + j * step;
        if (u.there && h < n) {
            a[j].bits = *(const u32x4 *)(x + h * xh + u.a);
            c[j].bits = *(const u32x4 *)(x + h * xh + u.b);
        }
    }
    Turn turn;
    turn.load(p.cos, p.sin, p.rotary ? position_of(p, b, t) : 0, p.table_rows, p.rotary, u, p.interleaved);
    float wa[8], wb[8];
    if (w) load_weight<T>(w, p.weight_f32, u, wa, wb);
#pragma unroll
    for (int j = 0; j < HPG; ++j) {
        const int h = first + j * step;
        float xa[8], xb[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { xa[e] = (float)a[j].e[e]; xb[e] = (float)c[j].e[e]; }
        if (w) norm_row<LPR>(xa, xb, wa, wb, p.inv_size, p.eps);
        if (u.turns) turn.turn<false>(xa, xb, p.interleaved);
#pragma unroll
        for (int e = 0; e < 8; ++e) { a[j].e[e] = (T)xa[e]; c[j].e[e] = (T)xb[e]; }
        if (u.there && h < n) {
            *(u32x4 *)(out + h * oh + u.a) = a[j].bits;
            *(u32x4 *)(out + h * oh + u.b) = c[j].bits;
        }
    }
}

// Gradients: a block takes items of one tensor, its lanes keep the weight's gradient of their sixteen elements over all of
// them, and the block's sum goes to the workspace.
template <typename T, int LPR, int HPG> __global__ __launch_bounds__(256) void rotate_back_kernel(const Params p) {
    const bool is_k = blockIdx.x >= p.blocks_q;
    const Rows &r = is_k ? p.k : p.q;
    const uint32_t block = is_k ? blockIdx.x - p.blocks_q : blockIdx.x, blocks = is_k ? gridDim.x - p.blocks_q : p.blocks_q;
    const uint32_t items = is_k ? p.items_k : p.items_q, magic = is_k ? p.k_magic : p.q_magic;
    const int shift = is_k ? p.k_shift : p.q_shift;
    const Unit u(threadIdx.x % LPR, p.size, p.rotary);
    float wa[8], wb[8], da[8], db[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) da[e] = db[e] = 0.f;
    if (r.w) load_weight<T>(r.w, p.weight_f32, u, wa, wb);
    for (uint64_t item = block * (256 / LPR) + threadIdx.x / LPR; item < items; item += (uint64_t)blocks * (256 / LPR)) {
        const uint32_t row = quotient((uint32_t)item, magic, shift), first = (uint32_t)item - row * r.groups;
        const uint32_t b = quotient(row, p.tokens_magic, p.tokens_shift), t = row - b * p.tokens;
        const T *x = (const T *)r.x + b * r.xb + t * r.xt, *dy = (const T *)r.dy + b * r.yb + t * r.yt;
        T *out = (T *)r.out + b * r.ob + t * r.ot;
        Chunk<T> xa[HPG], xb[HPG], ya[HPG], yb[HPG];
#pragma unroll
        for (int j = 0; j < HPG; ++j) {
            xa[j].bits = xb[j].bits = ya[j].bits = yb[j].bits = u32x4{0, 0, 0, 0};
            const int h = first + j * r.groups;
            if (u.there && h < r.heads) {
                ya[j].bits = *(const u32x4 *)(dy + h * r.yh + u.a);
                yb[j].bits = *(const u32x4 *)(dy + h * r.yh + u.b);
                if (r.w) {
                    xa[j].bits = *(const u32x4 *)(x + h * r.xh + u.a);
                    xb[j].bits = *(const u32x4 *)(x + h * r.xh + u.b);
                }
            }
        }
        Turn turn;
        turn.load(p.cos, p.sin, p.rotary ? position_of(p, b, t) : 0, p.table_rows, p.rotary, u, p.interleaved);
#pragma unroll
        for (int j = 0; j < HPG; ++j) {
            const int h = first + j * r.groups;
            float ga[8], gb[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) { ga[e] = (float)ya[j].e[e]; gb[e] = (float)yb[j].e[e]; }
            if (u.turns) turn.turn<true>(ga, gb, p.interleaved);
            if (r.w) {
                float squares = 0.f, products = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float a = (float)xa[j].e[e], c = (float)xb[j].e[e];
                    squares += a * a + c * c;
                    products += ga[e] * wa[e] * a + gb[e] * wb[e] * c;
                }
                const float inv = 1.0f / sqrtf(row_sum<LPR>(squares) * p.inv_size + p.eps);
                const float mean = row_sum<LPR>(products) * p.inv_size * inv * inv;
                // a head that is not there, whose rows are zeros here, would add 0 * NaN where a position is outside of the tables
                if (h < r.heads) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float a = (float)xa[j].e[e], c = (float)xb[j].e[e];
                        da[e] += ga[e] * (a * inv);
                        db[e] += gb[e] * (c * inv);
                        ga[e] = inv * (ga[e] * wa[e] - a * mean);
                        gb[e] = inv * (gb[e] * wb[e] - c * mean);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) { ya[j].e[e] = (T)ga[e]; yb[j].e[e] = (T)gb[e]; }
            if (u.there && h < r.heads) {
                *(u32x4 *)(out + h * r.oh + u.a) = ya[j].bits;
                *(u32x4 *)(out + h * r.oh + u.b) = yb[j].bits;
            }
        }
    }
    if (!r.w) return;
    __shared__ float part[256 * 16];
    if (u.there) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            part[threadIdx.x / LPR * p.size + u.a + e] = da[e];
            part[threadIdx.x / LPR * p.size + u.b + e] = db[e];
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.size; c += 256) {
        float sum = 0.f;
        for (int g = 0; g < 256 / LPR; ++g) sum += part[g * p.size + c];
        p.partial[(int64_t)blockIdx.x * p.size + c] = sum;
    }
}

// Sums the blocks' parts of sixteen elements of a weight's gradient: 64 slices of the blocks, each in order, then the slices.
__global__ __launch_bounds__(1024) void weight_sum_kernel(const float *partial, int size, uint32_t blocks_q, uint32_t blocks_k, float *dq, float *dk) {
    float *out = blockIdx.y ? dk : dq;
    if (!out) return;
    const float *src = partial + (blockIdx.y ? (int64_t)blocks_q * size : 0);
    const uint32_t n = blockIdx.y ? blocks_k : blocks_q;
    const int c = blockIdx.x * 16 + threadIdx.x % 16, slice = threadIdx.x / 16;
    float sum = 0.f;
    for (uint32_t b = slice; b < n; b += 64) sum += src[(int64_t)b * size + c];
    __shared__ float part[1024];
    part[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < 16) {
        sum = 0.f;
        for (int s = 0; s < 64; ++s) sum += part[s * 16 + threadIdx.x];
        out[c] = sum;
    }
}

struct Plan {
    Params p;
    int lanes, hpg;
    uint32_t blocks, blocks_k;
    bool nothing;
    int64_t workspace;
};

// Blocks of the backward kernel that are resident at once, by its registers (3 x 256: 4 x 4096 tokens of 32 heads of 64 in 41.1 us; with
// 2 x 256 44.5, with 4 x 256 47.8).
constexpr uint32_t kMostBlocks = 3 * kComputeUnits;

// Checks a call and lays it out.  MCF_OK or an error status.
int plan(const mcf_norm_rotate_call *c, bool back, Plan *o) {
    set_last_error("");
    if (!c) return MCF_EINVAL;
    if (c->dtype != MCF_F16 && c->dtype != MCF_BF16) return MCF_EUNSUPPORTED;
    if (c->batch < 0 || c->tokens < 0 || c->q_heads < 0 || c->k_heads < 0 || c->size <= 0 || !(c->eps >= 0.0)) return MCF_EINVAL;
    if (c->size % 16 != 0 || c->size > 512) { set_last_error("the size of a head is a multiple of 16 up to 512"); return MCF_EUNSUPPORTED; }
    int st = check_tables(c->rotary, c->size, c->table_rows, c->cos, c->sin);
    if (st != MCF_OK) return st;
    if (c->positions && c->position_bytes != 4 && c->position_bytes != 8) return MCF_EINVAL;
    if (c->positions && ((uintptr_t)c->positions % c->position_bytes != 0)) return MCF_EALIGN;
    if (c->position_batch != 0 && c->position_batch != c->tokens) return MCF_EINVAL;
    for (const void *w : {c->q_weight, c->k_weight})
        if ((uintptr_t)w % 16 != 0) return MCF_EALIGN;
    const int64_t rows = c->batch > 0 && c->tokens > (1ll << 31) / c->batch ? 1ll << 32 : c->batch * c->tokens;
    const struct { const mcf_rows *r; int64_t n; bool written; } args[] = {
        {&c->q, c->q_heads, false}, {&c->k, c->k_heads, false}, {&c->q_out, c->q_heads, true}, {&c->k_out, c->k_heads, true}, {&c->dq, c->q_heads, false}, {&c->dk, c->k_heads, false}};
    for (int i = 0; i < (back ? 6 : 4); ++i)
        if ((st = check_rows(*args[i].r, c->batch, c->tokens, args[i].n, c->size, args[i].written)) != MCF_OK) return st;
    if (back && ((c->q_weight && c->q_heads > 0 && !c->dq_weight) || (c->k_weight && c->k_heads > 0 && !c->dk_weight))) return MCF_EINVAL;
    const int64_t all = c->q_heads + c->k_heads;
    // 32-bit item numbers, and a grid of 256-lane blocks whose lanes HIP counts in 32 bits
    if (c->q_heads >= 1 << 20 || c->k_heads >= 1 << 20 || rows >= (1ll << 31) || rows * (all > 0 ? all : 1) * row_lanes(c->size) >= (1ll << 32) - 65536 ||
        rows * all >= (1ll << 31)) {
        set_last_error("too many rows for one call");
        return MCF_EUNSUPPORTED;
    }
    o->nothing = rows == 0 || all == 0;
    o->lanes = row_lanes(c->size);
    // Heads of a token share its cosines and sines: four of them an item where that still leaves eight waves a compute unit, one otherwise
    // (40 heads of 128, bf16, 8192 tokens: 32.2 us by fours, 33.7 by ones; 4 x 4096 tokens of 32 heads of 64: 24.7 and 27.1; 1024 tokens of
    // 40 heads: 7.1 and 6.1).  The gradients take two, whose registers leave three blocks a unit.
    const int64_t waves = rows * all * o->lanes / 64;
    o->hpg = back ? 2 : waves >= 4 * 8 * kComputeUnits ? 4 : 1;
    Params &p = o->p;
    const auto set = [&](Rows &r, const mcf_rows &x, const mcf_rows &y, const mcf_rows &out, const void *w, int64_t n) {
        r.x = x.data; r.dy = y.data; r.out = out.data; r.w = w;
        r.xb = x.stride[0]; r.xt = x.stride[1]; r.xh = x.stride[2];
        r.yb = y.stride[0]; r.yt = y.stride[1]; r.yh = y.stride[2];
        r.ob = out.stride[0]; r.ot = out.stride[1]; r.oh = out.stride[2];
        r.heads = (int32_t)n;
        r.groups = (int32_t)((n + o->hpg - 1) / o->hpg);
    };
    set(p.q, c->q, c->dq, c->q_out, c->q_weight, c->q_heads);
    set(p.k, c->k, c->dk, c->k_out, c->k_weight, c->k_heads);
    p.cos = c->cos; p.sin = c->sin; p.positions = c->positions;
    p.position_batch = c->position_batch; p.table_rows = c->table_rows;
    p.partial = nullptr;
    p.eps = (float)c->eps; p.inv_size = 1.0f / (float)c->size;
    p.position_bytes = c->position_bytes; p.weight_f32 = c->weight_f32 != 0; p.interleaved = c->interleaved != 0;
    p.size = (int32_t)c->size; p.rotary = (int32_t)c->rotary;
    p.tokens = (uint32_t)c->tokens;
    p.row_items = (uint32_t)(p.q.groups + p.k.groups);
    p.items = (uint32_t)(rows * p.row_items);
    p.items_q = (uint32_t)(rows * p.q.groups); p.items_k = (uint32_t)(rows * p.k.groups);
    division_magic(p.tokens, &p.tokens_magic, &p.tokens_shift);
    division_magic(p.row_items, &p.row_magic, &p.row_shift);
    division_magic((uint32_t)p.q.groups, &p.q_magic, &p.q_shift);
    division_magic((uint32_t)p.k.groups, &p.k_magic, &p.k_shift);
    const uint32_t per_block = 256 / o->lanes;
    o->blocks_k = 0; o->workspace = 0; p.blocks_q = 0;
    if (o->nothing) { o->blocks = 0; return MCF_OK; }
    if (!back) {
        o->blocks = (p.items + per_block - 1) / per_block;
        return MCF_OK;
    }
    // one round or two of the lanes' items: as few blocks as share them evenly (1500 tokens of 40 heads of 128: 16.2 us, by all that are resident
    // 18.4, by a block an item 19.3); more: all that are resident
    const uint32_t most_q = (p.items_q + per_block - 1) / per_block, most_k = (p.items_k + per_block - 1) / per_block, most = most_q + most_k;
    const uint32_t rounds = (most + kMostBlocks - 1) / kMostBlocks;
    const auto share = [&](uint32_t n) { return rounds <= 2 ? (n + rounds - 1) / rounds : n == 0 ? 0u : n <= most / kMostBlocks ? 1u : (uint32_t)((uint64_t)kMostBlocks * n / most); };
    p.blocks_q = share(most_q);
    o->blocks_k = share(most_k);
    o->blocks = p.blocks_q + o->blocks_k;
    if (c->q_weight || c->k_weight) o->workspace = (int64_t)o->blocks * c->size * 4;
    return MCF_OK;
}

// launch(kernel<T, LPR>) for the call's type and lanes of a row
template <typename F> void by_type(int dtype, int lanes, F &&f) {
    const auto with = [&](auto t) {
        if (lanes == 4) f(t, std::integral_constant<int, 4>());
        else if (lanes == 8) f(t, std::integral_constant<int, 8>());
        else if (lanes == 16) f(t, std::integral_constant<int, 16>());
        else f(t, std::integral_constant<int, 32>());
    };
    if (dtype == MCF_F16) with((_Float16)0);
    else with((__bf16)0);
}

int launched() {
    const hipError_t err = hipGetLastError();
    if (err == hipSuccess) return MCF_OK;
    set_last_error(hipGetErrorString(err));
    return MCF_ELAUNCH;
}

} // namespace
} // namespace heads

int check_norm_rotate(const mcf_norm_rotate_call *c, bool back) {
    heads::Plan l;
    return heads::plan(c, back, &l);
}

} // namespace mcf

using namespace mcf;

extern "C" int mcf_norm_rotate(const mcf_norm_rotate_call *c, void *stream) {
    heads::Plan l;
    const int st = heads::plan(c, false, &l);
    if (st != MCF_OK || l.nothing) return st;
    heads::by_type(c->dtype, l.lanes, [&](auto t, auto lanes) {
        typedef decltype(t) T;
        if (l.hpg == 4) hipLaunchKernelGGL((heads::rotate_kernel<T, lanes(), 4>), dim3(l.blocks), dim3(256), 0, (hipStream_t)stream, l.p);
        else hipLaunchKernelGGL((heads::rotate_kernel<T, lanes(), 1>), dim3(l.blocks), dim3(256), 0, (hipStream_t)stream, l.p);
    });
    return heads::launched();
}

extern "C" int mcf_norm_rotate_backward_workspace(const mcf_norm_rotate_call *c, int64_t *bytes) {
    heads::Plan l;
    if (!bytes) return MCF_EINVAL;
    const int st = heads::plan(c, true, &l);
    *bytes = st == MCF_OK ? l.workspace : 0;
    return st;
}

extern "C" int mcf_norm_rotate_backward(const mcf_norm_rotate_call *c, void *workspace, int64_t workspace_bytes, void *stream) {
    heads::Plan l;
    const int st = heads::plan(c, true, &l);
    if (st != MCF_OK) return st;
    if (l.workspace > 0 && (!workspace || workspace_bytes < l.workspace || (uintptr_t)workspace % 16 != 0)) return MCF_EINVAL;
    l.p.partial = (float *)workspace;
    if (!l.nothing) {
        heads::by_type(c->dtype, l.lanes, [&](auto t, auto lanes) {
            typedef decltype(t) T;
            hipLaunchKernelGGL((heads::rotate_back_kernel<T, lanes(), 2>), dim3(l.blocks), dim3(256), 0, (hipStream_t)stream, l.p);
        });
        const int launched = heads::launched();
        if (launched != MCF_OK) return launched;
    }
    // (without rows the sums are zeros; a tensor without heads has no gradient to write)
    float *dq = c->q_weight ? c->dq_weight : nullptr, *dk = c->k_weight ? c->dk_weight : nullptr;
    if (!dq && !dk) return MCF_OK;
    hipLaunchKernelGGL(heads::weight_sum_kernel, dim3((unsigned)c->size / 16, 2), dim3(1024), 0, (hipStream_t)stream, l.p.partial, (int)c->size, l.p.blocks_q,
                       l.blocks_k, dq, dk);
    return heads::launched();
}
