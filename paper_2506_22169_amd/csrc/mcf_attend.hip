// Attention over the paged cache (include/mcf_cache.h): checks, the choice of kernel and split, and the kernel that joins
// the chunks of a tile.
#include <hip/hip_runtime.h>

#include <initializer_list>
#include <type_traits>

#include "attend.hpp"
#include "head_rows.hpp"

namespace mcf {
namespace attend {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// out = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i over the parts of a tile, for `at_once` of its rows; a lane takes four elements of a row.  One
// row: its lanes form slices, each takes every slices-th part, and the sums are added in the slices' order.  Several: a lane takes all parts of
// its row in order, eight asked for at once.  Bound by latency: 4 to 6 us for the parts of 64 sequences' tiles (20 MB), 7 for 5 x 8 rows of 256 parts.
template <typename T> __global__ __launch_bounds__(256) void join_kernel(const Params p, int size, int at_once) {
    const uint32_t groups = (uint32_t)(p.part_rows + at_once - 1) / at_once, block = blockIdx.x / groups;
    const int row0 = (int)(blockIdx.x - block * groups) * at_once, h = (int)(block % (uint32_t)p.heads);
    if (p.by_tile && block / (uint32_t)p.heads >= (uint32_t)*p.tiles) return; // (tiles < slots: the grid ends within the room for them)
    const Split t = p.splits[block];
    if (t.parts == 0 || t.rows <= row0) return;
    const int quads = size / 4, unit = threadIdx.x / quads, d = 4 * (threadIdx.x - unit * quads), row = at_once == 1 ? row0 : row0 + unit;
    const auto at = [&](int i) __attribute__((always_inline)) {
        return ((int64_t)(i == 0 ? t.first : t.second + (i - 1) * t.step) * p.heads + h) * p.part_rows + row;
    };
    // (a reference of -inf: nothing seen, zeros, or NaN)
    const auto times = [](float from, float to) __attribute__((always_inline)) { return from == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(from - to); };
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    if (at_once == 1) {
        const int slices = 256 / quads;
        for (int i = threadIdx.x & 63; i < t.parts; i += 256) { // (behind the last part one of them again)
            float x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = p.part_ml[2 * at(i + 64 * k < t.parts ? i + 64 * k : i)];
            m = fmaxf(m, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
        }
        for (int x = 1; x < 64; x *= 2) m = fmaxf(m, __shfl_xor(m, x));
        if (unit < slices) {
#pragma unroll 4
            for (int i = unit; i < t.parts; i += slices) {
                const int64_t a = at(i);
                const float w = times(p.part_ml[2 * a], m);
                l += p.part_ml[2 * a + 1] * w;
                o += *(const f32x4 *)(p.part + a * size + d) * w;
            }
        }
        __shared__ f32x4 part[256];
        __shared__ float sum[256];
        part[threadIdx.x] = o;
        sum[threadIdx.x] = l;
        __syncthreads();
        if (unit != 0) return;
        for (int i = 1; i < slices; ++i) {
            o += part[threadIdx.x + i * quads];
            l += sum[threadIdx.x + i * quads];
        }
    } else {
        if (unit >= at_once || row >= t.rows) return;
        for (int i = 0; i < t.parts; i += 8) {
            f32x2 ml[8];
            f32x4 x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) { // (behind the last part the first of them again)
                const int64_t a = at(i + k < t.parts ? i + k : i);
                ml[k] = *(const f32x2 *)(p.part_ml + 2 * a);
                x[k] = *(const f32x4 *)(p.part + a * size + d);
            }
            float top = m;
#pragma unroll
            for (int k = 0; k < 8; ++k) top = fmaxf(top, ml[k][0]);
            const float by = times(m, top);
            m = top;
            l *= by;
            o *= by;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (i + k >= t.parts) break;
                const float w = times(ml[k][0], m);
                l += ml[k][1] * w;
                o += x[k] * w;
            }
        }
    }
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const int r = t.row + row, token = (int)quotient(r, p.group_magic, p.group_shift), head = r - token * p.group;
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (T)(o[e] * inv);
    *(T4 *)((T *)p.out + (int64_t)(t.token + token) * p.ot + (int64_t)(h * p.group + head) * p.oh + d) = y;
}

// Keys of a sequence, in bytes, that one block of eight waves goes through: 500 tokens of 128 take 9.5 us (in pieces 11.9), 600 10.6 (12.9), 1000
// 12.6 (11.8); 1000 of 64 10.6 (13.0).
constexpr int64_t kShort = 96 << 10;

struct Plan {
    Params p;
    int tile_rows;          // 16, 32, 48, 64: attend_rows.hpp; 128, 256: attend_tiles.hpp
    unsigned tiles, blocks; // an upper bound of the tiles; 0 blocks: nothing to do
    int waves;              // of a block of few rows
    int64_t workspace;      // what a split call wants
    int64_t places;         // of parts there
};

// Blocks that are resident at once, by the registers (attend_rows.hpp: waves_per_simd; attend_tiles.hpp: two waves a SIMD).
inline int64_t resident_blocks(int tile_rows, int64_t size) {
    if (tile_rows > 64) return kComputeUnits * (tile_rows == 128 ? 2 : 1);
    return kComputeUnits * waves_per_simd((int)size, tile_rows / 16);
}

int plan(const mcf_attention_call *c, bool may_split, Plan *o) {
    set_last_error("");
    if (!c) return MCF_EINVAL;
    if (c->dtype != MCF_F16 && c->dtype != MCF_BF16) return MCF_EUNSUPPORTED;
    const mcf_kv_cache &m = c->cache;
    int st = check_cache(m);
    if (st == MCF_OK) st = check_sequences(c->seq);
    if (st != MCF_OK) return st;
    if (!(c->scale - c->scale == 0.f)) return MCF_EINVAL; // NaN, infinity
    if (c->q_heads < 0 || (c->q_heads > 0 && (m.heads == 0 || c->q_heads % m.heads != 0))) {
        set_last_error("the heads of the queries are a multiple of the cache's");
        return MCF_EINVAL;
    }
    const int64_t tokens = c->seq.tokens, batch = c->seq.batch;
    if ((st = heads::check_rows(c->q, 1, tokens, c->q_heads, m.size, false)) != MCF_OK) return st;
    if ((st = heads::check_rows(c->out, 1, tokens, c->q_heads, m.size, true)) != MCF_OK) return st;
    o->blocks = 0; o->workspace = 0;
    if (tokens == 0 || batch == 0 || c->q_heads == 0) return MCF_OK;
    const int64_t group = c->q_heads / m.heads;
    if (group > 1 << 16 || tokens * group >= (1ll << 31) - 65536) { set_last_error("too many rows for one call"); return MCF_EUNSUPPORTED; }
    // The rows that a sequence brings in the mean decide the tile.  Where both kernels could: 16 sequences of 16 tokens against 4000, 32 heads on 8
    // (64 rows), take 43 us with the few rows' kernel and 48 with the other for heads of 64, 86 and 67 for heads of 128 (48 rows: 67 both;
    // 5 tokens of 16 heads on 2 of 64 against 130000, 40 rows: 26 and 74).
    const int64_t rows = (tokens * group + batch - 1) / batch;
    const int R = o->tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 48 && m.size <= 128 ? 48 : rows <= 64 && m.size <= 64 ? 64 : rows <= 128 ? 128 : 256;
    const int64_t tiles = tokens * group / R + (batch < tokens ? batch : tokens);
    int64_t slots = resident_blocks(R, m.size) / m.heads;
    o->waves = 4;
    bool split = may_split;
    if (R > 64) {
        // two chunks a tile at least, of tokens that are worth the parts' way through memory (256 rows of 128: 10 us) and a second kernel
        split = split && slots >= 2 * tiles && c->seq.table_width * m.page_size > 1024;
        if (!split) slots = tiles;
    } else {
        // no more pieces than the longest sequences that the table holds would give; the line in 31 bits
        const int64_t reach = m.pages ? c->seq.table_width * m.page_size : 0;
        const int64_t most = tiles * (reach / kUnit + 2);
        if (slots < 1) slots = 1;
        if (slots > (most + kLeast - 1) / kLeast) slots = (most + kLeast - 1) / kLeast;
        // a tile a block of eight waves where the table ends early and there are units for all: one launch instead of two
        if (R == 16 && reach * m.size <= kShort && tiles * m.heads <= kComputeUnits) { split = false; o->waves = 8; }
        split = split && most < 1ll << 31;
        if (!split) slots = tiles;
    }
    const int64_t places = R > 64 ? slots : 2 * slots; // of parts in the workspace
    if (slots * m.heads >= 1ll << 23) { set_last_error("too many rows for one call"); return MCF_EUNSUPPORTED; } // (2^32 lanes)
    Params &p = o->p;
    p.seq = device_sequences(c->seq, m.page_size);
    if (m.pages == 0) p.seq.capacity = 0;
    p.q = c->q.data; p.out = c->out.data;
    p.qt = c->q.stride[1]; p.qh = c->q.stride[2]; p.ot = c->out.stride[1]; p.oh = c->out.stride[2];
    p.k = (const uint8_t *)m.k; p.v = (const uint8_t *)m.v; p.k_scale = m.k_scale; p.v_scale = m.v_scale;
    p.k_page = m.k_stride[0]; p.k_head = m.k_stride[1]; p.v_page = m.v_stride[0]; p.v_head = m.v_stride[1];
    p.ks_page = m.k_scale_stride; p.vs_page = m.v_scale_stride;
    p.part = p.part_ml = nullptr;
    p.splits = nullptr; p.tiles = nullptr;
    p.c = c->scale * 1.44269504088896341f;
    p.causal = c->causal != 0; p.split = split; p.by_tile = split && R <= 64 && batch <= 64 && tiles < slots;
    p.pages = (int32_t)m.pages; p.heads = (int32_t)m.heads; p.group = (int32_t)group;
    p.page_log = m.page_size == 16 ? 4 : m.page_size == 32 ? 5 : m.page_size == 64 ? 6 : 7;
    p.part_rows = c->seq.starts ? R : group < R ? (int)group : R;
    p.slots = (uint32_t)slots;
    division_magic((uint32_t)group, &p.group_magic, &p.group_shift);
    o->tiles = (unsigned)tiles;
    o->blocks = (unsigned)(slots * m.heads);
    o->places = places * m.heads;
    if (split) o->workspace = o->places * p.part_rows * (m.size + 2) * 4 + (int64_t)o->blocks * sizeof(Split) + 16;
    return MCF_OK;
}

} // namespace

static int launch_join(const Params &p, int dtype, int size, int tile_rows, unsigned tiles, unsigned blocks, void *stream) {
    // a row a block where a tile has many parts (all lanes share them out), else as many rows as the lanes hold
    const int at_once = tile_rows <= 64 && p.slots >= 8 * tiles ? 1 : 256 / (size / 4);
    const dim3 grid((p.by_tile ? tiles * p.heads : blocks) * ((p.part_rows + at_once - 1) / at_once)), block(256);
    if (dtype == MCF_F16) hipLaunchKernelGGL((join_kernel<_Float16>), grid, block, 0, (hipStream_t)stream, p, size, at_once);
    else hipLaunchKernelGGL((join_kernel<__bf16>), grid, block, 0, (hipStream_t)stream, p, size, at_once);
    return (int)hipGetLastError();
}

} // namespace attend

int check_attention(const mcf_attention_call *c) {
    attend::Plan l;
    return attend::plan(c, true, &l);
}

} // namespace mcf

using namespace mcf;

extern "C" int mcf_cache_attention_workspace(const mcf_attention_call *c, int64_t *bytes) {
    attend::Plan l;
    if (!bytes) return MCF_EINVAL;
    const int st = attend::plan(c, true, &l);
    *bytes = st == MCF_OK ? l.workspace : 0;
    return st;
}

extern "C" int mcf_cache_attention(const mcf_attention_call *c, void *workspace, int64_t workspace_bytes, void *stream) {
    attend::Plan l;
    int st = attend::plan(c, true, &l);
    if (st != MCF_OK || l.blocks == 0) return st;
    if (l.workspace > 0) {
        if (!workspace || workspace_bytes < l.workspace) st = attend::plan(c, false, &l);
        else if ((uintptr_t)workspace % 16 != 0) return MCF_EALIGN;
        if (st != MCF_OK) return st;
    }
    attend::Params &p = l.p;
    if (l.workspace > 0) {
        p.part = (float *)workspace;
        p.part_ml = p.part + l.places * p.part_rows * c->cache.size;
        p.tiles = (int32_t *)(p.part_ml + 2 * l.places * p.part_rows);
        p.splits = (attend::Split *)(p.tiles + 4);
    }
    const int size = (int)c->cache.size;
    const bool f16 = c->dtype == MCF_F16;
    int err;
    if (l.tile_rows <= 64) err = (f16 ? attend::launch_rows_f16 : attend::launch_rows_bf16)(p, size, l.tile_rows / 16, l.waves, l.blocks, stream);
    else err = (f16 ? attend::launch_tiles_f16 : attend::launch_tiles_bf16)(p, size, l.tile_rows / 32, l.blocks, stream);
    if (err == hipSuccess && l.workspace > 0 && p.slots > 1) err = attend::launch_join(p, c->dtype, size, l.tile_rows, l.tiles, l.blocks, stream);
    if (err == hipSuccess) return MCF_OK;
    set_last_error(hipGetErrorString((hipError_t)err));
    return MCF_ELAUNCH;
}
