// Attention over the paged cache of 8 bits: arguments of its kernels, and how the work of a call is laid out over blocks.
//
// The rows of a sequence for one head of the cache are its tokens' query heads of that group, token by token: row r is
// query head r % group of token r / group.  Rows go to blocks in tiles of R; the tokens that a tile sees are split into
// chunks where tiles are few.  A slot is one chunk of one tile, a block one slot of one head.
//
// How long sequences are only the device knows, so the blocks find their work themselves; the host gives numbers of blocks.
//
// Few rows (attend_rows.hpp).  All tiles' tokens, in units of kUnit and one unit more for each tile (what it costs beside its
// tokens), form one line, that the blocks of a head cut into equal pieces: a block goes through the tiles that its piece touches.  A
// tile that lies in one piece is written by its block; of the others the block leaves a part in the workspace (at most two a block:
// its first tile and its last).
//
// Many rows (attend_tiles.hpp).  A block takes one chunk of one tile.  With S slots for a head, T tiles and W = sum of tiles
// times tokens
//     chunk = W / (S - T), rounded up      =>      sum over tiles of ceil(tokens / chunk) <= W / chunk + T <= S.
//
// The block that leaves a tile's first part also notes where the others will stand (Split), and a second kernel joins them: a block
// for each block that there was, or, where tiles are fewer (and sequences no more than a wave finds the number of a tile for), for each tile.
#pragma once
#include "sequences.hpp"

namespace mcf {
namespace attend {

constexpr int kUnit = 128; // tokens that pieces and chunks are multiples of
constexpr int kLeast = 2;  // units of a piece, at least

// attend_rows.hpp: waves that a SIMD's registers hold (left to itself the compiler spends them on fewer, and the loads in flight are what the kernel waits for).
constexpr int waves_per_simd(int D, int NB) { return NB == 1 ? (D <= 64 ? 4 : D <= 128 ? 3 : 2) : NB == 2 ? (D <= 64 ? 3 : D <= 128 ? 2 : 1) : D <= 64 ? 2 : 1; }

// A tile in parts: how many (0: none), where the first and the second stand and the step from there; its first row and the rows.
struct Split {
    int32_t parts, first, second, step, token, row, rows, pad;
};

struct Params {
    Sequences seq;
    const void *q;
    void *out;
    int64_t qt, qh, ot, oh;
    const uint8_t *k, *v;
    const float *k_scale, *v_scale;
    int64_t k_page, k_head, v_page, v_head;
    int64_t ks_page, vs_page;
    float *part;     // [places * heads][part_rows][size]: what a part leaves
    float *part_ml;  // [places * heads][part_rows][2]: its reference exponent and its sum
    Split *splits;   // [slots * heads]: the tile whose first part the block wrote; with by_tile [tiles * heads]: every tile's
    int32_t *tiles;  // with by_tile: how many there are
    float c;         // scale * log2(e)
    int32_t causal, split, by_tile;
    int32_t pages, heads, group, page_log;
    int32_t part_rows;
    uint32_t slots; // blocks of a head (few rows, split: pieces)
    uint32_t group_magic;
    int32_t group_shift;
};

__device__ __forceinline__ uint32_t quotient(uint32_t n, uint32_t magic, int shift) { return magic ? __umulhi(n, magic) >> shift : n; }

__device__ __forceinline__ int64_t wave_sum(int64_t x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor((long long)x, d);
    return x;
}

template <int R> __device__ __forceinline__ uint32_t tiles_of(const Params &p, const Sequence &s) {
    return (uint32_t)(((int64_t)s.rows * p.group + R - 1) / R);
}

// What a row sees: tokens 0 .. limit - 1.
__device__ __forceinline__ int limit_of(const Params &p, const Sequence &s, int token) { // token: of the sequence's rows
    const int n = s.length - s.rows + token + 1;
    return !p.causal || n > s.seen ? s.seen : n < 0 ? 0 : n;
}

// Whether any element of a lane's query is not finite, from the largest magnitudes of both halves of its words.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 larger_halves(u16x2 most, uint32_t w) { return __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, w & 0x7fff7fff)); }
template <bool F16> __device__ __forceinline__ bool not_finite(u16x2 most) { return (most[0] > most[1] ? most[0] : most[1]) >= (F16 ? 0x7c00 : 0x7f80); }

// V's scale (its bits) in two factors: a power of two that goes into V as it is widened, and the rest, which the weights have in their exponent.
// bf16 takes any power of two, fp16 those under which e4m3 stays exact (2^-9 to 448): 2^-15 to 2^7.  Rests of fp16 are held to 2^-45, where results cannot
// tell the values from zeros (448 * 2^-60; a weight of more range would leave the sum of the softmax nothing of such tokens), and to 2^119, whose
// reciprocal is still a normal number.  Scales that are not finite give any rest.
template <bool F16> __device__ __forceinline__ uint32_t scale_in_v(uint32_t scale) {
    const uint32_t power = scale & 0x7f800000, low = 0x38000000, high = 0x43000000;
    return !F16 ? power : power < low ? low : power < high ? power : high;
}
template <bool F16> __device__ __forceinline__ uint32_t scale_in_weights(uint32_t scale) {
    if (!F16) return (scale & 0x7fffff) | 0x3f800000;
    const uint32_t held = scale < 0x21800000 ? 0x21800000 : scale < 0x7e800000 ? scale : 0x7e800000; // 2^-60, 2^126
    return held - scale_in_v<true>(held) + 0x3f800000;
}

// ---- few rows: pieces of the line ----
__device__ __forceinline__ uint32_t units_of(const Sequence &s) { return (uint32_t)(s.seen + kUnit - 1) / kUnit + 1; }
// Piece j of the line: its first unit and the one behind it, and where the first lies: the sequence and the units before it there.
// False: beyond the line.  Up to 64 sequences are read once, a lane each (two passes over more of them).  The host holds the line of ascending
// starts below 2^31 units; others may bring more (the sums stop at 2^32 - 1), and then nothing is computed.
template <int R> __device__ __forceinline__ bool find_piece(const Params &p, uint32_t j, uint32_t *piece, uint32_t *at, uint32_t *end, int *b, uint32_t *rest, Sequence *s,
                                           uint32_t *tiles_before, uint32_t *all_tiles) {
    const int lane = threadIdx.x & 63;
    const auto units = [&](const Sequence &q) __attribute__((always_inline)) { return tiles_of<R>(p, q) * units_of(q); };
    const auto cut = [&](uint32_t total) __attribute__((always_inline)) {
        if (total >> 31) { *all_tiles = 0; return false; }
        const uint32_t n = (total + p.slots - 1) / p.slots;
        *piece = n < kLeast ? kLeast : n;
        *at = j * *piece;
        *end = *at + *piece < total ? *at + *piece : total;
        return *at < total;
    };
    if (p.seq.batch <= 64) {
        Sequence q = {0, 0, 0, 0};
        if (lane < p.seq.batch) q = sequence(p.seq, lane);
        const uint32_t n = units(q), tiles = tiles_of<R>(p, q);
        uint32_t upto = n, tiles_upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t x = __shfl_up(upto, d), y = __shfl_up(tiles_upto, d);
            if (lane >= d) { upto = __builtin_elementwise_add_sat(upto, x); tiles_upto += y; }
        }
        *all_tiles = __builtin_amdgcn_readlane(tiles_upto, 63);
        if (!cut(__builtin_amdgcn_readlane(upto, 63))) return false;
        const int i = __builtin_ctzll(__ballot(*at - (upto - n) < n));
        *b = i;
        *rest = *at - (__builtin_amdgcn_readlane(upto, i) - __builtin_amdgcn_readlane(n, i));
        *tiles_before = __builtin_amdgcn_readlane(tiles_upto, i) - __builtin_amdgcn_readlane(tiles, i);
        *s = {__builtin_amdgcn_readlane(q.first, i), __builtin_amdgcn_readlane(q.rows, i), __builtin_amdgcn_readlane(q.length, i), __builtin_amdgcn_readlane(q.seen, i)};
        return true;
    }
    uint32_t n = 0;
    for (int i = lane; i < p.seq.batch; i += 64) n = __builtin_elementwise_add_sat(n, units(sequence(p.seq, i)));
#pragma unroll
    for (int d = 1; d < 64; d *= 2) n = __builtin_elementwise_add_sat(n, (uint32_t)__shfl_xor(n, d));
    if (!cut(__builtin_amdgcn_readfirstlane(n)) || !locate(*at, p.seq.batch, [&](int i) __attribute__((always_inline)) -> uint32_t { return units(sequence(p.seq, i)); }, b, rest))
        return false;
    *b = __builtin_amdgcn_readfirstlane(*b);
    *rest = __builtin_amdgcn_readfirstlane(*rest);
    *s = sequence(p.seq, *b);
    return true;
}
// The token at which unit x of a tile begins (the first unit has none).
__device__ __forceinline__ int first_token(uint32_t x) { return x > 0 ? (int)(x - 1) * kUnit : 0; }

// ---- many rows: chunks ----
template <int R> __device__ __forceinline__ int chunk_of(const Params &p) {
    if (!p.split) return 0x7fffff80;
    const int lane = threadIdx.x & 63;
    int64_t work = 0, tiles = 0;
    for (int b = lane; b < p.seq.batch; b += 64) {
        const Sequence s = sequence(p.seq, b);
        const uint32_t n = tiles_of<R>(p, s);
        tiles += n;
        work += (int64_t)n * s.seen;
    }
    work = wave_sum(work);
    tiles = wave_sum(tiles);
    const int64_t room = (int64_t)p.slots - tiles;
    if (room <= 0) return 0x7fffff80;
    const int64_t chunk = ((work + room - 1) / room + kUnit - 1) / kUnit * kUnit;
    return chunk < kUnit ? kUnit : chunk < 0x7fffff80 ? (int)chunk : 0x7fffff80;
}
__device__ __forceinline__ uint32_t chunks_of(const Sequence &s, int chunk) { return s.seen > chunk ? (uint32_t)((s.seen - 1) / chunk) + 1 : 1u; }

// Tiles of a sequence whose last row sees more than x tokens (x < 0: all of them); these are its last.
template <int R> __device__ __forceinline__ uint32_t tiles_beyond(const Params &p, const Sequence &s, int x) {
    const uint32_t tiles = tiles_of<R>(p, s);
    if (x < 0) return tiles;
    if (x >= s.seen) return 0;
    if (!p.causal) return tiles;
    const int y = x - (s.length - s.rows); // token y of its rows sees y + 1 + length - rows
    if (y < 0) return tiles;
    const uint32_t first = (uint32_t)((int64_t)y * p.group / R);
    return y < s.rows && first < tiles ? tiles - first : 0;
}

// Tile number `slot` of all tiles (of up to 64 sequences) by what they see, the most first, in 64 classes: a unit's last block is short then.
template <int R> __device__ __forceinline__ bool locate_longest(const Params &p, uint32_t slot, int *b, uint32_t *tile, Sequence *s) {
    const int lane = threadIdx.x & 63;
    Sequence q = {0, 0, 0, 0};
    if (lane < p.seq.batch) q = sequence(p.seq, lane);
    int most = q.seen;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) { const int x = __shfl_xor(most, d); most = x > most ? x : most; }
    const auto of = [&](const Sequence &x, int i) __attribute__((always_inline)) -> Sequence {
        return {__builtin_amdgcn_readlane(x.first, i), __builtin_amdgcn_readlane(x.rows, i), __builtin_amdgcn_readlane(x.length, i), __builtin_amdgcn_readlane(x.seen, i)};
    };
    const auto border = [&](int i) __attribute__((always_inline)) { return i == 63 ? -1 : (int)((int64_t)most * (63 - i) >> 6); };
    uint32_t upto = 0; // tiles beyond this lane's border
    for (int i = 0; i < p.seq.batch; ++i) upto += tiles_beyond<R>(p, of(q, i), border(lane));
    const uint64_t hit = __ballot(upto > slot);
    if (!hit) return false;
    const int c = __builtin_ctzll(hit);
    const uint32_t before = c > 0 ? tiles_beyond<R>(p, q, border(c - 1)) : 0, n = tiles_beyond<R>(p, q, border(c)) - before;
    slot -= c > 0 ? __builtin_amdgcn_readlane(upto, c - 1) : 0;
    uint32_t sum = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t x = __shfl_up(sum, d);
        if (lane >= d) sum += x;
    }
    const int i = __builtin_ctzll(__ballot(slot - (sum - n) < n));
    *s = of(q, i);
    *b = i;
    *tile = tiles_of<R>(p, *s) - 1 - __builtin_amdgcn_readlane(before, i) - (slot - (__builtin_amdgcn_readlane(sum, i) - __builtin_amdgcn_readlane(n, i)));
    return true;
}

int launch_rows_f16(const Params &p, int size, int row_blocks, int waves, unsigned blocks, void *stream);  // returns hipError_t as int
int launch_rows_bf16(const Params &p, int size, int row_blocks, int waves, unsigned blocks, void *stream);
int launch_tiles_f16(const Params &p, int size, int waves, unsigned blocks, void *stream);
int launch_tiles_bf16(const Params &p, int size, int waves, unsigned blocks, void *stream);

} // namespace attend
} // namespace mcf
