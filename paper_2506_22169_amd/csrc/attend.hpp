// Attention over the paged cache of 8 bits: arguments of its kernels, and how the work of a call is laid out over blocks.
//
// The rows of a sequence for one head of the cache are its tokens' query heads of that group, token by token: row r is
// query head r % group of token r / group.  Rows go to blocks in tiles of R; the tokens that a tile sees are split into
// chunks where tiles are few.  A slot is one chunk of one tile, a block one slot of one head.
//
// How long sequences are only the device knows, so the blocks find their slot themselves: the host gives a number of slots
// S that leaves room for chunks beside the tiles, and with T tiles and W = sum of tiles times tokens
//     chunk = W / (S - T), rounded up      =>      sum over tiles of ceil(tokens / chunk) <= W / chunk + T <= S.
// Sequences of any mix of lengths are cut into equal pieces that way, and a block holds one piece of one tile only.
#pragma once
#include "sequences.hpp"

namespace mcf {
namespace attend {

constexpr int kStep = 128;     // chunks are multiples of this many tokens

struct Params {
    Sequences seq;
    const void *q;
    void *out;
    int64_t qt, qh, ot, oh;
    const uint8_t *k, *v;
    const float *k_scale, *v_scale;
    int64_t k_page, k_head, v_page, v_head;
    int64_t ks_page, vs_page;
    float *part;     // [slots * heads][part_rows][size]: what a chunk leaves
    float *part_ml;  // [slots * heads][part_rows][2]: its reference exponent and its sum
    float c;         // scale * log2(e)
    int32_t causal, split;
    int32_t pages, heads, group, page_log;
    int32_t part_rows;
    uint32_t slots;
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

// Tokens of a chunk.
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
    const int64_t chunk = ((work + room - 1) / room + kStep - 1) / kStep * kStep;
    return chunk < kStep ? kStep : chunk < 0x7fffff80 ? (int)chunk : 0x7fffff80;
}
__device__ __forceinline__ uint32_t chunks_of(const Sequence &s, int chunk) { return s.seen > chunk ? (uint32_t)((s.seen - 1) / chunk) + 1 : 1u; }

// What a row sees: tokens 0 .. limit - 1.
__device__ __forceinline__ int limit_of(const Params &p, const Sequence &s, int token) { // token: of the sequence's rows
    const int n = s.length - s.rows + token + 1;
    return !p.causal || n > s.seen ? s.seen : n < 0 ? 0 : n;
}

int launch_rows_f16(const Params &p, int size, int row_blocks, unsigned blocks, void *stream);  // returns hipError_t as int
int launch_rows_bf16(const Params &p, int size, int row_blocks, unsigned blocks, void *stream);
int launch_tiles_f16(const Params &p, int size, int waves, unsigned blocks, void *stream);
int launch_tiles_bf16(const Params &p, int size, int waves, unsigned blocks, void *stream);
int launch_join(const Params &p, int dtype, int size, int tile_rows, unsigned tiles, void *stream);

} // namespace attend
} // namespace mcf
