// The sequences of a call on the device (mcf_sequences): which rows belong to a sequence, and which sequence a block
// of work belongs to.  starts, lengths and table are the caller's device memory: every number from there is held to the
// bounds of the buffers before it becomes an address.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/mcf_cache.h"
#include "mcf_internal.h"

namespace mcf {

struct Sequences {
    const int32_t *starts, *lengths, *table;
    int64_t table_stride;
    int32_t batch, tokens, table_width;
    int32_t capacity; // tokens that a row of the table reaches, at most 2^31 - 1
};

struct Sequence {
    int first, rows; // its rows in the token tensors
    int length;      // its tokens, those rows the last of them (fewer than rows: the first rows have no place)
    int seen;        // tokens that the table reaches
};

__device__ __forceinline__ Sequence sequence(const Sequences &s, int b) {
    Sequence q;
    if (s.starts) {
        const int lo = s.starts[b], hi = s.starts[b + 1];
        q.first = lo < 0 ? 0 : lo > s.tokens ? s.tokens : lo;
        const int end = hi < 0 ? 0 : hi > s.tokens ? s.tokens : hi;
        q.rows = end > q.first ? end - q.first : 0;
    } else {
        q.first = b;
        q.rows = b < s.tokens ? 1 : 0;
    }
    const int n = s.lengths[b];
    q.length = n > 0 ? n : 0;
    q.seen = q.length < s.capacity ? q.length : s.capacity;
    return q;
}

// The sequence that number `slot` belongs to where sequence b has count(b) of them, and its number within that sequence.
// By a whole wave, 64 sequences at a time; every lane gets the answer.  False: beyond the last.
template <typename F> __device__ __forceinline__ bool locate(uint32_t slot, int batch, F count, int *b, uint32_t *rest) {
    const int lane = threadIdx.x & 63;
    for (int b0 = 0; b0 < batch; b0 += 64) {
        const uint32_t n = b0 + lane < batch ? count(b0 + lane) : 0u;
        uint32_t upto = n; // inclusive sum
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t x = __shfl_up(upto, d);
            if (lane >= d) upto += x;
        }
        const uint64_t hit = __ballot(slot - (upto - n) < n);
        if (hit) {
            const int at = __builtin_ctzll(hit);
            *b = b0 + at;
            *rest = slot - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(n, at));
            return true;
        }
        slot -= __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// The same with the sequence itself, of which up to 64 are read once.
template <typename F> __device__ __forceinline__ bool locate_sequence(const Sequences &all, uint32_t slot, F count, int *b, uint32_t *rest, Sequence *s) {
    if (all.batch > 64) {
        if (!locate(slot, all.batch, [&](int i) __attribute__((always_inline)) { return count(sequence(all, i)); }, b, rest)) return false;
        *b = __builtin_amdgcn_readfirstlane(*b);
        *s = sequence(all, *b);
        return true;
    }
    const int lane = threadIdx.x & 63;
    Sequence q = {0, 0, 0, 0};
    if (lane < all.batch) q = sequence(all, lane);
    const uint32_t n = count(q);
    uint32_t upto = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
    }
    const uint64_t hit = __ballot(slot - (upto - n) < n);
    if (!hit) return false;
    const int i = __builtin_ctzll(hit);
    *b = i;
    *rest = slot - (__builtin_amdgcn_readlane(upto, i) - __builtin_amdgcn_readlane(n, i));
    *s = {__builtin_amdgcn_readlane(q.first, i), __builtin_amdgcn_readlane(q.rows, i), __builtin_amdgcn_readlane(q.length, i), __builtin_amdgcn_readlane(q.seen, i)};
    return true;
}

// The sequence that row t belongs to (starts ascending), -1: none.
__device__ __forceinline__ int sequence_of_row(const Sequences &s, int t) {
    if (!s.starts) return t < s.batch ? t : -1;
    int lo = 0, hi = s.batch; // the last b with starts[b] <= t
    while (lo < hi) {
        const int mid = lo + ((hi - lo + 1) >> 1);
        if (s.starts[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo < s.batch && s.starts[lo] <= t && t < s.starts[lo + 1] ? lo : -1;
}

inline int check_sequences(const mcf_sequences &s) {
    if (s.batch < 0 || s.tokens < 0 || s.table_width < 0) return MCF_EINVAL;
    if (s.batch > (1 << 24) || s.tokens >= (1ll << 31) - 1024 || s.table_width >= 1ll << 31) return MCF_EUNSUPPORTED;
    if (s.batch > 0 && (!s.lengths || (s.table_width > 0 && !s.table))) return MCF_EINVAL;
    if (!s.starts && s.tokens != s.batch) return MCF_EINVAL;
    if (((uintptr_t)s.starts | (uintptr_t)s.lengths | (uintptr_t)s.table) % 4 != 0) return MCF_EALIGN;
    if (s.batch > 1 && s.table_stride < 0) return MCF_EINVAL;
    if (s.table_stride >= 1ll << 40) return MCF_EUNSUPPORTED;
    return MCF_OK;
}

inline Sequences device_sequences(const mcf_sequences &s, int64_t page_size) {
    Sequences o;
    o.starts = s.starts; o.lengths = s.lengths; o.table = s.table;
    o.table_stride = s.table_stride;
    o.batch = (int32_t)s.batch; o.tokens = (int32_t)s.tokens; o.table_width = (int32_t)s.table_width;
    const int64_t reach = s.table_width * page_size;
    o.capacity = (int32_t)(reach < (1ll << 31) - 1024 ? reach : (1ll << 31) - 1024);
    return o;
}

// The cache as a kernel sees it: sizes and strides checked, in elements (bytes).
inline int check_cache(const mcf_kv_cache &c) {
    if (c.pages < 0 || c.heads < 0) return MCF_EINVAL;
    if (c.page_size != 16 && c.page_size != 32 && c.page_size != 64 && c.page_size != 128) {
        set_last_error("pages hold 16, 32, 64 or 128 tokens");
        return MCF_EUNSUPPORTED;
    }
    if (c.size != 64 && c.size != 80 && c.size != 96 && c.size != 128 && c.size != 192 && c.size != 256) {
        set_last_error("the cache holds heads of 64, 80, 96, 128, 192 or 256");
        return MCF_EUNSUPPORTED;
    }
    if (c.pages >= 1ll << 31 || c.heads >= 1 << 20) return MCF_EUNSUPPORTED;
    if (c.pages == 0 || c.heads == 0) return MCF_OK;
    if (!c.k || !c.v || !c.k_scale || !c.v_scale) return MCF_EINVAL;
    if (((uintptr_t)c.k | (uintptr_t)c.v) % 16 != 0 || ((uintptr_t)c.k_scale | (uintptr_t)c.v_scale) % 4 != 0) return MCF_EALIGN;
    const int64_t tile = c.page_size * c.size;
    for (const int64_t *s : {c.k_stride, c.v_stride}) {
        const int64_t sp = c.pages > 1 ? s[0] : 0, sh = c.heads > 1 ? s[1] : 0;
        if (sp % 16 != 0 || sh % 16 != 0) return MCF_EALIGN;
        if (sp < 0 || sh < 0 || sp >= 1ll << 32 || sh >= (1ll << 60) / c.heads) return MCF_EUNSUPPORTED; // (page numbers times 32 bits)
        // pages and heads may lie in either order, but not on top of one another
        const bool heads_inside = sh <= sp || c.pages == 1;
        const int64_t in = heads_inside ? sh : sp, n_in = heads_inside ? c.heads : c.pages, outer = heads_inside ? sp : sh, n_out = heads_inside ? c.pages : c.heads;
        if (n_in > 1 && in < tile) return MCF_EINVAL;
        if (n_out > 1 && outer < (n_in > 1 ? in * (n_in - 1) : 0) + tile) return MCF_EINVAL;
    }
    if (c.pages > 1 && (c.k_scale_stride < c.heads || c.v_scale_stride < c.heads)) return MCF_EINVAL;
    if (c.k_scale_stride >= 1ll << 30 || c.v_scale_stride >= 1ll << 30) return MCF_EUNSUPPORTED;
    return MCF_OK;
}

} // namespace mcf
