// The paged cache: where the tokens of the streams lie (paged_append.hip, paged_attention.hip).
//
// cache [n_pages][H][page][D]: a page holds `page` (a power of two, at least 32) consecutive positions of one
// stream, head by head, so that a head's share of a page is one run of bytes. Entry i of a stream's row of the
// page table is the page of its positions [i page, (i + 1) page). Pages of 8 bits have a scale for each 32
// positions of a head: [n_pages][H][page / 32] bytes, 2^(byte - 127).
//
// That is how pools lie that come without a layout. With one, pages, heads and positions are any distances apart, and a
// position's D elements alone lie together. Such pools have kernels of their own: in those for contiguous ones the distances are
// numbers in the code. [pages][page][H][D] in 8 bits beside contiguous: 4680 queries on 28080 keys 920 us and 877, 10800
// tokens of 40 heads appended 65 and 61, one query on 37440 keys 26.7 and 24.8; but 64 single tokens of up to 16384 keys, 8
// heads, 332 and 258. A head's rows are 1024 bytes apart there, a power of two, and few workgroups then ask few of the
// memory's channels: with rows of 1152 bytes 260, with key_parts = 3 instead of the one part that is chosen 261. The
// choice does not know the layout, since the workspace's size does not. Other heads in turn on each XCD: 338.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"

namespace revisit {

constexpr int kScaleBlock = 32;    // positions that share a scale
constexpr int kScaleLow = -100;    // smallest exponent that is written: 2^-110, the smallest value, is far above what bf16 flushes

typedef const __attribute__((address_space(4))) int32_t const_i32;  // memory that does not change while the kernel runs

// Element i of a list that no output overlaps: a scalar load where i is uniform.
__device__ __forceinline__ int32_t listed(const int32_t* list, int64_t i) { return reinterpret_cast<const_i32*>((uintptr_t)list)[i]; }

// Positions that stream s holds, within what its row of the table can hold.
__device__ __forceinline__ int held_of(const PagedSeqs& q, int s) { return min(max(listed(q.kv_len, s), 0), q.max_pages << q.page_log2); }

// First token of stream s among the call's and how many it has. Lists that are not ascending give no access out of range.
__device__ __forceinline__ int2 tokens_of(const PagedSeqs& q, int s) {
    if (!q.cu) return make_int2(s * q.per, q.per);
    const int a = min(max(listed(q.cu, s), 0), q.n_tokens);
    return make_int2(a, max(min(listed(q.cu, (int64_t)s + 1), q.n_tokens), a) - a);
}

// Page of entry i of stream s, or -1: outside the table's row or the pool.
__device__ __forceinline__ int page_of(const PagedSeqs& q, int s, int i) {
    if (i >= q.max_pages) return -1;
    const int p = listed(q.page_table, (int64_t)s * q.max_pages + i);
    return p < q.n_pages ? p : -1;
}

// Byte of a strided pool at which position (block) `row` of a head's page begins.
__device__ __forceinline__ int64_t strided_at(const PagedStrides& s, int page, int head, int row) { return page * s.page + head * s.head + row * s.row; }

// Stream s and its item `in` that a call's unit stands for, where stream s has count(s) items; s = -1 past the
// last. The whole wave takes part: 64 streams at a time, whose counts are added up across its lanes.
struct StreamItem {
    int s, in;
};
template <class Count>
__device__ __forceinline__ StreamItem find_item(int B, int unit, Count count) {
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int base = 0; base < B; base += 64) {
        const int s = base + lane;
        const int c = s < B ? count(s) : 0;
        int sum = c;
#pragma unroll
        for (int off = 1; off < 64; off *= 2) {
            const int x = __shfl_up(sum, off);
            sum += lane >= off ? x : 0;
        }
        const unsigned long long past = __ballot(before + sum > unit);
        if (past) {
            const int l = __ffsll((long long)past) - 1;
            return StreamItem{base + l, unit - before - __builtin_amdgcn_readlane(sum - c, l)};
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return StreamItem{-1, 0};
}

// Stream and tile of `rows` (query, head of the group) rows that number `tile` of a key head's tiles stands for. A stream's
// tiles come in falling order: the last queries of a causal prompt have the most keys, and start first.
__device__ __forceinline__ StreamItem row_tile(const PagedAttentionArgs& a, int rows, int tile) {
    const PagedSeqs& q = a.seqs;
    auto count = [&](int s) { return (tokens_of(q, s).y * a.G + rows - 1) / rows; };
    StreamItem it;
    if (q.cu) {
        it = find_item(q.B, tile, count);
        if (it.s < 0) return it;
    } else {
        const int each = (q.per * a.G + rows - 1) / rows;
        it.s = tile / each;
        it.in = tile - it.s * each;
    }
    it.in = count(it.s) - 1 - it.in;
    return it;
}

// floats of a part's result of a tile: O [rows][D], maxima [rows], sums [rows]
__host__ __device__ constexpr int paged_part_floats(int rows, int D) { return rows * (D + 2); }

// 2^(byte - 127) of a scale: byte 0 counts as 1, 255 is NaN
__device__ __forceinline__ float scale_value(int byte) { return byte == 255 ? NAN : __uint_as_float((uint32_t)max(byte, 1) << 23); }

// two e4m3 values (the low or high half of x) times a power of two, as bf16: exact
template <bool kHigh>
__device__ __forceinline__ uint32_t widen2(uint32_t x, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, kHigh));
}

// Which values of a word are not finite, by their top bits: e4m3 with all seven bits set, bf16 and fp32 with an exponent
// of ones. Under a scale of 2^120 and more (bytes from 247 on) codes from 2^(255 - byte) on stand for 2^128 and more, which are
// infinities in bf16, and under a NaN scale none is finite: odd_codes(scale) is what is added to the seven bits of each
// code, so that it passes into the top one. spread: all bits of those values.
constexpr uint32_t kOddCodes = 0x01010101u;
__device__ __forceinline__ uint32_t odd_codes(float scale) {
    const int byte = (int)(__float_as_uint(scale) >> 23);  // 255: NaN
    const int from = max(0x80 - ((262 - byte) << 3), 1);   // (262 - byte) << 3 is the code of 2^(255 - byte)
    return (uint32_t)(byte == 255 ? 0x80 : from) * kOddCodes;
}
template <int T>
__device__ __forceinline__ uint32_t not_finite(uint32_t x, uint32_t odd = kOddCodes) {
    if constexpr (T == kPagedFp8) return ((x & 0x7f7f7f7fu) + odd) & 0x80808080u;
    else if constexpr (T == kPagedBf16) return ((x & 0x7fff7fffu) + 0x00800080u) & 0x80008000u;
    else return ((x & 0x7fffffffu) + 0x00800000u) & 0x80000000u;
}
template <int T>
__device__ __forceinline__ uint32_t spread(uint32_t top) {
    if constexpr (T == kPagedFp8) return (top >> 7) * 0xffu;
    else if constexpr (T == kPagedBf16) return (top >> 15) * 0xffffu;
    else return top ? ~0u : 0u;
}
// Element d of a stored row (8 bits: without its scale).
template <int T>
__device__ __forceinline__ float stored(const uint8_t* row, int d) {
    if constexpr (T == kPagedFp8) return __builtin_amdgcn_cvt_f32_fp8(row[d], 0);
    else if constexpr (T == kPagedBf16) return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(row)[d] << 16);
    else return reinterpret_cast<const float*>(row)[d];
}

}  // namespace revisit
