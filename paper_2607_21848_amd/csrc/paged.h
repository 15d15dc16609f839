// The paged cache: where the tokens of the streams lie (paged_append.hip, paged_attention.hip).
//
// cache [n_pages][H][page][D]: a page holds `page` (a power of two, at least 32) consecutive positions of one
// stream, head by head, so that a head's share of a page is one run of bytes. Entry i of a stream's row of the
// page table is the page of its positions [i page, (i + 1) page). Pages of 8 bits have a scale for each 32
// positions of a head: [n_pages][H][page / 32] bytes, 2^(byte - 127).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"

namespace revisit {

constexpr int kScaleBlock = 32;    // positions that share a scale
constexpr int kScaleLow = -100;    // smallest exponent that is written: 2^-110, the smallest value, is far above what bf16 flushes
constexpr int kScaleHigh = 120;    // largest one that an fp32 value needs

// Positions that stream s holds, within what its row of the table can hold.
__device__ __forceinline__ int held_of(const PagedSeqs& q, int s) { return min(max(q.kv_len[s], 0), q.max_pages << q.page_log2); }

// First token of stream s among the call's and how many it has. Lists that are not ascending give no access out of range.
__device__ __forceinline__ int2 tokens_of(const PagedSeqs& q, int s) {
    if (!q.cu) return make_int2(s * q.per, q.per);
    const int a = min(max(q.cu[s], 0), q.n_tokens);
    return make_int2(a, max(min(q.cu[s + 1], q.n_tokens), a) - a);
}

// Page of entry i of stream s, or -1: outside the table's row or the pool.
__device__ __forceinline__ int page_of(const PagedSeqs& q, int s, int i) {
    if (i >= q.max_pages) return -1;
    const int p = q.page_table[(int64_t)s * q.max_pages + i];
    return p < q.n_pages ? p : -1;
}

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

}  // namespace revisit
