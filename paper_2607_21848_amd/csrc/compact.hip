// The move of a cache's kept units into a smaller one (compact_kv).
//
// A stream: every kept byte is read once and written once, so the kernel is
// bound by HBM. One 256-thread block moves 1024 vectors of 16 bytes of one
// layer's keys or values, four per thread with all loads in flight first; a
// vector's unit, and with it its source row, comes from the selection. Keys whose
// unit moves to another frame position have their temporal pairs turned
// (rope.h); everything else is copied bit for bit.
//
// Measured: 12 of 18 frames of 1560 tokens, 12 heads, D 128, 30 layers, bf16, keys turned, weights
// too (7.0 GB): 1.22 ms, 5.7 TB/s, a plain copy of this card 4.9; with an angle per
// pair and vector in place of move_unit's table 2.1 ms. Half of 7019 tokens, each head its own, 8 fp32 layers
// (697 MB) with their choice: 129 us, 5.4 TB/s.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "internal.h"
#include "rope.h"

namespace revisit {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 256;
constexpr int kVecs = 4;
constexpr int kSpan = kBlock * kVecs;

__device__ __forceinline__ floatx2 turn(floatx2 p, CosSin r) { return floatx2{p[0] * r.c - p[1] * r.s, p[0] * r.s + p[1] * r.c}; }

// turns the first n of a vector's pairs
template <int ES, class At>
__device__ __forceinline__ void turn_vec(u32x4& w, At cs, int n) {
#pragma unroll
    for (int q = 0; q < 8 / ES; ++q) {
        if (q >= n) continue;
        const CosSin r = cs[q];
        if constexpr (ES == 2) {
            w[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector(
                turn(floatx2{__uint_as_float(w[q] << 16), __uint_as_float(w[q] & 0xffff0000u)}, r), bf16x2));
        } else {
            const floatx2 p = turn(floatx2{__uint_as_float(w[2 * q]), __uint_as_float(w[2 * q + 1])}, r);
            w[2 * q] = __float_as_uint(p[0]);
            w[2 * q + 1] = __float_as_uint(p[1]);
        }
    }
}

// One block's vectors of a layer's keys or values. ES: bytes of an element; kTurn: keys whose temporal pairs may turn.
template <int ES, bool kTurn>
__device__ __forceinline__ void move(const CompactArgs& a, const CompactFreq& f, const void* src_base, void* dst_base, int layer, unsigned b) {
    constexpr int kElems = 16 / ES, kPairs = kElems / 2;
    const int32_t* sel = a.sel + (int64_t)layer * a.sel_heads * a.keep;
    const int head_vecs = a.D / kElems, row_vecs = a.H * head_vecs;
    const int64_t n_vecs = (int64_t)a.keep * a.unit * row_vecs;
    const double inv_row_vecs = 1.0 / row_vecs;
    const u32x4* src = static_cast<const u32x4*>(src_base) + (int64_t)layer * a.src_rows * row_vecs;
    u32x4* dst = static_cast<u32x4*>(dst_base) + ((int64_t)layer * a.dst_rows + a.dst_row0) * row_vecs;
    const int64_t v0 = (int64_t)b * kSpan + threadIdx.x;
    u32x4 buf[kVecs];
    int from[kVecs], to[kVecs], part[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int64_t v = v0 + i * kBlock;
        from[i] = -1;
        to[i] = part[i] = 0;
        buf[i] = u32x4{0, 0, 0, 0};
        if (v >= n_vecs) continue;
        // (v + 1/2) / n truncates to v / n exactly below 2^50: its error is under v 2^-51 / n,
        // its distance from a whole number at least 1 / (2 n)
        const int r = (int)(((double)v + 0.5) * inv_row_vecs);  // output row
        const int c = (int)(v - (int64_t)r * row_vecs);
        const int h = c / head_vecs;
        part[i] = c - h * head_vecs;
        to[i] = (int)(((double)r + 0.5) * a.inv_unit);
        const int u = sel[(a.sel_heads > 1 ? h : 0) * (int64_t)a.keep + to[i]];
        if (u < 0 || u >= a.n_units) continue;  // no such unit: the destination stays as it is
        from[i] = u;
        buf[i] = __builtin_nontemporal_load(src + ((int64_t)u * a.unit + (r - (int64_t)to[i] * a.unit)) * row_vecs + c);
    }
    if constexpr (kTurn) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
            const int p0 = part[i] * kPairs;
            if (from[i] < 0 || p0 >= a.n_t) continue;
            const double was = a.src_pos ? (double)a.src_pos[from[i]] : (double)from[i] * a.step;
            const double delta = (double)a.dst_pos + (double)to[i] * a.step - was;
            if (delta == 0.0) continue;  // stays where it was: bit for bit
            CosSin cs[kPairs];
#pragma unroll
            for (int q = 0; q < kPairs; ++q)
                if (p0 + q < a.n_t) cs[q] = quarter_turns(delta * f.quarter[p0 + q]);
            turn_vec<ES>(buf[i], cs, a.n_t - p0);
        }
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
        if (from[i] >= 0) __builtin_nontemporal_store(buf[i], dst + v0 + i * kBlock);
}

// Large units that all heads share: a unit's rows are one run of bytes in both caches, so
// block `b` moves 1024 vectors of one unit, by one offset, with one table of
// angles for its keys.
template <int ES, bool kTurn>
__device__ __forceinline__ void move_unit(const CompactArgs& a, const CompactFreq& f, const void* src_base, void* dst_base, int layer,
                                          unsigned b, unsigned parts, CosSin* table) {
    constexpr int kElems = 16 / ES, kPairs = kElems / 2;
    const int to = (int)(b / parts), part = (int)(b - (unsigned)to * parts);
    const int u = a.sel[(int64_t)layer * a.keep + to];
    if (u < 0 || u >= a.n_units) return;  // no such unit: the destination stays as it is (uniform)
    const int head_vecs = a.D / kElems, row_vecs = a.H * head_vecs;
    const int64_t unit_vecs = (int64_t)a.unit * row_vecs;
    const u32x4* src = static_cast<const u32x4*>(src_base) + ((int64_t)layer * a.src_rows + (int64_t)u * a.unit) * row_vecs;
    u32x4* dst = static_cast<u32x4*>(dst_base) + ((int64_t)layer * a.dst_rows + a.dst_row0 + (int64_t)to * a.unit) * row_vecs;
    const int64_t v0 = (int64_t)part * kSpan + threadIdx.x;
    u32x4 buf[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int64_t v = v0 + i * kBlock;
        buf[i] = v < unit_vecs ? __builtin_nontemporal_load(src + v) : u32x4{0, 0, 0, 0};
    }
    if constexpr (kTurn) {
        const double was = a.src_pos ? (double)a.src_pos[u] : (double)u * a.step;
        const double delta = (double)a.dst_pos + (double)to * a.step - was;
        if (delta != 0.0) {  // uniform; a unit that stays where it was is copied bit for bit
            if ((int)threadIdx.x < a.n_t) table[threadIdx.x] = quarter_turns(delta * f.quarter[threadIdx.x]);
            __syncthreads();
            int m = (int)(v0 % head_vecs);
            const int m_step = kBlock % head_vecs;
#pragma unroll
            for (int i = 0; i < kVecs; ++i) {
                const int p0 = m * kPairs;
                if (p0 < a.n_t) turn_vec<ES>(buf[i], table + p0, a.n_t - p0);
                m += m_step;
                if (m >= head_vecs) m -= head_vecs;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int64_t v = v0 + i * kBlock;
        if (v < unit_vecs) __builtin_nontemporal_store(buf[i], dst + v);
    }
}

// KS, VS: bytes of a key's and a value's element; kUnits: move_unit, else move. Blocks per
// layer: k_blocks, v_blocks and w_blocks.
template <int KS, int VS, bool kUnits>
__global__ __launch_bounds__(kBlock) void compact_kernel(CompactArgs a, CompactFreq f, unsigned k_blocks, unsigned v_blocks,
                                                         unsigned w_blocks, unsigned blocks) {
    __shared__ CosSin table[kUnits ? kRotaryMaxPairs : 1];
    const unsigned block = row_block();
    if (block >= blocks) return;  // grid padding (uniform)
    const unsigned per_layer = k_blocks + v_blocks + w_blocks;
    const int layer = (int)(block / per_layer);
    unsigned b = block - (unsigned)layer * per_layer;
    auto run = [&](auto es, auto turned, const void* src, void* dst, unsigned n_blocks) {
        constexpr int ES = decltype(es)::value;
        constexpr bool kTurn = decltype(turned)::value;
        if constexpr (kUnits) move_unit<ES, kTurn>(a, f, src, dst, layer, b, n_blocks / (unsigned)a.keep, table);
        else move<ES, kTurn>(a, f, src, dst, layer, b);
    };
    using K = std::integral_constant<int, KS>;
    using V = std::integral_constant<int, VS>;
    if (b < k_blocks) {
        if constexpr (KS > 1) {
            if (a.n_t > 0) return run(K{}, std::true_type{}, a.src_k, a.dst_k, k_blocks);
        }
        return run(K{}, std::false_type{}, a.src_k, a.dst_k, k_blocks);
    }
    b -= k_blocks;
    if (b < v_blocks) return run(V{}, std::false_type{}, a.src_v, a.dst_v, v_blocks);
    b -= v_blocks;
    // weights: [layer][head][token]
    const int64_t kept = (int64_t)a.keep * a.unit;
    const int32_t* sel = a.sel + (int64_t)layer * a.sel_heads * a.keep;
    for (int i = 0; i < kVecs; ++i) {
        const int64_t e = (int64_t)b * kSpan + i * kBlock + threadIdx.x;
        if (e >= kept * a.H) break;
        const int h = (int)(((double)e + 0.5) * a.inv_kept);
        const int64_t r = e - h * kept;
        const int to = (int)(((double)r + 0.5) * a.inv_unit);
        const int u = sel[(a.sel_heads > 1 ? h : 0) * (int64_t)a.keep + to];
        if (u < 0 || u >= a.n_units) continue;
        a.dst_w[((int64_t)layer * a.H + h) * a.dst_w_cols + a.dst_row0 + r] =
            a.src_w[((int64_t)layer * a.H + h) * a.src_w_cols + (int64_t)u * a.unit + (r - (int64_t)to * a.unit)];
    }
}

// Units of at least one block's vectors that all heads share go by move_unit. (Smaller
// ones would leave its blocks partly empty.)
bool by_unit(const CompactArgs& a) {
    return a.sel_heads == 1 && (int64_t)a.unit * a.H * a.D * a.k_bytes / 16 >= kSpan;
}
// blocks of one layer's keys, values and weights
int64_t blocks_of(const CompactArgs& a, int bytes) {
    const int64_t unit_vecs = (int64_t)a.unit * a.H * a.D * bytes / 16;
    if (by_unit(a)) return a.keep * ((unit_vecs + kSpan - 1) / kSpan);
    return (a.keep * unit_vecs + kSpan - 1) / kSpan;
}
int64_t weight_blocks(const CompactArgs& a) { return a.src_w ? ((int64_t)a.keep * a.unit * a.H + kSpan - 1) / kSpan : 0; }

}  // namespace

double compact_blocks(const CompactArgs& a) {
    return (double)a.n_layers * ((double)blocks_of(a, a.k_bytes) + (double)blocks_of(a, a.v_bytes) + (double)weight_blocks(a));
}

hipError_t launch_compact(const CompactArgs& a, const CompactFreq& f, hipStream_t stream) {
    const unsigned kb = (unsigned)blocks_of(a, a.k_bytes), vb = (unsigned)blocks_of(a, a.v_bytes), wb = (unsigned)weight_blocks(a);
    const unsigned blocks = (unsigned)a.n_layers * (kb + vb + wb);  // the caller keeps compact_blocks(a) below 2^31
    if (blocks == 0) return hipSuccess;
    const dim3 grid = grid_rows(blocks), block(kBlock);
    const bool units = by_unit(a);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, f, kb, vb, wb, blocks); };
    if (a.k_bytes == 1) units ? go(compact_kernel<1, 2, true>) : go(compact_kernel<1, 2, false>);
    else if (a.k_bytes == 2) units ? go(compact_kernel<2, 2, true>) : go(compact_kernel<2, 2, false>);
    else units ? go(compact_kernel<4, 4, true>) : go(compact_kernel<4, 4, false>);
    return hipGetLastError();
}

}  // namespace revisit
