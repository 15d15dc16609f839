// The move of a cache's kept units into a smaller one (compact_kv).
//
// A stream: every kept byte is read once and written once, so the kernel is
// bound by HBM. One 256-thread block moves 1024 vectors of 16 bytes of one
// layer's keys or values, four per thread with all loads in flight first; a
// vector's unit, and with it its source row, comes from the selection. Keys whose
// unit moves to another frame position have their temporal pairs turned
// (rope.h); everything else is copied bit for bit.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

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
            u32x4& w = buf[i];
#pragma unroll
            for (int q = 0; q < kPairs; ++q) {
                if (p0 + q >= a.n_t) continue;
                const CosSin cs = quarter_turns(delta * f.quarter[p0 + q]);
                if constexpr (ES == 2) {
                    w[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector(
                        turn(floatx2{__uint_as_float(w[q] << 16), __uint_as_float(w[q] & 0xffff0000u)}, cs), bf16x2));
                } else {
                    const floatx2 p = turn(floatx2{__uint_as_float(w[2 * q]), __uint_as_float(w[2 * q + 1])}, cs);
                    w[2 * q] = __float_as_uint(p[0]);
                    w[2 * q + 1] = __float_as_uint(p[1]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
        if (from[i] >= 0) __builtin_nontemporal_store(buf[i], dst + v0 + i * kBlock);
}

// KS, VS: bytes of a key's and a value's element
template <int KS, int VS>
__global__ __launch_bounds__(kBlock) void compact_kernel(CompactArgs a, CompactFreq f, unsigned k_blocks, unsigned v_blocks,
                                                         unsigned w_blocks, unsigned blocks) {
    const unsigned block = row_block();
    if (block >= blocks) return;  // grid padding (uniform)
    const unsigned per_layer = k_blocks + v_blocks + w_blocks;
    const int layer = (int)(block / per_layer);
    unsigned b = block - (unsigned)layer * per_layer;
    if (b < k_blocks) {
        if constexpr (KS > 1) {
            if (a.n_t > 0) return move<KS, true>(a, f, a.src_k, a.dst_k, layer, b);
        }
        return move<KS, false>(a, f, a.src_k, a.dst_k, layer, b);
    }
    b -= k_blocks;
    if (b < v_blocks) return move<VS, false>(a, f, a.src_v, a.dst_v, layer, b);
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

// blocks of one layer's keys, values and weights
int64_t blocks_of(const CompactArgs& a, int bytes) { return ((int64_t)a.keep * a.unit * a.H * a.D * bytes / 16 + kSpan - 1) / kSpan; }
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
    if (a.k_bytes == 1) hipLaunchKernelGGL((compact_kernel<1, 2>), grid, block, 0, stream, a, f, kb, vb, wb, blocks);
    else if (a.k_bytes == 2) hipLaunchKernelGGL((compact_kernel<2, 2>), grid, block, 0, stream, a, f, kb, vb, wb, blocks);
    else hipLaunchKernelGGL((compact_kernel<4, 4>), grid, block, 0, stream, a, f, kb, vb, wb, blocks);
    return hipGetLastError();
}

}  // namespace revisit
