// Rotary position embedding over time, row and column (rotary_embed).
//
// Pair i of a head (elements 2i, 2i+1) belongs to one axis' band and is turned
// by the angle position * theta^(-j / n) of that axis, j its index in the band
// of n pairs. Every byte of x is read once and written once, so the kernel is
// bound by HBM: one 256-thread block moves 1024 vectors of 16 bytes, four per
// thread with all loads in flight first, and while they are it computes the cos
// and sin of its tokens' angles, one per (token, pair), into a table in LDS that
// all heads of the token share. Angles, cos and sin are evaluated in double and
// rounded once to fp32 (rope.h); products and sums are fp32, rounded once to the
// output's type.
//
// Measured: q and k of 10800 tokens, 40 heads, D 128, bf16 to e4m3 (332 MB): 61.7 us, 5.4 TB/s, a
// plain copy of this card 4.9; 4680 tokens of 12 heads out of packed rows (58 MB) 10.5 us (15.0 with
// the 76 registers that the compiler takes by itself, six waves per SIMD); one token 3.3 us on the
// device, 9 a call.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "internal.h"
#include "rope.h"

namespace revisit {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kBlock = 256;
constexpr int kVecs = 4;                  // 16-byte vectors per thread
constexpr int kSpan = kBlock * kVecs;

// (x, y) of a pair as fp32, turned
__device__ __forceinline__ floatx2 turn(floatx2 p, CosSin r) { return floatx2{p[0] * r.c - p[1] * r.s, p[0] * r.s + p[1] * r.c}; }

__device__ __forceinline__ uint32_t pack_bf16(floatx2 p) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2)); }

// beyond the largest e4m3 value (448) the nearest value is that one; NaN stays NaN
__device__ __forceinline__ float e4m3_range(float x) { return x > 448.0f ? 448.0f : (x < -448.0f ? -448.0f : x); }

template <int kIn, bool kFp8>
__global__ __launch_bounds__(kBlock, 8) void rotary_kernel(RotaryArgs a, RotaryFreq f, unsigned blocks_q, unsigned blocks) {
    extern __shared__ CosSin table[];  // [tokens of the block][pairs]
    const unsigned block = row_block();
    if (block >= blocks) return;  // grid padding (uniform)
    const RotaryTensor& t = block < blocks_q ? a.t[0] : a.t[1];
    constexpr int kElems = 16 / kIn, kPairs = kElems / 2;
    const int64_t v0 = (int64_t)(block < blocks_q ? block : block - blocks_q) * kSpan;
    const int row_vecs = t.H * a.D / kElems, head_vecs = a.D / kElems;
    const int64_t n_vecs = (int64_t)a.n_tokens * row_vecs;
    // (v + 1/2) / row_vecs truncates to v / row_vecs exactly below 2^50: its error is
    // under v 2^-52 / row_vecs, its distance from a whole number at least 1 / (2 row_vecs)
    auto token_of = [&](int64_t v) -> int { return (int)(((double)v + 0.5) * t.inv_row_vecs); };
    const int first = token_of(v0);
    const int last = token_of(min(v0 + kSpan, n_vecs) - 1);

    u32x4 buf[kVecs];
    int tok[kVecs], col[kVecs];
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int64_t v = v0 + threadIdx.x + i * kBlock;
        tok[i] = token_of(v);
        col[i] = (int)(v - (int64_t)tok[i] * row_vecs);
        buf[i] = u32x4{0, 0, 0, 0};
        if (v < n_vecs)
            buf[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(t.x) +
                                                                               (int64_t)tok[i] * t.x_row_bytes) + col[i]);
    }

    const int P = a.n_t + a.n_y + a.n_x;
    const int entries = (last - first + 1) * P;
    for (int e = threadIdx.x; e < entries; e += kBlock) {
        const int r = (int)(((float)e + 0.5f) * a.inv_pairs);  // at most 4608 entries: exact
        const int pair = e - r * P;
        const int token = first + r;
        const int axis = pair < a.n_t ? 0 : (pair < a.n_t + a.n_y ? 1 : 2);
        double at;
        if (a.pos) {
            at = (double)a.pos[(int64_t)token * 3 + axis];
        } else {
            const int frame = (int)(((double)token + 0.5) * a.inv_hw);
            const int in = token - frame * a.hw;
            const int y = (int)(((double)in + 0.5) * a.inv_w);
            at = axis == 0 ? (double)a.t0 + (double)frame : (axis == 1 ? (double)y : (double)(in - y * a.w));
        }
        CosSin cs = quarter_turns(at * f.quarter[pair]);
        if (a.inverse) cs.s = -cs.s;
        table[e] = cs;
    }
    __syncthreads();

#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
        const int64_t v = v0 + threadIdx.x + i * kBlock;
        if (v >= n_vecs) continue;
        const int p0 = (col[i] % head_vecs) * kPairs;
        const CosSin* cs = table + (tok[i] - first) * P + p0;
        uint8_t* o = static_cast<uint8_t*>(t.o) + (int64_t)tok[i] * t.o_row_bytes;
        u32x4 w = buf[i];
        if constexpr (kFp8) {
            u32x2 out;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t word = 0;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int q = 2 * j + h;
                    floatx2 p = {__uint_as_float(w[q] << 16), __uint_as_float(w[q] & 0xffff0000u)};
                    if (p0 + q < P) p = turn(p, cs[q]);
                    const float x = e4m3_range(p[0] * t.scale), y = e4m3_range(p[1] * t.scale);
                    word = h ? __builtin_amdgcn_cvt_pk_fp8_f32(x, y, word, true) : __builtin_amdgcn_cvt_pk_fp8_f32(x, y, word, false);
                }
                out[j] = word;
            }
            __builtin_nontemporal_store(out, reinterpret_cast<u32x2*>(o) + col[i]);
        } else {
#pragma unroll
            for (int q = 0; q < kPairs; ++q) {
                if (p0 + q >= P) continue;  // behind the last band: copied
                if constexpr (kIn == 2) {
                    w[q] = pack_bf16(turn(floatx2{__uint_as_float(w[q] << 16), __uint_as_float(w[q] & 0xffff0000u)}, cs[q]));
                } else {
                    const floatx2 p = turn(floatx2{__uint_as_float(w[2 * q]), __uint_as_float(w[2 * q + 1])}, cs[q]);
                    w[2 * q] = __float_as_uint(p[0]);
                    w[2 * q + 1] = __float_as_uint(p[1]);
                }
            }
            __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(o) + col[i]);
        }
    }
}

int64_t blocks_of(const RotaryArgs& a, int which) {
    if (!a.t[which].x) return 0;
    const int64_t vecs = (int64_t)a.n_tokens * (a.t[which].H * (int64_t)a.D * a.esize / 16);
    return (vecs + kSpan - 1) / kSpan;
}

}  // namespace

int64_t rotary_blocks(const RotaryArgs& a) { return blocks_of(a, 0) + blocks_of(a, 1); }

hipError_t launch_rotary(const RotaryArgs& a, const RotaryFreq& f, hipStream_t stream) {
    const unsigned blocks_q = (unsigned)blocks_of(a, 0), blocks = (unsigned)rotary_blocks(a);
    if (blocks == 0) return hipSuccess;
    // tokens that a block of kSpan vectors touches at most, and their table
    int rows = 1;
    for (int i = 0; i < 2; ++i) {
        if (!a.t[i].x) continue;
        const int row_vecs = a.t[i].H * a.D * a.esize / 16;
        const int touched = (kSpan + row_vecs - 2) / row_vecs + 1;
        rows = touched > rows ? touched : rows;
    }
    const unsigned lds = (unsigned)(rows * (a.n_t + a.n_y + a.n_x) * sizeof(CosSin));
    const dim3 grid = grid_rows(blocks), block(kBlock);
    if (a.fp8_out) hipLaunchKernelGGL((rotary_kernel<2, true>), grid, block, lds, stream, a, f, blocks_q, blocks);
    else if (a.esize == 2) hipLaunchKernelGGL((rotary_kernel<2, false>), grid, block, lds, stream, a, f, blocks_q, blocks);
    else hipLaunchKernelGGL((rotary_kernel<4, false>), grid, block, lds, stream, a, f, blocks_q, blocks);
    return hipGetLastError();
}

}  // namespace revisit
