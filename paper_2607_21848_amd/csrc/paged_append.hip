// New keys and values of several streams into the pages of their cache (append_paged_kv).
//
// Keys are turned by the rotary embedding of their position (time, row, column) on the way, as rotary_embed turns
// them; values are copied. Pages of 8 bits: the 32 positions of a block share a scale per head, keys and
// values each their own. It is a power of two, the least that brings the block's largest finite value to 448 or below
// (but 2^-100 at least): e4m3 is a floating format, so the rounding of its normal values does not depend on a power of
// two, a code times its scale is a bf16 value exactly, and a block that grows rounds again only what falls below
// the new scale's smallest normal value. Where a block held positions before, its scale only grows, and their codes
// are rounded to the new one.
//
// Every input byte is read once and every output byte written once: bound by HBM. One wave takes a (block of 32
// positions, head), so that it has what a scale depends on in its registers: all loads leave first, the
// angles' cos and sin, which the four heads of a workgroup share, are computed while they are in flight.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "internal.h"
#include "paged.h"
#include "rope.h"

namespace revisit {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;  // heads of a workgroup

__device__ __forceinline__ floatx2 turn(floatx2 p, CosSin r) { return floatx2{p[0] * r.c - p[1] * r.s, p[0] * r.s + p[1] * r.c}; }

__device__ __forceinline__ uint32_t pack_bf16(floatx2 p) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2)); }

// bits of |x| where x is finite, else 0
__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// what is not finite is stored as NaN: e4m3 has no infinity, and its largest value would hide one
__device__ __forceinline__ float nan_if_not_finite(float x) { return finite_bits(x) == (__float_as_uint(x) & 0x7fffffffu) ? x : NAN; }

// least e in [kScaleLow, kScaleHigh] with m <= 448 2^e, m >= 0 by its bits: 448 = 1.75 2^8
__device__ __forceinline__ int scale_exponent(uint32_t m) {
    const int e = (int)(m >> 23) - 127 - 8 + ((m & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, kScaleLow);
}

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // e in [-126, 127]

__device__ __forceinline__ uint32_t pack_e4m3(floatx2 a, floatx2 b) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a[0], a[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(b[0], b[1], lo, true);
}

// Codes of `rows` positions, rounded again from the scale 2^was to 2^now.
template <int D>
__device__ __forceinline__ void round_again(uint8_t* codes, int rows, int was, int now, int lane) {
    constexpr int kLanes = D / 8, kRows = 64 / kLanes;
    const float f = was - now < -126 ? 0.0f : power_of_two(was - now);
    for (int r = lane / kLanes; r < rows; r += kRows) {
        u32x2* p = reinterpret_cast<u32x2*>(codes + r * D) + lane % kLanes;
        u32x2 w = *p;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const floatx2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
            w[i] = pack_e4m3(floatx2{a[0] * f, a[1] * f}, floatx2{b[0] * f, b[1] * f});
        }
        *p = w;
    }
}

template <int D, int ES, bool kFp8>
__global__ __launch_bounds__(64 * kWaves, D == 128 ? 3 : 4) void append_kernel(PagedAppendArgs a, PagedFreq f, unsigned blocks) {
    constexpr int kElems = 16 / ES, kPairs = kElems / 2;      // of a lane's vector
    constexpr int kLanes = D / kElems, kRows = 64 / kLanes;   // lanes of a row, rows of a load
    constexpr int kLoads = kScaleBlock / kRows;
    __shared__ CosSin table[kScaleBlock * (D / 2)];  // [new row of the block][pair]
    __shared__ int at[kScaleBlock][3];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const PagedSeqs& q = a.seqs;
    const unsigned block = row_block();
    // the streams' new lengths
    if (a.out_len) {
        const int64_t stride = (int64_t)gridDim.x * gridDim.y * (64 * kWaves);
        for (int64_t s = (int64_t)block * (64 * kWaves) + tid; s < q.B; s += stride) {
            const int n = tokens_of(q, (int)s).y, held = held_of(q, (int)s);
            a.out_len[s] = (int)min((int64_t)held + n, (int64_t)(q.max_pages << q.page_log2));
        }
    }
    if (block >= blocks) return;  // grid padding (uniform)
    const int groups = (a.H + kWaves - 1) / kWaves;
    const int piece = (int)(block / (unsigned)groups);
    const int head = (int)(block - (unsigned)piece * (unsigned)groups) * kWaves + wave;

    // the stream's piece: one block of 32 positions that its new tokens touch
    auto pieces = [&](int s) -> int {
        const int n = tokens_of(q, s).y;
        return n > 0 ? (held_of(q, s) % kScaleBlock + n + kScaleBlock - 1) / kScaleBlock : 0;
    };
    StreamItem it;
    if (q.cu) {
        it = find_item(q.B, piece, pieces);
        if (it.s < 0) return;
    } else {  // room for the most pieces that q.per tokens can touch
        const int most = (q.per + 2 * kScaleBlock - 2) / kScaleBlock;
        it.s = piece / most;
        it.in = piece - it.s * most;
        if (it.in >= pieces(it.s)) return;
    }
    const int held = held_of(q, it.s);
    const int2 tok = tokens_of(q, it.s);
    const int start = held / kScaleBlock * kScaleBlock + it.in * kScaleBlock;
    const int lo = max(held - start, 0), hi = (int)min((int64_t)held + tok.y - start, (int64_t)kScaleBlock);  // its new rows
    const int page = page_of(q, it.s, start >> q.page_log2);
    if (page < 0) return;  // nowhere to store them (uniform)
    const int row0 = start & ((1 << q.page_log2) - 1);
    const bool live = head < a.H;

    // row r of the block is token tok.x + start + r - held
    const int64_t first = (int64_t)tok.x + start - held;
    const int r_lane = lane / kLanes, c_lane = lane % kLanes;
    u32x4 x[2][kLoads];
    auto load = [&](int which) {
        const uint8_t* src = static_cast<const uint8_t*>(which ? a.v : a.k) + (size_t)head * D * ES + 16 * c_lane;
        const int64_t row = which ? a.v_row_bytes : a.k_row_bytes;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = i * kRows + r_lane;
            x[which][i] = u32x4{0, 0, 0, 0};
            if (live && r >= lo && r < hi) x[which][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + (first + r) * row));
        }
    };
    load(0);
    if constexpr (ES == 2) load(1);

    const int P = a.n_t + a.n_y + a.n_x;
    if (tid < kScaleBlock && tid >= lo && tid < hi) {
        if (a.pos) {
#pragma unroll
            for (int j = 0; j < 3; ++j) at[tid][j] = a.pos[(first + tid) * 3 + j];
        } else {
            const int c = start + tid, frame = c / a.hw, in = c - frame * a.hw, y = in / a.w;
            at[tid][0] = frame;
            at[tid][1] = y;
            at[tid][2] = in - y * a.w;
        }
    }
    __syncthreads();
    const double t0 = a.pos ? 0.0 : (double)a.t0;
    for (int e = tid; e < (hi - lo) * P; e += 64 * kWaves) {
        const int r = (int)(((float)e + 0.5f) * a.inv_pairs);  // at most 2048 entries: exact
        const int pair = e - r * P;
        const int axis = pair < a.n_t ? 0 : (pair < a.n_t + a.n_y ? 1 : 2);
        table[e] = quarter_turns(((double)at[lo + r][axis] + (axis == 0 ? t0 : 0.0)) * f.quarter[pair]);
    }
    __syncthreads();
    if (!live) return;

    const size_t slot = ((size_t)page * a.H + head) << q.page_log2;  // first position of the head's page
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        if constexpr (ES == 4) {
            if (which == 1) load(1);
        }
        uint8_t* out = static_cast<uint8_t*>(which ? a.cache_v : a.cache_k) + (slot + row0) * (size_t)(D * (kFp8 ? 1 : ES));
        floatx2 p[kFp8 ? kLoads : 1][kPairs];
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = i * kRows + r_lane;
            const bool ok = r >= lo && r < hi;
            const CosSin* cs = table + (ok ? r - lo : 0) * P;
            floatx2* pi = p[kFp8 ? i : 0];
            u32x4& w = x[which][i];
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                if constexpr (ES == 2) pi[j] = floatx2{__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u)};
                else pi[j] = floatx2{__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1])};
                const int pair = c_lane * kPairs + j;
                const bool turned = which == 0 && pair < P;
                if (turned && ok) pi[j] = turn(pi[j], cs[pair]);
                if constexpr (kFp8) {
                    most = max(most, max(finite_bits(pi[j][0]), finite_bits(pi[j][1])));
                } else if (turned) {
                    if constexpr (ES == 2) {
                        w[j] = pack_bf16(pi[j]);
                    } else {
                        w[2 * j] = __float_as_uint(pi[j][0]);
                        w[2 * j + 1] = __float_as_uint(pi[j][1]);
                    }
                }
            }
            if constexpr (!kFp8) {
                if (ok) *reinterpret_cast<u32x4*>(out + r * (D * ES) + 16 * c_lane) = w;
            }
        }
        if constexpr (kFp8) {
#pragma unroll
            for (int off = 1; off < 64; off *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, off));
            int e = scale_exponent(most);
            uint8_t* scale = (which ? a.scale_v : a.scale_k) + ((slot + row0) / kScaleBlock);
            if (lo > 0) {
                const int was = min((int)*scale, kScaleHigh + 127) - 127;
                if (e > was) round_again<D>(out, lo, was, e, lane);
                e = max(e, was);
            }
            const float inv = power_of_two(-e);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int r = i * kRows + r_lane;
                u32x2 w;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const floatx2 u = p[i][2 * j], v = p[i][2 * j + 1];
                    w[j] = pack_e4m3(floatx2{nan_if_not_finite(u[0] * inv), nan_if_not_finite(u[1] * inv)},
                                     floatx2{nan_if_not_finite(v[0] * inv), nan_if_not_finite(v[1] * inv)});
                }
                if (r >= lo && r < hi) *reinterpret_cast<u32x2*>(out + r * D + 8 * c_lane) = w;
            }
            if (lane == 0) *scale = (uint8_t)(e + 127);
        }
    }
}

}  // namespace

// Pieces (blocks of 32 positions of a stream) that the new tokens touch at most: each holds one of them, and a
// stream's n are in at most (n + 62) / 32.
int64_t paged_append_blocks(const PagedAppendArgs& a) {
    const PagedSeqs& q = a.seqs;
    const int64_t groups = (a.H + kWaves - 1) / kWaves;
    if (q.n_tokens == 0) return 0;
    if (!q.cu) return (int64_t)q.B * ((q.per + 2 * kScaleBlock - 2) / kScaleBlock) * groups;
    const int64_t streams = q.B < q.n_tokens ? q.B : q.n_tokens;
    const int64_t most = (q.n_tokens + streams * (2 * kScaleBlock - 2)) / kScaleBlock;
    return (most < q.n_tokens ? most : q.n_tokens) * groups;
}

hipError_t launch_paged_append(const PagedAppendArgs& a, const PagedFreq& f, hipStream_t stream) {
    const unsigned blocks = (unsigned)paged_append_blocks(a);
    if (blocks == 0 && !a.out_len) return hipSuccess;
    const dim3 grid = blocks ? grid_rows(blocks) : dim3(1), block(64 * kWaves);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, f, blocks); };
    if (a.D == 128) {
        if (a.dtype == kPagedFp8) launch(append_kernel<128, 2, true>);
        else if (a.dtype == kPagedBf16) launch(append_kernel<128, 2, false>);
        else launch(append_kernel<128, 4, false>);
    } else {
        if (a.dtype == kPagedFp8) launch(append_kernel<64, 2, true>);
        else if (a.dtype == kPagedBf16) launch(append_kernel<64, 2, false>);
        else launch(append_kernel<64, 4, false>);
    }
    return hipGetLastError();
}

}  // namespace revisit
