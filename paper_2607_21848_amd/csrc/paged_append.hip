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
// angles' cos and sin, which the four heads of a workgroup share, are computed while they are in flight. A chunk's
// waves are all resident at once, so its time is one wave's: few instructions, and few waits one after the other.
// Lengths and pages come by scalar loads; largest values are found two bf16 at a time; a conversion takes the scale
// along. 10800 tokens of 40 heads of 128 into 8 bits 65.6 us (5.05 TB/s), 4680 of 12 heads 12.5 us, a token of each of
// 128 streams 7.7. Workgroups of eight waves: 70.5, 20.8 and 9.4 (of 65, 16 and 8.7 with four at that step).

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "internal.h"
#include "paged.h"
#include "rope.h"

namespace revisit {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short shortx2 __attribute__((ext_vector_type(2)));
typedef unsigned short ushortx2 __attribute__((ext_vector_type(2)));

constexpr int kWaves = 4;  // heads of a workgroup
// Largest value that is stored: a code times its scale below 2^128. What is finite above it would get, under 2^120 or more, the
// code of 2^128, which no bf16 holds; it is stored as this, less than half a step of e4m3 (2^-4 of it) away.
constexpr float kLargest = 0x1.ep127f;

__device__ __forceinline__ floatx2 turn(floatx2 p, CosSin r) { return floatx2{p[0] * r.c - p[1] * r.s, p[0] * r.s + p[1] * r.c}; }

__device__ __forceinline__ uint32_t pack_bf16(floatx2 p) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2)); }

// bits of |x| where x is finite, else 0
__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// least e >= kScaleLow with m <= 448 2^e, m >= 0 by its bits: 448 = 1.75 2^8. At most 120.
__device__ __forceinline__ int scale_exponent(uint32_t m) {
    const int e = (int)(m >> 23) - 127 - 8 + ((m & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, kScaleLow);
}

__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }  // e in [-126, 127]

// Four codes of values over a power of two, to nearest even; NaN, infinities and what would pass 464 give NaN (all finite bf16
// values and two million fp32 ones, over powers of two from 2^-100 to 2^120, gave what a product and a conversion give).
__device__ __forceinline__ uint32_t pack_e4m3(floatx2 a, floatx2 b, float scale) {
    const shortx2 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(shortx2{0, 0}, a[0], a[1], scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(lo, b[0], b[1], scale, true));
}
__device__ __forceinline__ uint32_t pack_e4m3(uint32_t a, uint32_t b, float scale) {  // of bf16 pairs
    const shortx2 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(shortx2{0, 0}, __builtin_bit_cast(bf16x2, a), scale, false);
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_bit_cast(bf16x2, b), scale, true));
}

// Codes of `rows` positions `step` bytes apart, rounded again from the scale 2^was to 2^now.
template <int D>
__device__ __forceinline__ void round_again(uint8_t* codes, int64_t step, int rows, int was, int now, int lane) {
    constexpr int kLanes = D / 8, kRows = 64 / kLanes;
    const float f = was - now < -126 ? 0.0f : power_of_two(was - now);
    for (int r = lane / kLanes; r < rows; r += kRows) {
        u32x2* p = reinterpret_cast<u32x2*>(codes + r * step) + lane % kLanes;
        u32x2 w = *p;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const floatx2 a = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
            w[i] = pack_e4m3(floatx2{a[0] * f, a[1] * f}, floatx2{b[0] * f, b[1] * f}, 1.0f);
        }
        *p = w;
    }
}

template <int D, int ES, bool kFp8, bool kStrided>
__global__ __launch_bounds__(64 * kWaves, D == 128 ? 3 : 4) void append_kernel(PagedAppendArgs a, PagedFreq f, unsigned blocks) {
    constexpr int kElems = 16 / ES, kPairs = kElems / 2;      // of a lane's vector
    constexpr int kLanes = D / kElems, kRows = 64 / kLanes;   // lanes of a row, rows of a load
    constexpr int kLoads = kScaleBlock / kRows;
    __shared__ CosSin table[kScaleBlock * (D / 2)];  // by axis, run of new rows with one place on it, pair of its band
    __shared__ double freq[D / 2];
    __shared__ double place[3][kScaleBlock];         // of an axis' runs
    __shared__ int4 row_at[kScaleBlock];             // where a row's angles of each axis begin
    __shared__ int ends[3];                          // of the axes' entries

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const PagedSeqs& q = a.seqs;
    const unsigned block = row_block();
    if (block >= blocks) {  // behind the pieces: the streams' new lengths
        const int64_t s = (int64_t)(block - blocks) * (64 * kWaves) + tid;
        if (a.out_len && s < q.B)
            a.out_len[s] = (int)min((int64_t)held_of(q, (int)s) + tokens_of(q, (int)s).y, (int64_t)(q.max_pages << q.page_log2));
        return;
    }
    // What the angles need is loaded before the rows, and all of it without branches around it, so that the waits are by
    // count and the rows stay in flight.
    const int P = a.n_t + a.n_y + a.n_x;
    const double own_freq = f.quarter[min(tid, D / 2 - 1)];
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
    const int row0 = start & ((1 << q.page_log2) - 1);
    const bool live = head < a.H;
    const int head_in = min(head, a.H - 1);

    // row r of the block is token tok.x + start + r - held
    const int64_t first = (int64_t)tok.x + start - held;
    int at[3] = {0, 0, 0};  // lane r of the first wave: the place of row r
    const bool placed = tid < kScaleBlock && tid >= lo && tid < hi;
    if (a.pos && placed) {
#pragma unroll
        for (int j = 0; j < 3; ++j) at[j] = a.pos[(first + tid) * 3 + j];
    }
    const int r_lane = lane / kLanes, c_lane = lane % kLanes;
    // the lane's row of load i; beside the new rows one of them, which changes no maximum and is not stored
    auto row_in = [&](int i) -> int { return min(max(i * kRows + r_lane, lo), hi - 1); };
    u32x4 x[2][kLoads];
    auto load = [&](int which) {
        const uint8_t* src = static_cast<const uint8_t*>(which ? a.v : a.k) + (size_t)head_in * D * ES + 16 * c_lane;
        const int64_t row = which ? a.v_row_bytes : a.k_row_bytes;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            x[which][i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + (first + row_in(i)) * row));
        }
    };
    load(0);
    if constexpr (ES == 2) load(1);
    if (page < 0) return;  // nowhere to store them (uniform)
    constexpr int kOut = kFp8 ? D : D * ES;  // bytes of a stored row
    const size_t slot = ((size_t)page * a.H + head_in) << q.page_log2;  // first position of the head's page
    // the block's first position in a cache, its scale, and the bytes from position to position
    auto block_at = [&](int which) -> uint8_t* {
        uint8_t* cache = static_cast<uint8_t*>(which ? a.cache_v : a.cache_k);
        if constexpr (kStrided) return cache + strided_at(which ? a.layout.v : a.layout.k, page, head_in, row0);
        else return cache + (slot + row0) * kOut;
    };
    auto scale_at = [&](int which) -> uint8_t* {
        uint8_t* scale = which ? a.scale_v : a.scale_k;
        if constexpr (kStrided) return scale + strided_at(which ? a.layout.scale_v : a.layout.scale_k, page, head_in, row0 / kScaleBlock);
        else return scale + (slot + row0) / kScaleBlock;
    };
    auto step_of = [&](int which) -> int64_t {
        if constexpr (kStrided) return which ? a.layout.v.row : a.layout.k.row;
        else return kOut;
    };
    uint8_t was[2] = {0, 0};  // the block's scales
    if constexpr (kFp8) {
        was[0] = *scale_at(0);
        was[1] = *scale_at(1);
    }
    if (tid < P) freq[tid] = own_freq;

    // The rows of a piece share most of their places on two of the axes: an angle is computed once per run of rows with
    // one place (32 tokens of a 30 x 52 grid: some 750 of 2048).
    if (wave == 0) {
        if (!a.pos) {
            const int c = start + lane, frame = c / a.hw, in = c - frame * a.hw, y = in / a.w;
            at[0] = frame;
            at[1] = y;
            at[2] = in - y * a.w;
        }
        const int n[3] = {a.n_t, a.n_y, a.n_x};
        int from[3], total = 0;
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            const int before = __shfl_up(at[j], 1);
            const bool starts = placed && (lane == lo || at[j] != before);
            const unsigned long long runs = __ballot(starts);
            const int run = __popcll(runs & ((2ull << lane) - 1)) - 1;
            if (starts) place[j][run] = (double)at[j] + (j == 0 && !a.pos ? (double)a.t0 : 0.0);
            from[j] = total + run * n[j];
            total += __popcll(runs) * n[j];
            if (lane == 0) ends[j] = total;
        }
        if (placed) row_at[lane] = make_int4(from[0], from[1], from[2], 0);
    }
    __syncthreads();
    {
        const int e0 = ends[0], e1 = ends[1], e2 = ends[2];
        for (int e = tid; e < e2; e += 64 * kWaves) {
            const int axis = e < e0 ? 0 : (e < e1 ? 1 : 2);
            const int i = e - (axis == 0 ? 0 : (axis == 1 ? e0 : e1)), n = axis == 0 ? a.n_t : (axis == 1 ? a.n_y : a.n_x);
            const int run = (int)(((float)i + 0.5f) * (axis == 0 ? a.inv_pairs[0] : (axis == 1 ? a.inv_pairs[1] : a.inv_pairs[2])));  // at most 2048 entries: exact
            table[e] = quarter_turns(place[axis][run] * freq[(axis > 0 ? a.n_t : 0) + (axis > 1 ? a.n_y : 0) + i - run * n]);
        }
    }
    __syncthreads();
    if (!live) return;
    // the lane's pairs: which axis each is of, and its place in that band
    int axis_of[kPairs], in_band[kPairs];
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        const int pair = c_lane * kPairs + j;
        axis_of[j] = pair < a.n_t ? 0 : (pair < a.n_t + a.n_y ? 1 : (pair < P ? 2 : 3));
        in_band[j] = axis_of[j] == 3 ? 0 : pair - (axis_of[j] > 0 ? a.n_t : 0) - (axis_of[j] > 1 ? a.n_y : 0);
    }

    // The lane's part of load i as pairs, turned to the row's position; pairs behind the last band as they are.
    auto turned = [&](int i, floatx2 (&p)[kPairs]) __attribute__((always_inline)) {
        const int4 angles = row_at[row_in(i)];
        const u32x4 w = x[0][i];
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            if constexpr (ES == 2) p[j] = floatx2{__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u)};
            else p[j] = floatx2{__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1])};
            const floatx2 t = turn(p[j], table[(axis_of[j] == 0 ? angles.x : (axis_of[j] == 1 ? angles.y : angles.z)) + in_band[j]]);
            p[j] = axis_of[j] < 3 ? t : p[j];
        }
    };
    auto is_new = [&](int i) -> bool { return i * kRows + r_lane >= lo && i * kRows + r_lane < hi; };
    // the lane's part of load i in a cache
    const size_t to_lane = (slot + row0 + r_lane) * (size_t)kOut + (kOut / kLanes) * c_lane;
    auto lane_at = [&](int which, int i) -> uint8_t* {
        if constexpr (kStrided) return block_at(which) + r_lane * step_of(which) + (kOut / kLanes) * c_lane + i * (kRows * step_of(which));
        else return static_cast<uint8_t*>(which ? a.cache_v : a.cache_k) + to_lane + i * (kRows * kOut);
    };
    if constexpr (kFp8) {
        // a block's codes from its largest value's bits: word(i, scale) is the lane's part of load i
        auto store = [&](int which, uint32_t most, auto word) __attribute__((always_inline)) {
#pragma unroll
            for (int off = 1; off < 64; off *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, off));
            int e = scale_exponent(most);
            if (lo > 0) {  // byte 0 counts as 1; 255, NaN, stays, and so do the codes that are there
                const int old = max((int)was[which], 1) - 127;
                if (e > old) round_again<D>(block_at(which), step_of(which), lo, old, e, lane);
                e = max(e, old);
            }
            const float to = power_of_two(min(e, 127));
            const uint32_t lost = e > 127 ? 0x7f7f7f7fu : 0u;  // beside a NaN scale codes are NaN too
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const u32x2 w = word(i, to) | lost;
                if (is_new(i)) *reinterpret_cast<u32x2*>(lane_at(which, i)) = w;
            }
            if (lane == 0) *scale_at(which) = (uint8_t)(e + 127);
        };
        // Largest values: of keys by fp32, of values by the bits of two bf16 at a time. Where one is not finite (bf16 with an
        // exponent of ones, or a turned pair past fp32), the others are looked at one by one.
        {
            floatx2 p[kLoads][kPairs];
            float top = 0.0f;
            ushortx2 bits = {0, 0};
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
#pragma unroll
                for (int j = 0; j < kPairs; ++j) bits = __builtin_elementwise_max(bits, __builtin_bit_cast(ushortx2, x[0][i][j] & 0x7fff7fffu));
                turned(i, p[i]);
#pragma unroll
                for (int j = 0; j < kPairs; ++j) top = fmaxf(top, fmaxf(fabsf(p[i][j][0]), fabsf(p[i][j][1])));
                if (i & 1) __builtin_amdgcn_sched_barrier(0);  // the angles of two loads at a time
            }
            if (__any(max(bits[0], bits[1]) >= 0x7f80 || top == INFINITY)) {
                uint32_t most = 0;
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
#pragma unroll
                    for (int j = 0; j < kPairs; ++j)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            most = max(most, finite_bits(p[i][j][h]));
                            __builtin_amdgcn_sched_barrier(0);  // one mask at a time
                        }
                top = __uint_as_float(most);
            }
            if (__any(top > kLargest)) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
#pragma unroll
                    for (int j = 0; j < kPairs; ++j)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float x = p[i][j][h], c = fminf(fmaxf(x, -kLargest), kLargest);
                            p[i][j][h] = fabsf(x) < INFINITY ? c : x;
                            __builtin_amdgcn_sched_barrier(0);  // one mask at a time
                        }
            }
            store(0, __float_as_uint(top), [&](int i, float to) -> u32x2 { return u32x2{pack_e4m3(p[i][0], p[i][1], to), pack_e4m3(p[i][2], p[i][3], to)}; });
        }
        ushortx2 bits = {0, 0};
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
#pragma unroll
            for (int j = 0; j < kPairs; ++j) bits = __builtin_elementwise_max(bits, __builtin_bit_cast(ushortx2, x[1][i][j] & 0x7fff7fffu));
        if (__any(max(bits[0], bits[1]) >= 0x7f80)) {
            bits = ushortx2{0, 0};
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    const uint32_t bad = spread<kPagedBf16>(not_finite<kPagedBf16>(x[1][i][j]));
                    bits = __builtin_elementwise_max(bits, __builtin_bit_cast(ushortx2, x[1][i][j] & ~bad & 0x7fff7fffu));
                }
        }
        if (__any(max(bits[0], bits[1]) > __float_as_uint(kLargest) >> 16)) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    // the sign and the magnitude, or the largest one where the magnitude is between it and infinity
                    const uint32_t w = x[1][i][j], inf = spread<kPagedBf16>(not_finite<kPagedBf16>(w));
                    const uint32_t least = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(ushortx2, w & 0x7fff7fffu), ushortx2{0x7f70, 0x7f70}));
                    x[1][i][j] = (w & (inf | 0x80008000u)) | (least & ~inf);
                }
        }
        store(1, (uint32_t)max(bits[0], bits[1]) << 16, [&](int i, float to) -> u32x2 {
            return u32x2{pack_e4m3(x[1][i][0], x[1][i][1], to), pack_e4m3(x[1][i][2], x[1][i][3], to)};
        });
    } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            floatx2 p[kPairs];
            turned(i, p);
            u32x4 w = x[0][i];
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                if (axis_of[j] == 3) continue;  // copied
                if constexpr (ES == 2) {
                    w[j] = pack_bf16(p[j]);
                } else {
                    w[2 * j] = __float_as_uint(p[j][0]);
                    w[2 * j + 1] = __float_as_uint(p[j][1]);
                }
            }
            if (is_new(i)) *reinterpret_cast<u32x4*>(lane_at(0, i)) = w;
        }
        if constexpr (ES == 4) load(1);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            if (is_new(i)) *reinterpret_cast<u32x4*>(lane_at(1, i)) = x[1][i];
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
    const unsigned lengths = a.out_len ? (unsigned)((a.seqs.B + 64 * kWaves - 1) / (64 * kWaves)) : 0;
    if (blocks + lengths == 0) return hipSuccess;
    const dim3 grid = grid_rows(blocks + lengths), block(64 * kWaves);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, f, blocks); };
    auto by_type = [&](auto d_tag, auto strided_tag) {
        constexpr int D = decltype(d_tag)::value;
        constexpr bool S = decltype(strided_tag)::value;
        if (a.dtype == kPagedFp8) launch(append_kernel<D, 2, true, S>);
        else if (a.dtype == kPagedBf16) launch(append_kernel<D, 2, false, S>);
        else launch(append_kernel<D, 4, false, S>);
    };
    auto by_layout = [&](auto d_tag) {
        if (a.strided) by_type(d_tag, std::true_type{});
        else by_type(d_tag, std::false_type{});
    };
    if (a.D == 128) by_layout(std::integral_constant<int, 128>{});
    else by_layout(std::integral_constant<int, 64>{});
    return hipGetLastError();
}

}  // namespace revisit
