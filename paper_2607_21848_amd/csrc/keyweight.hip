// Attention weight of every key (attention_key_weight):
//     out[h][k] = decay prev[h][k] + sum_p exp(A_pk - LSE_p),
// A the biased logits of biased_chunk_attention and LSE what that call returned.
//
// A wave owns blocks of 32 keys of one head and computes the logit tiles S = Q K^T
// with 32x32 MFMAs: queries are the M dimension, its keys the N dimension (held in
// registers), so a lane holds one key and 16 queries of each tile and a key's
// sum stays in its lane until the end, where the two wave halves meet: 16 weights
// of a tile are added first, then 16 or 18 tiles, then those sums, all in fp32 (n tiles
// one after the other would round n times at the sum's own size, up to n 2^-24 in all). No
// atomics: the same call gives the same bits. Blocks of 32 keys never cross a frame,
// so one retrieved frame's correspondences serve the whole block.
//
// Per logit: 256 flops of the product on the matrix cores, and one FMA, one
// exponential and one addition. The exponential carries a clamp to [0, 1] for
// free, which also turns the NaN of a row without an LSE into 0.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <numeric>
#include <type_traits>

#include "internal.h"

namespace revisit {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// -LSE log2 e, rounded once: log2 e alone in fp32 is 1.9e-8 off, which would make every weight too large by 1.3e-8 of the LSE
__device__ __forceinline__ float row_constant(float lse) {
    constexpr double kLog2e = 1.4426950408889634;
    constexpr float kHi = (float)kLog2e, kLo = (float)(kLog2e - (double)kHi);
    return -fmaf(lse, kHi, lse * kLo);
}
constexpr int kWaves = 4;
constexpr int kFewQueries = 32;
constexpr int kKeys = 32;  // keys of a block
constexpr int kTypeF32 = 2, kTypeFp8 = 3;  // REVISIT_F32, REVISIT_FP8_QK

// Accumulator row held by register i of a lane in wave half `hh` (32x32 MFMA).
__device__ __forceinline__ int acc_row(int hh, int i) { return 8 * (i >> 2) + 4 * hh + (i & 3); }

// ---------------------------------------------------------------------------
// bf16 and fp8 kernel: v_mfma_f32_32x32x16_bf16 (32 cycles), D = 128. A wave holds
// two blocks of keys (64 registers of operands), so that each query row read from LDS
// serves two products; the four waves of a workgroup share steps of 64 queries,
// which travel through registers into a ring of three steps in LDS (16-byte chunks
// swizzled: no bank conflicts); two workgroups per compute unit.
//
// The loop is half a step deep in software: the products of the next 32 queries
// alternate with the exponentials of the present ones, one MFMA to two of them (32
// cycles of matrix core to about as many of VALU), operands are read four products
// ahead, global loads a step ahead. What keeps it so: an empty asm on the running sum per
// group (without one the compiler moves the exponentials behind all MFMAs), scheduling
// fences, the keys' loads waited for before the loop, and three steps per
// iteration, so that every LDS address is a constant.
//
// Bound by matrix cores and VALU together at the chip's power limit (1.86 GHz):
// 12 heads of 4680 x 28080 without bias 391 us, 1032 TFLOP/s, where a large bf16 product
// reaches 1350 to 1390; MFMA 50 to 55% and VALU 60 to 70% of the cycles. With a third of the frames
// biased 440 us: the bias is two MFMAs per tile, and all that a biased tile does more adds to the time. On the way there:
// 32 keys per wave and queries from global memory 1458 (biased); 64 keys, LDS, no order of its own 536; products beside
// exponentials 470; query parts by rounds 441; ring addresses as constants and one wave per frame for the bias,
// one MFMA then, 416.
// Block 0's products before block 1's, with sums, exponentials and exponents of three groups in one
// slot so that nothing waits: 405 against 395 without bias, not kept.
//
// fp8: the fp8 matrix cores align the products of a few contraction indices to
// the largest and drop what lies 13 bits below it (measured on the device), which is
// no fp32 sum: a weight was outside the bound that fp32 sums keep. The values are turned to bf16, which holds
// e4m3 exactly, on their way into LDS and multiplied there: 357 us without bias, 409 with, at the size above.
// ---------------------------------------------------------------------------
template <int V>
using Int = std::integral_constant<int, V>;

constexpr int kD = 128;
constexpr int kStep = 64;                    // queries of a step
constexpr int kRowBytes = kD * 2;
constexpr int kStepBytes = kStep * kRowBytes;
constexpr int kSumSteps = 9;                 // steps whose weights are added up by themselves

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// Position of 16-byte chunk c of row r: 16 rows that read one chunk together touch 16 different positions, and so
// do the eight threads that write a row's even (or odd) chunks, modulo 8.
__device__ __forceinline__ int chunk_at(int r, int c) { return r * kRowBytes + ((c ^ (c >> 3) ^ (r & 15)) << 4); }

__device__ __forceinline__ uint32_t bf16_bits(float x) { return (uint32_t)__builtin_bit_cast(unsigned short, (__bf16)x); }
__device__ __forceinline__ uint32_t pack2(uint32_t lo, uint32_t hi) { return lo | (hi << 16); }
// x = hi + mid + lo exactly, three bf16 pieces of an fp32 value
__device__ __forceinline__ void split3(float x, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
    hi = bf16_bits(x);
    const float r = x - __uint_as_float(hi << 16);
    mid = bf16_bits(r);
    lo = bf16_bits(r - __uint_as_float(mid << 16));
}
constexpr uint32_t kOne = 0x3f80u;  // 1.0 in bf16

// e4m3 words -> bf16 pairs, exactly
__device__ __forceinline__ u32x4 wide(uint32_t a, uint32_t b) {
    auto pair = [](uint32_t w, auto hi) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, decltype(hi)::value));
    };
    return u32x4{pair(a, std::false_type{}), pair(a, std::true_type{}), pair(b, std::false_type{}), pair(b, std::true_type{})};
}

// Bias products. The matrix cores also make the bias gamma |a - u|^2, gamma = -lambda / (2 sigma^2 scale), a the token
// centre of a key and u a query's correspondence, and the products q k are added to it. Written out in fp32 as gamma (|a|^2 -
// 2 a.u + |u|^2) it would cancel where a key lies beside the correspondence and has the weight: logits off by
// 2e-6 at 30 x 52 tokens, sigma 2, and 1.1e-4 at 256 x 256 (rms; largest 5e-4). So u is taken apart into the token centre g
// next to it and the rest f, and gamma into a number c of 6 bits and the rest e: with T = 2 a, G = 2 g whole numbers
// counted from the middle of the grid, and sums over both axes,
//     gamma |a - u|^2 = c [sum T^2/4 - sum T G/2 + sum G^2/4]
//                       + [sum e T^2/4 - sum T (e G/2 + gamma f) + sum (e G^2/4 + gamma f (G + f))].
// On a grid of up to 256 tokens a side the terms of the first bracket and their partial sums are whole quarters of c's
// last place, below 2^24 of them, so that one MFMA adds them up without rounding; the second one's are small
// (n^2 / 256 + n / 2 times gamma on n tokens) and round like that: logits off by 2e-7 and less at 30 x 52 and 45 x 80, 1e-6 at
// 256 x 256, of which the exponential's argument alone makes 1e-7. What has more bits than a bf16 holds is cut into pieces
// that hold it. A lane has the x axis in the first half of the contraction (hh 0), the y axis in the second, and a sum
// over both in one of them:
//     key side    hh 0  [c sum T^2/4 (3 pieces), 0, T, T, T, *]    [T, T, T, e sum T^2/4 (3 pieces), 0, 0]
//                 hh 1  [1, 1, 1, 0, T, T, T, *]                   [T, T, T, 1, 1, 1, 0, 0]
//     query side  hh 0  [1, 1, 1, 0, -c G/2 (2 pieces), 0, 0]      [-(e G/2 + gamma f) (3 pieces), 1, 1, 1, 0, 0]
//                 hh 1  [c sum G^2/4 (3), 0, -c G/2 (2), 0, 0]     [the same (3), the last sum (3), 0, 0]
// A query without a correspondence has zeros. (With |a - u|^2 added up unscaled, u in 256ths first, and multiplied by gamma
// in the registers, nothing is left of the error, but 18 biased frames take 5% longer.)
struct BiasScale {
    float gamma, c, e;
};
__device__ __forceinline__ BiasScale bias_scale(float gamma) {
    // (to nearest; beyond the largest, down)
    uint32_t c = (__float_as_uint(gamma) + 0x20000u) & 0xfffc0000u;
    if ((c & 0x7f800000u) == 0x7f800000u) c = __float_as_uint(gamma) & 0xfffc0000u;
    return BiasScale{gamma, __uint_as_float(c), gamma - __uint_as_float(c)};
}
typedef unsigned int u32x6 __attribute__((ext_vector_type(6)));
struct KeySide {
    u32x6 words;  // the first product's operand in words 0 to 3, the second's in 2 to 5
};
__device__ __forceinline__ KeySide key_side(BiasScale b, int t, int w, int h, int hh) {
    const int ky = t / w;
    const float x = (float)(2 * (t - ky * w) + 1 - w), y = (float)(2 * ky + 1 - h);
    const float sq = 0.25f * (x * x + y * y);  // 17 bits
    uint32_t ch = kOne, cm = kOne, cl = kOne, eh = kOne, em = kOne, el = kOne;
    if (hh == 0) {
        split3(b.c * sq, ch, cm, cl);
        split3(b.e * sq, eh, em, el);
    }
    const uint32_t T = bf16_bits(hh ? y : x);
    return KeySide{u32x6{pack2(ch, cm), cl, pack2(T, T), pack2(T, eh), pack2(em, el), 0}};
}
struct QuerySide {
    u32x4 exact, rest;  // operands of the two products
};
// u: the correspondence's coordinate on this lane's axis of last + 1 tokens; ok: there is one (the same in both halves)
__device__ __forceinline__ QuerySide query_side(BiasScale b, float u, float last, bool ok, int hh) {
    auto both = [](float v) -> float {  // the sum over the axes
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return __uint_as_float(s[0]) + __uint_as_float(s[1]);
    };
    const float cell = fminf(fmaxf(floorf(u), 0.0f), last);
    const float f = (u - cell) - 0.5f, G = 2.0f * cell - last, q = 0.25f * (G * G);
    uint32_t ch = kOne, cm = kOne, cl = kOne, eh = kOne, em = kOne, el = kOne, lh, lm, ll;
    const float c = b.c * both(q), e = both(fmaf(b.e, q, (b.gamma * f) * (G + f)));
    if (hh) {
        split3(c, ch, cm, cl);
        split3(e, eh, em, el);
    }
    split3(-fmaf(b.gamma, f, b.e * (0.5f * G)), lh, lm, ll);
    const float lin = -0.5f * b.c * G;  // 14 bits
    const uint32_t lin_hi = bf16_bits(lin), lin_lo = bf16_bits(lin - __uint_as_float(lin_hi << 16));
    QuerySide s;
    s.exact = u32x4{pack2(ch, cm), cl, pack2(lin_hi, lin_lo), 0};
    s.rest = u32x4{pack2(lh, lm), pack2(ll, eh), pack2(em, el), 0};
    return ok ? s : QuerySide{u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
}
// a tile's bias
__device__ __forceinline__ floatx16 bias_tile(const QuerySide& q, const KeySide& k) {
    const u32x4 exact = __builtin_shufflevector(k.words, k.words, 0, 1, 2, 3), rest = __builtin_shufflevector(k.words, k.words, 2, 3, 4, 5);
    const floatx16 d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(q.exact), as_bf16x8(exact), floatx16{0}, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(q.rest), as_bf16x8(rest), d, 0, 0, 0);
}

// A block of 32 keys: where it is, and what its bias goes by.
struct KeyBlock {
    int frame;
    int64_t key0;
    int keys;     // of it within the frame; 0: no such block
    int slot;     // retrieved frame, -1: unbiased
    int in0;      // first key within the frame
};
__device__ __forceinline__ KeyBlock key_block(const KeyWeightArgs& a, int kb, bool bias) {
    KeyBlock b;
    b.frame = kb / a.frame_blocks;
    b.in0 = (kb - b.frame * a.frame_blocks) * kKeys;
    b.keys = kb < a.n_blocks ? min(kKeys, a.hw - b.in0) : 0;
    b.key0 = (int64_t)b.frame * a.hw + b.in0;
    b.slot = -1;
    if (bias && b.keys > 0) {
        const int s = __builtin_amdgcn_readfirstlane(a.slot[b.frame]);
        if (s >= 0 && s < a.S) b.slot = s;
    }
    return b;
}

// kFrames: frames that the blocks of a workgroup may lie in (2 or 4), 0: no bias.
template <bool kFp8, int kFrames>
__global__ __launch_bounds__(64 * kWaves, 2) void key_weight_bf16_kernel(KeyWeightArgs a, unsigned n_items) {
    constexpr bool kBias = kFrames > 0;
    __shared__ __attribute__((aligned(256))) uint8_t lds_q[3 * kStepBytes];
    __shared__ floatx4 lds_row[3 * kStep / 4];  // -LSE log2 e of the step's queries
    __shared__ float lds_total[2][kWaves][64];  // each lane's two sums
    // query side of the bias products: [ring of two][frame][half of the step][lane]
    __shared__ u32x4 lds_exact[kBias ? 2 * kFrames : 1][2][kBias ? 64 : 1];
    __shared__ uint32_t lds_rest[kBias ? 2 * kFrames : 1][2][kBias ? 64 : 1][3];

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hh = lane >> 5, n = lane & 31;
    const unsigned block = row_block();
    const unsigned item = xcd_item(block, n_items);
    if (block >= xcd_grid(n_items) || item >= n_items) return;  // grid padding (uniform, before any barrier)
    // item = (head, query part, group of key blocks)
    const int per_wave = a.wave_blocks, per_group = per_wave * kWaves;
    const int groups = (a.n_blocks + per_group - 1) / per_group;
    const int g = (int)(item % (unsigned)groups);
    const int hp = (int)(item / (unsigned)groups);
    const int hd = hp / a.parts, part = hp - hd * a.parts;
    const int n_tiles = (a.Lq + 31) / 32;
    const int t0 = (int)((int64_t)part * n_tiles / a.parts), t1 = (int)((int64_t)(part + 1) * n_tiles / a.parts);
    const int q_end = min(a.Lq, t1 * 32);

    constexpr int kSize = kFp8 ? 1 : 2;
    const int64_t row_bytes = (int64_t)a.H * kD * kSize;
    const uint8_t* Qg = static_cast<const uint8_t*>(a.q) + (int64_t)hd * kD * kSize;
    const uint8_t* Kg = static_cast<const uint8_t*>(a.k) + (int64_t)hd * kD * kSize;

    // this thread's share of a step's queries: kLoads 16-byte loads
    constexpr int kChunks = kD * kSize / 16;                   // per query
    constexpr int kLoads = kStep * kChunks / (64 * kWaves);
    u32x4 stage[kLoads];
    float stage_lse = 0.0f;
    // A step that would run past the last query is moved back to end with it (its
    // rows before q0 then have no weight to give again), so that the loads' offsets
    // (below 2^30) are the same for every step; fewer queries than a step repeat the last.
    const int last_base = max(0, a.Lq - kStep);
    auto base_of = [&](int q0) -> int { return min(q0, last_base); };
    uint32_t off[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int e = tid + i * 64 * kWaves;
        off[i] = (uint32_t)(min(e / kChunks, a.Lq - 1) * (int)row_bytes + 16 * (e % kChunks));
    }
    const int my_query = min(lane, a.Lq - 1);
    auto fetch = [&](int q0) {
        const uint8_t* base = Qg + base_of(q0) * row_bytes;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) stage[i] = *reinterpret_cast<const u32x4*>(base + off[i]);
        stage_lse = a.lse[(int64_t)hd * a.Lq + base_of(q0) + my_query];
        __builtin_amdgcn_sched_barrier(0);
    };
    auto put = [&](int q0, int to, int to_row) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int e = tid + i * 64 * kWaves;
            const int r = e / kChunks, c = e % kChunks;
            if constexpr (kFp8) {
                *reinterpret_cast<u32x4*>(lds_q + to + chunk_at(r, 2 * c)) = wide(stage[i][0], stage[i][1]);
                *reinterpret_cast<u32x4*>(lds_q + to + chunk_at(r, 2 * c + 1)) = wide(stage[i][2], stage[i][3]);
            } else {
                *reinterpret_cast<u32x4*>(lds_q + to + chunk_at(r, c)) = stage[i];
            }
        }
        // a query past the end, or one without an LSE, has no weight to give
        const int q = base_of(q0) + lane;
        __builtin_amdgcn_sched_barrier(0);  // the registers are loaded again only after this
        if (wave == 0) reinterpret_cast<float*>(lds_row + to_row)[lane] = q >= q0 && q < q_end && __builtin_isfinite(stage_lse) ? row_constant(stage_lse) : -INFINITY;
    };
    if (t0 < t1) fetch(t0 * 32);

    // this wave's keys: two blocks of 32
    KeyBlock kb[2];
    bf16x8 kf[2][kD / 16];
    KeySide kside[2];
    const BiasScale scale = bias_scale(-a.gamma);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        kb[b] = key_block(a, b < per_wave ? g * per_group + wave * per_wave + b : a.n_blocks, kBias);
        const uint8_t* row = Kg + (kb[b].keys > 0 ? kb[b].key0 + min(n, kb[b].keys - 1) : 0) * row_bytes;
#pragma unroll
        for (int j = 0; j < kD / 16; ++j) {
            if constexpr (kFp8) {
                const u32x2 v = *reinterpret_cast<const u32x2*>(row + 16 * j + 8 * hh);
                kf[b][j] = as_bf16x8(wide(v[0], v[1]));
            } else {
                kf[b][j] = as_bf16x8(*reinterpret_cast<const u32x4*>(row + 32 * j + 16 * hh));
            }
        }
        if constexpr (kBias) kside[b] = key_side(scale, kb[b].in0 + n, a.w, a.h, hh);
    }
    // The query side of the frames that the workgroup's blocks lie in (counted from its first
    // block's): a wave makes that of half a step (32 queries) for every other frame, each lane one query's on its axis. What
    // one step reads, its own second half and the next step's first, is made in the step before it (turn t: the
    // sides that step t reads), so that two turns are held.
    constexpr int kMade = kBias ? kFrames / 2 : 1;  // frames of a wave
    const int frame0 = g * per_group / a.frame_blocks;
    const int last_block = min((g + 1) * per_group, a.n_blocks) - 1;
    const int half = wave & 1;
    int made[kMade];  // retrieved frames whose side this wave makes, -1: none
#pragma unroll
    for (int i = 0; i < kMade; ++i) {
        made[i] = -1;
        const int f = frame0 + 2 * i + (wave >> 1);
        if (kBias && f <= last_block / a.frame_blocks) {
            const int s = a.slot[f];
            if (s >= 0 && s < a.S) made[i] = __builtin_amdgcn_readfirstlane(s);
        }
    }
    float corr_u[kMade];
    int corr_i[kMade];
    auto fetch_corr = [&](int turn) {
        int last = a.Lq - 1;
        asm volatile("" : "+s"(last));  // (no register for what is made of it here)
        const uint32_t corr_at = 4u * (uint32_t)min(32 * half + n, last);  // bytes of a correspondence's index
#pragma unroll
        for (int i = 0; i < kMade; ++i) {
            if (made[i] < 0) continue;
            const int64_t row = (int64_t)made[i] * a.Lq + base_of(t0 * 32 + max(turn + 1 - half, 0) * kStep);  // uniform
            corr_u[i] = *reinterpret_cast<const float*>(reinterpret_cast<const uint8_t*>(a.corr_uv + 2 * row) + (2u * corr_at + 4u * hh));
            corr_i[i] = *reinterpret_cast<const int32_t*>(reinterpret_cast<const uint8_t*>(a.corr_idx + row) + corr_at);
        }
    };
    auto make_bias = [&](int turn) {
        int w = a.w, h = a.h;
        asm volatile("" : "+s"(w), "+s"(h));  // (nor here)
        const float bias_last = (float)((hh ? h : w) - 1);
#pragma unroll
        for (int i = 0; i < kMade; ++i) {
            if (made[i] < 0) continue;
            // a correspondence whose x (the first half's) is NaN is none
            const float x = __uint_as_float(__builtin_amdgcn_permlane32_swap(__float_as_uint(corr_u[i]), __float_as_uint(corr_u[i]), false, false)[0]);
            const QuerySide q = query_side(scale, corr_u[i], bias_last, corr_i[i] >= 0 && !__builtin_isnan(x), hh);
            const int at = (turn & 1) * kFrames + 2 * i + (wave >> 1);
            lds_exact[at][half][lane] = q.exact;
#pragma unroll
            for (int k = 0; k < 3; ++k) lds_rest[at][half][lane][k] = q.rest[k];
        }
    };
    // this wave's blocks: whether they are biased, and by which of the frames' sides
    const int bias0 = kb[0].slot < 0 ? -1 : kb[0].frame - frame0, bias1 = kb[1].slot < 0 ? -1 : kb[1].frame - frame0;

    const int n_steps = (t1 - t0 + 1) / 2;
    const int q_begin = t0 * 32;
    float sum[2] = {0.0f, 0.0f};
    lds_total[0][wave][lane] = lds_total[1][wave][lane] = 0.0f;
    floatx16 accA[2], accB[2];
    u32x4 qf[4];     // queries of the next four products
    floatx4 rc[2];   // row constants of the next eight exponentials
    int q_lane[kD / 16];  // chunk 2 j + hh of this lane's row
#pragma unroll
    for (int j = 0; j < kD / 16; ++j) {
        q_lane[j] = chunk_at(n, 2 * j + hh);
        asm volatile("" : "+v"(q_lane[j]));  // one register each: not put together anew for the last steps
    }
    auto read_q = [&](int rows, int j) { qf[j & 3] = *reinterpret_cast<const u32x4*>(lds_q + q_lane[j] + rows); };
    auto read_rc = [&](int row, int i) { rc[i & 1] = lds_row[hh + row + 2 * i]; };
    constexpr int kHalf = 32 * kRowBytes, kRow = kStep / 4;  // half a step's rows; a step's row constants, in quads

    // two exponentials of block b's tile `from`: weights 2 e and 2 e + 1 of a lane, added to s
    auto exps = [&](const floatx16* from, int b, int e, float& s) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 2 * e; i < 2 * e + 2; ++i) {
            // a probability: at most 1, and 0 where the row has no LSE whatever its logits are
            const float x = __builtin_amdgcn_exp2f(fmaf(from[b][i], a.c_log2, rc[(i >> 2) & 1][i & 3]));
            s += fminf(fmaxf(x, 0.0f), 1.0f);
        }
        asm volatile("" : "+v"(s));  // keeps the exponentials here
        __builtin_amdgcn_sched_barrier(0);
    };
    auto product = [&](floatx16* to, int b, int j) __attribute__((always_inline)) {
        to[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(qf[j & 3]), kf[b][j], to[b], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    // The first products of a half (qf[0]), on top of the bias where a block has one. `meanwhile` is called with 0 while
    // the bias's operands are read and with 1 beside the first block's matrix instructions. (Branches are uniform per wave.)
    auto first_products = [&](floatx16* to, int turn, int which, auto meanwhile) __attribute__((always_inline)) {
        const int frame[2] = {bias0, bias1};
        QuerySide side[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (frame[b] < 0) continue;
            const int at = (turn & 1) * kFrames + frame[b];
            const uint32_t* rest = lds_rest[at][which][lane];
            side[b] = QuerySide{lds_exact[at][which][lane], u32x4{rest[0], rest[1], rest[2], 0}};
        }
        __builtin_amdgcn_sched_barrier(0);
        meanwhile(0);
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (frame[b] >= 0) {
                to[b] = bias_tile(side[b], kside[b]);
                product(to, b, 0);
            } else {
                to[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(qf[0]), kf[b][0], floatx16{0}, 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (b == 0) meanwhile(1);
        }
    };

    // Half of a step: the products of the next half (rows) beside the exponentials of
    // this one (row constants row), one MFMA to two of them. Operands are read four
    // products, row constants eight exponentials ahead: past the end, those of the half after.
    auto do_half = [&](auto last_tag, floatx16* cur, floatx16* next, auto rows, auto rows_after, auto row, auto row_after,
                       int turn, auto turn_half) __attribute__((always_inline)) {
        constexpr bool kLast = decltype(last_tag)::value;
        float s0 = 0.0f, s1 = 0.0f;
        auto exps_read = [&](int e) __attribute__((always_inline)) {  // row constants after their last use
            if (e & 1) {
                if (e < 4) read_rc(row, (e >> 1) + 2);
                else if constexpr (!kLast) read_rc(row_after, (e >> 1) - 2);
            }
        };
        if constexpr (kLast || !kBias) {
            if constexpr (!kLast) next[0] = next[1] = floatx16{0};
#pragma unroll
            for (int j = 0; j < kD / 16; ++j) {
                if constexpr (!kLast) product(next, 0, j);
                exps(cur, 0, j, s0);
                if constexpr (!kLast) product(next, 1, j);
                exps(cur, 1, j, s1);
                if constexpr (!kLast) read_q(j < 4 ? rows : rows_after, (j + 4) & 7);
                exps_read(j);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            first_products(next, turn, turn_half, [&](int b) __attribute__((always_inline)) {
                if (b == 0) exps(cur, 0, 0, s0);
                else exps(cur, 1, 0, s1);
            });
            read_q(rows, 4);
#pragma unroll
            for (int j = 1; j < kD / 16; ++j) {
                product(next, 0, j);
                exps(cur, 0, j, s0);
                product(next, 1, j);
                exps(cur, 1, j, s1);
                read_q(j < 4 ? rows : rows_after, (j + 4) & 7);
                exps_read(j);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        sum[0] += s0;
        sum[1] += s1;
    };

    if (n_steps > 0) {
        put(q_begin, 0, 0);
        if constexpr (kBias) {
            fetch_corr(-1);
            make_bias(-1);
        }
        fetch(q_begin + kStep);
        if constexpr (kBias) fetch_corr(0);
        // the keys are waited for here: at their first use below the wait would drain the
        // next step's query loads too, every time round the loop
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int j = 0; j < kD / 16; ++j) asm volatile("" : "+v"(kf[b][j]));
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) read_q(0, j);
        if constexpr (kBias) first_products(accA, -1, 0, [](int) {});
        else accA[0] = accA[1] = floatx16{0};
#pragma unroll
        for (int j = 0; j < kD / 16; ++j) {
            if (!kBias || j > 0) {
#pragma unroll
                for (int b = 0; b < 2; ++b) accA[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(qf[j & 3]), kf[b][j], accA[b], 0, 0, 0);
            }
            read_q(j < 4 ? 0 : kHalf, (j + 4) & 7);
        }
        read_rc(0, 0);
        read_rc(0, 1);
        put(q_begin + kStep, kStepBytes, kRow);
        fetch(q_begin + 2 * kStep);
        if constexpr (kBias) {
            make_bias(0);
            fetch_corr(1);
        }
        __syncthreads();
        // At the top of step s: accA holds the logits of its first half, qf the first queries of
        // its second, buffer s + 1 the next step, the stage registers the loads of step s + 2
        // (buffers s mod 3).
        // (ring: s mod 3, and the two behind it)
        auto step = [&](int s, auto ring0, auto ring1, auto ring2) __attribute__((always_inline)) {
            do_half(std::false_type{}, accA, accB, ring0 * kStepBytes + kHalf, ring1 * kStepBytes, ring0 * kRow, ring0 * kRow + kRow / 2, s, 1);
            if (s + 2 < n_steps) {
                put(q_begin + (s + 2) * kStep, ring2 * kStepBytes, ring2 * kRow);
                fetch(q_begin + (s + 3) * kStep);  // past the last step: in bounds, for nothing
            }
            if constexpr (kBias) {
                make_bias(s + 1);
                fetch_corr(s + 2);
            }
            do_half(std::false_type{}, accB, accA, ring1 * kStepBytes, ring1 * kStepBytes + kHalf, ring0 * kRow + kRow / 2, ring1 * kRow, s, 0);
            __syncthreads();
        };
        // three steps at a time, so that the ring's addresses are constants
        int s = 0;
        for (; s + 3 < n_steps; s += 3) {
            step(s, Int<0>{}, Int<1>{}, Int<2>{});
            step(s + 1, Int<1>{}, Int<2>{}, Int<0>{});
            step(s + 2, Int<2>{}, Int<0>{}, Int<1>{});
            if (s % kSumSteps == kSumSteps - 3) {  // (s is a multiple of 3)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    lds_total[b][wave][lane] += sum[b];
                    sum[b] = 0.0f;
                }
            }
        }
        for (int r = 0; s + 1 < n_steps; ++s, ++r) step(s, r, r == 2 ? 0 : r + 1, r == 0 ? 2 : r - 1);
        const int ring = s % 3, q0 = ring * kStepBytes, r0 = ring * kRow;
        do_half(std::false_type{}, accA, accB, q0 + kHalf, q0, r0, r0 + kRow / 2, s, 1);
        do_half(std::true_type{}, accB, accA, 0, 0, r0 + kRow / 2, 0, 0, 0);
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        sum[b] += lds_total[b][wave][lane];
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum[b]), __float_as_uint(sum[b]), false, false);
        const float s = __uint_as_float(p[0]) + __uint_as_float(p[1]);
        if (hh == 0 && n < kb[b].keys) {
            const int64_t o = (int64_t)hd * a.Lk + kb[b].key0 + n;
            if (a.parts > 1) a.partial[(int64_t)part * a.H * a.Lk + o] = s;
            else a.out[o] = a.prev ? fmaf(a.decay, a.prev[o], s) : s;
        }
    }
}

// ---------------------------------------------------------------------------
// bf16 and fp8 kernel for at most kFewQueries queries, one tile: the keys are read
// once and nothing is used twice, so it is bound by HBM, and small waves (32 keys
// each, no ring, no barrier) keep more loads in flight than the kernel above. One
// query of 12 heads against 37440 keys (115 MB, not in any cache): 26.9 us, 4.4 TB/s,
// against 30 there; for 60 queries in two tiles it would take 42 us against 34.
// All loads leave before the first is waited for (35 us without that), and the
// keys pass through L1 (non-temporal loads, 46 us: each line is met by four of them).
// ---------------------------------------------------------------------------
template <bool kFp8, bool kBias>
__global__ __launch_bounds__(64 * kWaves) void key_weight_few_kernel(KeyWeightArgs a, unsigned n_items) {
    __shared__ floatx4 lds_row[kWaves][8];  // -LSE log2 e of the queries, for each wave its own
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int hh = lane >> 5, n = lane & 31;
    const unsigned block = row_block();
    const unsigned item = xcd_item(block, n_items);
    if (block >= xcd_grid(n_items) || item >= n_items) return;  // grid padding (uniform)
    const int groups = (a.n_blocks + kWaves - 1) / kWaves;
    const int hd = (int)(item / (unsigned)groups);
    const KeyBlock kb = key_block(a, (int)(item - (unsigned)hd * (unsigned)groups) * kWaves + wave, kBias);
    if (kb.keys == 0) return;  // uniform per wave; no barrier below
    // A lane's share of a row in loads of 16 bytes; of an fp8 load the first eight elements
    // go to one MFMA step and the rest to the next (any numbering of the contraction
    // will do that queries and keys share).
    constexpr int kSize = kFp8 ? 1 : 2, kLoads = kD * kSize / 32;
    const int64_t row_bytes = (int64_t)a.H * kD * kSize;
    const uint8_t* kr = static_cast<const uint8_t*>(a.k) + (kb.key0 + min(n, kb.keys - 1)) * row_bytes + (int64_t)hd * kD * kSize + 16 * hh;
    const uint8_t* Qg = static_cast<const uint8_t*>(a.q) + (int64_t)hd * kD * kSize + 16 * hh;
    // the correspondence first: its bias is made while the keys are on their way
    const int q = max(min(n, a.Lq - 1), 0);
    float corr_u = 0.0f;
    int corr_i = -1;
    if (kBias && kb.slot >= 0 && a.Lq > 0) {
        const int64_t o = (int64_t)kb.slot * a.Lq + q;
        corr_u = a.corr_uv[2 * o + hh];
        corr_i = a.corr_idx[o];
    }
    u32x4 kraw[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) kraw[j] = *reinterpret_cast<const u32x4*>(kr + 32 * j);
    auto operand = [](const u32x4* raw, int step) -> bf16x8 {
        if constexpr (kFp8) return as_bf16x8(wide(raw[step >> 1][2 * (step & 1)], raw[step >> 1][2 * (step & 1) + 1]));
        else return as_bf16x8(raw[step]);
    };
    float sum = 0.0f;
    if (a.Lq > 0) {
        const uint8_t* qr = Qg + q * row_bytes;
        u32x4 qraw[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j) qraw[j] = *reinterpret_cast<const u32x4*>(qr + 32 * j);
        const float lse = a.lse[(int64_t)hd * a.Lq + q];
        __builtin_amdgcn_sched_barrier(0);  // all loads leave before the first is waited for
        floatx16 acc = floatx16{0};
        if (kBias && kb.slot >= 0) {
            // a correspondence whose x (the first half's) is NaN is none
            const float x = __uint_as_float(__builtin_amdgcn_permlane32_swap(__float_as_uint(corr_u), __float_as_uint(corr_u), false, false)[0]);
            const BiasScale scale = bias_scale(-a.gamma);
            const QuerySide side = query_side(scale, corr_u, (float)((hh ? a.h : a.w) - 1), corr_i >= 0 && !__builtin_isnan(x), hh);
            acc = bias_tile(side, key_side(scale, kb.in0 + n, a.w, a.h, hh));
        }
        // a query past the end, or one without an LSE, has no weight to give; both halves write the same
        reinterpret_cast<float*>(lds_row[wave])[n] = n < a.Lq && __builtin_isfinite(lse) ? row_constant(lse) : -INFINITY;
#pragma unroll
        for (int j = 0; j < kD / 16; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(qraw, j), operand(kraw, j), acc, 0, 0, 0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int i = 0; i < 16; ++i)
            sum += fminf(fmaxf(__builtin_amdgcn_exp2f(fmaf(acc[i], a.c_log2, lds_row[wave][2 * (i >> 2) + hh][i & 3])), 0.0f), 1.0f);
    }
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    sum = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    if (hh == 0 && n < kb.keys) {
        const int64_t o = (int64_t)hd * a.Lk + kb.key0 + n;
        a.out[o] = a.prev ? fmaf(a.decay, a.prev[o], sum) : sum;
    }
}

// ---------------------------------------------------------------------------
// fp32 kernel: v_mfma_f32_32x32x2_f32 (64 cycles each), so bound by the matrix
// cores as long as nothing waits (12 heads of 4680 x 28080, D 128: 3.13 ms, 129 of the 154 TFLOP/s
// that a large fp32 product reaches; with the bias 3.28). A wave owns 32 keys; while the products of one
// tile of 32 queries use up the query registers, the next tile's rows are loaded
// into them from global memory (no LDS, no barrier: a tile's 4096 cycles at D =
// 128 cover the loads), and the tile before has its exponentials and its bias, evaluated directly,
// differences first, between the MFMAs (2000 x 9360, against a form that loaded each tile when it
// came to it: 735 -> 541 us with the bias). The four loads of a row's 128-byte line leave together:
// one at a time, as its registers came free, each met the line anew in L1, 3.39 ms and 3.63. Queries
// shared by the workgroup through LDS instead: 3.18 and 3.33, not kept.
// ---------------------------------------------------------------------------

template <int D, bool kBias>
__global__ __launch_bounds__(64 * kWaves, 2) void key_weight_f32_kernel(KeyWeightArgs a, unsigned n_items) {
    // per query of two tiles: u^ x, y, -lambda log2 e / (2 sigma^2) or 0, -LSE log2 e
    __shared__ float4 lds_row[kWaves][2][32];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int hh = lane >> 5, n = lane & 31;
    const unsigned block = row_block();
    const unsigned item = xcd_item(block, n_items);
    if (block >= xcd_grid(n_items) || item >= n_items) return;  // grid padding (uniform)
    // item = (head, query part, group of kWaves key blocks)
    const int groups = (a.n_blocks + kWaves - 1) / kWaves;
    const int g = (int)(item % (unsigned)groups);
    const int hp = (int)(item / (unsigned)groups);
    const int hd = hp / a.parts, part = hp - hd * a.parts;
    const KeyBlock kb = key_block(a, g * kWaves + wave, kBias);
    if (kb.keys == 0) return;  // uniform per wave; no barrier below

    constexpr int kG = D / 8;  // MFMA step 4 g + i takes element 8 g + 4 hh + i: 16 bytes of a row serve four
    const int64_t row_bytes = (int64_t)a.H * D * 4;
    const uint8_t* Qg = static_cast<const uint8_t*>(a.q) + (int64_t)hd * D * 4;
    floatx4 kf[kG], qf[kG];
    {
        const uint8_t* row = static_cast<const uint8_t*>(a.k) + (kb.key0 + min(n, kb.keys - 1)) * row_bytes + (int64_t)hd * D * 4 + 16 * hh;
#pragma unroll
        for (int j = 0; j < kG; ++j) kf[j] = *reinterpret_cast<const floatx4*>(row + 32 * j);
    }
    const int ky_i = (kb.in0 + n) / a.w;
    const float kx = (float)(kb.in0 + n - ky_i * a.w) + 0.5f, ky = (float)ky_i + 0.5f;

    const int n_tiles = (a.Lq + 31) / 32;
    const int t0 = (int)((int64_t)part * n_tiles / a.parts), t1 = (int)((int64_t)(part + 1) * n_tiles / a.parts);
    // query row of this lane in tile t; rows past the last repeat it
    auto q_row = [&](int t) -> int { return min(t * 32 + n, a.Lq - 1); };
    auto q_at = [&](int t) -> const uint8_t* { return Qg + q_row(t) * row_bytes + 16 * hh; };
    // a tile's row data: loaded a tile ahead, made into what the exponentials take when its turn comes
    float row_lse = 0.0f;
    float2 row_u = {0.0f, 0.0f};
    int row_i = -1;
    auto fetch_row = [&](int t) {
        const int q = q_row(t);
        row_lse = a.lse[(int64_t)hd * a.Lq + q];
        if (kBias && kb.slot >= 0) {
            row_u = reinterpret_cast<const float2*>(a.corr_uv)[(int64_t)kb.slot * a.Lq + q];
            row_i = a.corr_idx[(int64_t)kb.slot * a.Lq + q];
        }
    };
    auto make_row = [&](int t) -> float4 {
        float4 r = {0.0f, 0.0f, 0.0f, -INFINITY};
        // a query past the end, or one without an LSE, has no weight to give
        if (t * 32 + n < a.Lq && __builtin_isfinite(row_lse)) r.w = row_constant(row_lse);
        if (kBias && row_i >= 0 && !__builtin_isnan(row_u.x)) {
            r.x = row_u.x;
            r.y = row_u.y;
            r.z = -a.gamma2;
        }
        return r;
    };
    float sum = 0.0f, group = 0.0f, part_sum = 0.0f;  // of all tiles, of up to 16 of them, of one
    // the weight of logit i of a tile whose rows lie in `rows`; the next one's row is read meanwhile
    float4 ahead;
    auto unit = [&](const floatx16& acc, const float4* rows, int i) {
        const float4 r = ahead;
        if (i < 15) ahead = rows[acc_row(hh, i + 1)];
        float x = fmaf(acc[i], a.c_log2, r.w);
        if constexpr (kBias) {
            const float dx = kx - r.x, dy = ky - r.y;
            x = fmaf(r.z, dx * dx + dy * dy, x);
        }
        // a probability: at most 1, and 0 where the row has no LSE whatever its logits are
        part_sum += fminf(fmaxf(__builtin_amdgcn_exp2f(x), 0.0f), 1.0f);
        asm volatile("" : "+v"(part_sum));  // keeps it between its MFMAs
    };
    // tile t's products into `acc`, tile t - 1's exponentials from `before`
    auto tile = [&](auto first_tag, int t, floatx16& acc, const floatx16& before) __attribute__((always_inline)) {
        constexpr bool kFirst = decltype(first_tag)::value;
        const float4* rows = lds_row[wave][(t - 1) & 1];
        lds_row[wave][t & 1][n] = make_row(t);  // both halves write the same; this wave reads it in tile t + 1
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (t + 1 < t1) fetch_row(t + 1);
        const uint8_t* next = q_at(t + 1 < t1 ? t + 1 : t);
        acc = floatx16{0};
        part_sum = 0.0f;
        if constexpr (!kFirst) ahead = rows[acc_row(hh, 0)];
        constexpr int kUnits = 16 / kG;  // logits of the tile before per four MFMAs
#pragma unroll
        for (int j = 0; j < kG; ++j) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(qf[j][i], kf[j][i], acc, 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (!kFirst) {
                    if (i % (4 / kUnits) == 0) unit(before, rows, j * kUnits + i / (4 / kUnits));
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if (j % 4 == 3) {  // a row's whole line of 128 bytes at once
#pragma unroll
                for (int i = j - 3; i <= j; ++i) qf[i] = *reinterpret_cast<const floatx4*>(next + 32 * i);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        group += part_sum;
    };
    if (t0 < t1) {
        floatx16 accA, accB;
        const uint8_t* first = q_at(t0);
#pragma unroll
        for (int j = 0; j < kG; ++j) qf[j] = *reinterpret_cast<const floatx4*>(first + 32 * j);
        fetch_row(t0);
        // the keys are waited for here, not at their first use in the loop
#pragma unroll
        for (int j = 0; j < kG; ++j) asm volatile("" : "+v"(kf[j]));
        tile(std::true_type{}, t0, accA, accB);
        int t = t0 + 1;
        for (; t + 1 < t1; t += 2) {
            tile(std::false_type{}, t, accB, accA);
            tile(std::false_type{}, t + 1, accA, accB);
            if (((t - t0) & 15) == 15) {
                sum += group;
                group = 0.0f;
            }
        }
        if (t < t1) {
            tile(std::false_type{}, t, accB, accA);
            accA = accB;
        }
        part_sum = 0.0f;
        ahead = lds_row[wave][(t1 - 1) & 1][acc_row(hh, 0)];
#pragma unroll
        for (int i = 0; i < 16; ++i) unit(accA, lds_row[wave][(t1 - 1) & 1], i);
        sum += group + part_sum;
    }
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    sum = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    if (hh == 0 && n < kb.keys) {
        const int64_t o = (int64_t)hd * a.Lk + kb.key0 + n;
        if (a.parts > 1) a.partial[(int64_t)part * a.H * a.Lk + o] = sum;
        else a.out[o] = a.prev ? fmaf(a.decay, a.prev[o], sum) : sum;
    }
}

// out = decay prev + the parts' sums, in the order of the parts
__global__ __launch_bounds__(256) void key_weight_merge(const float* partial, const float* prev, float decay, float* out,
                                                        int64_t n, int parts) {
    const int64_t i = (int64_t)row_block() * 256 + threadIdx.x;
    if (i >= n) return;
    float sum = 0.0f;
    for (int p = 0; p < parts; ++p) sum += partial[p * n + i];
    out[i] = prev ? fmaf(decay, prev[i], sum) : sum;
}

// Frames that the blocks of a workgroup lie in, at most: workgroups start at multiples of
// gcd(their blocks, a frame's blocks) within a frame. 2 for frames of 4 and 6 and of 7 blocks and more, else 3 or 4.
int group_frames(const KeyWeightArgs& a) {
    const int group = a.wave_blocks * kWaves, step = std::gcd(group, a.frame_blocks);
    return 1 + (group - step + a.frame_blocks - 1) / a.frame_blocks;
}

bool few_queries(const KeyWeightArgs& a) { return a.Lq <= kFewQueries; }

}  // namespace

void key_weight_plan(KeyWeightArgs& a) {
    // without a bias the frames do not matter: all keys are one
    if (a.S == 0) {
        a.hw = a.Lk;
        a.w = a.Lk;
    }
    a.frame_blocks = (a.hw + kKeys - 1) / kKeys;
    a.n_blocks = a.frame_blocks * (a.Lk / a.hw);
    // a wave takes two blocks; where frames are single blocks, one, so that a workgroup meets four at most
    a.wave_blocks = a.type == kTypeF32 || few_queries(a) || (a.S > 0 && a.frame_blocks == 1) ? 1 : 2;
}

int64_t key_weight_items(const KeyWeightArgs& a) {
    const int per_group = a.wave_blocks * kWaves;  // key blocks of a workgroup
    return ((int64_t)a.n_blocks + per_group - 1) / per_group * a.H * a.parts;
}

// Workgroups that a compute unit has room for, by the kernels' registers: fp32 at D 64, at D 128, bf16 / fp8.
constexpr int kPlacesF32D64 = 4, kPlacesF32D128 = 2, kPlacesBf16 = 2;

int32_t key_weight_parts(const KeyWeightArgs& a, int32_t cus) {
    if (a.Lq < 256) return 1;  // a part's own start (its keys, its first queries) would cost more than it saves
    KeyWeightArgs b = a;
    b.parts = 1;
    const int64_t items = key_weight_items(b), tiles = (a.Lq + 31) / 32;
    // Estimated time in steps of 64 queries: the rounds that the workgroups make on the chip's places,
    // each as long as a part plus its start. The last round leaves k workgroups on a compute unit, which share it and take
    // about k / places of a full one. Workgroups with a bias take a quarter longer than those without, and
    // which come last is chance: a fifth of a part more. With parts, the merge. Chosen against the best of 1 to 16
    // parts, us: fp32, D 128, 3 heads of 1560 x 28080 309, 309; 12 of 1170 x 4680 167, 167; D 64, 2 of 3321 x 9963 90, 90;
    // 3 of 1560 x 28080 167, 165 (places and step time of one size for both D chose 325, 180, 103 and 181); bf16, half of
    // 6 frames of 3600 biased, 12 heads of 10800 queries 810, 803 (without the fifth 860).
    const bool f32 = a.type == kTypeF32;
    const int64_t places = !f32 ? kPlacesBf16 : (a.D == 64 ? kPlacesF32D64 : kPlacesF32D128), slots = cus * places;
    const double start = f32 ? 1.0 : 2.3, step_us = f32 ? (a.D == 64 ? 9.0 : 8.0) : (a.S > 0 ? 2.1 : 1.8);
    const int64_t least = f32 ? 1 : 4;  // tiles of a part: an fp32 one takes 4 us, as long as a whole start
    double best = 0.0;
    int32_t parts = 1;
    for (int32_t p = 1; p <= 16 && (p == 1 || tiles / p >= least); ++p) {
        const int64_t n = items * p, last = (n % slots + cus - 1) / cus;
        const double rounds = (double)(n / slots) + (last > 0 ? ((double)last + 0.2) / ((double)places + 0.2) : 0.0);
        double t = (rounds + (!f32 && a.S > 0 ? 0.2 : 0.0)) * (start + (double)((tiles + p - 1) / p) / 2);
        if (p > 1) t += (3.0 + (double)p * a.H * a.Lk * 4 / 4e6) / step_us;
        if (p == 1 || t < best) {
            best = t;
            parts = p;
        }
    }
    return parts;
}

hipError_t launch_key_weight(const KeyWeightArgs& a, hipStream_t stream) {
    const unsigned n_items = (unsigned)key_weight_items(a);
    const dim3 grid = grid_rows(xcd_grid(n_items)), block(64 * kWaves);
    const bool bias = a.S > 0;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, n_items); };
    if (a.type == kTypeF32) {
        if (a.D == 64) bias ? go(key_weight_f32_kernel<64, true>) : go(key_weight_f32_kernel<64, false>);
        else bias ? go(key_weight_f32_kernel<128, true>) : go(key_weight_f32_kernel<128, false>);
    } else if (few_queries(a)) {
        if (a.type == kTypeFp8) bias ? go(key_weight_few_kernel<true, true>) : go(key_weight_few_kernel<true, false>);
        else bias ? go(key_weight_few_kernel<false, true>) : go(key_weight_few_kernel<false, false>);
    } else if (a.type == kTypeFp8) {
        if (!bias) go(key_weight_bf16_kernel<true, 0>);
        else group_frames(a) <= 2 ? go(key_weight_bf16_kernel<true, 2>) : go(key_weight_bf16_kernel<true, 4>);
    } else {
        if (!bias) go(key_weight_bf16_kernel<false, 0>);
        else group_frames(a) <= 2 ? go(key_weight_bf16_kernel<false, 2>) : go(key_weight_bf16_kernel<false, 4>);
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.parts > 1) {
        const int64_t n = (int64_t)a.H * a.Lk;
        hipLaunchKernelGGL(key_weight_merge, grid_rows((unsigned)((n + 255) / 256)), dim3(256), 0, stream, a.partial, a.prev, a.decay,
                           a.out, n, a.parts);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace revisit
