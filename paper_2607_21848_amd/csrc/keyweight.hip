// Attention weight of every key (attention_key_weight):
//     out[h][k] = decay prev[h][k] + sum_p exp(A_pk - LSE_p),
// A the biased logits of biased_chunk_attention and LSE what that call returned.
//
// A wave owns 32 keys of one head and computes the logit tiles S = Q K^T with
// 32x32 MFMAs: queries are the M dimension, its keys the N dimension (held in
// registers), so a lane holds one key and 16 queries of each tile and a key's
// sum stays in its lane until the end, where the two wave halves meet. No atomics:
// the same call gives the same bits. Blocks of 32 keys never cross a frame, so
// one retrieved frame's correspondences serve the whole block.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "internal.h"

namespace revisit {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWaves = 4;
constexpr int kKeys = 32;  // keys of a block
constexpr int kTypeF32 = 2, kTypeFp8 = 3;  // REVISIT_F32, REVISIT_FP8_QK

// Accumulator row held by register i of a lane in wave half `hh` (32x32 MFMA).
__device__ __forceinline__ int acc_row(int hh, int i) { return 8 * (i >> 2) + 4 * hh + (i & 3); }

// ---------------------------------------------------------------------------
// bf16 and fp8 kernel.
// ---------------------------------------------------------------------------
constexpr int kD = 128;
constexpr int kStep = 64;                    // queries of a step
constexpr int kRowBytes = kD * 2;
constexpr int kStepBytes = kStep * kRowBytes;

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// Position of 16-byte chunk c of row r: 16 rows that read one chunk together touch 16 different positions.
__device__ __forceinline__ int chunk_at(int r, int c) { return r * kRowBytes + ((c ^ (((r & 3) << 2) | ((r >> 2) & 3))) << 4); }

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

// A block of 32 keys: where it is, and what its bias goes by.
struct KeyBlock {
    int64_t key0;
    int keys;     // of it within the frame; 0: no such block
    int slot;     // retrieved frame, -1: unbiased
    int in0;      // first key within the frame
};
__device__ __forceinline__ KeyBlock key_block(const KeyWeightArgs& a, int kb, bool bias) {
    KeyBlock b;
    const int frame = kb / a.frame_blocks;
    b.in0 = (kb - frame * a.frame_blocks) * kKeys;
    b.keys = kb < a.n_blocks ? min(kKeys, a.hw - b.in0) : 0;
    b.key0 = (int64_t)frame * a.hw + b.in0;
    b.slot = -1;
    if (bias && b.keys > 0) {
        const int s = a.slot[frame];
        if (s >= 0 && s < a.S) b.slot = s;
    }
    return b;
}

template <bool kFp8, bool kBias>
__global__ __launch_bounds__(64 * kWaves, 2) void key_weight_bf16_kernel(KeyWeightArgs a, unsigned n_items) {
    __shared__ __attribute__((aligned(16))) uint8_t lds_q[2][kStepBytes];
    __shared__ __attribute__((aligned(16))) float lds_row[2][kStep];  // -LSE log2 e of the step's queries

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hh = lane >> 5, n = lane & 31;
    const unsigned block = row_block();
    const unsigned item = xcd_item(block, n_items);
    if (block >= xcd_grid(n_items) || item >= n_items) return;  // grid padding (uniform, before any barrier)
    // item = (head, query part, group of key blocks)
    const int groups = (a.n_blocks + 2 * kWaves - 1) / (2 * kWaves);
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
    auto fetch = [&](int q0) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int e = tid + i * 64 * kWaves;
            const int q = min(q0 + e / kChunks, a.Lq - 1);
            stage[i] = *reinterpret_cast<const u32x4*>(Qg + q * row_bytes + 16 * (e % kChunks));
        }
        if (tid < kStep) stage_lse = a.lse[(int64_t)hd * a.Lq + min(q0 + tid, a.Lq - 1)];
    };
    auto put = [&](int q0, int buf) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int e = tid + i * 64 * kWaves;
            const int r = e / kChunks, c = e % kChunks;
            if constexpr (kFp8) {
                *reinterpret_cast<u32x4*>(lds_q[buf] + chunk_at(r, 2 * c)) = wide(stage[i][0], stage[i][1]);
                *reinterpret_cast<u32x4*>(lds_q[buf] + chunk_at(r, 2 * c + 1)) = wide(stage[i][2], stage[i][3]);
            } else {
                *reinterpret_cast<u32x4*>(lds_q[buf] + chunk_at(r, c)) = stage[i];
            }
        }
        // a query past the end, or one without an LSE, has no weight to give
        if (tid < kStep) lds_row[buf][tid] = q0 + tid < q_end && __builtin_isfinite(stage_lse) ? -stage_lse * kLog2e : -INFINITY;
    };
    if (t0 < t1) fetch(t0 * 32);

    // this wave's keys: two blocks of 32
    KeyBlock kb[2];
    bf16x8 kf[2][kD / 16];
    bf16x8 kbias[2];  // key side of the bias products
    const float cx = 0.5f * (float)a.w, cy = 0.5f * (float)a.h;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        kb[b] = key_block(a, (g * kWaves + wave) * 2 + b, kBias);
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
        if constexpr (kBias) {
            const int t = kb[b].in0 + n, ky = t / a.w;
            const float at = hh ? ((float)ky + 0.5f) - cy : ((float)(t - ky * a.w) + 0.5f) - cx;
            const uint32_t twice = bf16_bits(2.0f * at);  // exact: a half-integer below 128
            uint32_t ph, pm, pl;
            split3(-a.gamma * (at * at), ph, pm, pl);
            kbias[b] = as_bf16x8(u32x4{pack2(twice, twice), pack2(twice, ph), pack2(pm, pl), hh ? kOne : pack2(kOne, kOne)});
        }
    }
    // query side of the bias products of 32 queries from q0 on, for retrieved frame s
    auto query_bias = [&](int s, int q0) -> bf16x8 {
        const int64_t o = (int64_t)s * a.Lq + min(q0 + n, a.Lq - 1);
        const float2 u = reinterpret_cast<const float2*>(a.corr_uv)[o];
        u32x4 v = u32x4{0, 0, 0, 0};
        if (a.corr_idx[o] >= 0 && !__builtin_isnan(u.x)) {
            const float ux = u.x - cx, uy = u.y - cy;
            uint32_t ah, am, al, zh, zm, zl;
            split3(a.gamma * (hh ? uy : ux), ah, am, al);
            split3(-a.gamma * (ux * ux + uy * uy), zh, zm, zl);
            v = u32x4{pack2(ah, am), pack2(al, kOne), pack2(kOne, kOne), hh ? zl : pack2(zh, zm)};
        }
        return as_bf16x8(v);
    };

    float sum[2] = {0.0f, 0.0f};
    int buf = 0;
    if (t0 < t1) put(t0 * 32, 0);
    __syncthreads();
    for (int t = t0; t < t1; t += 2, buf ^= 1) {
        const bool more = t + 2 < t1;
        if (more) fetch((t + 2) * 32);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            if (half && t + 1 >= t1) break;  // uniform
            floatx16 acc[2] = {floatx16{0}, floatx16{0}};
            if constexpr (kBias) {
                if (kb[0].slot >= 0 || kb[1].slot >= 0) {  // uniform per wave
                    bf16x8 qb = as_bf16x8(u32x4{0, 0, 0, 0});
                    if (kb[0].slot >= 0) {
                        qb = query_bias(kb[0].slot, (t + half) * 32);
                        acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qb, kbias[0], acc[0], 0, 0, 0);
                    }
                    if (kb[1].slot >= 0) {
                        if (kb[1].slot != kb[0].slot) qb = query_bias(kb[1].slot, (t + half) * 32);
                        acc[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qb, kbias[1], acc[1], 0, 0, 0);
                    }
                }
            }
            const uint8_t* rows = lds_q[buf];
#pragma unroll
            for (int j = 0; j < kD / 16; ++j) {
                const bf16x8 qf = as_bf16x8(*reinterpret_cast<const u32x4*>(rows + chunk_at(32 * half + n, 2 * j + hh)));
                acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[0][j], acc[0], 0, 0, 0);
                acc[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qf, kf[1][j], acc[1], 0, 0, 0);
            }
            floatx4 rc[4];  // queries 8 i + 4 hh ..
#pragma unroll
            for (int i = 0; i < 4; ++i) rc[i] = *reinterpret_cast<const floatx4*>(&lds_row[buf][32 * half + 8 * i + 4 * hh]);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float s = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    // a probability: at most 1, and 0 where the row has no LSE whatever its logits are
                    const float e = __builtin_amdgcn_exp2f(fmaf(acc[b][i], a.c_log2, rc[i >> 2][i & 3]));
                    s += fminf(fmaxf(e, 0.0f), 1.0f);
                }
                sum[b] += s;
            }
        }
        if (more) put((t + 2) * 32, buf ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
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
// fp32 kernel.
// ---------------------------------------------------------------------------

// Row of D elements, lane half hh's share: MFMA step 4 g + i takes element 8 g + 4 hh + i.
template <int D>
struct Row {
    floatx4 v[D / 8];
    __device__ __forceinline__ void load(const uint8_t* row, int hh) {
#pragma unroll
        for (int j = 0; j < D / 8; ++j) v[j] = *reinterpret_cast<const floatx4*>(row + 32 * j + 16 * hh);
    }
};

template <int D, bool kBias>
__global__ __launch_bounds__(64 * kWaves) void key_weight_f32_kernel(KeyWeightArgs a, unsigned n_items) {
    __shared__ float4 lds_row[kWaves][32];  // per query: u^ x, y, -gamma log2e or 0, -LSE log2e

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
    const int kb = g * kWaves + wave;
    if (kb >= a.n_blocks) return;  // uniform per wave; no barrier below
    const int frame = kb / a.frame_blocks;
    const int in0 = (kb - frame * a.frame_blocks) * kKeys;  // first key within the frame
    const int keys = min(kKeys, a.hw - in0);
    const int64_t key0 = (int64_t)frame * a.hw + in0;

    constexpr int kSize = 4;
    const int64_t row_bytes = (int64_t)a.H * D * kSize;
    Row<D> kf, qf;
    kf.load(static_cast<const uint8_t*>(a.k) + (key0 + min(n, keys - 1)) * row_bytes + (int64_t)hd * D * kSize, hh);
    int s = -1;
    if constexpr (kBias) {
        s = a.slot[frame];
        if (s >= a.S) s = -1;
    }
    const int ky_i = (in0 + n) / a.w;
    const float kx = (float)(in0 + n - ky_i * a.w) + 0.5f, ky = (float)ky_i + 0.5f;

    const int n_tiles = (a.Lq + 31) / 32;
    const int t0 = (int)((int64_t)part * n_tiles / a.parts), t1 = (int)((int64_t)(part + 1) * n_tiles / a.parts);
    float sum = 0.0f;
    for (int t = t0; t < t1; ++t) {
        const int q = t * 32 + n;
        const int q_in = min(q, a.Lq - 1);
        qf.load(static_cast<const uint8_t*>(a.q) + (int64_t)q_in * row_bytes + (int64_t)hd * D * kSize, hh);
        float4 row = {0.0f, 0.0f, 0.0f, -INFINITY};
        const float lse = a.lse[(int64_t)hd * a.Lq + q_in];
        // a query past the end, or one without an LSE, has no weight to give
        if (q < a.Lq && __builtin_isfinite(lse)) row.w = -lse * kLog2e;
        if (kBias && s >= 0) {
            const int64_t o = (int64_t)s * a.Lq + q_in;
            const float2 u = reinterpret_cast<const float2*>(a.corr_uv)[o];
            if (a.corr_idx[o] >= 0 && !__builtin_isnan(u.x)) {
                row.x = u.x;
                row.y = u.y;
                row.z = -a.gamma2;
            }
        }
        __builtin_amdgcn_wave_barrier();
        lds_row[wave][n] = row;  // both halves write the same
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        floatx16 acc = floatx16{0};
#pragma unroll
        for (int j = 0; j < D / 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(qf.v[j][i], kf.v[j][i], acc, 0, 0, 0);
        float part_sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float4 r = lds_row[wave][acc_row(hh, i)];
            float x = fmaf(acc[i], a.c_log2, r.w);
            if (kBias && s >= 0) {
                const float dx = kx - r.x, dy = ky - r.y;
                if (r.z != 0.0f) x = fmaf(r.z, dx * dx + dy * dy, x);
            }
            // a probability: at most 1, and 0 where the row has no LSE whatever its logits are
            part_sum += fminf(fmaxf(__builtin_amdgcn_exp2f(x), 0.0f), 1.0f);
        }
        sum += part_sum;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
    sum = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    if (hh == 0 && n < keys) {
        const int64_t o = (int64_t)hd * a.Lk + key0 + n;
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

}  // namespace

void key_weight_plan(KeyWeightArgs& a) {
    // without a bias the frames do not matter: all keys are one
    if (a.S == 0) {
        a.hw = a.Lk;
        a.w = a.Lk;
    }
    a.frame_blocks = (a.hw + kKeys - 1) / kKeys;
    a.n_blocks = a.frame_blocks * (a.Lk / a.hw);
}

int64_t key_weight_items(const KeyWeightArgs& a) {
    const int per_group = a.type == kTypeF32 ? kWaves : 2 * kWaves;  // key blocks of a workgroup
    return ((int64_t)a.n_blocks + per_group - 1) / per_group * a.H * a.parts;
}

int32_t key_weight_parts(const KeyWeightArgs& a, int32_t cus) {
    KeyWeightArgs b = a;
    b.parts = 1;
    const int64_t items = key_weight_items(b), want = 4 * (int64_t)cus;
    const int64_t tiles = (a.Lq + 31) / 32;
    int64_t parts = (want + items - 1) / items;
    parts = parts < tiles / 4 ? parts : tiles / 4;  // four query tiles a part at least
    return (int32_t)(parts < 1 ? 1 : (parts > kKeyWeightMaxParts ? kKeyWeightMaxParts : parts));
}

hipError_t launch_key_weight(const KeyWeightArgs& a, hipStream_t stream) {
    const unsigned n_items = (unsigned)key_weight_items(a);
    const dim3 grid = grid_rows(xcd_grid(n_items)), block(64 * kWaves);
    const bool bias = a.S > 0;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, n_items); };
    if (a.type == kTypeF32) {
        if (a.D == 64) bias ? go(key_weight_f32_kernel<64, true>) : go(key_weight_f32_kernel<64, false>);
        else bias ? go(key_weight_f32_kernel<128, true>) : go(key_weight_f32_kernel<128, false>);
    } else if (a.type == kTypeFp8) {
        bias ? go(key_weight_bf16_kernel<true, true>) : go(key_weight_bf16_kernel<true, false>);
    } else {
        bias ? go(key_weight_bf16_kernel<false, true>) : go(key_weight_bf16_kernel<false, false>);
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
