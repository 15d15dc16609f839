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
constexpr int kKeys = 32;  // keys of a wave

// Accumulator row held by register i of a lane in wave half `hh` (32x32 MFMA).
__device__ __forceinline__ int acc_row(int hh, int i) { return 8 * (i >> 2) + 4 * hh + (i & 3); }

// Operand of one row of D elements: lane half hh's share.
template <int kType, int D>
struct Row;
template <int D>
struct Row<1, D> {  // bf16: step j takes elements 16 j + 8 hh ..
    u32x4 v[D / 16];
    __device__ __forceinline__ void load(const uint8_t* row, int hh) {
#pragma unroll
        for (int j = 0; j < D / 16; ++j) v[j] = *reinterpret_cast<const u32x4*>(row + 32 * j + 16 * hh);
    }
};
template <int D>
struct Row<2, D> {  // fp32: step 4 g + i takes element 8 g + 4 hh + i
    floatx4 v[D / 8];
    __device__ __forceinline__ void load(const uint8_t* row, int hh) {
#pragma unroll
        for (int j = 0; j < D / 8; ++j) v[j] = *reinterpret_cast<const floatx4*>(row + 32 * j + 16 * hh);
    }
};
// fp8: the e4m3 values as bf16, which holds them exactly. The fp8 matrix cores drop what
// lies 13 bits below the largest product of a few (measured on the device), far
// from an fp32 sum; the bf16 ones keep 24 bits.
template <int D>
struct Row<3, D> {
    u32x4 v[D / 16];
    __device__ __forceinline__ void load(const uint8_t* row, int hh) {
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            const u32x2 b = *reinterpret_cast<const u32x2*>(row + 16 * j + 8 * hh);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                v[j][2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b[i], 1.0f, false));
                v[j][2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b[i], 1.0f, true));
            }
        }
    }
};
template <int kType, int D>
__device__ __forceinline__ floatx16 product(const Row<kType, D>& q, const Row<kType, D>& k) {
    floatx16 s = floatx16{0};
    if constexpr (kType == 2) {
#pragma unroll
        for (int j = 0; j < D / 8; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) s = __builtin_amdgcn_mfma_f32_32x32x2f32(q.v[j][i], k.v[j][i], s, 0, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, q.v[j]), __builtin_bit_cast(bf16x8, k.v[j]), s, 0, 0, 0);
    }
    return s;
}

template <int kType, int D, bool kBias>
__global__ __launch_bounds__(64 * kWaves) void key_weight_kernel(KeyWeightArgs a, unsigned n_items) {
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

    constexpr int kSize = kType == 1 ? 2 : (kType == 2 ? 4 : 1);
    const int64_t row_bytes = (int64_t)a.H * D * kSize;
    Row<kType, D> kf, qf;
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
        const floatx16 acc = product<kType, D>(qf, kf);
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

template <int kType, int D>
void launch(const KeyWeightArgs& a, unsigned n_items, hipStream_t stream) {
    const dim3 grid = grid_rows(xcd_grid(n_items)), block(64 * kWaves);
    if (a.S > 0) hipLaunchKernelGGL((key_weight_kernel<kType, D, true>), grid, block, 0, stream, a, n_items);
    else hipLaunchKernelGGL((key_weight_kernel<kType, D, false>), grid, block, 0, stream, a, n_items);
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
    return (int64_t)((a.n_blocks + kWaves - 1) / kWaves) * a.H * a.parts;
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
    if (a.type == 1) launch<1, 128>(a, n_items, stream);
    else if (a.type == 3) launch<3, 128>(a, n_items, stream);
    else if (a.D == 64) launch<2, 64>(a, n_items, stream);
    else launch<2, 128>(a, n_items, stream);
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
