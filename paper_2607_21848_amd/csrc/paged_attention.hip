// Attention over a paged cache (paged_chunk_attention).
//
// Per stream and head, O = softmax(scale Q K^T + lambda B) V over the keys that a query sees, with one pass over
// keys and values: a running maximum and sum, the sums rescaled where the maximum grows. Rows of a tile are
// (query, head of the group that shares a key head) pairs, so a key is read once for the whole group.
//
// Keys and values of 8 bits are widened to bf16 with their scale, which is a power of two: exactly. The 8-bit
// matrix cores would not give an fp32 sum of products (they drop what lies 13 bits below a group's largest).
//
// The wave kernel. Tiles of 16 or 32 rows against 32 keys; a wave works by itself, without a barrier until the
// end, and loads its operands straight from the pages into registers in the matrix cores' layout: with 16x16
// MFMAs a lane of S^T = K Q^T supplies 8 head dims of a key, of O^T = V^T P^T one head dim of 8 keys. Both
// contractions may number their index at will as long as both operands agree, so a lane's head dims are
// consecutive bytes of the key's row, the 8 keys of a lane are those whose probabilities its own accumulators
// hold (no exchange between lanes), and the head dim of row m and block db is (D / 16) m + db, so that a lane's value
// bytes are consecutive too; two keys' bytes are interleaved by byte permutes before they are widened. For few
// queries it is bound by HBM: a wave has the next tile's keys and values in flight while it works on this one's.

#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "paged.h"

namespace revisit {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kTK = 32;               // keys of a tile: those that share a scale
constexpr float kRescaleSlack = 8.0f;  // a maximum may grow by 2^8 before the sums are rescaled

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{a, b}, bf16x2));
}
__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// Sizes of a tile's loads, by element type and head size.
template <int D, int T>
struct Shape {
    static constexpr int kES = T == kPagedFp8 ? 1 : (T == kPagedBf16 ? 2 : 4);
    static constexpr int kRowBytes = D * kES;
    static constexpr int kDb = D / 16;                // blocks of 16 head dims
    static constexpr int kKLoads = kRowBytes / 64;    // 16-byte loads of a lane per 16 keys
    static constexpr int kVBytes = kDb * kES;         // of a lane and key
    static constexpr int kVWords = kVBytes / 4;
};

template <int N>
struct Words;
template <>
struct Words<1> {
    typedef uint32_t type;
};
template <>
struct Words<2> {
    typedef u32x2 type;
};
template <>
struct Words<4> {
    typedef u32x4 type;
};

// bias of a query beside the frame at hand
struct Corr {
    float ng;  // -gamma, or 0 where the frame is not retrieved or the correspondence not accepted
    float ux, uy;
};

struct PagedBias {
    const int32_t* slot;  // of the stream's frames
    const float* corr_uv;
    const int32_t* corr_idx;
    int max_frames, S, n_tokens;
    float ng;
};

constexpr int kManyWaves = 8;   // of a workgroup where there are few
constexpr int kCorrFrames = 16, kSlotFrames = 256;  // retrieved and key frames whose correspondences and slots are kept in LDS

// Two waves per SIMD where the registers do for it (fp32 at D = 64, 1170 queries on 7020 keys: one 283 us, two 271; at D = 128
// two would need each tile's keys and values loaded when their turn comes, 544 us with one and 561 with two so). The MFMAs
// accumulate in the registers that vector instructions read (-amdgpu-mfma-vgpr-form, set for this file): 1170 biased fp32
// queries at D = 128 543 us without, 514 with. Loads put between the products by hand instead of by the compiler: 528.
template <int D, int T, int NQ, bool kBias, int kW, bool kStrided>
__global__ __launch_bounds__(64 * kW, kW > 4 || (T == kPagedF32 ? D == 64 : NQ == 1) ? 2 : 1) void paged_wave_kernel(PagedAttentionArgs a, float c_log2) {
    using Sh = Shape<D, T>;
    constexpr int kRows = 16 * NQ;
    constexpr int kDb = Sh::kDb;
    constexpr bool kF32 = T == kPagedF32;
    // Few rows leave the matrix cores idle: their probabilities go in as two bf16 values each, off by 2^-17 (a single
    // one, 2^-9, made outputs of a few heavy keys 1.6 times as far off as their own rounding does). Tiles of 32 rows keep
    // one, like the tile kernel's: 30 queries on 37440 8-bit keys 26.6 us, with two 29.2.
    constexpr bool kFine = !kF32 && NQ == 1;
    // The next tile's keys leave behind this one's logits, its values behind this one's product, where the registers hold both
    // beside each other (1170 fp32 queries on 7020 keys, when it was taken: 606 us without, 567 with).
    constexpr bool kAhead = !kF32 || NQ == 2 || D == 64 || kW == 4;
    __shared__ float lds_o[kW][kDb * 64 * 4];  // of one block of 16 rows
    __shared__ float lds_m[kW][kRows], lds_l[kW][kRows];
    __shared__ int lds_token[kRows], lds_head[kRows];
    __shared__ floatx4 lds_q[kF32 ? NQ * D / 16 : 1][64];  // fp32 queries: the lane's vector of four steps

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int m = lane & 15, grp = lane >> 4;
    const PagedSeqs& sq = a.seqs;
    const int G = a.G;

    // unit = (key head, part, tile), tiles fastest: the tiles that read the same keys run on one XCD
    const unsigned n_units = (unsigned)a.tiles * (unsigned)a.Hk * (unsigned)a.parts;
    const unsigned block = row_block();
    const unsigned unit = xcd_item(block, n_units);
    if (block >= xcd_grid(n_units) || unit >= n_units) return;  // grid padding (uniform, before any barrier)
    const int tile = (int)(unit % (unsigned)a.tiles);
    const int hp = (int)(unit / (unsigned)a.tiles);
    const int hk = hp / a.parts, part = hp - hk * a.parts;
    const StreamItem it = row_tile(a, kRows, tile);
    if (it.s < 0) return;
    const int s = it.s;
    const int2 tok = tokens_of(sq, s);
    const int n_rows = tok.y * G;  // at most 2^30

    // the lane's query rows (column m of block nq)
    int token[NQ], head[NQ], vis[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
        const int r = it.in * kRows + 16 * nq + m, t = r / G;
        token[nq] = r < n_rows ? tok.x + t : -1;
        head[nq] = hk * G + r - t * G;
    }
    // queries: step (u, v) of a lane takes the head dims that its key vector u holds in elements 8 v .. (fp32: 4 v ..)
    constexpr int kSteps = kF32 ? 1 : D / 32;
    u32x4 qf[kF32 ? 1 : NQ][kSteps];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
        const int64_t row = (int64_t)max(token[nq], 0) * a.q_row + (int64_t)head[nq] * D;
        if constexpr (kF32) {
            for (int u = wave; u < D / 16; u += kW) {
                floatx4 v = floatx4{0, 0, 0, 0};
                if (token[nq] >= 0) v = *reinterpret_cast<const floatx4*>(static_cast<const float*>(a.q) + row + 16 * u + 4 * grp);
                lds_q[nq * (D / 16) + u][lane] = v;
            }
        } else {
#pragma unroll
            for (int st = 0; st < kSteps; ++st) {
                const int d = T == kPagedFp8 ? 64 * (st >> 1) + 16 * grp + 8 * (st & 1) : 32 * st + 8 * grp;
                qf[nq][st] = u32x4{0, 0, 0, 0};
                if (token[nq] >= 0) qf[nq][st] = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) + row + d);
            }
        }
    }

    // how many keys each sees
    const int held = held_of(sq, s);
    int seen = 0, seen_min = INT32_MAX;
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
        vis[nq] = held;
        if (token[nq] >= 0) {
            if (a.visible) vis[nq] = min(held, max(a.visible[token[nq]], 0));
            seen = max(seen, vis[nq]);
            seen_min = min(seen_min, vis[nq]);
        }
    }
    if (a.visible) {
#pragma unroll
        for (int off = 1; off < 16; off *= 2) {
            seen = max(seen, __shfl_xor(seen, off));
            seen_min = min(seen_min, __shfl_xor(seen_min, off));
        }
    } else {
        seen = seen_min = held;
    }
    seen = __builtin_amdgcn_readfirstlane(seen);
    seen_min = __builtin_amdgcn_readfirstlane(seen_min);

    const int n_tiles = (seen + kTK - 1) / kTK;
    const int t_begin = (int)((int64_t)part * n_tiles / a.parts), t_end = (int)((int64_t)(part + 1) * n_tiles / a.parts);
    if constexpr (kF32) __syncthreads();

    // A tile's page entry, by a scalar load: as a vector load it would wait for the keys and values in flight before it.
    const const_i32* pages = reinterpret_cast<const const_i32*>((uintptr_t)(sq.page_table + (int64_t)s * sq.max_pages));
    auto entry_of = [&](int t) -> int { return pages[__builtin_amdgcn_readfirstlane((t * kTK) >> sq.page_log2)]; };
    // the operands of a tile's keys and values
    using VVec = typename Words<(Sh::kVWords > 4 ? 4 : Sh::kVWords)>::type;
    constexpr int kVHalves = Sh::kVWords > 4 ? 2 : 1;
    struct Tile {
        u32x4 kr[2][Sh::kKLoads];
        VVec vr[8][kVHalves];
        int k_byte, v_byte;  // the scales, converted where they are used: sooner would wait for the loads
        int t, page;
    };
    const int in_page = (1 << sq.page_log2) - 1;
    // where a tile's rows of a cache and its scale are, and the bytes from row to row
    auto tile_row = [&](int t, int page) -> size_t { return (((size_t)page * a.Hk + hk) << sq.page_log2) + ((t * kTK) & in_page); };
    auto tile_at = [&](const void* cache, const PagedStrides& st, int t, int page) -> const uint8_t* {
        if constexpr (kStrided) return static_cast<const uint8_t*>(cache) + strided_at(st, page, hk, (t * kTK) & in_page);
        else return static_cast<const uint8_t*>(cache) + tile_row(t, page) * Sh::kRowBytes;
    };
    auto scale_of = [&](const uint8_t* scale, const PagedStrides& st, int t, int page) -> int {
        if constexpr (kStrided) return scale[strided_at(st, page, hk, ((t * kTK) & in_page) / kScaleBlock)];
        else return scale[tile_row(t, page) / kScaleBlock];
    };
    auto step_of = [&](const PagedStrides& st) -> int64_t {
        if constexpr (kStrided) return st.row;
        else return Sh::kRowBytes;
    };
    auto load_k = [&](Tile& b, int t, int page) {
        const uint8_t* base = tile_at(a.cache_k, a.layout.k, t, page);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int u = 0; u < Sh::kKLoads; ++u)
                b.kr[i][u] = *reinterpret_cast<const u32x4*>(base + (16 * i + m) * step_of(a.layout.k) + 64 * u + 16 * grp);
        if constexpr (T == kPagedFp8) b.k_byte = scale_of(a.scale_k, a.layout.scale_k, t, page);
    };
    // key of the lane's element j
    auto key_of = [&](int j) -> int { return 16 * (j >> 2) + 4 * grp + (j & 3); };
    auto load_v = [&](Tile& b, int t, int page) {
        const uint8_t* base = tile_at(a.cache_v, a.layout.v, t, page);
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int u = 0; u < kVHalves; ++u) {
                // fp32 at D 128: head dims 64 u + 4 m .., else kDb m ..
                const int off = kVHalves == 2 ? 256 * u + 16 * m : Sh::kVBytes * m;
                b.vr[j][u] = *reinterpret_cast<const VVec*>(base + key_of(j) * step_of(a.layout.v) + off);
            }
        if constexpr (T == kPagedFp8) b.v_byte = scale_of(a.scale_v, a.layout.scale_v, t, page);
    };

    // head dim of row 4 grp + i, block db
    auto dim = [&](int i, int db) -> int { return kVHalves == 2 ? 64 * (db >> 2) + 4 * (4 * grp + i) + (db & 3) : kDb * (4 * grp + i) + db; };
    floatx4 O[NQ][kDb];
    float m_run[NQ], l_run[NQ], m_thr[NQ];
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
#pragma unroll
        for (int db = 0; db < kDb; ++db) O[nq][db] = floatx4{0, 0, 0, 0};
        m_run[nq] = -FLT_MAX;
        m_thr[nq] = -INFINITY;
        l_run[nq] = 0.0f;
    }

    const int hw = a.h * a.w;
    // (p + 1/2) / w truncates to p / w exactly below 2^20 tokens of a frame: its error is under p 2^-22 / w, its
    // distance from a whole number at least 1 / (2 w)
    const float inv_w = 1.0f / (float)a.w;
    auto grid_row = [&](int p) -> int { return kF32 && hw > (1 << 20) ? p / a.w : (int)(((float)p + 0.5f) * inv_w); };
    Corr corr[NQ];
    int corr_f = -1;
    // What a new frame needs waits in LDS: loaded when the frame changes, it made the tiles in flight be waited for, too (30
    // queries on 7020 8-bit keys, 3 of their 18 frames retrieved, in one part: 97 us, from LDS 92); and the arguments of
    // frames past those that are kept, in scalar registers, made the compiler spill some.
    __shared__ PagedBias lds_b;
    __shared__ float2 lds_corr[kBias ? kCorrFrames : 1][kRows];  // NaN: rejected
    __shared__ int lds_slot[kBias ? kSlotFrames : 1];
    if constexpr (kBias) {
        const int* slots = a.slot + (int64_t)s * a.max_frames;
        if (threadIdx.x == 0) lds_b = PagedBias{slots, a.corr_uv, a.corr_idx, a.max_frames, a.S, sq.n_tokens, -a.gamma};
        for (int f = threadIdx.x; f < min(a.max_frames, kSlotFrames); f += 64 * kW) lds_slot[f] = slots[f];
        for (int e = threadIdx.x; e < min(a.S, kCorrFrames) * kRows; e += 64 * kW) {
            const int r = it.in * kRows + e % kRows;
            float2 u = make_float2(NAN, NAN);
            if (r < n_rows) {
                const int64_t o = (int64_t)(e / kRows) * sq.n_tokens + tok.x + r / G;
                if (a.corr_idx[o] >= 0) u = reinterpret_cast<const float2*>(a.corr_uv)[o];
            }
            lds_corr[e / kRows][e % kRows] = u;
        }
        __syncthreads();
    }
    auto frame_corr = [&](int f) {
        corr_f = f;
        const PagedBias c = lds_b;
        const int slot = f >= c.max_frames ? -1 : (f < kSlotFrames ? lds_slot[f] : c.slot[f]);
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            corr[nq] = Corr{0.0f, 0.0f, 0.0f};
            if (slot < 0 || slot >= c.S) continue;
            float2 u = make_float2(NAN, NAN);
            if (slot < kCorrFrames) {
                u = lds_corr[slot][16 * nq + m];
            } else if (token[nq] >= 0) {
                const int64_t o = (int64_t)slot * c.n_tokens + token[nq];
                if (c.corr_idx[o] >= 0) u = reinterpret_cast<const float2*>(c.corr_uv)[o];
            }
            if (!__builtin_isnan(u.x)) corr[nq] = Corr{c.ng, u.x, u.y};
        }
    };

    // this wave's next tile whose page is there: at `cursor` or behind it; `entry` is the cursor's
    int cursor = t_begin + wave, entry = cursor < t_end ? entry_of(cursor) : 0;
    auto take = [&](Tile& b) {
        while (cursor < t_end && (unsigned)entry >= (unsigned)sq.n_pages) {
            cursor += kW;
            if (cursor < t_end) entry = entry_of(cursor);
        }
        b.t = cursor;
        b.page = entry;
        cursor += kW;
        if (cursor < t_end) entry = entry_of(cursor);
    };

    // works on the tile in b and fills b with the next one to take: each of its loads leaves as soon as its registers are free
    auto work = [&](Tile& b) __attribute__((always_inline)) {
        const int t = b.t, page = b.page, k0 = t * kTK;
        const bool masked = k0 + kTK > seen_min;  // some query does not see all of the tile's keys
        if constexpr (!kAhead) load_k(b, t, page);
        take(b);
        const bool more = b.t < t_end;
        const int t_load = more ? b.t : t, page_load = more ? b.page : page;  // without another it is loaded again and not used
        auto value_word = [&](int j, int u, int w) -> uint32_t {
            if constexpr (Sh::kVWords == 1) return b.vr[j][0];
            else return b.vr[j][u][w];
        };

        // S^T = K Q^T, the bias as the accumulators' start
        floatx4 S[NQ][2];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
            for (int i = 0; i < 2; ++i) S[nq][i] = floatx4{0, 0, 0, 0};
        if constexpr (kBias) {
            const int span = min(kTK, seen - k0);
            int f = k0 / hw, first = k0 - f * hw;  // frame, and the tile's first key within it
            for (;;) {
                if (f != corr_f) frame_corr(f);
                bool any = false;
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq) any = any || corr[nq].ng != 0.0f;
                if (__any(any)) {
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int p = first + 16 * half + 4 * grp + i;
                            const bool in = p >= 0 && p < hw;
                            const int ky = grid_row(p);
                            const float x = (float)(p - ky * a.w) + 0.5f, y = (float)ky + 0.5f;
#pragma unroll
                            for (int nq = 0; nq < NQ; ++nq) {
                                const float dx = x - corr[nq].ux, dy = y - corr[nq].uy;
                                S[nq][half][i] = in ? corr[nq].ng * (dx * dx + dy * dy) : S[nq][half][i];
                            }
                            __builtin_amdgcn_sched_barrier(0);  // one mask at a time
                        }
                }
                if (first + span <= hw) break;  // the frame holds the tile's last key
                ++f;
                first -= hw;
            }
        }
        if constexpr (kF32) {
#pragma unroll
            for (int u = 0; u < D / 16; ++u) {
                floatx4 qv[NQ];
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq) qv[nq] = lds_q[nq * (D / 16) + u][lane];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                        for (int half = 0; half < 2; ++half)
                            S[nq][half] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(floatx4, b.kr[half][u])[i], qv[nq][i], S[nq][half], 0, 0, 0);
            }
        } else {
            const float k_scale = T == kPagedFp8 ? scale_value(b.k_byte) : 1.0f;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int st = 0; st < kSteps; ++st) {
                    u32x4 w;
                    if constexpr (T == kPagedFp8) {
                        const uint32_t x = b.kr[half][st >> 1][2 * (st & 1)], y = b.kr[half][st >> 1][2 * (st & 1) + 1];
                        w = u32x4{widen2<false>(x, k_scale), widen2<true>(x, k_scale), widen2<false>(y, k_scale), widen2<true>(y, k_scale)};
                    } else {
                        w = b.kr[half][st];
                    }
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq)
                        S[nq][half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), as_bf16x8(qf[nq][st]), S[nq][half], 0, 0, 0);
                }
        }
        if constexpr (kAhead) load_k(b, t_load, page_load);
        else load_v(b, t, page);

        // softmax: the lane's eight logits of each of its columns
        u32x4 pf[NQ], pl[1];
#pragma unroll
        for (int nq = 0; nq < NQ; ++nq) {
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (masked && k0 + key_of(j) >= vis[nq]) S[nq][j >> 2][j & 3] = -INFINITY;
                mx = fmaxf(mx, S[nq][j >> 2][j & 3]);
            }
            if (__any(mx > m_thr[nq])) {
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float m_new = fmaxf(m_run[nq], mx * c_log2);
                const float alpha = __builtin_amdgcn_exp2f(m_run[nq] - m_new);
                l_run[nq] *= alpha;
#pragma unroll
                for (int db = 0; db < kDb; ++db) O[nq][db] *= alpha;
                m_run[nq] = m_new;
                m_thr[nq] = (m_new + kRescaleSlack) / c_log2;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float p = __builtin_amdgcn_exp2f(fmaf(S[nq][j >> 2][j & 3], c_log2, -m_run[nq]));
                S[nq][j >> 2][j & 3] = p;
                l_run[nq] += p;
            }
            if constexpr (!kF32)
                pf[nq] = u32x4{pack_bf16(S[nq][0][0], S[nq][0][1]), pack_bf16(S[nq][0][2], S[nq][0][3]),
                               pack_bf16(S[nq][1][0], S[nq][1][1]), pack_bf16(S[nq][1][2], S[nq][1][3])};
            if constexpr (kFine) {
#pragma unroll
                for (int jp = 0; jp < 4; ++jp)
                    pl[0][jp] = pack_bf16(S[nq][jp >> 1][2 * (jp & 1)] - __uint_as_float(pf[nq][jp] << 16),
                                           S[nq][jp >> 1][2 * (jp & 1) + 1] - __uint_as_float(pf[nq][jp] & 0xffff0000u));
            }
        }

        float v_scale = T == kPagedFp8 ? scale_value(b.v_byte) : 1.0f;
        // values behind the stream's last key may be anything: none of them
        if (k0 + kTK > held) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int u = 0; u < kVHalves; ++u)
                    if (k0 + key_of(j) >= held) b.vr[j][u] = VVec{};
        }
        // A query's weight of a key that it does not see is 0, and 0 times a value that is not finite would be NaN. Where
        // a masked tile holds such values, they are taken out of the operands, and the queries that see their
        // keys get them one by one. So they do where a probability is two numbers, whose second one may be 0 or have
        // the other sign (8 bits are infinite under scales from 2^120 on alone).
        if (masked || (kFine && (T == kPagedBf16 || v_scale >= 0x1p120f))) {
            const uint32_t odd = T == kPagedFp8 ? odd_codes(v_scale) : 0u;
            uint32_t bad = 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int u = 0; u < kVHalves; ++u)
#pragma unroll
                    for (int w = 0; w < Sh::kVWords / kVHalves; ++w) bad |= not_finite<T>(value_word(j, u, w), odd);
            if (__builtin_expect(__any(bad != 0), 0)) {
                const uint8_t* base = tile_at(a.cache_v, a.layout.v, t, page);
#pragma unroll 1
                for (int key = 0; key < min(kTK, held - k0); ++key) {
                    const int j = 4 * (key >> 4) + (key & 3), from = 16 * ((key >> 2) & 3) + m;
                    float p[NQ];
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq) {
                        p[nq] = 0.0f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) p[nq] = i == j ? S[nq][i >> 2][i & 3] : p[nq];
                        p[nq] = __shfl(p[nq], from);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int db = 0; db < kDb; ++db) {
                            const float x = stored<T>(base + key * step_of(a.layout.v), dim(i, db)) * v_scale;
#pragma unroll
                            for (int nq = 0; nq < NQ; ++nq)
                                if (!(fabsf(x) < INFINITY) && k0 + key < vis[nq]) O[nq][db][i] += p[nq] * x;
                            __builtin_amdgcn_sched_barrier(0);  // one mask at a time
                        }
                }
                if (v_scale != v_scale) v_scale = 1.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int u = 0; u < kVHalves; ++u) {
                        if constexpr (Sh::kVWords == 1) {
                            b.vr[j][0] &= ~spread<T>(not_finite<T>(b.vr[j][0], odd));
                        } else {
#pragma unroll
                            for (int w = 0; w < Sh::kVWords / kVHalves; ++w) b.vr[j][u][w] &= ~spread<T>(not_finite<T>(b.vr[j][u][w], odd));
                        }
                    }
            }
        }
        // O^T += V^T P^T
        if constexpr (kF32) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int nq = 0; nq < NQ; ++nq)
#pragma unroll
                    for (int db = 0; db < kDb; ++db)
                        O[nq][db] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(value_word(j, db / 4, db % 4)), S[nq][j >> 2][j & 3], O[nq][db], 0, 0, 0);
        } else {
            constexpr int kPer = 4 / Sh::kES;  // blocks of head dims that a word of the lane's value bytes holds
#pragma unroll
            for (int w = 0; w < Sh::kVWords; ++w) {
                u32x4 vf[kPer];  // their operands, keys in pairs
#pragma unroll
                for (int jp = 0; jp < 4; ++jp) {
                    const uint32_t x = value_word(2 * jp, 0, w), y = value_word(2 * jp + 1, 0, w);
                    if constexpr (T == kPagedFp8) {
                        // bytes of the two keys side by side: (x0 y0 x1 y1), (x2 y2 x3 y3)
                        const uint32_t lo = __builtin_amdgcn_perm(y, x, 0x05010400), hi = __builtin_amdgcn_perm(y, x, 0x07030602);
                        vf[0][jp] = widen2<false>(lo, v_scale);
                        vf[1][jp] = widen2<true>(lo, v_scale);
                        vf[2][jp] = widen2<false>(hi, v_scale);
                        vf[3][jp] = widen2<true>(hi, v_scale);
                    } else {
                        vf[0][jp] = __builtin_amdgcn_perm(y, x, 0x05040100);
                        vf[1][jp] = __builtin_amdgcn_perm(y, x, 0x07060302);
                    }
                }
#pragma unroll
                for (int i = 0; i < kPer; ++i)
#pragma unroll
                    for (int nq = 0; nq < NQ; ++nq)
                        O[nq][kPer * w + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[i]), as_bf16x8(pf[nq]), O[nq][kPer * w + i], 0, 0, 0);
                if constexpr (kFine) {
#pragma unroll
                    for (int i = 0; i < kPer; ++i)
                        O[0][kPer * w + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[i]), as_bf16x8(pl[0]), O[0][kPer * w + i], 0, 0, 0);
                }
            }
        }
        if constexpr (kAhead) load_v(b, t_load, page_load);
    };

    Tile now;
    take(now);
    if (kAhead && now.t < t_end) {
        load_k(now, now.t, now.page);
        load_v(now, now.t, now.page);
    }
    // 8 bits and few rows: two tiles in flight (one: 37440 keys of 12 heads 36.1 us, two: 29.5)
    if constexpr (T == kPagedFp8 && NQ == 1) {
        if (now.t < t_end) {
            Tile then;
            take(then);
            const bool more = then.t < t_end;
            load_k(then, more ? then.t : now.t, more ? then.page : now.page);
            load_v(then, more ? then.t : now.t, more ? then.page : now.page);
            for (;;) {
                work(now);
                if (then.t >= t_end) break;
                work(then);
                if (now.t >= t_end) break;
            }
        }
    } else {
        while (now.t < t_end) work(now);
    }

    // the waves' sums meet in LDS: thread (l, i) adds up what lane l holds in register i of every block, which are
    // consecutive head dims of column l % 16
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
        l_run[nq] += __shfl_xor(l_run[nq], 16);
        l_run[nq] += __shfl_xor(l_run[nq], 32);
        if (grp == 0) {
            lds_m[wave][16 * nq + m] = m_run[nq];
            lds_l[wave][16 * nq + m] = l_run[nq];
            if (wave == 0) {
                lds_token[16 * nq + m] = token[nq];
                lds_head[16 * nq + m] = head[nq];
            }
        }
    }
#pragma unroll
    for (int nq = 0; nq < NQ; ++nq) {
        if (nq > 0) __syncthreads();  // the block before has been read
#pragma unroll
        for (int db = 0; db < kDb; ++db) *reinterpret_cast<floatx4*>(&lds_o[wave][(db * 64 + lane) * 4]) = O[nq][db];
        __syncthreads();
        if (threadIdx.x >= 256) continue;
        const int l = threadIdx.x >> 2, i = threadIdx.x & 3, col = 16 * nq + (l & 15);
        const int to = lds_token[col];
        float M = -FLT_MAX, L = 0.0f;
#pragma unroll
        for (int w = 0; w < kW; ++w) M = fmaxf(M, lds_m[w][col]);
        float x[kDb];
#pragma unroll
        for (int db = 0; db < kDb; ++db) x[db] = 0.0f;
#pragma unroll
        for (int w = 0; w < kW; ++w) {
            const float c = __builtin_amdgcn_exp2f(lds_m[w][col] - M);
            L = fmaf(c, lds_l[w][col], L);
#pragma unroll
            for (int db = 0; db < kDb; ++db) x[db] = fmaf(c, lds_o[w][(db * 64 + l) * 4 + i], x[db]);
        }
        // its head dims: blocks 4 b .. 4 b + 3 from first[b] on
        auto first = [&](int b) -> int { return kVHalves == 2 ? 64 * b + 4 * (4 * (l >> 4) + i) : kDb * (4 * (l >> 4) + i) + 4 * b; };
        if (a.parts > 1) {
            float* base = a.partial + ((size_t)((size_t)tile * a.Hk + hk) * a.parts + part) * paged_part_floats(kRows, D);
            if (l < 16 && i == 0) {
                base[kRows * D + col] = t_begin < t_end ? M : -INFINITY;
                base[kRows * D + kRows + col] = L;
            }
            if (t_begin < t_end && to >= 0) {
#pragma unroll
                for (int b = 0; b < kDb / 4; ++b)
                    *reinterpret_cast<floatx4*>(base + col * D + first(b)) = floatx4{x[4 * b], x[4 * b + 1], x[4 * b + 2], x[4 * b + 3]};
            }
        } else if (to >= 0) {
            // a query that sees no key: nothing, and an LSE of -inf
            const float inv = L == 0.0f ? 0.0f : 1.0f / L;
            const int head = lds_head[col];
            const size_t row = ((size_t)to * a.Hq + head) * D;
#pragma unroll
            for (int b = 0; b < kDb / 4; ++b) {
                const floatx4 v = floatx4{x[4 * b], x[4 * b + 1], x[4 * b + 2], x[4 * b + 3]} * inv;
                if constexpr (kF32) *reinterpret_cast<floatx4*>(static_cast<float*>(a.o) + row + first(b)) = v;
                else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + row + first(b)) = u32x2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
            }
            if (a.lse && l < 16 && i == 0) a.lse[(size_t)head * sq.n_tokens + to] = (M + log2f(L)) * kLn2;
        }
    }
}

// O = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p over the key parts of a tile's row: a part without keys has m = -inf
// and nothing else that counts. A workgroup takes kRowsPer rows, 256 / kRowsPer threads each: D / 4 of them hold a part's
// head dims, and as many parts are read at once as there are such groups; their maxima and sums meet in LDS. Bound by
// latency: four parts of a group are loaded at a time, maxima with the rest (12 rows of 12 parts 3.4 us, of 21 4.6; the maxima
// first and each part when its own is there took a quarter longer).
template <int D, bool kF32, int kRowsPer>
__global__ __launch_bounds__(256) void paged_merge_kernel(PagedAttentionArgs a, unsigned blocks) {
    constexpr int kLanes = D / 4, kThreads = 256 / kRowsPer, kGroups = kThreads / kLanes;
    __shared__ floatx4 lds_x[kGroups > 1 ? 256 : 1];
    __shared__ float lds_l[kGroups > 1 ? 256 / kLanes : 1], lds_m[kGroups > 1 ? 256 / kLanes : 1];
    const unsigned block = row_block();
    if (block >= blocks) return;
    const unsigned per = (unsigned)(a.rows / kRowsPer);
    const unsigned item = block / per;  // (tile, key head)
    const int r = (int)(block - item * per) * kRowsPer + (int)threadIdx.x / kThreads;
    const int g = (int)threadIdx.x % kThreads / kLanes, d = 4 * ((int)threadIdx.x % kLanes);
    const int tile = (int)(item / (unsigned)a.Hk), hk = (int)(item - (unsigned)tile * (unsigned)a.Hk);
    const PagedSeqs& sq = a.seqs;
    const StreamItem it = row_tile(a, a.rows, tile);
    if (it.s < 0) return;
    const int2 tok = tokens_of(sq, it.s);
    const int row = it.in * a.rows + r;
    const bool ok = row < tok.y * a.G;
    if (kRowsPer == 1 && !ok) return;  // uniform
    const int token = tok.x + row / a.G, head = hk * a.G + row % a.G;
    const size_t step = paged_part_floats(a.rows, D);
    const float* base = a.partial + (size_t)item * a.parts * step + r * D + d;
    const float* stat = a.partial + (size_t)item * a.parts * step + a.rows * D + r;
    float M = -INFINITY, L = 0.0f;
    floatx4 x = floatx4{0, 0, 0, 0};
    auto add = [&](float to, float m, float l, floatx4 v) {  // of a sum's maximum m; to >= m
        if (m == -INFINITY) return;
        const float c = __builtin_amdgcn_exp2f(m - to);
        L = fmaf(c, l, L);
        x += c * v;
    };
    if (ok) {
        constexpr int kBatch = 4;
        for (int p = g; p < a.parts; p += kBatch * kGroups) {
            float m[kBatch], l[kBatch], top = M;
            floatx4 v[kBatch];
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                const int at = min(p + i * kGroups, a.parts - 1);
                m[i] = stat[at * step];
                l[i] = stat[at * step + a.rows];
                v[i] = *reinterpret_cast<const floatx4*>(base + at * step);
            }
#pragma unroll
            for (int i = 0; i < kBatch; ++i) {
                if (p + i * kGroups >= a.parts) m[i] = -INFINITY;
                top = fmaxf(top, m[i]);
            }
            const float l_old = L;
            const floatx4 x_old = x;
            L = 0.0f;
            x = floatx4{0, 0, 0, 0};
            add(top, M, l_old, x_old);
#pragma unroll
            for (int i = 0; i < kBatch; ++i) add(top, m[i], l[i], v[i]);
            M = top;
        }
    }
    if constexpr (kGroups > 1) {
        lds_x[threadIdx.x] = x;
        if (d == 0) {
            lds_l[threadIdx.x / kLanes] = L;
            lds_m[threadIdx.x / kLanes] = M;
        }
        __syncthreads();
        if (g != 0) return;
        const int t0 = (int)threadIdx.x, g0 = t0 / kLanes;
#pragma unroll
        for (int i = 0; i < kGroups; ++i) M = fmaxf(M, lds_m[g0 + i]);
        L = 0.0f;
        x = floatx4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < kGroups; ++i) add(M, lds_m[g0 + i], lds_l[g0 + i], lds_x[t0 + i * kLanes]);
    }
    if (!ok) return;
    x *= L == 0.0f ? 0.0f : 1.0f / L;
    const size_t out = ((size_t)token * a.Hq + head) * D + d;
    if constexpr (kF32) *reinterpret_cast<floatx4*>(static_cast<float*>(a.o) + out) = x;
    else *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.o) + out) = u32x2{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
    if (a.lse && d == 0) a.lse[(size_t)head * sq.n_tokens + token] = L == 0.0f ? -INFINITY : (M + log2f(L)) * kLn2;
}

}  // namespace

size_t paged_plan(PagedAttentionArgs& a, int32_t key_parts, int32_t max_keys, int32_t cus) {
    const PagedSeqs& q = a.seqs;
    const int64_t streams = q.B < q.n_tokens ? q.B : q.n_tokens;
    const int64_t rows = streams ? (int64_t)q.n_tokens * a.G / streams : 0;  // of a stream and key head, on average
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(max_keys, (int64_t)q.max_pages << q.page_log2));
    const int64_t key_tiles = (most + kTK - 1) / kTK;
    auto tiles_of = [&](int64_t r) { return q.cu ? (int64_t)q.n_tokens * a.G / r + streams : q.B * (((int64_t)q.per * a.G + r - 1) / r); };
    // Up to 32 rows, and where a compute unit has no more than 32 tiles of 32 rows and keys to do, a wave for each range
    // of keys (12 heads of 128: 300 queries on 300 keys 10 us, 64 on 2000 17); else the tile kernel (15 and 19 us; but
    // 64 on 20000 37, for 50, and 1000 on 1000 31, for 42). That one has no fp32 form; at D = 128 its tiles are of 256
    // rows where a stream has more than 128 (200 queries on 20000 keys 58 us, for 61; 4680 on 28080 878, for 1264).
    if (rows <= 16) a.rows = 16;
    else if (rows <= 32 || a.dtype == kPagedF32 || tiles_of(32) * a.Hk * key_tiles <= 32 * (int64_t)cus) a.rows = 32;
    else a.rows = rows <= 128 || a.D == 64 ? 128 : 256;
    const int64_t tiles = tiles_of(a.rows);
    a.tiles = (int32_t)std::min<int64_t>(tiles, INT32_MAX);
    const int64_t units = std::max<int64_t>(1, tiles * a.Hk);
    // workgroups of many waves where there are fewer units than compute units
    a.many = a.rows == 16 && units < cus;
    int64_t parts = key_parts;
    if (parts == 0 && a.many) {
        // One workgroup per compute unit, four key tiles a part (a token, 12 heads of 8 bits: 1560 keys whole 14.5 us, in 12
        // parts 9.7; 12000 71.3 and, in 21, 13.5), but a range as short as a launch takes whole (300 keys 7.6 us, in two 8.9).
        parts = key_tiles <= (a.dtype == kPagedF32 ? 8 : 16) ? 1 : std::min<int64_t>(cus / units, key_tiles / 4);
    } else if (parts == 0) {
        // The number of parts with the least estimated time: the busiest compute unit's workgroups, one after the other (two
        // at a time for the tile kernel at D = 64), a time per 32-key step that was measured at each size of tile, 4 us for
        // a workgroup's start and end, and a merge (a launch, and the parts' results written and read). 12 heads of 8
        // bits on 20000 keys: 100 queries 401 us whole, 43 in 16 parts; 400 queries 551 whole, 89 in 9; 4680 queries on 28080
        // keys 878 whole, 911 in two. fp32: 200 queries on 4000 keys 141 us whole, 63 in 3; 800 284 and, in 4, 216;
        // 1170 on 7020 484 whole, 513 in two. 264 single rows on 30000 keys: 503 us whole, 375 in 4.
        const int64_t places = a.rows == 128 && a.D == 64 ? 2 * (int64_t)cus : cus;
        const double step = a.rows == 256 ? 0.9
                            : a.rows == 128 ? (a.D == 128 ? 0.65 : 0.72)
                            : a.rows == 32  ? (a.dtype == kPagedF32 ? 1.1 : 0.32)
                                            : (a.dtype == kPagedF32 ? 0.6 : 0.27);
        const int64_t most_parts = std::min<int64_t>(kPagedMaxParts, a.rows >= 128 ? key_tiles : key_tiles / 16);
        double best = INFINITY;
        for (int64_t n = 1; n == 1 || (n <= most_parts && units * n <= 4 * places); ++n) {
            const double rounds = (double)((units * n + places - 1) / places);
            double us = rounds * ((double)((key_tiles + n - 1) / n) * step + 4.0);
            if (n > 1) us += 3.0 + 0.0002 * (double)(units * n * a.rows);
            if (us < 0.985 * best) {
                best = us;
                parts = n;
            }
        }
    }
    a.parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(parts, kPagedMaxParts), key_tiles));
    return a.parts > 1 ? (size_t)tiles * a.Hk * a.parts * paged_part_floats(a.rows, a.D) * sizeof(float) : 0;
}

double paged_units(const PagedAttentionArgs& a) { return (double)a.tiles * a.Hk * a.parts; }

hipError_t launch_paged_attention(const PagedAttentionArgs& a, hipStream_t stream) {
    if (a.seqs.n_tokens == 0 || a.tiles == 0) return hipSuccess;
    const float c = a.softmax_scale * kLog2e;
    const dim3 grid = grid_rows(xcd_grid((unsigned)a.tiles * (unsigned)a.Hk * (unsigned)a.parts));
    auto wave = [&](auto d_tag, auto t_tag) {
        constexpr int D = decltype(d_tag)::value, T = decltype(t_tag)::value;
        auto launch = [&](auto nq_tag, auto bias_tag, auto w_tag) {
            constexpr int NQ = decltype(nq_tag)::value, W = decltype(w_tag)::value;
            constexpr bool B = decltype(bias_tag)::value;
            if (a.strided) hipLaunchKernelGGL((paged_wave_kernel<D, T, NQ, B, W, true>), grid, dim3(64 * W), 0, stream, a, c);
            else hipLaunchKernelGGL((paged_wave_kernel<D, T, NQ, B, W, false>), grid, dim3(64 * W), 0, stream, a, c);
        };
        auto rows = [&](auto bias_tag) {
            using W4 = std::integral_constant<int, 4>;
            if (a.rows == 16 && a.many) launch(std::integral_constant<int, 1>{}, bias_tag, std::integral_constant<int, kManyWaves>{});
            else if (a.rows == 16) launch(std::integral_constant<int, 1>{}, bias_tag, W4{});
            else launch(std::integral_constant<int, 2>{}, bias_tag, W4{});
        };
        hipError_t e;
        if (a.rows >= 128) {
            e = launch_paged_tiles(a, stream);
        } else {
            if (a.S > 0) rows(std::true_type{});
            else rows(std::false_type{});
            e = hipGetLastError();
        }
        if (e != hipSuccess || a.parts == 1) return e;
        // a workgroup per row where there are many parts to read
        auto merge = [&](auto per_tag) {
            constexpr int kRowsPer = decltype(per_tag)::value;
            const unsigned blocks = (unsigned)a.tiles * (unsigned)a.Hk * (unsigned)(a.rows / kRowsPer);
            hipLaunchKernelGGL((paged_merge_kernel<D, T == kPagedF32, kRowsPer>), grid_rows(blocks), dim3(256), 0, stream, a, blocks);
            return hipGetLastError();
        };
        return a.parts > 4 ? merge(std::integral_constant<int, 1>{}) : merge(std::integral_constant<int, 1024 / D>{});
    };
    auto by_type = [&](auto d_tag) {
        if (a.dtype == kPagedFp8) return wave(d_tag, std::integral_constant<int, kPagedFp8>{});
        if (a.dtype == kPagedBf16) return wave(d_tag, std::integral_constant<int, kPagedBf16>{});
        return wave(d_tag, std::integral_constant<int, kPagedF32>{});
    };
    return a.D == 128 ? by_type(std::integral_constant<int, 128>{}) : by_type(std::integral_constant<int, 64>{});
}

}  // namespace revisit
