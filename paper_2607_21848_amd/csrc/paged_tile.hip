// The tile kernel of paged_chunk_attention: 128 (query, head of the group) rows per workgroup, for chunks and prompts.
//
// Four waves of 32 rows each, 32-key tiles, two workgroups per compute unit. As in biased_chunk_attention's bf16
// kernel a wave computes the transposed logits S^T = K Q^T with 32x32x16 MFMAs, keys in the rows, so that a lane
// has 16 logits of one query and softmax needs one exchange with the other half of the wave, and with the K rows
// read in an order that makes a lane's probabilities the B operand of O^T = V^T P^T as they are.
//
// Keys and values come from the pages, where a head's share of a tile is one run of bytes: each thread loads its 16-byte
// pieces into registers, a step ahead, and writes them to LDS as bf16, 8-bit ones widened with their scale on the
// way (exactly: it is a power of two), so that the matrix cores see the same numbers whatever the pages hold.
// 256-byte (128-byte) rows with their 16-byte chunks at c ^ swz(row), which keeps the reads of both operands, V's
// through the transposing LDS load, off each other's banks.
//
// LDS holds a ring of two slots; slot t mod 2 carries K_t and V_{t-1}. Step j, after its one barrier, reads K_{j+1} and
// V_j from slot j + 1 mod 2 and refills slot j mod 2 with K_{j+2} and V_{j+1}: the logits of the next tile are computed
// beside the softmax of this one.
//
// The bias goes through the matrix cores in separable form, one more MFMA for a tile of a retrieved frame: as in
// biased_chunk_attention (attention.hip), where its factors are described.

#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "internal.h"
#include "paged.h"

namespace revisit {
namespace {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) shortx4 lds_shortx4;

constexpr int kTK = 32;
constexpr float kRescaleSlack = 8.0f;
constexpr int kGridSide = 256;  // token-grid rows / columns of the bias tables
constexpr int kCorrLds = 16;    // retrieved frames whose correspondences are staged in LDS

__device__ __forceinline__ bf16x8 as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

// Row of the key that A-operand row m takes: bits 2 and 3 exchanged.
__device__ __forceinline__ int perm_row(int m) { return (m & ~12) | ((m & 8) >> 1) | ((m & 4) << 1); }

// key of a lane's logit i within its tile
__device__ __forceinline__ int key_of(int hh, int i) { return 16 * (i >> 3) + 8 * hh + (i & 7); }

// chunk swizzle of LDS row r
template <int D>
__device__ __forceinline__ int swz(int r) { return D == 128 ? ((r & 3) << 2) | (((r >> 2) & 3) ^ (r & 1)) : (r >> 1) & 7; }

// max / sum of x over the lane and its partner in the other wave half
__device__ __forceinline__ float half_swap_max(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float half_swap_sum(float x) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
// max(a, b, c) in one instruction (a NaN among them is passed over)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm volatile("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

__device__ __forceinline__ uint32_t bf16_bits(float x) { return (uint32_t)__builtin_bit_cast(unsigned short, (__bf16)x); }
__device__ __forceinline__ uint32_t pack2(uint32_t lo, uint32_t hi) { return lo | (hi << 16); }
// x = hi + mid + lo exactly
__device__ __forceinline__ void split3(float x, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
    hi = bf16_bits(x);
    const float r1 = x - __uint_as_float(hi << 16);
    mid = bf16_bits(r1);
    lo = bf16_bits(r1 - __uint_as_float(mid << 16));
}

// Barrier without a fence: what the waves exchange through LDS is waited for by count, and loads in flight stay there.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

struct Geom {
    float gamma, cx, cy;  // lambda / (2 sigma^2 softmax_scale), the grid's centre
    int hw, w, h;
};

template <int D, int T, bool kBias, int kW>
__global__ __launch_bounds__(64 * kW, 2) void paged_tile_kernel(PagedAttentionArgs a, Geom g, float c_log2) {
    constexpr int kRowB = D * 2, kTileB = kTK * kRowB;      // in LDS
    constexpr int kStored = T == kPagedFp8 ? D : 2 * D;     // bytes of a row in the pages
    constexpr int kHalf = kTK * kStored / 16;               // 16-byte pieces of a K or V tile
    constexpr int kRows = 32 * kW, kThreads = 64 * kW;
    constexpr int kPieces = (2 * kHalf + kThreads - 1) / kThreads;  // of a thread
    constexpr int kKk = D / 16, kDb = D / 32;
    __shared__ __attribute__((aligned(1024))) uint8_t ring[2][2 * kTileB];
    __shared__ u32x4 lds_tab[2][kBias ? kGridSide : 1];     // key operands by column and by row
    __shared__ float2 lds_corr[kBias ? kCorrLds : 1][kRows];  // centred correspondences, NaN: rejected
    __shared__ int lds_block[512];
    __shared__ float lds_scale[2][T == kPagedFp8 ? 512 : 1];
    __shared__ int lds_seen[kW], lds_least[kW];
    __shared__ int lds_odd[2];  // V tile of a slot from which values that are not finite were taken out, or -1

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int hh = lane >> 5, n = lane & 31;
    const PagedSeqs& sq = a.seqs;
    const int G = a.G;

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

    // the lane's row, its query and how many keys it sees
    const int r = it.in * kRows + wave * 32 + n;
    const bool row_ok = r < n_rows;
    const int token = row_ok ? tok.x + r / G : -1, head = hk * G + r % G;
    u32x4 qf[kKk];  // head dims 16 kk + 8 hh ..
    {
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + (int64_t)max(token, 0) * a.q_row + (int64_t)head * D + 8 * hh;
#pragma unroll
        for (int kk = 0; kk < kKk; ++kk) qf[kk] = u32x4{0, 0, 0, 0};
        if (row_ok) {
#pragma unroll
            for (int kk = 0; kk < kKk; ++kk) qf[kk] = *reinterpret_cast<const u32x4*>(qp + 16 * kk);
        }
    }
    const int held = held_of(sq, s);
    int vis = held, seen = held, seen_min = held, least = held;  // seen_min: of the wave's rows, least: of the workgroup's
    if (a.visible) {
        if (row_ok) vis = min(held, max(a.visible[token], 0));
        seen = row_ok ? vis : 0;
        seen_min = row_ok ? vis : held;
#pragma unroll
        for (int off = 1; off < 32; off *= 2) {
            seen = max(seen, __shfl_xor(seen, off));
            seen_min = min(seen_min, __shfl_xor(seen_min, off));
        }
        if (lane == 0) {
            lds_seen[wave] = seen;
            lds_least[wave] = seen_min;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kW; ++w) {
            seen = max(seen, lds_seen[w]);
            least = min(least, lds_least[w]);
        }
    }
    least = __builtin_amdgcn_readfirstlane(least);
    seen = __builtin_amdgcn_readfirstlane(seen);
    seen_min = __builtin_amdgcn_readfirstlane(seen_min);
    const int n_tiles = (seen + kTK - 1) / kTK;
    const int t0 = (int)((int64_t)part * n_tiles / a.parts);
    const int nt = (int)((int64_t)(part + 1) * n_tiles / a.parts) - t0;  // this part's tiles

    // ---- the pages --------------------------------------------------------
    const int in_page = (1 << sq.page_log2) - 1;
    // Where the part's tiles lie, 256 at a time in LDS, the next 256 beside them (a scalar load in every step would make
    // each wait for LDS a wait for it, a vector load one for the pieces in flight): the block of 32 rows of the
    // caches, or -1 without a page (page 0's rows stand in for them, which nobody sees), and the scales.
    auto fetch_info = [&](int j) __attribute__((always_inline)) {  // of tiles j + tid, past the last one the last one's
        const int x = j + tid, pos = (t0 + min(x, nt - 1)) * kTK;
        const int entry = sq.page_table[(int64_t)s * sq.max_pages + (pos >> sq.page_log2)];
        const bool there = (unsigned)entry < (unsigned)sq.n_pages;
        const int block = (((there ? entry : 0) * a.Hk + hk) << (sq.page_log2 - 5)) + ((pos & in_page) >> 5);
        if constexpr (T == kPagedFp8) {
            lds_scale[0][x & 511] = scale_value(a.scale_k[block]);
            lds_scale[1][x & 511] = scale_value(a.scale_v[block]);
        }
        lds_block[x & 511] = there ? block : -1;
    };
    auto block_of = [&](int j) __attribute__((always_inline)) -> int { return lds_block[j & 511]; };
    u32x4 piece[kPieces];
    // pieces of the K tile in block bk and the V tile in block bv; piece p of a thread is number kThreads p + tid of K's
    // and then V's
    auto load = [&](int bk, int bv) __attribute__((always_inline)) {
        const uint8_t* kb = static_cast<const uint8_t*>(a.cache_k) + (size_t)(unsigned)max(bk, 0) * (kTK * kStored);
        const uint8_t* vb = static_cast<const uint8_t*>(a.cache_v) + (size_t)(unsigned)max(bv, 0) * (kTK * kStored);
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int i = kThreads * p + tid;
            if constexpr (kHalf % kThreads == 0) {
                const uint32_t off = 16 * (uint32_t)tid;
                piece[p] = *reinterpret_cast<const u32x4*>((kThreads * p >= kHalf ? vb + 16 * (kThreads * p - kHalf) : kb + 16 * kThreads * p) + off);
            } else {
                if (2 * kHalf % kThreads == 0 || i < 2 * kHalf) piece[p] = *reinterpret_cast<const u32x4*>(i >= kHalf ? vb + 16 * (i - kHalf) : kb + 16 * i);
            }
        }
    };
    // A weight of 0 times a value that is not finite would be NaN. In a tile that some row does not see all of, such
    // values (and whatever lies behind the stream's end) are left out here; the rows that see them get them one by
    // one (`odd_values`).
    auto store = [&](int which, float k_scale, float v_scale, int jv, int bv) __attribute__((always_inline)) {
        uint8_t* slot = ring[which];
        if (__builtin_expect((t0 + jv + 1) * kTK > least || bv < 0, 0)) {
            const float f = T == kPagedFp8 ? v_scale : 1.0f;
            uint32_t odd = 0;
#pragma unroll
            for (int p = 0; p < kPieces; ++p) {
                const int i = kThreads * p + tid - kHalf;
                if (i < 0 || (2 * kHalf % kThreads != 0 && i >= kHalf)) continue;
                const bool none = bv < 0 || (t0 + jv) * kTK + i / (kStored / 16) >= held;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t bad = f != f ? ~0u : spread<T>(not_finite<T>(piece[p][w]));
                    if (none) piece[p][w] = 0;
                    else odd |= bad;
                    piece[p][w] &= ~bad;
                }
            }
            if (f != f) v_scale = 1.0f;
            if (odd) lds_odd[which] = jv;
        }
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int i = kThreads * p + tid;
            if (2 * kHalf % kThreads != 0 && i >= 2 * kHalf) continue;
            const bool is_v = i >= kHalf;
            const int at = is_v ? i - kHalf : i;
            const int row = at / (kStored / 16), c = at % (kStored / 16);
            uint8_t* to = slot + (is_v ? kTileB : 0) + row * kRowB;
            if constexpr (T == kPagedFp8) {
                const float f = is_v ? v_scale : k_scale;
                u32x4 lo, hi;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    lo[2 * w] = widen2<false>(piece[p][w], f);
                    lo[2 * w + 1] = widen2<true>(piece[p][w], f);
                    hi[2 * w] = widen2<false>(piece[p][2 + w], f);
                    hi[2 * w + 1] = widen2<true>(piece[p][2 + w], f);
                }
                *reinterpret_cast<u32x4*>(to + (((2 * c) ^ swz<D>(row)) << 4)) = lo;
                *reinterpret_cast<u32x4*>(to + (((2 * c + 1) ^ swz<D>(row)) << 4)) = hi;
            } else {
                *reinterpret_cast<u32x4*>(to + ((c ^ swz<D>(row)) << 4)) = piece[p];
            }
        }
    };

    // LDS byte offsets of the lane's operand reads
    const int krow = perm_row(n);
    int koff[kKk];
#pragma unroll
    for (int kk = 0; kk < kKk; ++kk) koff[kk] = krow * kRowB + (((2 * kk + hh) ^ swz<D>(krow)) << 4);
    // transposing reads of V: lane t of 16-lane group q reads row 8 hh + t / 4 (+ 4) at columns 32 db + 16 (q % 2) + 4 (t % 4) ..
    int voff[2][kDb];
    {
        const int t16 = lane & 15, grp = lane >> 4;
        const int row0 = 8 * hh + (t16 >> 2), cc = 2 * (grp & 1) + ((t16 >> 1) & 1), byte = 8 * (t16 & 1);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int db = 0; db < kDb; ++db) {
                const int row = row0 + 4 * half;
                voff[half][db] = row * kRowB + (((4 * db + cc) ^ swz<D>(row)) << 4) + byte;
            }
    }

    // ---- bias ---------------------------------------------------------------
    const uint32_t one = 0x3f80u;
    const float inv_w = 1.0f / (float)g.w;
    const const_i32* slots = reinterpret_cast<const const_i32*>((uintptr_t)(a.slot + (int64_t)s * a.max_frames));
    auto slot_of = [&](int f) __attribute__((always_inline)) -> int {
        const int v = f < a.max_frames ? slots[__builtin_amdgcn_readfirstlane(f)] : -1;
        return v >= 0 && v < a.S ? v : -1;
    };
    if constexpr (kBias) {
        for (int i = tid; i < g.w + g.h; i += kThreads) {
            const bool col = i < g.w;
            const int k = col ? i : i - g.w;
            const float ac = ((float)k + 0.5f) - (col ? g.cx : g.cy);
            const uint32_t a2 = bf16_bits(2.0f * ac);
            uint32_t ph, pm, pl;
            split3(-g.gamma * (ac * ac), ph, pm, pl);
            lds_tab[col ? 0 : 1][k] = u32x4{pack2(a2, a2), pack2(a2, ph), pack2(pm, pl), col ? pack2(one, one) : one};
        }
        constexpr int kPer = kCorrLds * kRows / kThreads;
        int ci[kPer];
        float2 cu[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = tid + kThreads * i, f = e / kRows, row = it.in * kRows + e % kRows;
            ci[i] = -1;
            cu[i] = make_float2(0.0f, 0.0f);
            if (f < a.S && row < n_rows) {
                const int64_t o = (int64_t)f * sq.n_tokens + tok.x + row / G;
                ci[i] = a.corr_idx[o];
                cu[i] = reinterpret_cast<const float2*>(a.corr_uv)[o];
            }
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = tid + kThreads * i;
            lds_corr[e / kRows][e % kRows] = ci[i] >= 0 ? make_float2(cu[i].x - g.cx, cu[i].y - g.cy) : make_float2(NAN, NAN);
        }
    }
    // query-side operand of retrieved frame f: zeros where the correspondence is rejected
    auto query_operand = [&](int f) __attribute__((always_inline)) -> bf16x8 {
        float ux = NAN, uy = NAN;
        if (f < kCorrLds) {
            const float2 u = lds_corr[f][wave * 32 + n];
            ux = u.x;
            uy = u.y;
        } else if (row_ok) {
            const int64_t o = (int64_t)f * sq.n_tokens + token;
            if (a.corr_idx[o] >= 0) {
                const float2 u = reinterpret_cast<const float2*>(a.corr_uv)[o];
                ux = u.x - g.cx;
                uy = u.y - g.cy;
            }
        }
        u32x4 v = u32x4{0, 0, 0, 0};
        if (!__builtin_isnan(ux)) {
            uint32_t xh, xm, xl, zh, zm, zl;
            split3(g.gamma * (hh ? uy : ux), xh, xm, xl);
            split3(-g.gamma * (ux * ux + uy * uy), zh, zm, zl);
            v = u32x4{pack2(xh, xm), pack2(xl, one), pack2(one, one), hh ? zl : pack2(zh, zm)};
        }
        return as_bf16x8(v);
    };
    auto key_operand = [&](int p) __attribute__((always_inline)) -> u32x4 {  // in-frame position p
        const int ky = (int)(((float)p + 0.5f) * inv_w);
        return lds_tab[hh][hh ? ky : p - ky * g.w];
    };
    bf16x8 qcur = as_bf16x8(u32x4{0, 0, 0, 0});  // operand of the frame at hand
    int cur_f = -1, cur_s = -1;
    int blk_f = 0, blk_t = 0;  // frame and in-frame position of the next QK tile's first key
    if constexpr (kBias) {
        blk_f = t0 * kTK / g.hw;
        blk_t = t0 * kTK - blk_f * g.hw;
    }
    // 1: the tile lies in one retrieved frame (kop: the lane's key operand), 0: in one that is none, -1: across frames
    auto classify = [&](u32x4& kop) __attribute__((always_inline)) -> int {
        if (__builtin_expect(blk_t + kTK > g.hw, 0)) return -1;
        if (__builtin_expect(cur_f != blk_f, 0)) {
            cur_f = blk_f;
            cur_s = slot_of(blk_f);
            qcur = cur_s >= 0 ? query_operand(cur_s) : as_bf16x8(u32x4{0, 0, 0, 0});
        }
        if (cur_s < 0) return 0;
        kop = key_operand(blk_t + krow);
        return 1;
    };
    auto bias_add = [&](floatx16 x, int cls, const u32x4& kop) __attribute__((always_inline)) -> floatx16 {
        if (cls > 0) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kop), qcur, x, 0, 0, 0);
        if (__builtin_expect(cls < 0, 0)) {
            const int lane_f = blk_f + (blk_t + krow) / g.hw, lane_p = (blk_t + krow) % g.hw;
            for (int f = blk_f, first = -blk_t; first < kTK; ++f, first += g.hw) {
                const int sl = slot_of(f);
                if (sl < 0) continue;
                const bf16x8 qv = query_operand(sl);
                u32x4 kv = u32x4{0, 0, 0, 0};
                if (lane_f == f) kv = key_operand(lane_p);
                x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kv), qv, x, 0, 0, 0);
            }
        }
        blk_t += kTK;
        while (blk_t >= g.hw) {
            blk_t -= g.hw;
            ++blk_f;
        }
        return x;
    };

    // ---- state ----------------------------------------------------------------
    floatx16 O[kDb];
#pragma unroll
    for (int db = 0; db < kDb; ++db) O[db] = floatx16{0};
    float m_run = -FLT_MAX, m_thr = -INFINITY, l0 = 0.0f, l1 = 0.0f;

    // logits of tile j that a row does not see
    auto mask = [&](floatx16& S, int j, int block) __attribute__((always_inline)) {
        const int k0 = (t0 + j) * kTK, lim = block < 0 ? 0 : vis;
#pragma unroll
        for (int i = 0; i < 16; ++i) S[i] = k0 + key_of(hh, i) >= lim ? -INFINITY : S[i];
    };
    auto row_max = [&](const floatx16& S) __attribute__((always_inline)) -> float {
        float x = max3(S[0], S[1], S[2]);
#pragma unroll
        for (int i = 3; i < 15; i += 2) x = max3(x, S[i], S[i + 1]);
        return fmaxf(x, S[15]);
    };

    // the values of V tile j that `store` left out, for the rows that see them (probabilities in S)
    auto odd_values = [&](const floatx16& S, int j, int block) __attribute__((always_inline)) {
        const int k0 = (t0 + j) * kTK;
        const uint8_t* base = static_cast<const uint8_t*>(a.cache_v) + (size_t)(unsigned)block * (kTK * kStored);
        const float f = T == kPagedFp8 ? scale_value(a.scale_v[block]) : 1.0f;
#pragma unroll 1
        for (int key = 0; key < min(kTK, held - k0); ++key) {
            const int want = 8 * (key >> 4) + (key & 7);  // register of the lane that has its probability
            float p = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) p = i == want ? S[i] : p;
            p = __shfl(p, 32 * ((key >> 3) & 1) + n);
#pragma unroll
            for (int db = 0; db < kDb; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = stored<T>(base + key * kStored, 32 * db + 8 * (i >> 2) + 4 * hh + (i & 3)) * f;
                    if (!(fabsf(x) < INFINITY) && k0 + key < vis) O[db][i] += p * x;
                    __builtin_amdgcn_sched_barrier(0);  // one mask at a time
                }
        }
    };

    floatx16 Sa, Sb;
    float mx = -INFINITY;
    int b0 = 0, b1 = 0, b2 = 0;  // blocks of tiles j, j + 1 and j + 2

    // One step: softmax and P V of tile j, whose logits are in S_cur, beside the logits of tile j + 1.
    auto step = [&](int j, floatx16& S_cur, floatx16& S_next, auto slot_tag) __attribute__((always_inline)) {
        constexpr int kRefill = decltype(slot_tag)::value;
        const uint8_t* next = ring[1 - kRefill];
        lds_barrier();
        const bool more = j + 1 < nt;  // past the last tile its logits are computed again and not used
        const uint8_t* vt = next + kTileB;
        u32x4 kf[kKk];
        auto kread = [&](int kk) { kf[kk] = *reinterpret_cast<const u32x4*>(next + koff[kk]); };
        kread(0);
        kread(1);
        kread(2);
        const int b3_lane = block_of(j + 3);
        const float k_scale = T == kPagedFp8 ? lds_scale[0][(j + 2) & 511] : 1.0f, v_scale = T == kPagedFp8 ? lds_scale[1][(j + 1) & 511] : 1.0f;
        u32x4 kop = u32x4{0, 0, 0, 0};
        int cls = 0;
        if constexpr (kBias) cls = classify(kop);
        // rescale where a row's maximum has grown by more than the slack
        if (__builtin_expect(__any(mx > m_thr), 0)) {
            const float m_new = fmaxf(m_run, half_swap_max(mx) * c_log2);
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
            l0 *= alpha;
            l1 *= alpha;
#pragma unroll
            for (int db = 0; db < kDb; ++db) O[db] *= alpha;
            m_run = m_new;
            m_thr = (m_new + kRescaleSlack) / c_log2;
        }
        S_next = floatx16{0};
        uint32_t w4[2][4];
        auto unit = [&](int t, int e) {  // probabilities 8 t + 2 e and the next
            const int i = 8 * t + 2 * e;
            const float p0 = __builtin_amdgcn_exp2f(fmaf(S_cur[i], c_log2, -m_run));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(S_cur[i + 1], c_log2, -m_run));
            S_cur[i] = p0;
            S_cur[i + 1] = p1;
            w4[t][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{p0, p1}, __bf16 __attribute__((ext_vector_type(2)))));
            l0 += p0;
            l1 += p1;
        };
        shortx4 vlo[2][kDb], vhi[2][kDb];
        auto vread = [&](int t, int db) {
            const uint8_t* vp = vt + 16 * t * kRowB;
            vlo[t][db] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(vp + voff[0][db]));
            vhi[t][db] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(vp + voff[1][db]));
        };
        auto voperand = [&](int t, int db) -> bf16x8 {
            const u32x2 lo = __builtin_bit_cast(u32x2, vlo[t][db]), hi = __builtin_bit_cast(u32x2, vhi[t][db]);
            return as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]});
        };
        __builtin_amdgcn_sched_barrier(0);
        // the QK MFMAs of tile j + 1, K read three ahead, and the first V reads
#pragma unroll
        for (int kk = 0; kk < kKk; ++kk) {
            if (kk + 3 < kKk) kread(kk + 3);
            S_next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf[kk]), as_bf16x8(qf[kk]), S_next, 0, 0, 0);
            if (kk >= kKk - kDb) vread(0, kk - (kKk - kDb));
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (kBias) {
            S_next = bias_add(S_next, cls, kop);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int u = 0; u < 6; ++u) unit(u >> 2, u & 3);
        __builtin_amdgcn_sched_barrier(0);
        // the pieces of K_{j+2} and V_{j+1} go to LDS, those of the tiles behind them leave
        store(kRefill, k_scale, v_scale, min(j + 1, nt - 1), b1);
        const int b3 = __builtin_amdgcn_readfirstlane(b3_lane);
        load(b3, b2);
        __builtin_amdgcn_sched_barrier(0);
        const bf16x8 pf0 = as_bf16x8(u32x4{w4[0][0], w4[0][1], w4[0][2], w4[0][3]});
#pragma unroll
        for (int db = 0; db < kDb; ++db) {
            O[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(voperand(0, db), pf0, O[db], 0, 0, 0);
            if (db < 2) unit(1, 2 + db);
            vread(1, db);
            __builtin_amdgcn_sched_barrier(0);
        }
        const bf16x8 pf1 = as_bf16x8(u32x4{w4[1][0], w4[1][1], w4[1][2], w4[1][3]});
#pragma unroll
        for (int db = 0; db < kDb; ++db) {
            O[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(voperand(1, db), pf1, O[db], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (__builtin_expect((t0 + j + 2) * kTK > seen_min || b1 < 0, 0)) mask(S_next, j + 1, b1);
        mx = row_max(S_next);
        if (__builtin_expect((t0 + j + 1) * kTK > least, 0)) {
            asm volatile("" ::: "memory");  // lds_odd is read for such tiles alone
            if (lds_odd[1 - kRefill] == j) odd_values(S_cur, j, b0);
        }
        if (__builtin_expect(((j + 4) & 255) == 128, 0)) {
            if (tid < 256) fetch_info(((j + 4) & ~255) + 256);
        }
        if (!more) mx = -INFINITY;
        b0 = b1;
        b1 = b2;
        b2 = b3;
    };

    if (nt > 0) {
        if (tid < 256) fetch_info(0);
        if (tid < 2) lds_odd[tid] = -1;
        __syncthreads();
        auto scale = [&](int which, int j) -> float { return T == kPagedFp8 ? lds_scale[which][j] : 1.0f; };
        b0 = __builtin_amdgcn_readfirstlane(block_of(0));
        b1 = __builtin_amdgcn_readfirstlane(block_of(1));
        b2 = __builtin_amdgcn_readfirstlane(block_of(2));
        load(b0, b0);
        store(0, scale(0, 0), scale(1, 0), 0, b0);
        load(b1, b0);
        store(1, scale(0, 1), scale(1, 0), 0, b0);
        load(b2, b1);
        __syncthreads();
        u32x4 kop = u32x4{0, 0, 0, 0};
        int cls = 0;
        if constexpr (kBias) cls = classify(kop);
        Sa = floatx16{0};
#pragma unroll
        for (int kk = 0; kk < kKk; ++kk)
            Sa = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(ring[0] + koff[kk]), as_bf16x8(qf[kk]), Sa, 0, 0, 0);
        if constexpr (kBias) Sa = bias_add(Sa, cls, kop);
        if ((t0 + 1) * kTK > seen_min || b0 < 0) mask(Sa, 0, b0);
        mx = row_max(Sa);
        for (int j = 0;;) {
            step(j, Sa, Sb, std::integral_constant<int, 0>{});
            if (++j >= nt) break;
            step(j, Sb, Sa, std::integral_constant<int, 1>{});
            if (++j >= nt) break;
        }
    }

    const float l = half_swap_sum(l0 + l1);
    if (a.parts == 1) {
        if (!row_ok) return;
        // a row that sees no key: nothing, and an LSE of -inf
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        uint16_t* o = static_cast<uint16_t*>(a.o) + ((size_t)token * a.Hq + head) * D;
#pragma unroll
        for (int db = 0; db < kDb; ++db)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w[2];
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    w[j] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{O[db][4 * i + 2 * j] * inv, O[db][4 * i + 2 * j + 1] * inv},
                                                                               __bf16 __attribute__((ext_vector_type(2)))));
                *reinterpret_cast<u32x2*>(o + 32 * db + 8 * i + 4 * hh) = u32x2{w[0], w[1]};
            }
        if (a.lse && hh == 0) a.lse[(size_t)head * sq.n_tokens + token] = (m_run + log2f(l)) * 0.6931471805599453f;
    } else {
        float* base = a.partial + ((size_t)((size_t)tile * a.Hk + hk) * a.parts + part) * paged_part_floats(kRows, D);
        const int row = wave * 32 + n;
        if (hh == 0) {
            base[kRows * D + row] = nt > 0 ? m_run : -INFINITY;
            base[kRows * D + kRows + row] = l;
        }
        if (nt > 0 && row_ok) {
#pragma unroll
            for (int db = 0; db < kDb; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<float4*>(base + row * D + 32 * db + 8 * i + 4 * hh) =
                        make_float4(O[db][4 * i], O[db][4 * i + 1], O[db][4 * i + 2], O[db][4 * i + 3]);
        }
    }
}

}  // namespace

hipError_t launch_paged_tiles(const PagedAttentionArgs& a, hipStream_t stream) {
    const float c = a.softmax_scale * 1.4426950408889634f;
    const Geom g{a.gamma, 0.5f * (float)a.w, 0.5f * (float)a.h, a.h * a.w, a.w, a.h};
    const dim3 grid = grid_rows(xcd_grid((unsigned)a.tiles * (unsigned)a.Hk * (unsigned)a.parts)), block(2 * a.rows);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, g, c); };
    auto bias = [&](auto d_tag, auto t_tag) {
        constexpr int D = decltype(d_tag)::value, T = decltype(t_tag)::value;
        if (a.rows == 256) {
            if (a.S > 0) launch(paged_tile_kernel<D, T, true, 8>);
            else launch(paged_tile_kernel<D, T, false, 8>);
        } else {
            if (a.S > 0) launch(paged_tile_kernel<D, T, true, 4>);
            else launch(paged_tile_kernel<D, T, false, 4>);
        }
    };
    using Fp8 = std::integral_constant<int, kPagedFp8>;
    using Bf16 = std::integral_constant<int, kPagedBf16>;
    if (a.D == 128) {
        if (a.dtype == kPagedFp8) bias(std::integral_constant<int, 128>{}, Fp8{});
        else bias(std::integral_constant<int, 128>{}, Bf16{});
    } else {
        if (a.dtype == kPagedFp8) bias(std::integral_constant<int, 64>{}, Fp8{});
        else bias(std::integral_constant<int, 64>{}, Bf16{});
    }
    return hipGetLastError();
}

}  // namespace revisit
