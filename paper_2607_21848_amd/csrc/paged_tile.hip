// The tile kernel of paged_chunk_attention: 128 or 256 (query, head of the group) rows per workgroup, for chunks and
// prompts.
//
// Four waves of kQ blocks of 32 rows each, 32-key tiles. As in biased_chunk_attention's bf16 kernel a wave computes
// the transposed logits S^T = K Q^T with 32x32x16 MFMAs, keys in the rows, so that a lane has 16 logits of one query
// and softmax needs one exchange with the other half of the wave, and with the K rows read in an order that makes a
// lane's probabilities the B operand of O^T = V^T P^T as they are.
//
// Keys and values come from the pages, where a head's share of a tile is one run of bytes: each thread loads its 16-byte
// pieces into registers, a step ahead, and writes them to LDS as bf16, 8-bit ones widened with their scale on the
// way (exactly: it is a power of two), so that the matrix cores see the same numbers whatever the pages hold.
// 256-byte (128-byte) rows with their 16-byte chunks at c ^ swz(row), which keeps the reads of both operands, V's
// through the transposing LDS load, off each other's banks.
//
// LDS holds a ring of four slots; slot t mod 4 carries K_t and V_{t-1}. Step j computes the logits of tile j + 1 beside
// the softmax of tile j, and behind its one barrier P V of tile j beside the refilling of slot j + 3 mod 4.
//
// What bounds it is the vector work and the LDS traffic of a tile beside its MFMAs (matrix cores busy 38% of the time at
// 4680 x 28080 and 43% at 10800 x 43200): a piece of a tile is loaded, widened and stored once per
// workgroup and read by each of its waves, so that its share of a row falls with the rows of a wave and of a workgroup.
// Two blocks of 32 rows per wave (kQ = 2) need 500 registers, one wave per SIMD, and that the MFMAs accumulate in the
// registers that vector instructions read (-amdgpu-mfma-vgpr-form, set for this file: without it each logit is moved
// first, and it is 25 % slower); the order of a step is then fixed slot by slot, an MFMA and as much of the other work
// as runs beside it, since no second wave fills a gap. 4680 queries on 28080 8-bit keys, 12 heads of 128, biased: 880 us
// (920 TFLOP/s); eight waves of one block 1000, four waves of one block 1100 (two workgroups per compute unit). 10800
// on 43200, 40 heads: 9.45 ms (1010 TFLOP/s), 10.2 and 13.5. At D = 64 one block per wave is faster: 8 ragged prompts
// of up to 2000 on 4000 bf16 keys, 16 heads on 4: 107 us, with two 120.
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

// The kernel's arguments, read again: those that only rare blocks need would otherwise fill the scalar registers.
typedef const __attribute__((address_space(4))) PagedAttentionArgs* RareArgs;
__device__ __forceinline__ RareArgs rare_args() {
    auto p = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();  // the first argument
    asm volatile("" : "+s"(p));
    return (RareArgs)p;
}

template <int D, int T, bool kBias, int kQ, bool kStrided>
__global__ __launch_bounds__(256, kQ == 2 ? 1 : 2) void paged_tile_kernel(PagedAttentionArgs a, float c_log2) {
    constexpr int kRowB = D * 2, kTileB = kTK * kRowB;      // in LDS
    constexpr int kStored = T == kPagedFp8 ? D : 2 * D;     // bytes of a row in the pages
    constexpr int kHalf = kTK * kStored / 16;               // 16-byte pieces of a K or V tile
    constexpr int kW = 4, kRows = 32 * kQ * kW, kThreads = 64 * kW;
    constexpr int kPieces = (2 * kHalf + kThreads - 1) / kThreads;  // of a thread
    constexpr int kKk = D / 16, kDb = D / 32;
    __shared__ __attribute__((aligned(1024))) uint8_t ring[4][2 * kTileB];
    __shared__ u32x4 lds_tab[2][kBias ? kGridSide : 1];     // key operands by column and by row
    __shared__ float2 lds_corr[kBias ? kCorrLds : 1][kRows];  // centred correspondences, NaN: rejected
    __shared__ int lds_block[512];
    __shared__ int64_t lds_at[2][kStrided ? 512 : 1];       // strided pools: bytes at which a tile's keys and values begin
    __shared__ int2 lds_bias[kBias ? 512 : 1];              // slot (-1: unbiased, -2: across frames) and in-frame position of a tile
    __shared__ u32x4 lds_qop[kBias ? kW : 1][kQ][64];       // the waves' query operands of the frame at hand
    __shared__ float lds_scale[2][T == kPagedFp8 ? 512 : 1];
    __shared__ int lds_seen[kW], lds_least[kW];
    __shared__ int lds_odd[4];  // V tile of a slot from which values that are not finite were taken out, or -1

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

    // the lane's rows (one of each block of 32), their queries and how many keys they see
    int token[kQ], head[kQ], vis[kQ];
    u32x4 qf[kQ][kKk];  // head dims 16 kk + 8 hh ..
#pragma unroll
    for (int b = 0; b < kQ; ++b) {
        const int r = it.in * kRows + (wave * kQ + b) * 32 + n;
        token[b] = r < n_rows ? tok.x + r / G : -1;
        head[b] = hk * G + r % G;
        const uint16_t* qp = static_cast<const uint16_t*>(a.q) + (int64_t)max(token[b], 0) * a.q_row + (int64_t)head[b] * D + 8 * hh;
#pragma unroll
        for (int kk = 0; kk < kKk; ++kk) qf[b][kk] = u32x4{0, 0, 0, 0};
        if (token[b] >= 0) {
#pragma unroll
            for (int kk = 0; kk < kKk; ++kk) qf[b][kk] = *reinterpret_cast<const u32x4*>(qp + 16 * kk);
        }
    }
    const int held = held_of(sq, s);
    int seen = held, seen_min = held, least = held;  // seen_min: of the wave's rows, least: of the workgroup's
#pragma unroll
    for (int b = 0; b < kQ; ++b) vis[b] = held;
    if (a.visible) {
        seen = 0;
#pragma unroll
        for (int b = 0; b < kQ; ++b) {
            if (token[b] < 0) continue;
            vis[b] = min(held, max(a.visible[token[b]], 0));
            seen = max(seen, vis[b]);
            seen_min = min(seen_min, vis[b]);
        }
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
    // Where the part's tiles lie, 256 at a time in LDS, the next 256 beside them (a scalar load in every step would make
    // each wait for LDS a wait for it, a vector load one for the pieces in flight): the block of 32 rows of the
    // caches, or -1 without a page (page 0's rows stand in for them, which nobody sees), and the scales.
    auto slot_of = [&](int f) __attribute__((always_inline)) -> int {
        const RareArgs r = rare_args();
        const int v = f < r->max_frames ? r->slot[(int64_t)s * r->max_frames + f] : -1;
        return v >= 0 && v < r->S ? v : -1;
    };
    auto fetch_info = [&](int j) __attribute__((always_inline)) {  // of tiles j + tid, past the last one the last one's
        const RareArgs r = rare_args();
        const int x = j + tid, pos = (t0 + min(x, nt - 1)) * kTK;
        const int page_log2 = r->seqs.page_log2;
        const int entry = r->seqs.page_table[(int64_t)s * r->seqs.max_pages + (pos >> page_log2)];
        const bool there = (unsigned)entry < (unsigned)r->seqs.n_pages;
        const int page = there ? entry : 0, in_page = (pos & ((1 << page_log2) - 1)) >> 5;
        int block;
        if constexpr (kStrided) {
            block = (page << (page_log2 - 5)) + in_page;
            auto at = [&](const __attribute__((address_space(4))) PagedStrides& st, int row) -> int64_t { return page * st.page + hk * st.head + row * st.row; };
            lds_at[0][x & 511] = at(r->layout.k, in_page * kTK);
            lds_at[1][x & 511] = at(r->layout.v, in_page * kTK);
            if constexpr (T == kPagedFp8) {
                lds_scale[0][x & 511] = scale_value(r->scale_k[at(r->layout.scale_k, in_page)]);
                lds_scale[1][x & 511] = scale_value(r->scale_v[at(r->layout.scale_v, in_page)]);
            }
        } else {
            block = ((page * r->Hk + hk) << (page_log2 - 5)) + in_page;
            if constexpr (T == kPagedFp8) {
                lds_scale[0][x & 511] = scale_value(r->scale_k[block]);
                lds_scale[1][x & 511] = scale_value(r->scale_v[block]);
            }
        }
        lds_block[x & 511] = there ? block : -1;
        if constexpr (kBias) {
            const int hw = r->h * r->w, f = pos / hw, p = pos - f * hw;
            int sl = slot_of(f);
            if (p + kTK > hw) {
                for (int e = f + 1; e <= (pos + kTK - 1) / hw; ++e) sl = max(sl, slot_of(e));
                sl = sl >= 0 ? -2 : -1;
            }
            lds_bias[x & 511] = make_int2(sl, p);
        }
    };
    auto block_of = [&](int j) __attribute__((always_inline)) -> int { return lds_block[j & 511]; };
    u32x4 piece[kPieces];
    auto scalar = [](int64_t x) __attribute__((always_inline)) -> int64_t {  // the same in all of the wave
        return (int64_t)(((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32) | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
    };
    // pieces of the K tile in block bk and the V tile in block bv (of strided pools: at bytes ak and av); piece p of a thread is
    // number kThreads p + tid of K's and then V's
    auto load = [&](int bk, int bv, int64_t ak, int64_t av) __attribute__((always_inline)) {
        const uint8_t* kb = static_cast<const uint8_t*>(a.cache_k) + (kStrided ? ak : (int64_t)(unsigned)max(bk, 0) * (kTK * kStored));
        const uint8_t* vb = static_cast<const uint8_t*>(a.cache_v) + (kStrided ? av : (int64_t)(unsigned)max(bv, 0) * (kTK * kStored));
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int i = kThreads * p + tid;
            if constexpr (kStrided) {
                constexpr int kOf = kStored / 16;  // pieces of a row
                const bool is_v = kHalf % kThreads == 0 ? kThreads * p >= kHalf : i >= kHalf;
                const int64_t step = is_v ? a.layout.v.row : a.layout.k.row;
                if constexpr (kHalf % kThreads == 0) {
                    const int first = kThreads * p - (kThreads * p >= kHalf ? kHalf : 0);  // of the threads' pieces
                    piece[p] = *reinterpret_cast<const u32x4*>((is_v ? vb : kb) + first / kOf * step + (tid / kOf * step + 16 * (tid % kOf)));
                } else {
                    const int at = is_v ? i - kHalf : i;
                    if (2 * kHalf % kThreads == 0 || i < 2 * kHalf) piece[p] = *reinterpret_cast<const u32x4*>((is_v ? vb : kb) + at / kOf * step + 16 * (at % kOf));
                }
            } else if constexpr (kHalf % kThreads == 0) {
                const uint32_t off = 16 * (uint32_t)tid;
                piece[p] = *reinterpret_cast<const u32x4*>((kThreads * p >= kHalf ? vb + 16 * (kThreads * p - kHalf) : kb + 16 * kThreads * p) + off);
            } else {
                if (2 * kHalf % kThreads == 0 || i < 2 * kHalf) piece[p] = *reinterpret_cast<const u32x4*>(i >= kHalf ? vb + 16 * (i - kHalf) : kb + 16 * i);
            }
        }
    };
    // A weight of 0 times a value that is not finite would be NaN. In a tile that some row does not see all of, such
    // values (and whatever lies behind the stream's end) are left out here; the rows that see them get them one by
    // one (odd_values).
    auto leave_out = [&](int which, float& v_scale, int jv, int bv) __attribute__((always_inline)) {
        const uint32_t codes = T == kPagedFp8 ? odd_codes(v_scale) : 0u;
        uint32_t odd = 0;
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            const int i = kThreads * p + tid - kHalf;
            if (i < 0) continue;
            const bool none = bv < 0 || (t0 + jv) * kTK + i / (kStored / 16) >= held;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const uint32_t bad = spread<T>(not_finite<T>(piece[p][w], codes));
                if (none) piece[p][w] = 0;
                else odd |= bad;
                piece[p][w] &= ~bad;
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (v_scale != v_scale) v_scale = 1.0f;
        if (odd) lds_odd[which] = jv;
    };
    // half h of piece p, as bf16 (8-bit pages: 8 values; else the whole piece in half 0)
    auto put = [&](int which, int p, int h, float k_scale, float v_scale) __attribute__((always_inline)) {
        const int i = kThreads * p + tid;
        const bool is_v = kHalf % kThreads == 0 ? kThreads * p >= kHalf : i >= kHalf;
        const int at = is_v ? i - kHalf : i;
        const int row = at / (kStored / 16), c = at % (kStored / 16);
        uint8_t* to = ring[which] + (is_v ? kTileB : 0) + row * kRowB;
        if constexpr (T == kPagedFp8) {
            const float f = is_v ? v_scale : k_scale;
            *reinterpret_cast<u32x4*>(to + (((2 * c + h) ^ swz<D>(row)) << 4)) =
                u32x4{widen2<false>(piece[p][2 * h], f), widen2<true>(piece[p][2 * h], f), widen2<false>(piece[p][2 * h + 1], f),
                      widen2<true>(piece[p][2 * h + 1], f)};
        } else if (h == 0) {
            *reinterpret_cast<u32x4*>(to + ((c ^ swz<D>(row)) << 4)) = piece[p];
        }
    };
    auto put_all = [&](int which, float k_scale, float v_scale, int jv, int bv) __attribute__((always_inline)) {
        if ((t0 + jv + 1) * kTK > least || bv < 0) leave_out(which, v_scale, jv, bv);
#pragma unroll
        for (int p = 0; p < kPieces; ++p) {
            put(which, p, 0, k_scale, v_scale);
            put(which, p, 1, k_scale, v_scale);
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
    const float inv_w = 1.0f / (float)a.w;
    const int grid_w = a.w;
    if constexpr (kBias) {
        for (int i = tid; i < a.w + a.h; i += kThreads) {
            const bool col = i < a.w;
            const int k = col ? i : i - a.w;
            const float ac = ((float)k + 0.5f) - 0.5f * (float)(col ? a.w : a.h);
            const uint32_t a2 = bf16_bits(2.0f * ac);
            uint32_t ph, pm, pl;
            split3(-a.gamma * (ac * ac), ph, pm, pl);
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
            lds_corr[e / kRows][e % kRows] = ci[i] >= 0 ? make_float2(cu[i].x - 0.5f * (float)a.w, cu[i].y - 0.5f * (float)a.h) : make_float2(NAN, NAN);
        }
    }
    // query-side operand of retrieved frame f: zeros where the correspondence is rejected
    auto query_operand = [&](int f, int b) __attribute__((always_inline)) -> bf16x8 {
        const RareArgs r = rare_args();
        float ux = NAN, uy = NAN;
        if (f < kCorrLds) {
            const float2 u = lds_corr[f][(wave * kQ + b) * 32 + n];
            ux = u.x;
            uy = u.y;
        } else if (token[b] >= 0) {
            const int64_t o = (int64_t)f * r->seqs.n_tokens + token[b];
            if (r->corr_idx[o] >= 0) {
                const float2 u = reinterpret_cast<const float2*>(r->corr_uv)[o];
                ux = u.x - 0.5f * (float)r->w;
                uy = u.y - 0.5f * (float)r->h;
            }
        }
        u32x4 v = u32x4{0, 0, 0, 0};
        if (!__builtin_isnan(ux)) {
            uint32_t xh, xm, xl, zh, zm, zl;
            split3(r->gamma * (hh ? uy : ux), xh, xm, xl);
            split3(-r->gamma * (ux * ux + uy * uy), zh, zm, zl);
            v = u32x4{pack2(xh, xm), pack2(xl, one), pack2(one, one), hh ? zl : pack2(zh, zm)};
        }
        return as_bf16x8(v);
    };
    auto key_operand = [&](int p) __attribute__((always_inline)) -> u32x4 {  // in-frame position p
        const int ky = (int)(((float)p + 0.5f) * inv_w);
        return lds_tab[hh][hh ? ky : p - ky * grid_w];
    };
    int cur_s = -1;  // retrieved frame whose operands are in lds_qop
    // slot of a tile's frame (and position p in it) by what lds_bias has of it; the wave's query operands follow it
    auto classify = [&](int2 x, int& p) __attribute__((always_inline)) -> int {
        const int sl = __builtin_amdgcn_readfirstlane(x.x);
        p = x.y;
        if (__builtin_expect(sl >= 0 && sl != cur_s, 0)) {
            cur_s = sl;
#pragma unroll
            for (int b = 0; b < kQ; ++b) lds_qop[wave][b][lane] = __builtin_bit_cast(u32x4, query_operand(sl, b));
        }
        return sl;
    };
    // a tile across frames: its frames one by one
    auto bias_across = [&](floatx16 (&x)[kQ], int j) __attribute__((always_inline)) {
        const RareArgs r = rare_args();
        const int hw = r->h * r->w, pos = (t0 + min(j, nt - 1)) * kTK, f0 = pos / hw;
        const int lane_f = (pos + krow) / hw, lane_p = (pos + krow) - lane_f * hw;
        for (int f = f0; f <= (pos + kTK - 1) / hw; ++f) {
            const int sl = __builtin_amdgcn_readfirstlane(slot_of(f));
            if (sl < 0) continue;
            const u32x4 kv = lane_f == f ? key_operand(lane_p) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int b = 0; b < kQ; ++b) x[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kv), query_operand(sl, b), x[b], 0, 0, 0);
        }
    };

    // ---- state ----------------------------------------------------------------
    floatx16 O[kQ][kDb];
    float m_run[kQ], m_thr[kQ], l0[kQ], l1[kQ], mx[kQ];
#pragma unroll
    for (int b = 0; b < kQ; ++b) {
#pragma unroll
        for (int db = 0; db < kDb; ++db) O[b][db] = floatx16{0};
        m_run[b] = -FLT_MAX;
        m_thr[b] = mx[b] = -INFINITY;
        l0[b] = l1[b] = 0.0f;
    }

    // logits of tile j that a row does not see
    auto mask = [&](floatx16 (&S)[kQ], int j, int block) __attribute__((always_inline)) {
        const int k0 = (t0 + j) * kTK;
#pragma unroll
        for (int b = 0; b < kQ; ++b) {
            const int lim = block < 0 ? 0 : vis[b];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                S[b][i] = k0 + key_of(hh, i) >= lim ? -INFINITY : S[b][i];
                __builtin_amdgcn_sched_barrier(0);  // one mask at a time
            }
        }
    };
    // the values of V tile j that leave_out took out, for the rows that see them (probabilities in w4)
    auto odd_values = [&](const uint32_t (&w4)[kQ][2][4], int j, int block) __attribute__((always_inline)) {
        const int k0 = (t0 + j) * kTK;
        const RareArgs r = rare_args();
        const uint8_t* base;
        int64_t step = kStored, scale_at = block;
        if constexpr (kStrided) {
            const int shift = r->seqs.page_log2 - 5, page = block >> shift, in_page = block & ((1 << shift) - 1);
            base = static_cast<const uint8_t*>(r->cache_v) + lds_at[1][j & 511];
            step = r->layout.v.row;
            scale_at = page * r->layout.scale_v.page + hk * r->layout.scale_v.head + in_page * r->layout.scale_v.row;
        } else {
            base = static_cast<const uint8_t*>(r->cache_v) + (size_t)(unsigned)block * (kTK * kStored);
        }
        const float f = T == kPagedFp8 ? scale_value(r->scale_v[scale_at]) : 1.0f;
#pragma unroll 1
        for (int key = 0; key < min(kTK, held - k0); ++key) {
            const int want = 8 * (key >> 4) + (key & 7);  // register of the lane that has its probability
            float p[kQ];
            uint32_t sees[kQ];
#pragma unroll
            for (int b = 0; b < kQ; ++b) {
                p[b] = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t w = w4[b][i >> 3][(i >> 1) & 3];
                    p[b] = i == want ? __uint_as_float((i & 1) ? w & 0xffff0000u : w << 16) : p[b];
                }
                p[b] = __shfl(p[b], 32 * ((key >> 3) & 1) + n);
                sees[b] = k0 + key < vis[b] ? ~0u : 0u;
                asm volatile("" : "+v"(sees[b]));  // a mask in a vector register: scalar ones are rare
            }
#pragma unroll
            for (int db = 0; db < kDb; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float x = stored<T>(base + key * step, 32 * db + 8 * (i >> 2) + 4 * hh + (i & 3)) * f;
#pragma unroll
                    for (int b = 0; b < kQ; ++b) {
                        const float seen_x = __uint_as_float(__float_as_uint(x) & sees[b]);
                        if (!(fabsf(seen_x) < INFINITY)) O[b][db][i] += p[b] * seen_x;
                        __builtin_amdgcn_sched_barrier(0);  // one mask at a time
                    }
                }
        }
    };

    floatx16 Sa[kQ], Sb[kQ];
    int b0 = 0, b1 = 0, b2 = 0, b3 = 0;  // blocks of tiles j .. j + 3
    u32x4 kf[kKk];  // K operands of the next tile

    // One step: softmax and P V of tile j, whose logits are in S_cur, beside the logits of tile j + 1. The order is
    // fixed slot by slot: each slot is one MFMA and as much of the other work as runs beside it.
    auto step = [&](int j, floatx16 (&S_cur)[kQ], floatx16 (&S_next)[kQ], auto slot_tag) __attribute__((always_inline)) {
        // slot t mod 4 holds K_t and V_{t-1}
        constexpr int kStep = decltype(slot_tag)::value, kNext = (kStep + 1) & 3, kRefill = (kStep + 3) & 3;
        const uint8_t* next = ring[kNext];
        const bool more = j + 1 < nt;  // past the last tile its logits are computed again and not used
        const uint8_t* vt = next + kTileB;
        auto kread = [&](int kk) { kf[kk] = *reinterpret_cast<const u32x4*>(next + koff[kk]); };
        int2 bias_at = make_int2(-1, 0);
        if constexpr (kBias) {
            bias_at = lds_bias[(j + 1) & 511];
            __builtin_amdgcn_sched_barrier(0);  // the first of the step's reads: it is the one that is waited for
        }
        const int b4_lane = block_of(j + 4);
        float k_scale = T == kPagedFp8 ? lds_scale[0][(j + 3) & 511] : 1.0f, v_scale = T == kPagedFp8 ? lds_scale[1][(j + 2) & 511] : 1.0f;
        int bias_slot = -1, bias_p = 0;
        if constexpr (kBias) bias_slot = classify(bias_at, bias_p);
        u32x4 kop = u32x4{0, 0, 0, 0}, qop[kQ];
        // rescale where a row's maximum has grown by more than the slack
        bool grown = false;
#pragma unroll
        for (int b = 0; b < kQ; ++b) grown = grown || mx[b] > m_thr[b];
        if (__builtin_expect(__any(grown), 0)) {
#pragma unroll
            for (int b = 0; b < kQ; ++b) {
                const float m_new = fmaxf(m_run[b], half_swap_max(mx[b]) * c_log2);
                const float alpha = __builtin_amdgcn_exp2f(m_run[b] - m_new);
                l0[b] *= alpha;
                l1[b] *= alpha;
#pragma unroll
                for (int db = 0; db < kDb; ++db) O[b][db] *= alpha;
                m_run[b] = m_new;
                m_thr[b] = (m_new + kRescaleSlack) / c_log2;
            }
        }
        uint32_t w4[kQ][2][4];
        // Probabilities 2 (u % 8) and the next of block u / 8, each as one bf16 number: outputs of N(0, 1) values are off by
        // 0.0021 of their size then, where rounding them to bf16 leaves 0.0017. A second number, as in the wave kernel's
        // tiles of 16 rows, is a second product here: 4680 queries on 28080 keys 878 us and 1248, ragged prompts at D = 64 105
        // and 143.
        auto unit = [&](int u) __attribute__((always_inline)) {
            const int b = u >> 3, t = (u >> 2) & 1, e = u & 3, i = 8 * t + 2 * e;
            const float p0 = __builtin_amdgcn_exp2f(fmaf(S_cur[b][i], c_log2, -m_run[b]));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(S_cur[b][i + 1], c_log2, -m_run[b]));
            w4[b][t][e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{p0, p1}, __bf16 __attribute__((ext_vector_type(2)))));
            l0[b] += p0;
            l1[b] += p1;
            asm volatile("" : "+v"(l0[b]), "+v"(l1[b]), "+v"(w4[b][t][e]));  // here, not at the end of the step
        };
        shortx4 vlo[2][kDb], vhi[2][kDb];
        auto vread = [&](int t, int db) __attribute__((always_inline)) {
            const uint8_t* vp = vt + 16 * t * kRowB;
            vlo[t][db] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(vp + voff[0][db]));
            vhi[t][db] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4*)(vp + voff[1][db]));
        };
        auto voperand = [&](int t, int db) __attribute__((always_inline)) -> bf16x8 {
            const u32x2 lo = __builtin_bit_cast(u32x2, vlo[t][db]), hi = __builtin_bit_cast(u32x2, vhi[t][db]);
            return as_bf16x8(u32x4{lo[0], lo[1], hi[0], hi[1]});
        };
        __builtin_amdgcn_sched_barrier(0);
        // the QK MFMAs of tile j + 1 beside the softmax of tile j; K read three ahead, the first half of V at the end
        constexpr int kSlotsA = kKk * kQ, kUnits = 8 * kQ;
#pragma unroll
        for (int i = 0; i < kSlotsA; ++i) {
            const int kk = i / kQ, b = i % kQ;
            if (b == 0 && kk + 3 < kKk) kread(kk + 3);
            S_next[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kf[kk]), as_bf16x8(qf[b][kk]), kk == 0 ? floatx16{0} : S_next[b], 0, 0, 0);
#pragma unroll
            for (int u = i * kUnits / kSlotsA; u < (i + 1) * kUnits / kSlotsA; ++u) unit(u);
            if (b == 0 && kk >= kKk - kDb) vread(0, kk - (kKk - kDb));
            if (kBias && i == kSlotsA / 2 && bias_slot >= 0) {  // half of S_cur's registers are free by now
                kop = key_operand(bias_p + krow);
#pragma unroll
                for (int x = 0; x < kQ; ++x) qop[x] = lds_qop[wave][x][lane];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (kBias) {
            if (bias_slot >= 0) {
#pragma unroll
                for (int b = 0; b < kQ; ++b) S_next[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kop), as_bf16x8(qop[b]), S_next[b], 0, 0, 0);
            }
            if (__builtin_expect(bias_slot == -2, 0)) bias_across(S_next, j + 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        // P V of tile j beside the staging (the pieces of K_{j+3} and V_{j+2} go to LDS, those behind them leave) and the row maxima of tile j + 1
        int64_t at_k = 0, at_v = 0;
        if constexpr (kStrided) {
            at_k = lds_at[0][(j + 4) & 511];
            at_v = lds_at[1][(j + 3) & 511];
        }
        lds_barrier();  // slot kRefill was read two steps ago; what was written to the others is there
        const int jv = min(j + 2, nt - 1);
        if (__builtin_expect((t0 + jv + 1) * kTK > least || b2 < 0, 0)) leave_out(kRefill, v_scale, jv, b2);
        if (__builtin_expect((t0 + j + 2) * kTK > seen_min || b1 < 0, 0)) mask(S_next, j + 1, b1);
        const int b4 = __builtin_amdgcn_readfirstlane(b4_lane);
        if constexpr (kStrided) {
            at_k = scalar(at_k);
            at_v = scalar(at_v);
        }
        bf16x8 pf[kQ][2];
#pragma unroll
        for (int b = 0; b < kQ; ++b)
#pragma unroll
            for (int t = 0; t < 2; ++t) pf[b][t] = as_bf16x8(u32x4{w4[b][t][0], w4[b][t][1], w4[b][t][2], w4[b][t][3]});
        constexpr int kSlotsB = 2 * kDb * kQ, kPuts = 2 * kPieces;
#pragma unroll
        for (int i = 0; i < kSlotsB; ++i) {
            const int t = i / (kDb * kQ), db = i / kQ % kDb, b = i % kQ;
            O[b][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(voperand(t, db), pf[b][t], O[b][db], 0, 0, 0);
            if (t == 0 && b == 0) vread(1, db);
            // first half: the pieces; then the loads; second half: the maxima
            if (t == 0) {
#pragma unroll
                for (int x = i * kPuts / (kSlotsB / 2); x < (i + 1) * kPuts / (kSlotsB / 2); ++x) put(kRefill, x >> 1, x & 1, k_scale, v_scale);
                if (i == kSlotsB / 2 - 1) load(b4, b3, at_k, at_v);
            } else {
                const int slot = i - kSlotsB / 2, per = 16 * kQ / (kSlotsB / 2);  // logits of a slot
#pragma unroll
                for (int x = slot * per; x < (slot + 1) * per; x += 2) {
                    const int xb = x >> 4, xi = x & 15;
                    mx[xb] = xi == 0 ? max3(S_next[xb][0], S_next[xb][1], S_next[xb][1]) : max3(mx[xb], S_next[xb][xi], S_next[xb][xi + 1]);
                }
            }
            // the first K operands of the step behind: they are there since the barrier above
            if (i >= kSlotsB - 3) kf[i - (kSlotsB - 3)] = *reinterpret_cast<const u32x4*>(ring[(kStep + 2) & 3] + koff[i - (kSlotsB - 3)]);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (__builtin_expect((t0 + j + 1) * kTK > least, 0)) {
            asm volatile("" ::: "memory");  // lds_odd is read for such tiles alone
            if (lds_odd[kNext] == j) odd_values(w4, j, b0);
        }
        if constexpr (kStep == 3) {  // j + 5 is a multiple of 4 here
            if (__builtin_expect(((j + 5) & 255) == 128, 0)) fetch_info(((j + 5) & ~255) + 256);
        }
        if (!more) {
#pragma unroll
            for (int b = 0; b < kQ; ++b) mx[b] = -INFINITY;
        }
        b0 = b1;
        b1 = b2;
        b2 = b3;
        b3 = b4;
    };

    if (nt > 0) {
        fetch_info(0);
        if (tid < 4) lds_odd[tid] = -1;
        __syncthreads();
        auto scale = [&](int which, int j) -> float { return T == kPagedFp8 ? lds_scale[which][j] : 1.0f; };
        auto place = [&](int which, int j) -> int64_t { return kStrided ? scalar(lds_at[which][j]) : 0; };
        b0 = __builtin_amdgcn_readfirstlane(block_of(0));
        b1 = __builtin_amdgcn_readfirstlane(block_of(1));
        b2 = __builtin_amdgcn_readfirstlane(block_of(2));
        b3 = __builtin_amdgcn_readfirstlane(block_of(3));
        load(b0, b0, place(0, 0), place(1, 0));
        put_all(0, scale(0, 0), scale(1, 0), 0, b0);
        load(b1, b0, place(0, 1), place(1, 0));
        put_all(1, scale(0, 1), scale(1, 0), 0, b0);
        load(b2, b1, place(0, 2), place(1, 1));
        put_all(2, scale(0, 2), scale(1, 1), min(1, nt - 1), b1);
        load(b3, b2, place(0, 3), place(1, 2));
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < 3; ++kk) kf[kk] = *reinterpret_cast<const u32x4*>(ring[1] + koff[kk]);
#pragma unroll
        for (int b = 0; b < kQ; ++b) {
            Sa[b] = floatx16{0};
#pragma unroll
            for (int kk = 0; kk < kKk; ++kk)
                Sa[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(ring[0] + koff[kk]), as_bf16x8(qf[b][kk]), Sa[b], 0, 0, 0);
        }
        if constexpr (kBias) {
            int p = 0;
            const int sl = classify(lds_bias[0], p);
            if (sl >= 0) {
                const u32x4 kop = key_operand(p + krow);
#pragma unroll
                for (int b = 0; b < kQ; ++b) Sa[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kop), as_bf16x8(lds_qop[wave][b][lane]), Sa[b], 0, 0, 0);
            }
            if (sl == -2) bias_across(Sa, 0);
        }
        if ((t0 + 1) * kTK > seen_min || b0 < 0) mask(Sa, 0, b0);
#pragma unroll
        for (int b = 0; b < kQ; ++b) {
            mx[b] = Sa[b][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mx[b] = fmaxf(mx[b], Sa[b][i]);
        }
        for (int j = 0;;) {
            step(j, Sa, Sb, std::integral_constant<int, 0>{});
            if (++j >= nt) break;
            step(j, Sb, Sa, std::integral_constant<int, 1>{});
            if (++j >= nt) break;
            step(j, Sa, Sb, std::integral_constant<int, 2>{});
            if (++j >= nt) break;
            step(j, Sb, Sa, std::integral_constant<int, 3>{});
            if (++j >= nt) break;
        }
    }

#pragma unroll
    for (int b = 0; b < kQ; ++b) {
        asm volatile("" : "+v"(token[b]));  // no mask of the prologue's is kept for it
        const float l = half_swap_sum(l0[b] + l1[b]);
        if (a.parts == 1) {
            if (token[b] < 0) continue;
            // a row that sees no key: nothing, and an LSE of -inf
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            uint16_t* o = static_cast<uint16_t*>(a.o) + ((size_t)token[b] * a.Hq + head[b]) * D;
#pragma unroll
            for (int db = 0; db < kDb; ++db)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t w[2];
#pragma unroll
                    for (int x = 0; x < 2; ++x)
                        w[x] = __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{O[b][db][4 * i + 2 * x] * inv, O[b][db][4 * i + 2 * x + 1] * inv},
                                                                                   __bf16 __attribute__((ext_vector_type(2)))));
                    *reinterpret_cast<u32x2*>(o + 32 * db + 8 * i + 4 * hh) = u32x2{w[0], w[1]};
                }
            if (a.lse && hh == 0) a.lse[(size_t)head[b] * sq.n_tokens + token[b]] = (m_run[b] + log2f(l)) * 0.6931471805599453f;
        } else {
            float* base = a.partial + ((size_t)((size_t)tile * a.Hk + hk) * a.parts + part) * paged_part_floats(kRows, D);
            const int row = (wave * kQ + b) * 32 + n;
            if (hh == 0) {
                base[kRows * D + row] = nt > 0 ? m_run[b] : -INFINITY;
                base[kRows * D + kRows + row] = l;
            }
            if (nt > 0 && token[b] >= 0) {
#pragma unroll
                for (int db = 0; db < kDb; ++db)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<float4*>(base + row * D + 32 * db + 8 * i + 4 * hh) =
                            make_float4(O[b][db][4 * i], O[b][db][4 * i + 1], O[b][db][4 * i + 2], O[b][db][4 * i + 3]);
            }
        }
    }
}

}  // namespace

hipError_t launch_paged_tiles(const PagedAttentionArgs& a, hipStream_t stream) {
    const float c = a.softmax_scale * 1.4426950408889634f;
    const dim3 grid = grid_rows(xcd_grid((unsigned)a.tiles * (unsigned)a.Hk * (unsigned)a.parts)), block(256);
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, a, c); };
    auto bias = [&](auto d_tag, auto t_tag, auto q_tag) {
        constexpr int D = decltype(d_tag)::value, T = decltype(t_tag)::value, kQ = decltype(q_tag)::value;
        auto layout = [&](auto strided_tag) {
            constexpr bool kStrided = decltype(strided_tag)::value;
            if (a.S > 0) launch(paged_tile_kernel<D, T, true, kQ, kStrided>);
            else launch(paged_tile_kernel<D, T, false, kQ, kStrided>);
        };
        if (a.strided) layout(std::true_type{});
        else layout(std::false_type{});
    };
    auto rows = [&](auto t_tag) {
        using One = std::integral_constant<int, 1>;
        using Two = std::integral_constant<int, 2>;
        if (a.D == 64) bias(std::integral_constant<int, 64>{}, t_tag, One{});
        else if (a.rows == 128) bias(std::integral_constant<int, 128>{}, t_tag, One{});
        else bias(std::integral_constant<int, 128>{}, t_tag, Two{});
    };
    if (a.dtype == kPagedFp8) rows(std::integral_constant<int, kPagedFp8>{});
    else rows(std::integral_constant<int, kPagedBf16>{});
    return hipGetLastError();
}

}  // namespace revisit
