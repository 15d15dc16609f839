// The choice of what a cache keeps (select_kept): unit scores, then the largest of
// them in the order of their places.
//
// Scores. Every weight is read once: bound by HBM. A unit's weights are added in
// double by a group of lanes that fits its loads (one lane, 8, a wave or a
// workgroup; units of a few tokens go one to a lane, so that lanes read neighbouring
// words), four loads in flight; where few long units leave compute units idle, the
// heads are cut into parts whose sums meet in the choice. 30 sets of 18 frames of 1560
// tokens and 12 heads (40 MB) take 10.7 us, and their choice 3 to 4.
//
// Choice. One workgroup of 16 waves per set; a wave takes a contiguous range of units,
// eight rounds of 64 at a time. The keep-th largest score is found digit by digit
// over the scores as ordered unsigned numbers (kept in LDS), 12, 10 and 10 bits,
// with a histogram in LDS: the first digit holds sign, exponent and three bits, so
// that the usual scores spread over many bins, and the few units in the bin that it
// leaves are listed for the other two. Where a round's units all have the same digit (equal
// scores) one lane counts for all. With the threshold every wave knows how many it
// keeps, one barrier gives each its place, and the units are written in order. Long sets that
// leave compute units idle are shared out over workgroups, in three launches.
// Bound by its instructions (60 per round of 64 units and wave) on one compute unit
// per set: 96 sets of 37440 tokens 25 us, with the keys in registers and code unrolled over them 31, with
// four digits of 8 bits read from memory each time 98.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "internal.h"

namespace revisit {
namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kScoreBlock = 256;

// Sum of a unit's weights in vectors of VEC, G lanes a unit; grid.z = head part.
template <int G, int VEC>
__global__ __launch_bounds__(kScoreBlock) void unit_score_kernel(SelectArgs a, int64_t n_items, double inv_len) {
    constexpr int kUnits = kScoreBlock / G;
    const int64_t item = (int64_t)row_block() * kUnits + threadIdx.x / G;
    const int part = blockIdx.z;
    const int h0 = (int)((int64_t)part * a.heads / a.splits), h1 = (int)((int64_t)(part + 1) * a.heads / a.splits);
    const int64_t row = (int64_t)a.n_units * a.unit;
    double sum = 0.0;
    if (item < n_items) {
        const int64_t set = item / a.n_units, u = item - set * a.n_units;
        const float* w = a.weight + (set * a.heads + h0) * row + u * a.unit;
        const int len = a.unit / VEC;
        const int64_t total = (int64_t)(h1 - h0) * len;
        for (int64_t e0 = threadIdx.x % G; e0 < total; e0 += 4 * G) {
            float v[4][VEC];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t e = e0 + k * G;
                // (e + 1/2) / len truncates to e / len exactly below 2^50
                const int64_t h = len == 1 ? e : (int64_t)(((double)e + 0.5) * inv_len);
                const float* p = w + h * row + (e - h * len) * VEC;
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[k][i] = 0.0f;
                if (e < total) {
                    if constexpr (VEC == 4) {
                        const floatx4 x = *reinterpret_cast<const floatx4*>(p);
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[k][i] = x[i];
                    } else {
                        v[k][0] = *p;
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum += (double)v[k][i];
        }
    }
#pragma unroll
    for (int k = (G < 64 ? G : 64) / 2; k > 0; k /= 2) sum += __shfl_xor(sum, k);
    if constexpr (G > 64) {
        __shared__ double lds[G / 64];
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = sum;
        __syncthreads();
        sum = 0.0;
#pragma unroll
        for (int k = 0; k < G / 64; ++k) sum += lds[k];
    }
    if (threadIdx.x % G == 0 && item < n_items) a.unit_sum[(int64_t)part * n_items + item] = sum;
}

// fp32 as an unsigned number in the same order: NaN below all, -0 equal to 0; and back
__device__ __forceinline__ uint32_t ordered(float x) {
    if (__builtin_isnan(x)) return 0;
    const uint32_t u = __float_as_uint(x + 0.0f);  // -0 + 0 = 0
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float number(uint32_t k) {
    if (k == 0) return NAN;
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}

// Where a unit's score comes from: it is its one weight, the sums of unit_score_kernel, or (units of
// one token) the sum over the heads here.
enum class Score { kWeight, kSums, kHeads };

// score of unit u of a set
template <Score kFrom>
__device__ __forceinline__ float score_of(const SelectArgs& a, int64_t set, int64_t u) {
    const int64_t item = set * a.n_units + u;
    if constexpr (kFrom == Score::kWeight) {
        return a.weight[item];
    } else {
        double s = 0.0;
        if constexpr (kFrom == Score::kSums) {
            const int64_t n_items = (int64_t)a.sets * a.n_units;
            for (int p = 0; p < a.splits; ++p) s += a.unit_sum[(int64_t)p * n_items + item];
        } else {
            const float* w = a.weight + set * a.heads * a.n_units + u;
#pragma unroll 1
            for (int h = 0; h < a.heads; ++h) s += (double)w[(int64_t)h * a.n_units];
        }
        return (float)s;
    }
}

constexpr int kSelWaves = 16;
constexpr int kSelThreads = 64 * kSelWaves;
constexpr int kBins = 4096;
constexpr int kList = 2048;
constexpr int kEnds = 8;
constexpr size_t kSelLds = 128 << 10;  // of keys: with the histogram and the list below a compute unit's 160 KiB

// lanes below this one in a ballot
__device__ __forceinline__ unsigned lanes_below(uint64_t who) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
}

// one more in a bin of hist for every lane that is in; equal bins of a wave together
__device__ __forceinline__ void count_bin(unsigned* hist, bool in, unsigned bin, int lane) {
    const uint64_t who = __ballot(in);
    if (who == 0) return;
    const int leader = __builtin_ctzll(who);
    const unsigned bin0 = __builtin_amdgcn_readlane(bin, leader);
    if (__ballot(in && bin == bin0) == who) {
        if (lane == leader) atomicAdd(&hist[bin0], (unsigned)__popcll(who));
    } else if (in) {
        atomicAdd(&hist[bin], 1u);
    }
}

// The protected ends of a set, by threads `at` of `step`, eight loads in flight (a store between
// would hold the next load back).
template <Score kFrom>
__device__ __forceinline__ void protected_ends(const SelectArgs& a, int64_t set, int64_t at, int64_t step) {
    const int64_t ends = (int64_t)a.first + a.last;
    int32_t* out = a.out_idx + set * a.keep;
    float* out_score = a.out_score ? a.out_score + set * a.keep : nullptr;
    for (int64_t i0 = at; i0 < ends; i0 += step * kEnds) {
        float x[kEnds];
#pragma unroll
        for (int j = 0; j < kEnds; ++j) {
            const int64_t i = i0 + j * step;
            x[j] = out_score && i < ends ? score_of<kFrom>(a, set, i < a.first ? i : a.n_units - ends + i) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kEnds; ++j) {
            const int64_t i = i0 + j * step;
            if (i >= ends) break;
            const int64_t o = i < a.first ? i : a.keep - ends + i;
            out[o] = (int32_t)(i < a.first ? i : a.n_units - ends + i);
            if (out_score) out_score[o] = x[j];
        }
    }
}

// kLds: the keys to choose from lie in LDS after the first sweep; else every sweep reads the scores again.
template <bool kLds, Score kFrom>
__global__ __launch_bounds__(kSelThreads) void select_kernel(SelectArgs a) {
    extern __shared__ uint32_t keys[];  // kLds: [waves][rounds][64]
    __shared__ unsigned hist[kBins];
    __shared__ unsigned wave_sum[kSelWaves], found[3], wave_gt[kSelWaves], wave_eq[kSelWaves];
    __shared__ uint32_t list_key[kList];  // the units in the first digit's bin, where they fit, and their waves
    __shared__ uint8_t list_wave[kList];
    __shared__ unsigned list_n;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int32_t* out = a.out_idx + (int64_t)blockIdx.x * a.keep;
    float* out_score = a.out_score ? a.out_score + (int64_t)blockIdx.x * a.keep : nullptr;
    auto score = [&](int64_t unit) -> float { return score_of<kFrom>(a, blockIdx.x, unit); };
    const int from_last = a.n_units - a.last;
    protected_ends<kFrom>(a, blockIdx.x, tid, kSelThreads);
    const unsigned m = (unsigned)(a.keep - a.first - a.last);  // to choose from the units between
    if (m == 0) return;  // uniform
    // this wave's share of them: rounds of 64, `count` in all, from u0 on
    const int64_t open = (int64_t)from_last - a.first;
    const int rounds = (int)((open + kSelThreads - 1) / kSelThreads);
    const int64_t start = (int64_t)wave * rounds * 64, u0 = a.first + start;
    const int count = (int)max((int64_t)0, min((int64_t)rounds * 64, open - start));
    // f(unit's place in the wave, whether there is one, its key) for this lane's units, eight
    // rounds at a time with their loads in flight together
    auto sweep = [&](auto first_tag, auto f) {
        constexpr bool kFirst = decltype(first_tag)::value;
        constexpr int kBatch = 8;
        for (int r0 = 0; r0 < count; r0 += 64 * kBatch) {
            uint32_t k[kBatch];
            auto batch = [&](auto full_tag) __attribute__((always_inline)) {
                constexpr bool kFull = decltype(full_tag)::value;
                if constexpr (kLds && !kFirst) {
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) k[j] = kFull || r0 + j * 64 < count ? keys[start + r0 + j * 64 + lane] : 0u;
                } else {
                    float x[kBatch];
                    if constexpr (kFrom == Score::kHeads) {
                        double s[kBatch] = {};
                        const float* w = a.weight + (int64_t)blockIdx.x * a.heads * a.n_units + u0 + r0 + lane;
#pragma unroll 1
                        for (int h = 0; h < a.heads; ++h, w += a.n_units)
#pragma unroll
                            for (int j = 0; j < kBatch; ++j) s[j] += kFull || r0 + j * 64 + lane < count ? (double)w[j * 64] : 0.0;
#pragma unroll
                        for (int j = 0; j < kBatch; ++j) x[j] = (float)s[j];
                    } else {
#pragma unroll
                        for (int j = 0; j < kBatch; ++j) x[j] = kFull || r0 + j * 64 + lane < count ? score(u0 + r0 + j * 64 + lane) : 0.0f;
                    }
#pragma unroll
                    for (int j = 0; j < kBatch; ++j) {
                        k[j] = ordered(x[j]);
                        if (kLds && (kFull || r0 + j * 64 < count)) keys[start + r0 + j * 64 + lane] = k[j];
                    }
                }
#pragma unroll
                for (int j = 0; j < kBatch; ++j) {
                    if (kFull || r0 + j * 64 < count) f(r0 + j * 64 + lane, kFull || r0 + j * 64 + lane < count, k[j]);
                }
            };
            if (r0 + 64 * kBatch <= count) batch(std::true_type{});  // uniform
            else batch(std::false_type{});
        }
    };

    // the m-th largest: its leading digits so far, and how many equal to it are taken
    uint32_t prefix = 0, mask = 0;
    unsigned want = m;
    bool listed = false;
    if (tid == 0) list_n = 0;
#pragma unroll
    for (int digit = 0; digit < 3; ++digit) {
        constexpr int kShift[3] = {20, 10, 0};
        const int shift = kShift[digit], bins = digit == 0 ? kBins : 1024;
        for (int b = tid; b < bins; b += kSelThreads) hist[b] = 0;
        __syncthreads();
        auto count_in = [&](int, bool have, uint32_t k) { count_bin(hist, have && (k & mask) == prefix, (k >> shift) & (bins - 1), lane); };
        if (digit > 0 && listed) {
            for (unsigned i = tid - lane; i < list_n; i += kSelThreads) count_in(0, i + lane < list_n, list_key[(i + lane) % kList]);
        } else if (digit == 0) {
            sweep(std::true_type{}, count_in);
        } else {
            sweep(std::false_type{}, count_in);
        }
        __syncthreads();
        // each thread takes some bins, from the highest down: the one where the count from above reaches `want`
        const int per = bins / kSelThreads;
        unsigned own[kBins / kSelThreads], mine = 0;
#pragma unroll
        for (int b = 0; b < kBins / kSelThreads; ++b) {
            own[b] = b < per ? hist[bins - 1 - (tid * per + b)] : 0;
            mine += own[b];
        }
        unsigned upto = mine;  // of this wave's lanes up to this one
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const unsigned y = __shfl_up(upto, d);
            if (lane >= d) upto += y;
        }
        if (lane == 63) wave_sum[wave] = upto;
        __syncthreads();
        unsigned above = upto - mine;
        for (int w = 0; w < wave; ++w) above += wave_sum[w];
#pragma unroll
        for (int b = 0; b < kBins / kSelThreads; ++b) {
            if (b < per && above < want && above + own[b] >= want) {
                found[0] = (unsigned)(bins - 1 - (tid * per + b));
                found[1] = want - above;
                found[2] = own[b];
            }
            above += own[b];
        }
        __syncthreads();
        prefix |= __builtin_amdgcn_readfirstlane(found[0]) << shift;
        mask |= (unsigned)(bins - 1) << shift;
        want = __builtin_amdgcn_readfirstlane(found[1]);
        if (digit == 0 && __builtin_amdgcn_readfirstlane(found[2]) <= kList) {
            // few enough in the bin: they are listed, and the waves count what lies above it
            listed = true;
            unsigned gt = 0;
            sweep(std::false_type{}, [&](int, bool have, uint32_t k) {
                const uint32_t top = k & mask;
                gt += __popcll(__ballot(have && top > prefix));
                const bool in = have && top == prefix;
                const uint64_t who = __ballot(in);
                if (who == 0) return;
                unsigned at = 0;
                const int leader = __builtin_ctzll(who);
                if (lane == leader) at = atomicAdd(&list_n, (unsigned)__popcll(who));
                at = __builtin_amdgcn_readlane(at, leader) + lanes_below(who);
                if (in) {
                    list_key[at] = k;
                    list_wave[at] = (uint8_t)wave;
                }
            });
            if (lane == 0) {
                wave_gt[wave] = gt;
                wave_eq[wave] = 0;
            }
        }
    }

    // what each wave keeps: above the threshold, and equal to it
    if (listed) {
        for (unsigned i = tid; i < list_n; i += kSelThreads) {
            const uint32_t k = list_key[i];
            if (k > prefix) atomicAdd(&wave_gt[list_wave[i]], 1u);
            else if (k == prefix) atomicAdd(&wave_eq[list_wave[i]], 1u);
        }
    } else {
        unsigned gt = 0, eq = 0;
        sweep(std::false_type{}, [&](int, bool have, uint32_t k) {
            gt += __popcll(__ballot(have && k > prefix));
            eq += __popcll(__ballot(have && k == prefix));
        });
        if (lane == 0) {
            wave_gt[wave] = gt;
            wave_eq[wave] = eq;
        }
    }
    __syncthreads();
    unsigned at = a.first, eq_before = 0, eq_all = 0;
    for (int w = 0; w < kSelWaves; ++w) {
        if (w < wave) {
            at += wave_gt[w];
            eq_before += wave_eq[w];
        }
        eq_all += wave_eq[w];
    }
    at += min(eq_before, want);
    const bool all_equal = eq_all == want;  // nothing equal to the threshold is left out
    sweep(std::false_type{}, [&](int i, bool have, uint32_t k) {
        bool keep = have && k >= prefix;
        if (!all_equal) {
            const bool same = have && k == prefix;
            const uint64_t same_mask = __ballot(same);
            if (same) keep = eq_before + lanes_below(same_mask) < want;
            eq_before += __popcll(same_mask);
        }
        const uint64_t keep_mask = __ballot(keep);
        if (keep) {
            const unsigned o = at + lanes_below(keep_mask);
            out[o] = (int32_t)(u0 + i);
            if (out_score) out_score[o] = number(k);
        }
        at += __popcll(keep_mask);
    });
}

// ---------------------------------------------------------------------------
// Long sets: a set's units to choose from are shared out over workgroups, in shares of
// whole blocks of kWideUnits. Three launches: wide_count_kernel leaves every
// share's histogram of the first digit; wide_list_kernel finds from all of a
// set's the bin that holds the threshold and lists the keys in it, the shares' one
// behind the other; wide_write_kernel finds the threshold in the list
// (each workgroup for itself), how many the shares before its own keep, and
// writes its own. Nothing is added atomically outside a workgroup, so the
// workspace needs no clearing.
// ---------------------------------------------------------------------------
constexpr int kWideRounds = 4;
constexpr int kWideUnits = kSelThreads * kWideRounds;
constexpr int kWideGroups = 256;          // workgroups of a launch: one per compute unit
constexpr int64_t kWideFrom = 31000, kWideFromTwo = 50000;  // (wide_shares)
// where a workgroup is, and its set's part of the workspace: per share the histogram, its sums over
// 64 bins and the range of the listed keys, and the list
struct Wide {
    int64_t set, open, u0;  // u0: the share's first unit
    int share, shares, blocks;
    unsigned m;
    uint32_t *fine, *coarse, *range, *list;
};
__device__ __forceinline__ Wide wide_of(const SelectArgs& a) {
    Wide x;
    x.open = (int64_t)a.n_units - a.first - a.last;
    x.shares = a.shares;
    x.blocks = a.share_blocks;
    x.set = blockIdx.x / (unsigned)a.shares;
    x.share = (int)(blockIdx.x - (unsigned)x.set * (unsigned)a.shares);
    x.u0 = a.first + (int64_t)x.share * a.share_blocks * kWideUnits;
    x.m = (unsigned)(a.keep - a.first - a.last);
    x.fine = a.wide + x.set * a.shares * kBins;
    x.coarse = a.wide + (int64_t)a.sets * a.shares * kBins + x.set * a.shares * 64;
    x.range = a.wide + (int64_t)a.sets * a.shares * (kBins + 64) + x.set * a.shares * 2;
    x.list = a.wide + (int64_t)a.sets * a.shares * (kBins + 66) + x.set * a.n_units;
    return x;
}
// keys of block b of a share: k[j] of unit base + 64 j + lane of it, for those below `left`
template <Score kFrom>
__device__ __forceinline__ int64_t wide_load(const SelectArgs& a, const Wide& x, int b, int wave, int lane, uint32_t (&k)[kWideRounds],
                                             bool (&have)[kWideRounds]) {
    const int64_t u = x.u0 + (int64_t)b * kWideUnits + wave * 64 * kWideRounds;
    const int64_t left = a.first + x.open - u;
    float s[kWideRounds];
#pragma unroll
    for (int j = 0; j < kWideRounds; ++j) {
        have[j] = 64 * j + lane < left;
        s[j] = have[j] ? score_of<kFrom>(a, x.set, u + 64 * j + lane) : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < kWideRounds; ++j) k[j] = ordered(s[j]);
    return u;
}

template <Score kFrom>
__global__ __launch_bounds__(kSelThreads) void wide_count_kernel(SelectArgs a) {
    __shared__ __attribute__((aligned(16))) unsigned hist[kBins];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Wide x = wide_of(a);
    for (int b = tid; b < kBins; b += kSelThreads) hist[b] = 0;
    __syncthreads();
    for (int b = 0; b < x.blocks; ++b) {
        uint32_t k[kWideRounds];
        bool have[kWideRounds];
        wide_load<kFrom>(a, x, b, wave, lane, k, have);
#pragma unroll
        for (int j = 0; j < kWideRounds; ++j) count_bin(hist, have[j], k[j] >> 20, lane);
    }
    protected_ends<kFrom>(a, x.set, (int64_t)x.share * kSelThreads + tid, (int64_t)x.shares * kSelThreads);
    __syncthreads();
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    static_assert(kBins == 4 * kSelThreads, "four bins a thread");
    const u32x4 own = *reinterpret_cast<const u32x4*>(hist + 4 * tid);
    *reinterpret_cast<u32x4*>(x.fine + (int64_t)x.share * kBins + 4 * tid) = own;
    unsigned sum = own[0] + own[1] + own[2] + own[3];  // of 64 bins: 16 threads
#pragma unroll
    for (int d = 1; d < 16; d *= 2) sum += __shfl_xor(sum, d);
    if ((tid & 15) == 0) x.coarse[x.share * 64 + tid / 16] = sum;
}

// Of 64 bins in every share (lane's bin at p[share * stride + lane]): the one where the count from the
// highest down reaches `want`.
struct WideBin {
    unsigned bin, want;     // in 0..63; how many are taken from it
    unsigned all;           // units in it
    unsigned before, above_before;  // in the shares before this workgroup's: in it, and above it
};
__device__ __forceinline__ WideBin wide_find(const Wide& x, const uint32_t* p, int stride, unsigned want, unsigned (*lds)[2][64], int wave, int lane) {
    unsigned all = 0, before = 0;
    for (int s0 = wave; s0 < x.shares; s0 += kSelWaves * 4) {
        unsigned v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = s0 + i * kSelWaves;
            v[i] = s < x.shares ? p[(int64_t)s * stride + lane] : 0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            all += v[i];
            before += s0 + i * kSelWaves < x.share ? v[i] : 0;
        }
    }
    lds[wave][0][lane] = all;
    lds[wave][1][lane] = before;
    __syncthreads();
    all = before = 0;
#pragma unroll
    for (int w = 0; w < kSelWaves; ++w) {
        all += lds[w][0][lane];
        before += lds[w][1][lane];
    }
    unsigned from = all, before_from = before;  // of this bin and those above
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const unsigned y = __shfl_down(from, d), z = __shfl_down(before_from, d);
        if (lane + d < 64) {
            from += y;
            before_from += z;
        }
    }
    const int at = __builtin_ctzll(__ballot(from >= want && from - all < want));
    WideBin r;
    r.bin = at;
    r.all = __builtin_amdgcn_readlane(all, at);
    r.want = want - (__builtin_amdgcn_readlane(from, at) - r.all);
    r.before = __builtin_amdgcn_readlane(before, at);
    r.above_before = __builtin_amdgcn_readlane(before_from, at) - r.before;
    return r;
}
// the same of the first digit's bins
__device__ __forceinline__ WideBin wide_digit(const Wide& x, unsigned (*lds)[kSelWaves][2][64], int wave, int lane) {
    const WideBin c = wide_find(x, x.coarse, 64, x.m, lds[0], wave, lane);
    WideBin f = wide_find(x, x.fine + c.bin * 64, kBins, c.want, lds[1], wave, lane);
    f.bin += c.bin * 64;
    f.above_before += c.above_before;
    return f;
}

template <Score kFrom>
__global__ __launch_bounds__(kSelThreads) void wide_list_kernel(SelectArgs a) {
    __shared__ unsigned sums[2][kSelWaves][2][64];
    __shared__ unsigned list_n, lo, hi;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Wide x = wide_of(a);
    if (tid == 0) {
        list_n = 0;
        lo = ~0u;
        hi = 0;
    }
    const WideBin d = wide_digit(x, sums, wave, lane);  // (with barriers)
    uint32_t least = ~0u, most = 0;
    for (int b = 0; b < x.blocks; ++b) {
        uint32_t k[kWideRounds];
        bool have[kWideRounds];
        wide_load<kFrom>(a, x, b, wave, lane, k, have);
#pragma unroll
        for (int j = 0; j < kWideRounds; ++j) {
            const bool in = have[j] && k[j] >> 20 == d.bin;
            const uint64_t who = __ballot(in);
            if (who == 0) continue;
            const int leader = __builtin_ctzll(who);
            unsigned at = 0;
            if (lane == leader) at = atomicAdd(&list_n, (unsigned)__popcll(who));
            at = __builtin_amdgcn_readlane(at, leader) + lanes_below(who);
            if (in) {
                x.list[d.before + at] = k[j];
                least = min(least, k[j]);
                most = max(most, k[j]);
            }
        }
    }
#pragma unroll
    for (int s = 32; s > 0; s /= 2) {
        least = min(least, (uint32_t)__shfl_xor(least, s));
        most = max(most, (uint32_t)__shfl_xor(most, s));
    }
    if (lane == 0 && least <= most) {
        atomicMin(&lo, least);
        atomicMax(&hi, most);
    }
    __syncthreads();
    if (tid < 2) x.range[2 * x.share + tid] = tid ? hi : lo;
}

template <Score kFrom>
__global__ __launch_bounds__(kSelThreads) void wide_write_kernel(SelectArgs a) {
    __shared__ unsigned sums[2][kSelWaves][2][64];
    __shared__ unsigned hist[2][1024], wave_sum[2][kSelWaves], found[2][2], counts[2], range[2];
    __shared__ unsigned wave_gt[2][kSelWaves], wave_eq[2][kSelWaves];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Wide x = wide_of(a);
    static_assert(kSelThreads == 1024, "one bin a thread");
    hist[0][tid] = hist[1][tid] = 0;
    if (tid < 2) {
        counts[tid] = 0;
        range[tid] = tid ? 0u : ~0u;
    }
    const WideBin d = wide_digit(x, sums, wave, lane);  // (with barriers)
    for (int s = tid; s < x.shares; s += kSelThreads) {
        atomicMin(&range[0], x.range[2 * s]);
        atomicMax(&range[1], x.range[2 * s + 1]);
    }
    __syncthreads();
    // f(whether there is one, key) of the first n listed
    auto listed = [&](unsigned n, auto f) {
        for (unsigned i0 = tid - lane; i0 < n; i0 += 4 * kSelThreads) {
            uint32_t k[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = i0 + i * kSelThreads + lane < n ? x.list[i0 + i * kSelThreads + lane] : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) f(i0 + i * kSelThreads + lane < n, k[i]);
        }
    };
    // the m-th largest key, how many equal to it are taken, and of the listed keys before this
    // share's how many are larger and equal
    uint32_t prefix = __builtin_amdgcn_readfirstlane(range[0]);
    unsigned want = d.want, gt_before = 0, eq_before = d.before;
    bool all_equal = d.want == d.all;
    if (prefix != __builtin_amdgcn_readfirstlane(range[1])) {  // else all of them are equal
        prefix = d.bin << 20;
        uint32_t mask = 0xfffu << 20;
#pragma unroll
        for (int digit = 0; digit < 2; ++digit) {
            const int shift = digit == 0 ? 10 : 0;
            listed(d.all, [&](bool have, uint32_t k) { count_bin(hist[digit], have && (k & mask) == prefix, (k >> shift) & 1023, lane); });
            __syncthreads();
            const unsigned own = hist[digit][1023 - tid];  // thread t has the t-th highest bin
            unsigned upto = own;
#pragma unroll
            for (int s = 1; s < 64; s *= 2) {
                const unsigned y = __shfl_up(upto, s);
                if (lane >= s) upto += y;
            }
            if (lane == 63) wave_sum[digit][wave] = upto;
            __syncthreads();
            for (int w = 0; w < wave; ++w) upto += wave_sum[digit][w];
            if (upto >= want && upto - own < want) {
                found[digit][0] = (unsigned)(1023 - tid);
                found[digit][1] = want - (upto - own);
                if (digit == 1) range[0] = own;  // (read by all before the first digit's barriers)
            }
            __syncthreads();
            prefix |= __builtin_amdgcn_readfirstlane(found[digit][0]) << shift;
            mask |= 1023u << shift;
            want = __builtin_amdgcn_readfirstlane(found[digit][1]);
        }
        all_equal = __builtin_amdgcn_readfirstlane(range[0]) == want;
        unsigned gt = 0, eq = 0;
        listed(d.before, [&](bool have, uint32_t k) {
            gt += have && k > prefix;
            eq += have && k == prefix;
        });
#pragma unroll
        for (int s = 32; s > 0; s /= 2) {
            gt += __shfl_xor(gt, s);
            eq += __shfl_xor(eq, s);
        }
        if (lane == 0) {
            atomicAdd(&counts[0], gt);
            atomicAdd(&counts[1], eq);
        }
        __syncthreads();
        gt_before = __builtin_amdgcn_readfirstlane(counts[0]);
        eq_before = __builtin_amdgcn_readfirstlane(counts[1]);
    }
    int32_t* out = a.out_idx + x.set * a.keep;
    float* out_score = a.out_score ? a.out_score + x.set * a.keep : nullptr;
    // places of the keys above the threshold, and of those equal to it, as they come
    unsigned gt_at = a.first + d.above_before + gt_before, eq_at = eq_before;
    for (int b = 0; b < x.blocks; ++b) {
        uint32_t k[kWideRounds];
        bool have[kWideRounds];
        const int64_t u = wide_load<kFrom>(a, x, b, wave, lane, k, have);
        unsigned gt = 0, eq = 0;
#pragma unroll
        for (int j = 0; j < kWideRounds; ++j) {
            gt += __popcll(__ballot(have[j] && k[j] > prefix));
            eq += __popcll(__ballot(have[j] && k[j] == prefix));
        }
        if (lane == 0) {
            wave_gt[b & 1][wave] = gt;
            wave_eq[b & 1][wave] = eq;
        }
        __syncthreads();  // (one per block: the other half of the counts is read before the next)
        unsigned gt_here = gt_at, eq_here = eq_at;
        for (int w = 0; w < kSelWaves; ++w) {
            const unsigned g = wave_gt[b & 1][w], e = wave_eq[b & 1][w];
            gt_here += w < wave ? g : 0;
            eq_here += w < wave ? e : 0;
            gt_at += g;
            eq_at += e;
        }
        unsigned at = gt_here + min(eq_here, want);
#pragma unroll
        for (int j = 0; j < kWideRounds; ++j) {
            bool keep = have[j] && k[j] >= prefix;
            if (!all_equal) {
                const bool same = have[j] && k[j] == prefix;
                const uint64_t same_mask = __ballot(same);
                if (same) keep = eq_here + lanes_below(same_mask) < want;
                eq_here += __popcll(same_mask);
            }
            const uint64_t keep_mask = __ballot(keep);
            if (keep) {
                const unsigned o = at + lanes_below(keep_mask);
                out[o] = (int32_t)(u + 64 * j + lane);
                if (out_score) out_score[o] = number(k[j]);
            }
            at += __popcll(keep_mask);
        }
    }
}

// Up to 64 units, whose scores x the lanes of one wave hold: of those to choose from
// one is kept if fewer than m come before it.
__device__ __forceinline__ void select_few(const SelectArgs& a, int64_t set, int lane, float x) {
    const uint32_t k = ordered(x);
    const int hi = a.n_units - a.last, m = a.keep - a.first - a.last;
    int before = 0;
    for (int j = a.first; j < hi; ++j) {
        const uint32_t y = __builtin_amdgcn_readlane(k, j);
        before += y > k || (y == k && j < lane) ? 1 : 0;
    }
    const bool open = lane >= a.first && lane < hi;
    const bool keep = lane < a.n_units && (!open || before < m);
    const uint64_t kept = __ballot(keep);
    if (keep) {
        const int64_t o = set * a.keep + lanes_below(kept);
        a.out_idx[o] = lane;
        if (a.out_score) a.out_score[o] = x;
    }
}

template <Score kFrom>
__global__ __launch_bounds__(64) void select_few_kernel(SelectArgs a) {
    const int lane = threadIdx.x;
    select_few(a, blockIdx.x, lane, lane < a.n_units ? score_of<kFrom>(a, blockIdx.x, lane) : 0.0f);
}

// The same from the weights: wave w sums units w, w + 16, ...
__global__ __launch_bounds__(kSelThreads) void select_few_sums_kernel(SelectArgs a, double inv_unit) {
    __shared__ float score[64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t row = (int64_t)a.n_units * a.unit;
    const float* w = a.weight + (int64_t)blockIdx.x * a.heads * row;
    const int total = a.heads * a.unit;  // at most kFewWeights
    for (int u = wave; u < a.n_units; u += kSelWaves) {
        double sum = 0.0;
        for (int e0 = lane; e0 < total; e0 += 64 * 8) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int e = e0 + 64 * k;
                const int h = (int)(((double)e + 0.5) * inv_unit);
                v[k] = e < total ? w[h * row + (int64_t)u * a.unit + (e - h * a.unit)] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += (double)v[k];
        }
#pragma unroll
        for (int k = 32; k > 0; k /= 2) sum += __shfl_xor(sum, k);
        if (lane == 0) score[u] = (float)sum;
    }
    __syncthreads();
    if (wave == 0) select_few(a, blockIdx.x, lane, lane < a.n_units ? score[lane] : 0.0f);
}

template <int G, int VEC>
void launch_scores(const SelectArgs& a, hipStream_t stream) {
    const int64_t n = (int64_t)a.sets * a.n_units;
    const int64_t blocks = (n + kScoreBlock / G - 1) / (kScoreBlock / G);
    dim3 grid = grid_rows((unsigned)blocks);
    grid.z = (unsigned)a.splits;
    hipLaunchKernelGGL((unit_score_kernel<G, VEC>), grid, dim3(kScoreBlock), 0, stream, a, n, 1.0 / (a.unit / VEC));
}

}  // namespace

// How a choice gets its scores. Where a set has few weights its own workgroup adds
// them up: one launch instead of two (one head, 18 units of 390 tokens: 5.9 us
// a call instead of 8.8, 4.6 instead of 5.2 on the device). One compute unit reads
// more weights too slowly (12 heads, 18 units of 130 tokens: 9.4 us on the device, in two launches 6.9).
constexpr int64_t kFewWeights = 1 << 13;
enum class Plan { kWeights, kOwnHeads, kOwnUnits, kSums };

namespace {
Plan plan_of(const SelectArgs& a) {
    if (a.heads == 1 && a.unit == 1) return Plan::kWeights;
    if ((int64_t)a.n_units * a.unit <= kFewWeights / a.heads) {
        if (a.unit == 1) return Plan::kOwnHeads;
        if (a.n_units <= 64) return Plan::kOwnUnits;
    }
    return Plan::kSums;
}
}  // namespace

// Head parts of the scores: where there are fewer long units than two workgroups per
// compute unit of a large chip, the heads share them out.
int32_t select_splits(const SelectArgs& a) {
    const int64_t n = (int64_t)a.sets * a.n_units;
    if (plan_of(a) != Plan::kSums || n == 0 || n >= 512 || (int64_t)a.heads * a.unit < 8192) return 1;
    const int64_t want = (512 + n - 1) / n;
    return (int32_t)(want < a.heads ? want : a.heads);
}

// Shares of a long set, 0 where one workgroup chooses from all of it. Where its keys do not lie in LDS, that one takes 8 us and
// 0.5 to 0.6 ns per unit, the three launches 17 us and 4.3 per block of a share: up to one block each 21. They
// pay from n (1 - 1 / shares) = 31000 on, with two shares, whose blocks fill only half of the chip's time, from n = 100000. One
// workgroup against shares, us (spread scores; a tenth and a twentieth of the units protected): one or eight sets
// of 36000 22.5, 20.9; 51 of 42000 29.5, 26.1; 64 of 52000 35.3, 30.7; 85 of 52000 36.0, 34.7; 100 of 120000 90.0,
// 74.3; one of 140000 84, 24; of 1000000 657, 38. On the other side of the rule: one of 32700 21.5, 20.5; 51 of
// 36000 23.7, 25.7; 64 of 36000 23.9, 26.0; 85 of 42000 30.5, 30.8; 100 of 90000 57.8, 59.5.
// Scores that nearly all lie in one bin of the first digit (within an eighth of each other, but not equal) are all listed, and each
// workgroup searches the whole list: 30 sets of 40000 34.5, 48.3; 128 of 140000 118, 160; one of 131072 91, 71, of 1000000
// 700, 443. Equal scores are quicker than spread ones (one of 1000000 820, 26).
static int32_t wide_shares(const SelectArgs& a) {
    if (a.sets < 1 || a.sets > kWideGroups / 2) return 0;
    const int64_t n = a.n_units, most = (n + kWideUnits - 1) / kWideUnits;
    const int64_t shares = most < kWideGroups / a.sets ? most : kWideGroups / a.sets;
    return n * (shares - 1) > (shares == 2 ? kWideFromTwo : kWideFrom) * shares ? (int32_t)shares : 0;
}

// the workspace: unit sums in double, then what the workgroups of a long set share
static size_t sum_bytes(const SelectArgs& a) {
    return plan_of(a) == Plan::kSums ? (size_t)a.sets * a.n_units * select_splits(a) * sizeof(double) : 0;
}
size_t select_workspace_bytes(const SelectArgs& a) {
    size_t bytes = sum_bytes(a);
    if (const int32_t shares = wide_shares(a)) {
        bytes = (bytes + 15) / 16 * 16;
        bytes += ((size_t)a.sets * shares * (kBins + 66) + (size_t)a.sets * a.n_units) * sizeof(uint32_t);
    }
    return bytes;
}

hipError_t launch_select(const SelectArgs& a, hipStream_t stream) {
    const Plan plan = plan_of(a);
    if (plan == Plan::kOwnUnits) {
        hipLaunchKernelGGL(select_few_sums_kernel, dim3(a.sets), dim3(kSelThreads), 0, stream, a, 1.0 / a.unit);
        return hipGetLastError();
    }
    if (plan == Plan::kSums) {
        const bool vec = a.unit % 4 == 0 && (uintptr_t)a.weight % 16 == 0;
        // lanes for a unit by its loads, so that a lane has a few rounds of four; units of few tokens one lane
        // each, whose neighbours' words lie beside its own
        const int64_t loads = (int64_t)(a.heads / a.splits) * (vec ? a.unit / 4 : a.unit);
        if (a.unit < 8) launch_scores<1, 1>(a, stream);
        else if (loads >= 1024) vec ? launch_scores<256, 4>(a, stream) : launch_scores<256, 1>(a, stream);
        else if (loads >= 64) vec ? launch_scores<64, 4>(a, stream) : launch_scores<64, 1>(a, stream);
        else vec ? launch_scores<8, 4>(a, stream) : launch_scores<8, 1>(a, stream);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    auto run = [&](auto from) {
        constexpr Score kFrom = decltype(from)::value;
        if (a.n_units <= 64) {
            hipLaunchKernelGGL(select_few_kernel<kFrom>, dim3(a.sets), dim3(64), 0, stream, a);
            return;
        }
        const int64_t open = (int64_t)a.n_units - a.first - a.last;
        if (wide_shares(a) > 0) {
            if constexpr (kFrom != Score::kHeads) {
                SelectArgs b = a;
                b.wide = reinterpret_cast<uint32_t*>(reinterpret_cast<char*>(a.unit_sum) + (sum_bytes(a) + 15) / 16 * 16);
                b.shares = wide_shares(a);
                b.share_blocks = (int32_t)((open + (int64_t)b.shares * kWideUnits - 1) / ((int64_t)b.shares * kWideUnits));
                const dim3 grid(a.sets * b.shares);
                hipLaunchKernelGGL(wide_count_kernel<kFrom>, grid, dim3(kSelThreads), 0, stream, b);
                if (a.keep == a.first + a.last) return;  // nothing to choose
                hipLaunchKernelGGL(wide_list_kernel<kFrom>, grid, dim3(kSelThreads), 0, stream, b);
                hipLaunchKernelGGL(wide_write_kernel<kFrom>, grid, dim3(kSelThreads), 0, stream, b);
            }
            return;
        }
        const size_t lds = (size_t)((open + kSelThreads - 1) / kSelThreads) * kSelThreads * sizeof(uint32_t);
        // (the few weights of kHeads always fit)
        if (kFrom == Score::kHeads || lds <= kSelLds) hipLaunchKernelGGL((select_kernel<true, kFrom>), dim3(a.sets), dim3(kSelThreads), lds, stream, a);
        else if constexpr (kFrom != Score::kHeads) hipLaunchKernelGGL((select_kernel<false, kFrom>), dim3(a.sets), dim3(kSelThreads), 0, stream, a);
    };
    if (plan == Plan::kWeights) run(std::integral_constant<Score, Score::kWeight>{});
    else if (plan == Plan::kOwnHeads) run(std::integral_constant<Score, Score::kHeads>{});
    else run(std::integral_constant<Score, Score::kSums>{});
    return hipGetLastError();
}

}  // namespace revisit
