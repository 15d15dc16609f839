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
// keeps, one barrier gives each its place, and the units are written in order.
// Bound by its instructions (60 per round of 64 units and wave) on one compute unit
// per set: 96 sets of 37440 tokens 26 us, with the keys in registers and code unrolled over them 31, with
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
    // the protected ends, eight loads in flight (a store between would hold the next load back)
    const int from_last = a.n_units - a.last;
    for (int i0 = tid; i0 < a.first + a.last; i0 += kSelThreads * kEnds) {
        float x[kEnds];
#pragma unroll
        for (int j = 0; j < kEnds; ++j) {
            const int i = i0 + j * kSelThreads;
            x[j] = out_score && i < a.first + a.last ? score(i < a.first ? i : from_last + (i - a.first)) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < kEnds; ++j) {
            const int i = i0 + j * kSelThreads;
            if (i >= a.first + a.last) break;
            const int o = i < a.first ? i : a.keep - a.last + (i - a.first);
            out[o] = i < a.first ? i : from_last + (i - a.first);
            if (out_score) out_score[o] = x[j];
        }
    }
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
        auto count_in = [&](int, bool have, uint32_t k) {
            const bool in = have && (k & mask) == prefix;
            const uint64_t who = __ballot(in);
            if (who == 0) return;
            const unsigned bin = (k >> shift) & (bins - 1);
            const int leader = __builtin_ctzll(who);
            const unsigned bin0 = __builtin_amdgcn_readlane(bin, leader);
            if (__ballot(in && bin == bin0) == who) {
                if (lane == leader) atomicAdd(&hist[bin0], (unsigned)__popcll(who));
            } else if (in) {
                atomicAdd(&hist[bin], 1u);
            }
        };
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

size_t select_workspace_bytes(const SelectArgs& a) {
    return plan_of(a) == Plan::kSums ? (size_t)a.sets * a.n_units * select_splits(a) * sizeof(double) : 0;
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
