// The choice of what a cache keeps (select_kept): unit scores and the largest of
// them, in order.

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "internal.h"

namespace revisit {
namespace {

// Unit scores: the sum of a unit's weights over its tokens and the set's heads,
// in double (in any order it is within 2^-40 or so of the sum, so the one
// rounding to fp32 gives what a reader of the definition gets). One block per unit.
__global__ __launch_bounds__(256) void unit_score_kernel(SelectArgs a, unsigned n_items) {
    const unsigned item = row_block();
    if (item >= n_items) return;
    const unsigned set = item / (unsigned)a.n_units, u = item - set * (unsigned)a.n_units;
    const int64_t row = (int64_t)a.n_units * a.unit;
    const float* w = a.weight + (int64_t)set * a.heads * row + (int64_t)u * a.unit;
    double sum = 0.0;
    for (int h = 0; h < a.heads; ++h)
        for (int i = threadIdx.x; i < a.unit; i += 256) sum += (double)w[h * row + i];
    __shared__ double lds[256];
    lds[threadIdx.x] = sum;
    __syncthreads();
    for (int k = 128; k > 0; k /= 2) {
        if ((int)threadIdx.x < k) lds[threadIdx.x] += lds[threadIdx.x + k];
        __syncthreads();
    }
    if (threadIdx.x == 0) a.unit_score[item] = (float)lds[0];
}

// fp32 as an unsigned number in the same order: NaN below all, -0 equal to 0
__device__ __forceinline__ uint32_t ordered(float x) {
    if (__builtin_isnan(x)) return 0;
    uint32_t u = __float_as_uint(x);
    if (u == 0x80000000u) u = 0;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

constexpr int kSelThreads = 1024;

__global__ __launch_bounds__(kSelThreads) void select_kernel(SelectArgs a, const float* score) {
    __shared__ unsigned hist[256];
    __shared__ unsigned sh_digit, sh_want, wave_n[2][kSelThreads / 64];
    const int tid = threadIdx.x;
    const float* s = score + (int64_t)blockIdx.x * a.n_units;
    int32_t* out = a.out_idx + (int64_t)blockIdx.x * a.keep;
    float* out_score = a.out_score ? a.out_score + (int64_t)blockIdx.x * a.keep : nullptr;
    const int lo = a.first, hi = a.n_units - a.last;
    const unsigned m = (unsigned)(a.keep - a.first - a.last);  // to choose of [lo, hi)
    // the m-th largest of them, digit by digit; `want` of those equal to it are taken
    uint32_t prefix = 0, mask = 0;
    unsigned want = m;
    for (int shift = 24; shift >= 0 && m > 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i = lo + tid; i < hi; i += kSelThreads) {
            const uint32_t k = ordered(s[i]);
            if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            unsigned left = want;
            int d = 255;
            while (d > 0 && hist[d] < left) left -= hist[d--];
            sh_digit = d;
            sh_want = left;
        }
        __syncthreads();
        prefix |= sh_digit << shift;
        mask |= 255u << shift;
        want = sh_want;
        __syncthreads();
    }
    // the kept ones in order: all of the protected ends, what is above the threshold and the first `want` equal to it
    unsigned base = 0, equal = 0;
    for (int i0 = 0; i0 < a.n_units; i0 += kSelThreads) {
        const int i = i0 + tid;
        const bool in = i < a.n_units, open = in && i >= lo && i < hi;
        const uint32_t k = open ? ordered(s[i]) : 0;
        const bool eq = open && m > 0 && k == prefix;
        const uint64_t eq_mask = __ballot(eq);
        const int wv = tid >> 6, lane = tid & 63;
        const uint64_t below = ((uint64_t)1 << lane) - 1;
        if (lane == 0) wave_n[0][wv] = __popcll(eq_mask);
        __syncthreads();
        unsigned eq_before = equal + __popcll(eq_mask & below), eq_all = 0;
        for (int j = 0; j < kSelThreads / 64; ++j) {
            if (j < wv) eq_before += wave_n[0][j];
            eq_all += wave_n[0][j];
        }
        const bool keep = in && (!open || (m > 0 && (k > prefix || (eq && eq_before < want))));
        const uint64_t keep_mask = __ballot(keep);
        if (lane == 0) wave_n[1][wv] = __popcll(keep_mask);
        __syncthreads();
        unsigned at = base + __popcll(keep_mask & below), all = 0;
        for (int j = 0; j < kSelThreads / 64; ++j) {
            if (j < wv) at += wave_n[1][j];
            all += wave_n[1][j];
        }
        if (keep) {
            out[at] = i;
            if (out_score) out_score[at] = s[i];
        }
        base += all;
        equal += eq_all;
        __syncthreads();
    }
}

}  // namespace

bool select_sums(const SelectArgs& a) { return a.heads > 1 || a.unit > 1; }

size_t select_workspace_bytes(const SelectArgs& a) { return select_sums(a) ? (size_t)a.sets * a.n_units * sizeof(float) : 0; }

hipError_t launch_select(const SelectArgs& a, hipStream_t stream) {
    const float* score = a.weight;
    if (select_sums(a)) {
        const unsigned n = (unsigned)((int64_t)a.sets * a.n_units);
        hipLaunchKernelGGL(unit_score_kernel, grid_rows(n), dim3(256), 0, stream, a, n);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        score = a.unit_score;
    }
    hipLaunchKernelGGL(select_kernel, dim3(a.sets), dim3(kSelThreads), 0, stream, a, score);
    return hipGetLastError();
}

}  // namespace revisit
