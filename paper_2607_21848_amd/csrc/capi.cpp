// C entry points of librevisit: argument validation on the host, then the
// kernel launches on the caller's stream. The only state is a per-thread
// last-error string; scratch memory comes from the caller (workspace
// arguments sized by the rc_*_workspace_size queries). The streaming driver's
// entry points are in stream.cpp.

#include <math.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include <utility>

#include <hip/hip_runtime.h>

#include "../../include/revisit.h"
#include "internal.h"

namespace {

thread_local char g_last_error[512] = "";

int fail(int status, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
    va_end(ap);
    return status;
}

int launched(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(REVISIT_ERR_LAUNCH, "%s: launch failed: %s", what, hipGetErrorString(e));
    return REVISIT_OK;
}

bool finite(float x) { return isfinite(x); }

bool aligned(const void* ptr, uintptr_t bytes) { return ((uintptr_t)ptr % bytes) == 0; }

constexpr int64_t kMaxElems = (int64_t)1 << 40;
constexpr int kMaxFrames = 1024;
constexpr int kMaxGridSide = 256;  // token-grid rows / columns of the bf16 kernel's bias tables
constexpr int kMaxKeyParts = 64;
constexpr uintptr_t kWorkspaceAlign = 16;

// Checks a caller's workspace against the bytes a call needs.
int check_workspace(const char* fn, size_t need, const void* ws, size_t ws_bytes) {
    if (need == 0) return REVISIT_OK;
    if (ws_bytes < need)
        return fail(REVISIT_ERR_SHAPE, "%s: workspace of %zu bytes given, %zu needed", fn, ws_bytes, need);
    if (!ws) return fail(REVISIT_ERR_NULL, "%s: workspace is NULL (%zu bytes needed)", fn, need);
    if (!aligned(ws, kWorkspaceAlign)) return fail(REVISIT_ERR_SHAPE, "%s: workspace must be 16-byte aligned", fn);
    return REVISIT_OK;
}

// Compute units of the current device.
hipError_t device_compute_units(int* cus) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    return hipDeviceGetAttribute(cus, hipDeviceAttributeMultiprocessorCount, dev);
}

// Shape, dtype and key-part checks shared by biased_chunk_attention and
// rc_attention_workspace_size.
int check_attention_shape(const char* fn, int32_t dtype, int32_t Lq, int32_t Lk, int32_t H, int32_t D,
                          int32_t key_parts) {
    if (dtype != REVISIT_BF16 && dtype != REVISIT_F32 && dtype != REVISIT_FP8_QK)
        return fail(REVISIT_ERR_UNSUPPORTED, "%s: dtype %d not supported", fn, dtype);
    if ((dtype == REVISIT_BF16 || dtype == REVISIT_FP8_QK) && D != 128)
        return fail(REVISIT_ERR_UNSUPPORTED, "%s: bf16 / fp8 needs D = 128 (got %d)", fn, D);
    if (dtype == REVISIT_F32 && D != 64 && D != 128)
        return fail(REVISIT_ERR_UNSUPPORTED, "%s: fp32 needs D = 64 or 128 (got %d)", fn, D);
    if (Lq < 0 || Lk < 1 || H < 1) return fail(REVISIT_ERR_SHAPE, "%s: need Lq >= 0, Lk >= 1, H >= 1", fn);
    if (H > 65535) return fail(REVISIT_ERR_SHAPE, "%s: H > 65535", fn);
    if ((int64_t)Lk * H * D > kMaxElems || (int64_t)Lq * H * D > kMaxElems)
        return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    // (head, key part, 128-query tile) workgroups of the bf16 kernel: a 32-bit count
    if (((int64_t)Lq + 127) / 128 * H * kMaxKeyParts > ((int64_t)1 << 31))
        return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    if (key_parts < 0 || key_parts > kMaxKeyParts)
        return fail(REVISIT_ERR_PARAM, "%s: key_parts=%d outside [0, %d]", fn, key_parts, kMaxKeyParts);
    return REVISIT_OK;
}

// Key parts of the bf16 / fp8 kernel for this call (0 = automatic), and the
// workspace bytes they need. AttentionArgs needs only Lq, Lk, H and layers here.
int attention_parts(const char* fn, const revisit::AttentionArgs& a, int32_t key_parts, int32_t* parts,
                    size_t* bytes) {
    int32_t P = key_parts;
    if (P == 0) {
        int cus = 0;
        const hipError_t e = device_compute_units(&cus);
        if (e != hipSuccess) return fail(REVISIT_ERR_LAUNCH, "%s: device query failed: %s", fn, hipGetErrorString(e));
        P = revisit::attention_bf16_key_parts(a, cus);
    }
    const int32_t tiles = (a.Lk + 31) / 32;
    P = P < tiles ? P : tiles;  // at least one key tile per part
    *parts = P;
    *bytes = revisit::attention_bf16_workspace_bytes(a, P);
    return REVISIT_OK;
}

// Key parts whose workspace an automatic call has to bring at least (1: none).
int attention_least_parts(const char* fn, const revisit::AttentionArgs& a, int32_t* parts) {
    int cus = 0;
    const hipError_t e = device_compute_units(&cus);
    if (e != hipSuccess) return fail(REVISIT_ERR_LAUNCH, "%s: device query failed: %s", fn, hipGetErrorString(e));
    *parts = revisit::attention_bf16_least_parts(a, 2 * cus);
    return REVISIT_OK;
}

}  // namespace

namespace revisit {

int retrieve_with_slots(const char* fn, const float* bank_c2w, int32_t n_bank, const float* query_c2w,
                        const int32_t* query_chunk, int32_t n_query, float E, float w_v, float tau_c, float tau_v,
                        int32_t delta, int32_t first_candidate, int32_t k, int32_t* out_idx, float* out_score,
                        int32_t* out_count, int32_t frames_per_chunk, int32_t* out_frame_sel, const StreamSlotsArgs* slots,
                        void* workspace, size_t workspace_bytes, hipStream_t stream) {
    size_t need = 0;
    int st = rc_retrieve_workspace_size(n_bank, n_query, k, &need);
    if (st != REVISIT_OK) return st;
    if (!(finite(E) && E > 0.0f)) return fail(REVISIT_ERR_PARAM, "%s: E must be finite and > 0", fn);
    if (!finite(w_v) || !finite(tau_c) || !finite(tau_v))
        return fail(REVISIT_ERR_PARAM, "%s: w_v, tau_c and tau_v must be finite", fn);
    if (out_frame_sel && (frames_per_chunk < 1 || (int64_t)k * frames_per_chunk > (1 << 20)))
        return fail(REVISIT_ERR_PARAM, "%s: frames_per_chunk=%d invalid", fn, frames_per_chunk);
    if (n_query == 0) return REVISIT_OK;
    if (!query_c2w || !query_chunk || !out_idx || !out_count || (n_bank > 0 && !bank_c2w))
        return fail(REVISIT_ERR_NULL, "%s: required pointer is NULL", fn);
    // the scan reads the pose columns it needs as 8-byte pairs
    if (!aligned(bank_c2w, 8)) return fail(REVISIT_ERR_SHAPE, "%s: bank_c2w must be 8-byte aligned", fn);
    RetrieveArgs a{};
    a.bank_c2w = bank_c2w;
    a.n_bank = n_bank;
    a.query_c2w = query_c2w;
    a.query_chunk = query_chunk;
    a.n_query = n_query;
    a.E = (double)E;
    a.w_v = (double)w_v;
    a.tau_c = (double)tau_c;
    a.cos_tau_v = cos((double)tau_v);
    // above (tau_c E)^2 (1 + 1e-9) the definition's sqrt(x) / E exceeds tau_c: its two roundings move it by
    // 2^-52 of its value. fp32 tau_c and E keep the square between 1e-180 and 1e154 unless it is 0.
    a.reach2 = (a.tau_c * a.E) * (a.tau_c * a.E) * (1.0 + 1e-9);
    a.delta = delta;
    a.first_candidate = first_candidate;
    a.k = k;
    a.out_idx = out_idx;
    a.out_score = out_score;
    a.out_count = out_count;
    a.frames_per_chunk = frames_per_chunk;
    a.out_frame_sel = out_frame_sel;
    a.n_seg = revisit::retrieve_segments(n_bank);
    a.seg_s = nullptr;
    a.seg_j = nullptr;
    if (slots) {
        a.with_slots = 1;
        a.slots = *slots;
    }
    st = check_workspace(fn, need, workspace, workspace_bytes);
    if (st != REVISIT_OK) return st;
    if (a.n_seg > 0) {
        a.seg_s = static_cast<double*>(workspace);
        a.seg_j = reinterpret_cast<int32_t*>(a.seg_s + (size_t)a.n_seg * n_query * k);
    }
    return launched(launch_retrieve(a, stream), fn);
}

int fail_status(int status, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof(g_last_error), fmt, ap);
    va_end(ap);
    return status;
}
}  // namespace revisit

extern "C" {

const char* rc_status_string(int status) {
    switch (status) {
        case REVISIT_OK: return "ok";
        case REVISIT_ERR_NULL: return "null pointer";
        case REVISIT_ERR_SHAPE: return "bad shape";
        case REVISIT_ERR_UNSUPPORTED: return "unsupported";
        case REVISIT_ERR_PARAM: return "bad parameter";
        case REVISIT_ERR_LAUNCH: return "launch error";
        case REVISIT_ERR_MEMORY: return "out of memory";
        default: return "unknown status";
    }
}

const char* rc_last_error(void) { return g_last_error; }

int retrieve_chunks(const float* bank_c2w, int32_t n_bank, const float* query_c2w, const int32_t* query_chunk,
                    int32_t n_query, float E, float w_v, float tau_c, float tau_v, int32_t delta,
                    int32_t first_candidate, int32_t k, int32_t* out_idx, float* out_score, int32_t* out_count,
                    int32_t frames_per_chunk, int32_t* out_frame_sel, void* workspace, size_t workspace_bytes,
                    hipStream_t stream) {
    return revisit::retrieve_with_slots("retrieve_chunks", bank_c2w, n_bank, query_c2w, query_chunk, n_query, E, w_v, tau_c,
                                        tau_v, delta, first_candidate, k, out_idx, out_score, out_count, frames_per_chunk,
                                        out_frame_sel, nullptr, workspace, workspace_bytes, stream);
}

int rc_retrieve_workspace_size(int32_t n_bank, int32_t n_query, int32_t k, size_t* bytes) {
    if (!bytes) return fail(REVISIT_ERR_NULL, "rc_retrieve_workspace_size: bytes is NULL");
    *bytes = 0;
    if (n_bank < 0 || n_query < 0) return fail(REVISIT_ERR_SHAPE, "retrieve_chunks: negative n_bank or n_query");
    if (n_bank > (1 << 30)) return fail(REVISIT_ERR_SHAPE, "retrieve_chunks: n_bank=%d above 2^30", n_bank);
    if (k < 1 || k > REVISIT_MAX_K) return fail(REVISIT_ERR_PARAM, "retrieve_chunks: k=%d outside [1, %d]", k, REVISIT_MAX_K);
    const int32_t n_seg = revisit::retrieve_segments(n_bank);
    if (n_seg > 0 && (int64_t)n_seg * n_query * k > ((int64_t)1 << 31))
        return fail(REVISIT_ERR_SHAPE, "retrieve_chunks: n_bank * n_query too large");
    *bytes = n_seg > 0 ? revisit::retrieve_workspace_bytes(n_bank, n_query, k) : 0;
    return REVISIT_OK;
}

int reproject_correspondence(const float* tgt_depth, const float* tgt_c2w, const float* tgt_K,
                             const float* src_depth, const float* src_c2w, const float* src_K,
                             const int32_t* src_sel, int32_t n_src, int32_t B, int32_t Tq, int32_t S, int32_t h,
                             int32_t w, int32_t p, float eps, float* out_uv, int32_t* out_idx, hipStream_t stream) {
    if (B < 0 || Tq < 0 || S < 0 || h < 1 || w < 1 || p < 1)
        return fail(REVISIT_ERR_SHAPE, "reproject_correspondence: need B, Tq, S >= 0 and h, w, p >= 1");
    if ((int64_t)h * w * p * p > ((int64_t)1 << 28) || (int64_t)h * p > (1 << 20) || (int64_t)w * p > (1 << 20))
        return fail(REVISIT_ERR_SHAPE, "reproject_correspondence: frame too large");
    if ((int64_t)B * Tq * h * w > ((int64_t)1 << 31) - 1 || (int64_t)B * S * Tq * h * w > kMaxElems)
        return fail(REVISIT_ERR_SHAPE, "reproject_correspondence: problem too large");
    if (src_sel && n_src < 0) return fail(REVISIT_ERR_SHAPE, "reproject_correspondence: n_src < 0");
    if (S > 64) return fail(REVISIT_ERR_SHAPE, "reproject_correspondence: more than 64 source frames per problem");
    if (!(finite(eps) && eps >= 0.0f)) return fail(REVISIT_ERR_PARAM, "reproject_correspondence: eps must be finite and >= 0");
    if (B == 0 || Tq == 0 || S == 0) return REVISIT_OK;
    if (!tgt_depth || !tgt_c2w || !tgt_K || !out_uv || !out_idx)
        return fail(REVISIT_ERR_NULL, "reproject_correspondence: required pointer is NULL");
    if ((!src_sel || n_src > 0) && (!src_depth || !src_c2w || !src_K))
        return fail(REVISIT_ERR_NULL, "reproject_correspondence: source pointer is NULL");
    if (!aligned(out_uv, 8) || !aligned(out_idx, 4) || !aligned(tgt_depth, 4) || !aligned(src_depth, 4) ||
        !aligned(src_sel, 4))
        return fail(REVISIT_ERR_SHAPE, "reproject_correspondence: out_uv must be 8-byte aligned, arrays 4-byte");
    revisit::ReprojectArgs a;
    a.tgt_depth = tgt_depth;
    a.tgt_c2w = tgt_c2w;
    a.tgt_K = tgt_K;
    a.src_depth = src_depth;
    a.src_c2w = src_c2w;
    a.src_K = src_K;
    a.src_sel = src_sel;
    a.n_src = src_sel ? n_src : 0;
    a.B = B;
    a.Tq = Tq;
    a.S = S;
    a.h = h;
    a.w = w;
    a.p = p;
    a.eps = (double)eps;
    a.out_uv = out_uv;
    a.out_idx = out_idx;
    a.paired = 0;
    return launched(revisit::launch_reproject(a, stream), "reproject_correspondence");
}

int reproject_rotation(const float* tgt_c2w, const float* tgt_K, const float* src_c2w, const float* src_K,
                       const int32_t* src_sel, int32_t n_src, int32_t B, int32_t Tq, int32_t S, int32_t h, int32_t w,
                       int32_t p, float* out_uv, int32_t* out_idx, hipStream_t stream) {
    if (B < 0 || Tq < 0 || S < 0 || h < 1 || w < 1 || p < 1)
        return fail(REVISIT_ERR_SHAPE, "reproject_rotation: need B, Tq, S >= 0 and h, w, p >= 1");
    if ((int64_t)h * w > ((int64_t)1 << 28))
        return fail(REVISIT_ERR_SHAPE, "reproject_rotation: frame too large");
    if ((int64_t)B * Tq * h * w > ((int64_t)1 << 31) - 1 || (int64_t)B * S * Tq * h * w > kMaxElems)
        return fail(REVISIT_ERR_SHAPE, "reproject_rotation: problem too large");
    if (src_sel && n_src < 0) return fail(REVISIT_ERR_SHAPE, "reproject_rotation: n_src < 0");
    if (S > 64) return fail(REVISIT_ERR_SHAPE, "reproject_rotation: more than 64 source frames per problem");
    if (B == 0 || Tq == 0 || S == 0) return REVISIT_OK;
    if (!tgt_c2w || !tgt_K || !out_uv || !out_idx)
        return fail(REVISIT_ERR_NULL, "reproject_rotation: required pointer is NULL");
    if ((!src_sel || n_src > 0) && (!src_c2w || !src_K))
        return fail(REVISIT_ERR_NULL, "reproject_rotation: source pointer is NULL");
    if (!aligned(out_uv, 8) || !aligned(out_idx, 4) || !aligned(src_sel, 4))
        return fail(REVISIT_ERR_SHAPE, "reproject_rotation: out_uv must be 8-byte aligned, arrays 4-byte");
    revisit::ReprojectArgs a;
    a.tgt_depth = nullptr;
    a.tgt_c2w = tgt_c2w;
    a.tgt_K = tgt_K;
    a.src_depth = nullptr;
    a.src_c2w = src_c2w;
    a.src_K = src_K;
    a.src_sel = src_sel;
    a.n_src = src_sel ? n_src : 0;
    a.B = B;
    a.Tq = Tq;
    a.S = S;
    a.h = h;
    a.w = w;
    a.p = p;
    a.eps = 0.0;
    a.out_uv = out_uv;
    a.out_idx = out_idx;
    a.paired = aligned(out_uv, 16) && aligned(out_idx, 8);
    return launched(revisit::launch_rotation(a, stream), "reproject_rotation");
}

}  // extern "C"

namespace {

// Validation shared by both attention entry points: fills `a` for a launch,
// or returns a non-zero status. *nothing = true when there is nothing to do.
int prepare_attention(const char* fn, const void* q, const void* k, const void* v, void* o, float* lse, int32_t dtype,
                      int32_t Lq, int32_t Lk, int32_t H, int32_t D, int32_t h, int32_t w,
                      const int32_t* kv_frame_slot, const float* corr_uv, const int32_t* corr_idx, int32_t S,
                      float softmax_scale, float lambda, float sigma, int32_t key_parts, revisit::AttentionArgs& a,
                      bool* nothing) {
    *nothing = false;
    int st = check_attention_shape(fn, dtype, Lq, Lk, H, D, key_parts);
    if (st != REVISIT_OK) return st;
    if (h < 1 || w < 1 || S < 0) return fail(REVISIT_ERR_SHAPE, "%s: need h, w >= 1, S >= 0", fn);
    const int64_t hw = (int64_t)h * w;
    if (Lk % hw != 0) return fail(REVISIT_ERR_SHAPE, "%s: Lk=%d not a multiple of h*w=%lld", fn, Lk, (long long)hw);
    if (Lk / hw > kMaxFrames) return fail(REVISIT_ERR_SHAPE, "%s: more than %d KV frames", fn, kMaxFrames);
    if ((int64_t)S * Lq > kMaxElems) return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    if (!(finite(softmax_scale) && softmax_scale > 0.0f))
        return fail(REVISIT_ERR_PARAM, "%s: softmax_scale must be finite and > 0", fn);
    if (!(finite(sigma) && sigma > 0.0f)) return fail(REVISIT_ERR_PARAM, "%s: sigma must be finite and > 0", fn);
    if (!finite(lambda)) return fail(REVISIT_ERR_PARAM, "%s: lambda must be finite", fn);
    const float gamma = lambda / (2.0f * sigma * sigma * softmax_scale);
    if (!finite(gamma)) return fail(REVISIT_ERR_PARAM, "%s: lambda / (2 sigma^2 scale) overflows", fn);
    if (Lq == 0) {
        *nothing = true;
        return REVISIT_OK;
    }
    const bool bias = S > 0 && lambda != 0.0f;
    // the bf16 / fp8 kernel keeps per-column and per-row bias operands of the token grid in LDS
    if (bias && dtype != REVISIT_F32 && (h > kMaxGridSide || w > kMaxGridSide))
        return fail(REVISIT_ERR_SHAPE, "%s: bf16 / fp8 with bias needs h, w <= %d (got %d x %d)", fn, kMaxGridSide, h, w);
    if (!q || !k || !v || !o) return fail(REVISIT_ERR_NULL, "%s: q, k, v and o are required", fn);
    if (bias && (!kv_frame_slot || !corr_uv || !corr_idx))
        return fail(REVISIT_ERR_NULL, "%s: slot table and correspondence map are required when S > 0", fn);
    // the kernels move q/k/v/o rows in 16-byte vectors and u^ pairs in 8-byte ones
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) || !aligned(lse, 4) ||
        (bias && (!aligned(corr_uv, 8) || !aligned(corr_idx, 4) || !aligned(kv_frame_slot, 4))))
        return fail(REVISIT_ERR_SHAPE, "%s: q, k, v, o must be 16-byte aligned, corr_uv 8-byte", fn);
    a.q = q;
    a.k = k;
    a.v = v;
    a.o = o;
    a.lse = lse;
    a.Lq = Lq;
    a.Lk = Lk;
    a.H = H;
    a.D = D;
    a.h = h;
    a.w = w;
    a.slot = kv_frame_slot;
    a.corr_uv = corr_uv;
    a.corr_idx = corr_idx;
    a.S = bias ? S : 0;
    a.softmax_scale = softmax_scale;
    a.lambda = lambda;
    a.sigma = sigma;
    a.fp8_qk = dtype == REVISIT_FP8_QK;
    a.layers = 1;
    a.q_rows = 0;
    a.kv_rows = 0;
    return REVISIT_OK;
}

// The launch with the caller's workspace. The automatic split takes what the
// size query says, or, in a smaller workspace that holds at least the parts of
// attention_bf16_least_parts (none for short key ranges), as many parts as fit.
int run_attention(const char* fn, const revisit::AttentionArgs& a, int32_t dtype, int32_t key_parts, void* workspace,
                  size_t workspace_bytes, hipStream_t stream) {
    if (dtype == REVISIT_F32) return launched(revisit::launch_attention_f32(a, stream), fn);
    int32_t parts = 1;
    size_t need = 0;
    int st = attention_parts(fn, a, key_parts, &parts, &need);
    if (st != REVISIT_OK) return st;
    const bool usable = workspace && aligned(workspace, kWorkspaceAlign);
    if (need > 0 && key_parts == 0 && (workspace_bytes < need || !usable)) {
        int32_t fewest = 1;
        st = attention_least_parts(fn, a, &fewest);
        if (st != REVISIT_OK) return st;
        const size_t least = revisit::attention_bf16_workspace_bytes(a, fewest);
        if (least == 0 || (least <= workspace_bytes && usable)) {
            const size_t have = usable ? workspace_bytes : 0;
            while (parts > 1 && revisit::attention_bf16_workspace_bytes(a, parts) > have) --parts;
            need = 0;  // what remains fits
        }
    }
    st = check_workspace(fn, need, workspace, workspace_bytes);
    if (st != REVISIT_OK) return st;
    return launched(revisit::launch_attention_bf16(a, parts, static_cast<float*>(workspace), stream), fn);
}

}  // namespace

namespace revisit {

int attention_layers(const char* fn, const void* q, const void* k, const void* v, void* o, float* lse, int32_t dtype,
                     int32_t Lq, int32_t Lk, int32_t H, int32_t D, int32_t h, int32_t w, const int32_t* kv_frame_slot,
                     const float* corr_uv, const int32_t* corr_idx, int32_t S, float softmax_scale, float lambda,
                     float sigma, int32_t layers, int32_t q_rows, int32_t kv_rows, void* workspace,
                     size_t workspace_bytes, hipStream_t stream) {
    AttentionArgs a{};
    bool nothing = false;
    const int st = prepare_attention(fn, q, k, v, o, lse, dtype, Lq, Lk, H, D, h, w, kv_frame_slot, corr_uv, corr_idx, S,
                                     softmax_scale, lambda, sigma, 0, a, &nothing);
    if (st != REVISIT_OK || nothing) return st;
    a.layers = layers;
    a.q_rows = q_rows;
    a.kv_rows = kv_rows;
    return run_attention(fn, a, dtype, 0, workspace, workspace_bytes, stream);
}

int attention_layers_workspace(const char* fn, int32_t dtype, int32_t Lq, int32_t Lk, int32_t H, int32_t D,
                               int32_t layers, size_t* bytes) {
    *bytes = 0;
    const int st = check_attention_shape(fn, dtype, Lq, Lk, H, D, 0);
    if (st != REVISIT_OK || dtype == REVISIT_F32 || Lq == 0) return st;
    AttentionArgs a{};
    a.Lq = Lq;
    a.Lk = Lk;
    a.H = H;
    a.layers = layers;
    int32_t parts = 1;
    return attention_parts(fn, a, 0, &parts, bytes);
}

int32_t attention_max_layers(int32_t Lq, int32_t H, int32_t layers) {
    // 32-query items (fp32) or 128-query items in at most 16 parts (bf16, 256 threads each)
    const int64_t per_layer = (((int64_t)Lq + 31) / 32 + 16 * (((int64_t)Lq + 127) / 128)) * H;
    const int64_t most = (((int64_t)1 << 24) - kXcds) / (per_layer > 0 ? per_layer : 1);
    return most < 1 ? 1 : (int32_t)(most < layers ? most : layers);
}

}  // namespace revisit

extern "C" {

int biased_chunk_attention(const void* q, const void* k, const void* v, void* o, float* lse, int32_t dtype,
                           int32_t Lq, int32_t Lk, int32_t H, int32_t D, int32_t h, int32_t w,
                           const int32_t* kv_frame_slot, const float* corr_uv, const int32_t* corr_idx, int32_t S,
                           float softmax_scale, float lambda, float sigma, int32_t key_parts, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
    revisit::AttentionArgs a{};
    bool nothing = false;
    int st = prepare_attention("biased_chunk_attention", q, k, v, o, lse, dtype, Lq, Lk, H, D, h, w, kv_frame_slot,
                               corr_uv, corr_idx, S, softmax_scale, lambda, sigma, key_parts, a, &nothing);
    if (st != REVISIT_OK || nothing) return st;
    return run_attention("biased_chunk_attention", a, dtype, key_parts, workspace, workspace_bytes, stream);
}

int biased_chunk_attention_noalloc(const void* q, const void* k, const void* v, void* o, float* lse, int32_t dtype,
                                   int32_t Lq, int32_t Lk, int32_t H, int32_t D, int32_t h, int32_t w,
                                   const int32_t* kv_frame_slot, const float* corr_uv, const int32_t* corr_idx,
                                   int32_t S, float softmax_scale, float lambda, float sigma, int32_t key_parts,
                                   hipStream_t stream) {
    const char* fn = "biased_chunk_attention_noalloc";
    revisit::AttentionArgs a{};
    bool nothing = false;
    int st = prepare_attention(fn, q, k, v, o, lse, dtype, Lq, Lk, H, D, h, w, kv_frame_slot, corr_uv, corr_idx, S,
                               softmax_scale, lambda, sigma, key_parts, a, &nothing);
    if (st != REVISIT_OK || nothing) return st;
    if (dtype == REVISIT_F32) return launched(revisit::launch_attention_f32(a, stream), fn);
    int32_t parts = 1;
    size_t need = 0;
    st = attention_parts(fn, a, key_parts, &parts, &need);
    if (st != REVISIT_OK) return st;
    if (need > 0 && key_parts == 0) {
        // a call that can do without a workspace leaves the shared array alone
        int32_t least = 1;
        st = attention_least_parts(fn, a, &least);
        if (st != REVISIT_OK) return st;
        if (least == 1) {
            parts = 1;
            need = 0;
        }
    }
    if (need > revisit::kAttentionScratchBytes) {
        if (key_parts != 0)
            return fail(REVISIT_ERR_SHAPE, "%s: %d key parts need %zu bytes of scratch, more than the %zu bytes it holds "
                                           "(use fewer parts, or biased_chunk_attention with a workspace)",
                        fn, parts, need, revisit::kAttentionScratchBytes);
        // the automatic split, cut to the most parts whose partial results fit
        while (parts > 1 && revisit::attention_bf16_workspace_bytes(a, parts) > revisit::kAttentionScratchBytes)
            --parts;
        need = revisit::attention_bf16_workspace_bytes(a, parts);
    }
    float* scratch = nullptr;
    if (need > 0) {
        const hipError_t e = revisit::attention_scratch(&scratch);
        if (e != hipSuccess)
            return fail(REVISIT_ERR_LAUNCH, "%s: device address of the scratch array: %s", fn, hipGetErrorString(e));
    }
    return launched(revisit::launch_attention_bf16(a, parts, scratch, stream), fn);
}

int rc_attention_workspace_size(int32_t dtype, int32_t Lq, int32_t Lk, int32_t H, int32_t D, int32_t key_parts,
                                size_t* bytes) {
    if (!bytes) return fail(REVISIT_ERR_NULL, "rc_attention_workspace_size: bytes is NULL");
    *bytes = 0;
    const int st = check_attention_shape("rc_attention_workspace_size", dtype, Lq, Lk, H, D, key_parts);
    if (st != REVISIT_OK || dtype == REVISIT_F32 || Lq == 0) return st;
    revisit::AttentionArgs a{};
    a.Lq = Lq;
    a.Lk = Lk;
    a.H = H;
    a.layers = 1;
    int32_t parts = 1;
    return attention_parts("rc_attention_workspace_size", a, key_parts, &parts, bytes);
}

int pack_retrieved_kv(const void* store_k, const void* store_v, const int32_t* store_pos, int32_t n_store,
                      const int32_t* sel, int32_t n_sel, int32_t dst_pos, void* cache_k, void* cache_v,
                      int32_t dst_row0, int32_t cache_rows, int32_t n_layers, int32_t dtype, int32_t F, int32_t h,
                      int32_t w, int32_t H, int32_t D, int32_t rope_t_pairs, float rope_theta, hipStream_t stream) {
    if (dtype != REVISIT_BF16 && dtype != REVISIT_F32)
        return fail(REVISIT_ERR_UNSUPPORTED, "pack_retrieved_kv: dtype %d not supported", dtype);
    if (D < 8 || D > 512 || D % 8 != 0)
        return fail(REVISIT_ERR_UNSUPPORTED, "pack_retrieved_kv: D=%d (need a multiple of 8 in [8, 512])", D);
    if (n_store < 0 || n_sel < 0 || n_layers < 0 || F < 1 || h < 1 || w < 1 || H < 1 || dst_row0 < 0 || cache_rows < 0)
        return fail(REVISIT_ERR_SHAPE, "pack_retrieved_kv: need n_store, n_sel, n_layers, dst_row0, cache_rows >= 0 "
                                       "and F, h, w, H >= 1");
    const int64_t T = (int64_t)F * h * w;
    if (T > INT32_MAX) return fail(REVISIT_ERR_SHAPE, "pack_retrieved_kv: F*h*w too large");
    if ((int64_t)dst_row0 + (int64_t)n_sel * T > cache_rows)
        return fail(REVISIT_ERR_SHAPE, "pack_retrieved_kv: %d slots of %lld rows from row %d exceed cache_rows=%d", n_sel,
                    (long long)T, dst_row0, cache_rows);
    const int64_t row = (int64_t)H * D;
    if ((double)n_layers * n_store * T * row > (double)kMaxElems || (double)n_layers * cache_rows * row > (double)kMaxElems)
        return fail(REVISIT_ERR_SHAPE, "pack_retrieved_kv: store or cache too large");
    if (rope_t_pairs < 0 || rope_t_pairs > D / 2)
        return fail(REVISIT_ERR_PARAM, "pack_retrieved_kv: rope_t_pairs=%d outside [0, D/2]", rope_t_pairs);
    if (rope_t_pairs > 0 && !(finite(rope_theta) && rope_theta > 0.0f))
        return fail(REVISIT_ERR_PARAM, "pack_retrieved_kv: rope_theta must be finite and > 0");
    if (n_layers == 0 || n_sel == 0) return REVISIT_OK;
    if (!sel || !cache_k || !cache_v || (n_store > 0 && (!store_k || !store_v)))
        return fail(REVISIT_ERR_NULL, "pack_retrieved_kv: required pointer is NULL");
    // the kernel moves 16-byte vectors
    if (!aligned(store_k, 16) || !aligned(store_v, 16) || !aligned(cache_k, 16) || !aligned(cache_v, 16) ||
        !aligned(sel, 4) || !aligned(store_pos, 4))
        return fail(REVISIT_ERR_SHAPE, "pack_retrieved_kv: store and cache must be 16-byte aligned, sel and store_pos 4-byte");
    revisit::KvPackArgs a{};
    a.store_k = store_k;
    a.store_v = store_v;
    a.store_pos = store_pos;
    a.n_store = n_store;
    a.sel = sel;
    a.n_sel = n_sel;
    a.dst_pos = dst_pos;
    a.cache_k = cache_k;
    a.cache_v = cache_v;
    a.dst_row0 = dst_row0;
    a.cache_rows = cache_rows;
    a.n_layers = n_layers;
    a.esize = dtype == REVISIT_BF16 ? 2 : 4;
    a.F = F;
    a.T = (int32_t)T;
    a.H = H;
    a.D = D;
    a.n_t = rope_t_pairs;
    a.theta = (double)rope_theta;
    if (revisit::kvpack_blocks(a) > INT32_MAX) return fail(REVISIT_ERR_SHAPE, "pack_retrieved_kv: problem too large");
    return launched(revisit::launch_kvpack(a, stream), "pack_retrieved_kv");
}

int pool_token_depth(const float* depth, int32_t n_frames, int32_t h, int32_t w, int32_t p, float* out,
                     hipStream_t stream) {
    if (n_frames < 0 || h < 1 || w < 1 || p < 1)
        return fail(REVISIT_ERR_SHAPE, "pool_token_depth: need n_frames >= 0 and h, w, p >= 1");
    if ((int64_t)h * p > (1 << 20) || (int64_t)w * p > (1 << 20) ||
        (double)n_frames * h * w * p * p > (double)kMaxElems)
        return fail(REVISIT_ERR_SHAPE, "pool_token_depth: depth maps too large");
    if (n_frames == 0) return REVISIT_OK;
    if (!depth || !out) return fail(REVISIT_ERR_NULL, "pool_token_depth: depth and out are required");
    if (!aligned(depth, 4) || !aligned(out, 4)) return fail(REVISIT_ERR_SHAPE, "pool_token_depth: arrays must be 4-byte aligned");
    return launched(revisit::launch_pool_depth(depth, (int64_t)n_frames * h * w, h, w, p, out, stream), "pool_token_depth");
}

}  // extern "C"

namespace {

// Quarter turns per position of a band of n pairs: theta^(-j / n) radians. One power and products
// in long double (256 of them stay within 2^-55): 0.4 us for 22 pairs, as a power in double per pair,
// which is less exact, and against 7 for powers in long double.
void band_quarters(double theta, int n, double* out) {
    if (n == 0) return;
    const long double ratio = powl((long double)theta, -1.0L / n);
    long double q = 2.0L / 3.14159265358979323846264338327950288L;
    for (int j = 0; j < n; ++j, q *= ratio) out[j] = (double)q;
}

// whether two ranges share a byte (an empty one shares none)
bool overlap(const void* a, double a_bytes, const void* b, double b_bytes) {
    if (a_bytes == 0.0 || b_bytes == 0.0) return false;
    const double x = (double)(uintptr_t)a, y = (double)(uintptr_t)b;
    return x < y + b_bytes && y < x + a_bytes;
}

}  // namespace

extern "C" {

int rotary_embed(const void* q, int64_t q_row, const void* k, int64_t k_row, void* q_out, int64_t q_out_row, void* k_out,
                 int64_t k_out_row, int32_t dtype, int32_t n_tokens, int32_t Hq, int32_t Hk, int32_t D, const int32_t* pos,
                 int32_t t0, int32_t h, int32_t w, int32_t pairs_t, int32_t pairs_y, int32_t pairs_x, float theta,
                 int32_t inverse, float q_scale, float k_scale, hipStream_t stream) {
    const char* fn = "rotary_embed";
    if (dtype != REVISIT_BF16 && dtype != REVISIT_F32 && dtype != REVISIT_FP8_QK)
        return fail(REVISIT_ERR_UNSUPPORTED, "%s: dtype %d not supported", fn, dtype);
    if (D < 8 || D > 512 || D % 8 != 0)
        return fail(REVISIT_ERR_UNSUPPORTED, "%s: D=%d (need a multiple of 8 in [8, 512])", fn, D);
    if (n_tokens < 0 || Hq < 1 || Hq > 65535 || (k && (Hk < 1 || Hk > 65535)))
        return fail(REVISIT_ERR_SHAPE, "%s: need n_tokens >= 0 and 1 to 65535 heads", fn);
    if (pairs_t < 0 || pairs_y < 0 || pairs_x < 0 || (int64_t)pairs_t + pairs_y + pairs_x > D / 2)
        return fail(REVISIT_ERR_PARAM, "%s: bands of %d + %d + %d pairs in a head of %d", fn, pairs_t, pairs_y, pairs_x, D / 2);
    if (!(finite(theta) && theta > 0.0f)) return fail(REVISIT_ERR_PARAM, "%s: theta must be finite and > 0", fn);
    if (inverse != 0 && inverse != 1) return fail(REVISIT_ERR_PARAM, "%s: inverse=%d (0 or 1)", fn, inverse);
    const bool fp8 = dtype == REVISIT_FP8_QK;
    if (fp8 && !(finite(q_scale) && q_scale > 0.0f && finite(k_scale) && k_scale > 0.0f))
        return fail(REVISIT_ERR_PARAM, "%s: q_scale and k_scale must be finite and > 0", fn);
    if (!pos && (h < 1 || w < 1 || (int64_t)h * w > INT32_MAX))
        return fail(REVISIT_ERR_SHAPE, "%s: without positions the token grid is needed: h, w >= 1", fn);
    const int esize = dtype == REVISIT_F32 ? 4 : 2, osize = fp8 ? 1 : esize;
    revisit::RotaryArgs a{};
    const void* x[2] = {q, k};
    void* o[2] = {q_out, k_out};
    const int64_t x_row[2] = {q_row, k_row}, o_row[2] = {q_out_row, k_out_row};
    const int32_t heads[2] = {Hq, Hk};
    for (int i = 0; i < 2; ++i) {
        if (i == 1 && !k) break;
        const int64_t row = (int64_t)heads[i] * D;
        if ((double)n_tokens * (double)row > (double)kMaxElems) return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
        const int64_t most = kMaxElems / (n_tokens > 1 ? n_tokens : 1);
        if (x_row[i] < row || o_row[i] < row || x_row[i] > most || o_row[i] > most)
            return fail(REVISIT_ERR_SHAPE, "%s: a row stride is below the row's %lld elements or too large", fn, (long long)row);
        if (x_row[i] * esize % 16 != 0 || o_row[i] * osize % (16 * osize / esize) != 0)
            return fail(REVISIT_ERR_SHAPE, "%s: rows of q and k must start on 16 bytes (on 8 for fp8 output)", fn);
    }
    if (n_tokens == 0) return REVISIT_OK;
    if (!q || !q_out || (k && !k_out)) return fail(REVISIT_ERR_NULL, "%s: q and q_out (and k_out with k) are required", fn);
    if (!aligned(pos, 4)) return fail(REVISIT_ERR_SHAPE, "%s: pos must be 4-byte aligned", fn);
    for (int i = 0; i < 2; ++i) {
        if (i == 1 && !k) break;
        if (!aligned(x[i], 16) || !aligned(o[i], fp8 ? 8 : 16))
            return fail(REVISIT_ERR_SHAPE, "%s: q and k must be 16-byte aligned, outputs too (8-byte for fp8)", fn);
        const int64_t row = (int64_t)heads[i] * D;
        revisit::RotaryTensor& t = a.t[i];
        t.x = x[i];
        t.o = o[i];
        t.x_row_bytes = x_row[i] * esize;
        t.o_row_bytes = o_row[i] * osize;
        t.H = heads[i];
        t.scale = i ? k_scale : q_scale;
        t.inv_row_vecs = 16.0 / ((double)row * esize);
        // in place only element by element
        if (x[i] == o[i] ? (fp8 || x_row[i] != o_row[i]) : false)
            return fail(REVISIT_ERR_SHAPE, "%s: an output in its input's place needs the same type and rows", fn);
    }
    a.n_tokens = n_tokens;
    a.D = D;
    a.esize = esize;
    a.fp8_out = fp8;
    a.pos = pos;
    a.t0 = t0;
    a.hw = pos ? 1 : h * w;
    a.w = pos ? 1 : w;
    a.n_t = pairs_t;
    a.n_y = pairs_y;
    a.n_x = pairs_x;
    a.inverse = inverse;
    const int pairs = pairs_t + pairs_y + pairs_x;
    a.inv_pairs = pairs > 0 ? 1.0f / (float)pairs : 0.0f;
    a.inv_hw = 1.0 / a.hw;
    a.inv_w = 1.0 / a.w;
    if (revisit::rotary_blocks(a) > INT32_MAX) return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    revisit::RotaryFreq f;
    band_quarters((double)theta, pairs_t, f.quarter);
    band_quarters((double)theta, pairs_y, f.quarter + pairs_t);
    band_quarters((double)theta, pairs_x, f.quarter + pairs_t + pairs_y);
    return launched(revisit::launch_rotary(a, f, stream), fn);
}

}  // extern "C"

namespace {

// Shape, type and part checks shared by attention_key_weight and its workspace
// query; fills the plan of `a` and its parts.
int prepare_key_weight(const char* fn, int32_t dtype, int32_t Lq, int32_t Lk, int32_t H, int32_t D, int32_t h, int32_t w, int32_t S,
                       int32_t query_parts, revisit::KeyWeightArgs& a, size_t* bytes) {
    *bytes = 0;
    const int st = check_attention_shape(fn, dtype, Lq, Lk, H, D, 0);
    if (st != REVISIT_OK) return st;
    if (h < 1 || w < 1 || S < 0) return fail(REVISIT_ERR_SHAPE, "%s: need h, w >= 1, S >= 0", fn);
    if (Lq > (1 << 30)) return fail(REVISIT_ERR_SHAPE, "%s: Lq=%d above 2^30", fn, Lq);
    const int64_t hw = (int64_t)h * w;
    if (Lk % hw != 0) return fail(REVISIT_ERR_SHAPE, "%s: Lk=%d not a multiple of h*w=%lld", fn, Lk, (long long)hw);
    if (Lk / hw > kMaxFrames) return fail(REVISIT_ERR_SHAPE, "%s: more than %d KV frames", fn, kMaxFrames);
    if (S > 0 && dtype != REVISIT_F32 && (h > kMaxGridSide || w > kMaxGridSide))
        return fail(REVISIT_ERR_SHAPE, "%s: bf16 / fp8 with bias needs h, w <= %d (got %d x %d)", fn, kMaxGridSide, h, w);
    if (query_parts < 0 || query_parts > revisit::kKeyWeightMaxParts)
        return fail(REVISIT_ERR_PARAM, "%s: query_parts=%d outside [0, %d]", fn, query_parts, revisit::kKeyWeightMaxParts);
    a.type = dtype;
    a.Lq = Lq;
    a.Lk = Lk;
    a.H = H;
    a.D = D;
    a.hw = (int32_t)hw;
    a.h = h;
    a.w = w;
    a.S = S;
    revisit::key_weight_plan(a);
    a.parts = revisit::kKeyWeightMaxParts;
    if (revisit::key_weight_items(a) > INT32_MAX - revisit::kXcds) return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    a.parts = query_parts;
    if (a.parts == 0) {
        int cus = 0;
        const hipError_t e = device_compute_units(&cus);
        if (e != hipSuccess) return fail(REVISIT_ERR_LAUNCH, "%s: device query failed: %s", fn, hipGetErrorString(e));
        a.parts = revisit::key_weight_parts(a, cus);
    }
    const int32_t tiles = (int32_t)(((int64_t)Lq + 31) / 32);
    if (a.parts > tiles) a.parts = tiles > 1 ? tiles : 1;  // at least one tile of 32 queries per part
    *bytes = a.parts > 1 ? (size_t)a.parts * H * Lk * sizeof(float) : 0;
    return REVISIT_OK;
}

}  // namespace

extern "C" {

int rc_key_weight_workspace_size(int32_t dtype, int32_t Lq, int32_t Lk, int32_t H, int32_t D, int32_t h, int32_t w, int32_t S,
                                 int32_t query_parts, size_t* bytes) {
    if (!bytes) return fail(REVISIT_ERR_NULL, "rc_key_weight_workspace_size: bytes is NULL");
    revisit::KeyWeightArgs a{};
    return prepare_key_weight("rc_key_weight_workspace_size", dtype, Lq, Lk, H, D, h, w, S, query_parts, a, bytes);
}

int attention_key_weight(const void* q, const void* k, const float* lse, int32_t dtype, int32_t Lq, int32_t Lk, int32_t H, int32_t D,
                         int32_t h, int32_t w, const int32_t* kv_frame_slot, const float* corr_uv, const int32_t* corr_idx, int32_t S,
                         float softmax_scale, float lambda, float sigma, const float* prev, float decay, float* out,
                         int32_t query_parts, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    const char* fn = "attention_key_weight";
    if (!(finite(softmax_scale) && softmax_scale > 0.0f))
        return fail(REVISIT_ERR_PARAM, "%s: softmax_scale must be finite and > 0", fn);
    if (!(finite(sigma) && sigma > 0.0f)) return fail(REVISIT_ERR_PARAM, "%s: sigma must be finite and > 0", fn);
    if (!finite(lambda)) return fail(REVISIT_ERR_PARAM, "%s: lambda must be finite", fn);
    if (!finite(decay)) return fail(REVISIT_ERR_PARAM, "%s: decay must be finite", fn);
    const float gamma = lambda / (2.0f * sigma * sigma * softmax_scale), gamma2 = lambda / (2.0f * sigma * sigma);
    if (!finite(gamma) || !finite(gamma2)) return fail(REVISIT_ERR_PARAM, "%s: lambda / (2 sigma^2 scale) overflows", fn);
    revisit::KeyWeightArgs a{};
    size_t need = 0;
    const bool bias = S > 0 && lambda != 0.0f;
    int st = prepare_key_weight(fn, dtype, Lq, Lk, H, D, h, w, S < 0 ? S : (bias ? S : 0), query_parts, a, &need);
    if (st != REVISIT_OK) return st;
    if (bias && (double)S * Lq > (double)kMaxElems) return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    if (!k || !out || (Lq > 0 && (!q || !lse))) return fail(REVISIT_ERR_NULL, "%s: q, k, lse and out are required", fn);
    if (bias && (!kv_frame_slot || !corr_uv || !corr_idx) && Lq > 0)
        return fail(REVISIT_ERR_NULL, "%s: slot table and correspondence map are required when S > 0", fn);
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(lse, 4) || !aligned(prev, 4) || !aligned(out, 4) ||
        (bias && (!aligned(corr_uv, 8) || !aligned(corr_idx, 4) || !aligned(kv_frame_slot, 4))))
        return fail(REVISIT_ERR_SHAPE, "%s: q and k must be 16-byte aligned, corr_uv 8-byte, arrays of words 4-byte", fn);
    st = check_workspace(fn, need, workspace, workspace_bytes);
    if (st != REVISIT_OK) return st;
    if (Lq == 0) {  // no query: nothing of the bias is read
        a.S = 0;
        revisit::key_weight_plan(a);
    }
    a.q = q;
    a.k = k;
    a.lse = lse;
    a.prev = prev;
    a.out = out;
    a.partial = static_cast<float*>(workspace);
    a.slot = kv_frame_slot;
    a.corr_uv = corr_uv;
    a.corr_idx = corr_idx;
    a.c_log2 = (float)((double)softmax_scale * M_LOG2E);
    a.gamma = gamma;
    a.gamma2 = (float)((double)gamma2 * M_LOG2E);
    a.decay = decay;
    return launched(revisit::launch_key_weight(a, stream), fn);
}

}  // extern "C"

namespace {

int prepare_select(const char* fn, int32_t sets, int32_t heads, int32_t n_units, int32_t unit, revisit::SelectArgs& a, size_t* bytes) {
    *bytes = 0;
    if (sets < 0 || heads < 1 || n_units < 0 || unit < 1)
        return fail(REVISIT_ERR_SHAPE, "%s: need sets, n_units >= 0 and heads, unit >= 1", fn);
    if (n_units > (1 << 30) || (int64_t)n_units * unit > INT32_MAX || sets > (1 << 21) ||
        (int64_t)sets * n_units > INT32_MAX || (double)sets * heads * n_units * unit > (double)kMaxElems)
        return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    a.sets = sets;
    a.heads = heads;
    a.n_units = n_units;
    a.unit = unit;
    a.splits = revisit::select_splits(a);
    *bytes = revisit::select_workspace_bytes(a);
    return REVISIT_OK;
}

}  // namespace

extern "C" {

int rc_select_workspace_size(int32_t sets, int32_t heads, int32_t n_units, int32_t unit, size_t* bytes) {
    if (!bytes) return fail(REVISIT_ERR_NULL, "rc_select_workspace_size: bytes is NULL");
    revisit::SelectArgs a{};
    return prepare_select("rc_select_workspace_size", sets, heads, n_units, unit, a, bytes);
}

int select_kept(const float* weight, int32_t sets, int32_t heads, int32_t n_units, int32_t unit, int32_t keep, int32_t first,
                int32_t last, int32_t* out_idx, float* out_score, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    const char* fn = "select_kept";
    revisit::SelectArgs a{};
    size_t need = 0;
    int st = prepare_select(fn, sets, heads, n_units, unit, a, &need);
    if (st != REVISIT_OK) return st;
    if (first < 0 || last < 0 || (int64_t)first + last > keep || keep > n_units)
        return fail(REVISIT_ERR_PARAM, "%s: need first, last >= 0 and first + last <= keep <= n_units (got %d, %d, %d, %d)", fn, first,
                    last, keep, n_units);
    if (sets == 0 || keep == 0) return REVISIT_OK;
    if (!weight || !out_idx) return fail(REVISIT_ERR_NULL, "%s: weight and out_idx are required", fn);
    if (!aligned(weight, 4) || !aligned(out_idx, 4) || !aligned(out_score, 4))
        return fail(REVISIT_ERR_SHAPE, "%s: arrays must be 4-byte aligned", fn);
    st = check_workspace(fn, need, workspace, workspace_bytes);
    if (st != REVISIT_OK) return st;
    a.weight = weight;
    a.keep = keep;
    a.first = first;
    a.last = last;
    a.out_idx = out_idx;
    a.out_score = out_score;
    a.unit_sum = static_cast<double*>(workspace);
    return launched(revisit::launch_select(a, stream), fn);
}

int compact_kv(const void* src_k, const void* src_v, int32_t src_rows, const int32_t* sel, int32_t sel_heads, int32_t keep,
               int32_t unit, int32_t n_units, void* dst_k, void* dst_v, int32_t dst_rows, int32_t dst_row0, const float* src_weight,
               int32_t src_weight_cols, float* dst_weight, int32_t dst_weight_cols, int32_t n_layers, int32_t dtype, int32_t H,
               int32_t D, const int32_t* src_pos, int32_t dst_pos, int32_t frames_per_unit, int32_t rope_t_pairs, float rope_theta,
               hipStream_t stream) {
    const char* fn = "compact_kv";
    if (dtype != REVISIT_BF16 && dtype != REVISIT_F32 && dtype != REVISIT_FP8_QK)
        return fail(REVISIT_ERR_UNSUPPORTED, "%s: dtype %d not supported", fn, dtype);
    const bool fp8 = dtype == REVISIT_FP8_QK;
    const int step = fp8 ? 16 : 8;
    if (D < step || D > 512 || D % step != 0)
        return fail(REVISIT_ERR_UNSUPPORTED, "%s: D=%d (need a multiple of %d up to 512)", fn, D, step);
    if (n_layers < 0 || keep < 0 || n_units < 0 || unit < 1 || H < 1 || H > 65535 || src_rows < 0 || dst_rows < 0 || dst_row0 < 0)
        return fail(REVISIT_ERR_SHAPE, "%s: need n_layers, keep, n_units, rows >= 0, unit >= 1 and 1 to 65535 heads", fn);
    if (sel_heads != 1 && sel_heads != H) return fail(REVISIT_ERR_SHAPE, "%s: a selection for 1 or all %d heads (got %d)", fn, H, sel_heads);
    if ((int64_t)n_units * unit > src_rows)
        return fail(REVISIT_ERR_SHAPE, "%s: %d units of %d rows exceed src_rows=%d", fn, n_units, unit, src_rows);
    if ((int64_t)dst_row0 + (int64_t)keep * unit > dst_rows)
        return fail(REVISIT_ERR_SHAPE, "%s: %d units of %d rows from row %d exceed dst_rows=%d", fn, keep, unit, dst_row0, dst_rows);
    const double row = (double)H * D;
    if ((double)n_layers * src_rows * row > (double)kMaxElems || (double)n_layers * dst_rows * row > (double)kMaxElems ||
        (double)n_layers * sel_heads * keep > (double)kMaxElems)
        return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    if (rope_t_pairs < 0 || rope_t_pairs > D / 2) return fail(REVISIT_ERR_PARAM, "%s: rope_t_pairs=%d outside [0, D/2]", fn, rope_t_pairs);
    if (rope_t_pairs > 0) {
        if (fp8) return fail(REVISIT_ERR_UNSUPPORTED, "%s: fp8 keys are not turned (they would be rounded to 8 bits a second time)", fn);
        if (!(finite(rope_theta) && rope_theta > 0.0f)) return fail(REVISIT_ERR_PARAM, "%s: rope_theta must be finite and > 0", fn);
        if (frames_per_unit < 0) return fail(REVISIT_ERR_PARAM, "%s: frames_per_unit=%d", fn, frames_per_unit);
    }
    if ((src_weight == nullptr) != (dst_weight == nullptr))
        return fail(REVISIT_ERR_NULL, "%s: src_weight and dst_weight are given together or not at all", fn);
    if (src_weight) {
        if (src_weight_cols < (int64_t)n_units * unit || dst_weight_cols < (int64_t)dst_row0 + (int64_t)keep * unit)
            return fail(REVISIT_ERR_SHAPE, "%s: weight rows are shorter than the units' rows", fn);
        if ((double)n_layers * H * src_weight_cols > (double)kMaxElems || (double)n_layers * H * dst_weight_cols > (double)kMaxElems)
            return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    }
    if (n_layers == 0 || keep == 0) return REVISIT_OK;
    if (!sel || !dst_k || !dst_v || (n_units > 0 && (!src_k || !src_v)))
        return fail(REVISIT_ERR_NULL, "%s: required pointer is NULL", fn);
    if (!aligned(src_k, 16) || !aligned(src_v, 16) || !aligned(dst_k, 16) || !aligned(dst_v, 16) || !aligned(sel, 4) ||
        !aligned(src_pos, 4) || !aligned(src_weight, 4) || !aligned(dst_weight, 4))
        return fail(REVISIT_ERR_SHAPE, "%s: caches must be 16-byte aligned, arrays of words 4-byte", fn);
    revisit::CompactArgs a{};
    a.src_k = src_k;
    a.src_v = src_v;
    a.dst_k = dst_k;
    a.dst_v = dst_v;
    a.sel = sel;
    a.n_layers = n_layers;
    a.sel_heads = sel_heads;
    a.keep = keep;
    a.unit = unit;
    a.n_units = n_units;
    a.H = H;
    a.D = D;
    a.src_rows = src_rows;
    a.dst_rows = dst_rows;
    a.dst_row0 = dst_row0;
    a.k_bytes = fp8 ? 1 : (dtype == REVISIT_BF16 ? 2 : 4);
    a.v_bytes = dtype == REVISIT_F32 ? 4 : 2;
    a.src_w = src_weight;
    a.dst_w = dst_weight;
    a.src_w_cols = src_weight_cols;
    a.dst_w_cols = dst_weight_cols;
    a.src_pos = src_pos;
    a.dst_pos = dst_pos;
    a.step = frames_per_unit;
    a.n_t = rope_t_pairs;
    a.inv_unit = 1.0 / unit;
    a.inv_kept = 1.0 / ((double)keep * unit);
    // no destination within a source or another destination: bytes could be overwritten before another
    // block has read them, or written twice
    struct Range {
        const void* at;
        double bytes;
    };
    const double src_rows_all = (double)n_layers * src_rows * row, dst_rows_all = (double)n_layers * dst_rows * row;
    const Range dst[] = {{dst_k, dst_rows_all * a.k_bytes}, {dst_v, dst_rows_all * a.v_bytes},
                         {dst_weight, dst_weight ? 4.0 * n_layers * H * dst_weight_cols : 0.0}};
    const Range src[] = {{src_k, src_rows_all * a.k_bytes}, {src_v, src_rows_all * a.v_bytes},
                         {src_weight, src_weight ? 4.0 * n_layers * H * src_weight_cols : 0.0},
                         {sel, 4.0 * n_layers * sel_heads * keep},
                         {src_pos, src_pos && rope_t_pairs > 0 ? 4.0 * n_units : 0.0}};
    for (int i = 0; i < 3; ++i) {
        for (const Range& r : src)
            if (overlap(dst[i].at, dst[i].bytes, r.at, r.bytes)) return fail(REVISIT_ERR_SHAPE, "%s: source and destination overlap", fn);
        for (int j = 0; j < i; ++j)
            if (overlap(dst[i].at, dst[i].bytes, dst[j].at, dst[j].bytes)) return fail(REVISIT_ERR_SHAPE, "%s: destinations overlap", fn);
    }
    if (revisit::compact_blocks(a) > (double)INT32_MAX) return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    revisit::CompactFreq f;
    if (rope_t_pairs > 0) band_quarters((double)rope_theta, rope_t_pairs, f.quarter);
    return launched(revisit::launch_compact(a, f, stream), fn);
}

}  // extern "C"

namespace {

// What append_paged_kv and paged_chunk_attention check alike; fills `q`.
int check_paged(const char* fn, int32_t dtype, int32_t n_tokens, const int32_t* cu_tokens, int32_t B, const int32_t* kv_len,
                const int32_t* page_table, int32_t n_pages, int32_t page, int32_t max_pages, int32_t H, int32_t D,
                revisit::PagedSeqs& q) {
    if (dtype != REVISIT_BF16 && dtype != REVISIT_F32 && dtype != REVISIT_FP8_KV)
        return fail(REVISIT_ERR_UNSUPPORTED, "%s: dtype %d not supported", fn, dtype);
    if (D != 64 && D != 128) return fail(REVISIT_ERR_UNSUPPORTED, "%s: D = 64 or 128 (got %d)", fn, D);
    if (H < 1 || H > 65535) return fail(REVISIT_ERR_SHAPE, "%s: need 1 to 65535 heads", fn);
    if (n_tokens < 0 || n_tokens > (1 << 30) || B < 0 || B > (1 << 20) || n_pages < 0 || max_pages < 0)
        return fail(REVISIT_ERR_SHAPE, "%s: need 0 <= n_tokens <= 2^30, 0 <= B <= 2^20, n_pages, max_pages >= 0", fn);
    if (page < 32 || page > 4096 || (page & (page - 1)) != 0)
        return fail(REVISIT_ERR_SHAPE, "%s: page=%d is not a power of two in [32, 4096]", fn, page);
    if ((int64_t)max_pages * page > (1 << 30)) return fail(REVISIT_ERR_SHAPE, "%s: more than 2^30 positions in a stream", fn);
    if ((double)n_pages * page * H * D > (double)kMaxElems) return fail(REVISIT_ERR_SHAPE, "%s: cache too large", fn);
    if (!cu_tokens && (B ? n_tokens % B : n_tokens) != 0)
        return fail(REVISIT_ERR_SHAPE, "%s: %d tokens are not shared evenly by %d streams (cu_tokens is NULL)", fn, n_tokens, B);
    if (!aligned(cu_tokens, 4) || !aligned(kv_len, 4) || !aligned(page_table, 4))
        return fail(REVISIT_ERR_SHAPE, "%s: cu_tokens, kv_len and page_table must be 4-byte aligned", fn);
    q.cu = cu_tokens;
    q.kv_len = kv_len;
    q.page_table = page_table;
    q.n_tokens = n_tokens;
    q.B = B;
    q.per = B ? n_tokens / B : 0;
    q.n_pages = n_pages;
    q.max_pages = max_pages;
    q.page_log2 = __builtin_ctz((unsigned)page);
    return REVISIT_OK;
}

int check_paged_pointers(const char* fn, const revisit::PagedSeqs& q, int32_t dtype, const void* cache_k, const void* cache_v,
                         const uint8_t* scale_k, const uint8_t* scale_v) {
    if (!q.kv_len) return fail(REVISIT_ERR_NULL, "%s: kv_len is required", fn);
    if (q.max_pages > 0 && !q.page_table) return fail(REVISIT_ERR_NULL, "%s: page_table is required", fn);
    if (q.n_pages > 0 && (!cache_k || !cache_v)) return fail(REVISIT_ERR_NULL, "%s: cache_k and cache_v are required", fn);
    if (q.n_pages > 0 && dtype == REVISIT_FP8_KV && (!scale_k || !scale_v))
        return fail(REVISIT_ERR_NULL, "%s: pages of 8 bits need scale_k and scale_v", fn);
    if (!aligned(cache_k, 16) || !aligned(cache_v, 16)) return fail(REVISIT_ERR_SHAPE, "%s: cache_k and cache_v must be 16-byte aligned", fn);
    return REVISIT_OK;
}

// A range of memory that a call reads or writes.
struct Range {
    const char* name;
    const void* at;
    double bytes;
};

// Refuses a written range that shares a byte with a read one or with another written one (the first `known` of those apart from
// each other already).
int check_apart(const char* fn, const Range* written, int n_written, const Range* read, int n_read, int known = 0) {
    for (int i = 0; i < n_written; ++i) {
        if (!written[i].at) continue;
        for (int j = i + 1 < known ? known : i + 1; j < n_written; ++j)
            if (written[j].at && overlap(written[i].at, written[i].bytes, written[j].at, written[j].bytes))
                return fail(REVISIT_ERR_SHAPE, "%s: %s and %s overlap", fn, written[i].name, written[j].name);
        for (int j = 0; j < n_read; ++j)
            if (read[j].at && overlap(written[i].at, written[i].bytes, read[j].at, read[j].bytes))
                return fail(REVISIT_ERR_SHAPE, "%s: %s overlaps %s", fn, written[i].name, read[j].name);
    }
    return REVISIT_OK;
}

// A pool as runs of `run` bytes at at + i0 step[0] + i1 step[1] + i2 step[2], i_d < size[d], steps in falling order.
struct Runs {
    const void* at;
    int64_t size[3], step[3], run;
};

Runs runs_of(const void* at, int64_t pages, int64_t heads, int64_t rows, revisit::PagedStrides& s, int64_t run) {
    // a distance that nothing is apart by does not count
    if (pages <= 1) s.page = 0;
    if (heads <= 1) s.head = 0;
    if (rows <= 1) s.row = 0;
    Runs r{at, {pages, heads, rows}, {s.page, s.head, s.row}, run};
    auto order = [&](int i, int j) {
        if (r.step[i] > r.step[j] || (r.step[i] == r.step[j] && r.size[i] >= r.size[j])) return;
        std::swap(r.step[i], r.step[j]);
        std::swap(r.size[i], r.size[j]);
    };
    order(0, 1);
    order(1, 2);
    order(0, 1);
    return r;
}

// Bytes from the first to behind the last of the dimensions from d on.
double extent(const Runs& r, int d) {
    double e = (double)r.run;
    for (; d < 3; ++d) {
        if (r.size[d] == 0) return 0.0;
        e += (double)(r.size[d] - 1) * (double)r.step[d];
    }
    return e;
}

// Whether all runs are apart: each dimension's step spans what lies within it.
bool all_apart(const Runs& r) {
    for (int d = 0; d < 3; ++d)
        if (r.size[d] > 1 && (double)r.step[d] < extent(r, d + 1)) return false;
    return true;
}

// Whether runs of two pools, each all apart and the second one's `delta` bytes behind the first's, share a byte. Where an outer dimension
// is the same, only neighbours in it can (keys beside values in one tensor); else their extents decide.
bool share(const Runs& x, const Runs& y, int64_t delta, int d) {
    if (d == 3 || x.size[d] != y.size[d] || x.step[d] != y.step[d]) return (double)delta < extent(x, d) && (double)-delta < extent(y, d);
    if (x.size[d] <= 1) return share(x, y, delta, d + 1);
    int64_t t = -delta / x.step[d];
    if (t * x.step[d] > -delta) --t;  // floor
    for (int64_t i = t; i <= t + 1; ++i)
        if (i > -x.size[d] && i < x.size[d] && share(x, y, delta + i * x.step[d], d + 1)) return true;
    return false;
}

// The pools as the kernels take them: cache_k, cache_v and, of 8 bits, scale_k and scale_v.
struct Pools {
    Range whole[4];  // from the first to behind the last byte
    int count;
    bool strided;
    revisit::PagedLayout layout;  // in bytes, of strided ones
    Runs runs[4];
};

// Contiguous pools (given NULL, or a layout that says so) need no distances.
int check_layout(const char* fn, const revisit::PagedSeqs& q, int32_t dtype, int32_t H, int32_t D, const void* cache_k, const void* cache_v,
                 const uint8_t* scale_k, const uint8_t* scale_v, const rc_pool_layout* given, Pools& p) {
    const int64_t page = (int64_t)1 << q.page_log2, es = dtype == REVISIT_FP8_KV ? 1 : (dtype == REVISIT_F32 ? 4 : 2);
    const double positions = (double)q.n_pages * page * H;
    p.count = dtype == REVISIT_FP8_KV ? 4 : 2;
    p.whole[0] = Range{"cache_k", cache_k, positions * (D * es)};
    p.whole[1] = Range{"cache_v", cache_v, positions * (D * es)};
    p.whole[2] = p.count == 4 ? Range{"scale_k", scale_k, positions / 32} : Range{};
    p.whole[3] = p.count == 4 ? Range{"scale_v", scale_v, positions / 32} : Range{};
    p.strided = false;
    if (!given) return REVISIT_OK;
    const int64_t* const from[4] = {given->k, given->v, given->scale_k, given->scale_v};
    revisit::PagedStrides* const to[4] = {&p.layout.k, &p.layout.v, &p.layout.scale_k, &p.layout.scale_v};
    for (int i = 0; i < p.count; ++i) {
        const bool codes = i < 2;
        const int64_t size = codes ? es : 1, run = codes ? D * es : 1, rows = codes ? page : page / 32;
        for (int d = 0; d < 3; ++d)
            if (from[i][d] < 0 || from[i][d] > kMaxElems) return fail(REVISIT_ERR_SHAPE, "%s: a stride of %s is negative or too large", fn, p.whole[i].name);
        revisit::PagedStrides& s = *to[i];
        s = revisit::PagedStrides{from[i][0] * size, from[i][1] * size, from[i][2] * size};
        p.runs[i] = runs_of(p.whole[i].at, q.n_pages, H, rows, s, run);
        if (codes && (s.page % 16 != 0 || s.head % 16 != 0 || s.row % 16 != 0))
            return fail(REVISIT_ERR_SHAPE, "%s: positions of %s must start on 16 bytes", fn, p.whole[i].name);
        p.whole[i].bytes = extent(p.runs[i], 0);
        if (p.whole[i].bytes > (double)kMaxElems) return fail(REVISIT_ERR_SHAPE, "%s: %s spans too much memory", fn, p.whole[i].name);
        p.strided = p.strided || (q.n_pages > 1 && s.page != H * rows * run) || (H > 1 && s.head != rows * run) || (rows > 1 && s.row != run);
    }
    return REVISIT_OK;
}

// Shape checks and plan shared by paged_chunk_attention and its workspace query (H is Hk).
int plan_paged_attention(const char* fn, int32_t Hq, int32_t max_keys, int32_t key_parts, revisit::PagedAttentionArgs& a, size_t* bytes) {
    *bytes = 0;
    if (Hq < 1 || Hq > 65535 || Hq % a.Hk != 0)
        return fail(REVISIT_ERR_SHAPE, "%s: Hq=%d is not a multiple of Hk=%d in [1, 65535]", fn, Hq, a.Hk);
    a.Hq = Hq;
    a.G = Hq / a.Hk;
    if ((int64_t)a.seqs.n_tokens * a.G > (1 << 30) || (double)a.seqs.n_tokens * Hq * a.D > (double)kMaxElems)
        return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    if (max_keys < 0) return fail(REVISIT_ERR_PARAM, "%s: max_keys=%d", fn, max_keys);
    if (key_parts < 0 || key_parts > revisit::kPagedMaxParts)
        return fail(REVISIT_ERR_PARAM, "%s: key_parts=%d outside [0, %d]", fn, key_parts, revisit::kPagedMaxParts);
    if (a.seqs.n_tokens == 0 || a.seqs.B == 0) return REVISIT_OK;
    int cus = 256;
    const hipError_t e = device_compute_units(&cus);
    if (e != hipSuccess) {
        // without a device only a fixed split has a size
        if (key_parts == 0) return fail(REVISIT_ERR_LAUNCH, "%s: device query failed: %s", fn, hipGetErrorString(e));
        (void)hipGetLastError();
    }
    *bytes = revisit::paged_plan(a, key_parts, max_keys ? max_keys : INT32_MAX, cus);
    if (revisit::paged_units(a) > (double)(1 << 30)) return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    return REVISIT_OK;
}

}  // namespace

extern "C" {

int append_paged_kv_strided(const void* k, int64_t k_row, const void* v, int64_t v_row, int32_t dtype, int32_t n_tokens,
                            const int32_t* cu_tokens, int32_t B, const int32_t* kv_len, int32_t* out_len, void* cache_k, void* cache_v,
                            uint8_t* scale_k, uint8_t* scale_v, const int32_t* page_table, int32_t n_pages, int32_t page,
                            int32_t max_pages, int32_t H, int32_t D, const int32_t* pos, int32_t t0, int32_t h, int32_t w,
                            int32_t pairs_t, int32_t pairs_y, int32_t pairs_x, float theta, const rc_pool_layout* layout,
                            hipStream_t stream) {
    const char* fn = "append_paged_kv";
    revisit::PagedAppendArgs a{};
    int st = check_paged(fn, dtype, n_tokens, cu_tokens, B, kv_len, page_table, n_pages, page, max_pages, H, D, a.seqs);
    if (st != REVISIT_OK) return st;
    if (pairs_t < 0 || pairs_y < 0 || pairs_x < 0 || (int64_t)pairs_t + pairs_y + pairs_x > D / 2)
        return fail(REVISIT_ERR_PARAM, "%s: bands of %d + %d + %d pairs in a head of %d", fn, pairs_t, pairs_y, pairs_x, D / 2);
    if (!(finite(theta) && theta > 0.0f)) return fail(REVISIT_ERR_PARAM, "%s: theta must be finite and > 0", fn);
    const bool grid = !pos && pairs_t + pairs_y + pairs_x > 0;  // positions come from the token grid
    if (grid && (h < 1 || w < 1 || (int64_t)h * w > INT32_MAX))
        return fail(REVISIT_ERR_SHAPE, "%s: without positions the token grid is needed: h, w >= 1", fn);
    const int esize = dtype == REVISIT_F32 ? 4 : 2;
    const int64_t row = (int64_t)H * D, most = kMaxElems / (n_tokens > 1 ? n_tokens : 1);
    if (k_row < row || v_row < row || k_row > most || v_row > most)
        return fail(REVISIT_ERR_SHAPE, "%s: a row stride is below the row's %lld elements or too large", fn, (long long)row);
    if (k_row * esize % 16 != 0 || v_row * esize % 16 != 0) return fail(REVISIT_ERR_SHAPE, "%s: rows of k and v must start on 16 bytes", fn);
    if (B == 0 || (n_tokens == 0 && !out_len)) return REVISIT_OK;
    if (n_tokens > 0 && (!k || !v)) return fail(REVISIT_ERR_NULL, "%s: k and v are required", fn);
    st = check_paged_pointers(fn, a.seqs, dtype, cache_k, cache_v, scale_k, scale_v);
    if (st != REVISIT_OK) return st;
    if (!aligned(k, 16) || !aligned(v, 16)) return fail(REVISIT_ERR_SHAPE, "%s: k and v must be 16-byte aligned", fn);
    if (!aligned(out_len, 4) || !aligned(pos, 4)) return fail(REVISIT_ERR_SHAPE, "%s: out_len and pos must be 4-byte aligned", fn);
    Pools pools;
    st = check_layout(fn, a.seqs, dtype, H, D, cache_k, cache_v, scale_k, scale_v, layout, pools);
    if (st != REVISIT_OK) return st;
    for (int i = 0; i < pools.count && pools.strided; ++i) {
        const Runs& x = pools.runs[i];
        if (!all_apart(x)) return fail(REVISIT_ERR_SHAPE, "%s: positions of %s share memory", fn, pools.whole[i].name);
        for (int j = i + 1; j < pools.count; ++j)
            if (n_pages > 0 && share(x, pools.runs[j], (int64_t)((uintptr_t)pools.runs[j].at - (uintptr_t)x.at), 0))
                return fail(REVISIT_ERR_SHAPE, "%s: %s and %s overlap", fn, pools.whole[i].name, pools.whole[j].name);
    }
    const double in_k = n_tokens ? ((double)(n_tokens - 1) * k_row + row) * esize : 0.0,
                 in_v = n_tokens ? ((double)(n_tokens - 1) * v_row + row) * esize : 0.0;
    const Range written[] = {pools.whole[0], pools.whole[1], pools.whole[2], pools.whole[3], {"out_len", out_len, 4.0 * B}};
    const Range read[] = {{"k", k, in_k},
                          {"v", v, in_v},
                          {"cu_tokens", cu_tokens, 4.0 * (B + 1.0)},
                          {"kv_len", kv_len, 4.0 * B},
                          {"page_table", page_table, 4.0 * B * max_pages},
                          {"pos", pos, 12.0 * n_tokens}};
    st = check_apart(fn, written, 5, read, 6, pools.strided ? 4 : 0);
    if (st != REVISIT_OK) return st;
    a.k = k;
    a.v = v;
    a.k_row_bytes = k_row * esize;
    a.v_row_bytes = v_row * esize;
    a.cache_k = cache_k;
    a.cache_v = cache_v;
    a.scale_k = scale_k;
    a.scale_v = scale_v;
    a.strided = pools.strided;
    a.layout = pools.layout;
    a.out_len = out_len;
    a.dtype = dtype;
    a.H = H;
    a.D = D;
    a.pos = pos;
    a.t0 = t0;
    a.hw = grid ? h * w : 1;
    a.w = grid ? w : 1;
    a.n_t = pairs_t;
    a.n_y = pairs_y;
    a.n_x = pairs_x;
    a.inv_pairs[0] = pairs_t > 0 ? 1.0f / (float)pairs_t : 0.0f;
    a.inv_pairs[1] = pairs_y > 0 ? 1.0f / (float)pairs_y : 0.0f;
    a.inv_pairs[2] = pairs_x > 0 ? 1.0f / (float)pairs_x : 0.0f;
    if (revisit::paged_append_blocks(a) > (1 << 30)) return fail(REVISIT_ERR_SHAPE, "%s: problem too large", fn);
    revisit::PagedFreq f;
    band_quarters((double)theta, pairs_t, f.quarter);
    band_quarters((double)theta, pairs_y, f.quarter + pairs_t);
    band_quarters((double)theta, pairs_x, f.quarter + pairs_t + pairs_y);
    return launched(revisit::launch_paged_append(a, f, stream), fn);
}

int append_paged_kv(const void* k, int64_t k_row, const void* v, int64_t v_row, int32_t dtype, int32_t n_tokens,
                    const int32_t* cu_tokens, int32_t B, const int32_t* kv_len, int32_t* out_len, void* cache_k, void* cache_v,
                    uint8_t* scale_k, uint8_t* scale_v, const int32_t* page_table, int32_t n_pages, int32_t page, int32_t max_pages,
                    int32_t H, int32_t D, const int32_t* pos, int32_t t0, int32_t h, int32_t w, int32_t pairs_t, int32_t pairs_y,
                    int32_t pairs_x, float theta, hipStream_t stream) {
    return append_paged_kv_strided(k, k_row, v, v_row, dtype, n_tokens, cu_tokens, B, kv_len, out_len, cache_k, cache_v, scale_k, scale_v,
                                   page_table, n_pages, page, max_pages, H, D, pos, t0, h, w, pairs_t, pairs_y, pairs_x, theta, nullptr, stream);
}

int rc_paged_attention_workspace_size(int32_t dtype, int32_t n_tokens, int32_t ragged, int32_t B, int32_t Hq, int32_t Hk, int32_t D,
                                      int32_t page, int32_t max_pages, int32_t max_keys, int32_t key_parts, size_t* bytes) {
    const char* fn = "rc_paged_attention_workspace_size";
    if (!bytes) return fail(REVISIT_ERR_NULL, "%s: bytes is NULL", fn);
    *bytes = 0;
    static const int32_t list = 0;  // stands for a list; never read
    revisit::PagedAttentionArgs a{};
    const int st = check_paged(fn, dtype, n_tokens, ragged ? &list : nullptr, B, nullptr, nullptr, 0, page, max_pages, Hk, D, a.seqs);
    if (st != REVISIT_OK) return st;
    a.dtype = dtype;
    a.Hk = Hk;
    a.D = D;
    return plan_paged_attention(fn, Hq, max_keys, key_parts, a, bytes);
}

int paged_chunk_attention_strided(const void* q, int64_t q_row, const void* cache_k, const void* cache_v, const uint8_t* scale_k,
                                  const uint8_t* scale_v, void* o, float* lse, int32_t dtype, int32_t n_tokens, const int32_t* cu_tokens,
                                  int32_t B, const int32_t* kv_len, const int32_t* visible, const int32_t* page_table, int32_t n_pages,
                                  int32_t page, int32_t max_pages, int32_t Hq, int32_t Hk, int32_t D, int32_t h, int32_t w,
                                  const int32_t* kv_frame_slot, int32_t max_frames, const float* corr_uv, const int32_t* corr_idx, int32_t S,
                                  float softmax_scale, float lambda, float sigma, int32_t max_keys, int32_t key_parts, void* workspace,
                                  size_t workspace_bytes, const rc_pool_layout* layout, hipStream_t stream) {
    const char* fn = "paged_chunk_attention";
    revisit::PagedAttentionArgs a{};
    int st = check_paged(fn, dtype, n_tokens, cu_tokens, B, kv_len, page_table, n_pages, page, max_pages, Hk, D, a.seqs);
    if (st != REVISIT_OK) return st;
    a.dtype = dtype;
    a.Hk = Hk;
    a.D = D;
    size_t need = 0;
    st = plan_paged_attention(fn, Hq, max_keys, key_parts, a, &need);
    if (st != REVISIT_OK) return st;
    if (!(finite(softmax_scale) && softmax_scale > 0.0f)) return fail(REVISIT_ERR_PARAM, "%s: softmax_scale must be finite and > 0", fn);
    if (S < 0) return fail(REVISIT_ERR_SHAPE, "%s: S=%d", fn, S);
    const bool bias = S > 0 && lambda != 0.0f;
    if (S > 0 && !finite(lambda)) return fail(REVISIT_ERR_PARAM, "%s: lambda must be finite", fn);
    if (bias) {
        if (!(finite(sigma) && sigma > 0.0f)) return fail(REVISIT_ERR_PARAM, "%s: sigma must be finite and > 0", fn);
        a.gamma = lambda / (2.0f * sigma * sigma * softmax_scale);
        if (!finite(a.gamma)) return fail(REVISIT_ERR_PARAM, "%s: lambda / (2 sigma^2 softmax_scale) is not finite", fn);
        if (h < 1 || w < 1 || (int64_t)h * w > INT32_MAX) return fail(REVISIT_ERR_SHAPE, "%s: the bias needs a token grid: h, w >= 1", fn);
        if (dtype != REVISIT_F32 && (h > kMaxGridSide || w > kMaxGridSide))
            return fail(REVISIT_ERR_SHAPE, "%s: bf16 / 8 bits with bias needs h, w <= %d (got %d x %d)", fn, kMaxGridSide, h, w);
        if (max_frames < 0 || (double)S * n_tokens > (double)kMaxElems) return fail(REVISIT_ERR_SHAPE, "%s: max_frames=%d, S=%d", fn, max_frames, S);
    }
    const int64_t row = (int64_t)Hq * D, most = kMaxElems / (n_tokens > 1 ? n_tokens : 1);
    const int esize = dtype == REVISIT_F32 ? 4 : 2;
    if (q_row < row || q_row > most) return fail(REVISIT_ERR_SHAPE, "%s: q_row is below the row's %lld elements or too large", fn, (long long)row);
    if (q_row * esize % 16 != 0) return fail(REVISIT_ERR_SHAPE, "%s: rows of q must start on 16 bytes", fn);
    if (n_tokens == 0 || B == 0) return REVISIT_OK;
    if (!q || !o) return fail(REVISIT_ERR_NULL, "%s: q and o are required", fn);
    st = check_paged_pointers(fn, a.seqs, dtype, cache_k, cache_v, scale_k, scale_v);
    if (st != REVISIT_OK) return st;
    if (bias && ((max_frames > 0 && !kv_frame_slot) || !corr_uv || !corr_idx))
        return fail(REVISIT_ERR_NULL, "%s: the bias needs kv_frame_slot, corr_uv and corr_idx", fn);
    if (!aligned(q, 16) || !aligned(o, 16)) return fail(REVISIT_ERR_SHAPE, "%s: q and o must be 16-byte aligned", fn);
    if (!aligned(lse, 4) || !aligned(visible, 4) || (bias && (!aligned(kv_frame_slot, 4) || !aligned(corr_uv, 8) || !aligned(corr_idx, 4))))
        return fail(REVISIT_ERR_SHAPE, "%s: lse, visible, kv_frame_slot and corr_idx must be 4-byte, corr_uv 8-byte aligned", fn);
    Pools pools;
    st = check_layout(fn, a.seqs, dtype, Hk, D, cache_k, cache_v, scale_k, scale_v, layout, pools);
    if (st != REVISIT_OK) return st;
    const double out = (double)n_tokens * row * esize;
    const Range written[] = {{"o", o, out}, {"lse", lse, 4.0 * Hq * n_tokens}, {"workspace", need ? workspace : nullptr, (double)need}};
    const Range read[] = {{"q", q, ((double)(n_tokens - 1) * q_row + row) * esize},
                          pools.whole[0],
                          pools.whole[1],
                          pools.whole[2],
                          pools.whole[3],
                          {"cu_tokens", cu_tokens, 4.0 * (B + 1.0)},
                          {"kv_len", kv_len, 4.0 * B},
                          {"visible", visible, 4.0 * n_tokens},
                          {"page_table", page_table, 4.0 * B * max_pages},
                          {"kv_frame_slot", bias ? kv_frame_slot : nullptr, 4.0 * B * max_frames},
                          {"corr_uv", bias ? corr_uv : nullptr, 8.0 * S * n_tokens},
                          {"corr_idx", bias ? corr_idx : nullptr, 4.0 * S * n_tokens}};
    st = check_apart(fn, written, 3, read, 12);
    if (st != REVISIT_OK) return st;
    st = check_workspace(fn, need, workspace, workspace_bytes);
    if (st != REVISIT_OK) return st;
    a.q = q;
    a.q_row = q_row;
    a.cache_k = cache_k;
    a.cache_v = cache_v;
    a.scale_k = scale_k;
    a.scale_v = scale_v;
    a.strided = pools.strided;
    a.layout = pools.layout;
    a.o = o;
    a.lse = lse;
    a.visible = visible;
    a.h = h;
    a.w = w;
    a.slot = kv_frame_slot;
    a.max_frames = max_frames;
    a.corr_uv = corr_uv;
    a.corr_idx = corr_idx;
    a.S = bias ? S : 0;
    a.softmax_scale = softmax_scale;
    if (n_pages == 0) a.seqs.max_pages = 0;  // nobody has a key; the kernels take page 0 to be there
    a.partial = static_cast<float*>(workspace);
    return launched(revisit::launch_paged_attention(a, stream), fn);
}

int paged_chunk_attention(const void* q, int64_t q_row, const void* cache_k, const void* cache_v, const uint8_t* scale_k,
                          const uint8_t* scale_v, void* o, float* lse, int32_t dtype, int32_t n_tokens, const int32_t* cu_tokens, int32_t B,
                          const int32_t* kv_len, const int32_t* visible, const int32_t* page_table, int32_t n_pages, int32_t page,
                          int32_t max_pages, int32_t Hq, int32_t Hk, int32_t D, int32_t h, int32_t w, const int32_t* kv_frame_slot,
                          int32_t max_frames, const float* corr_uv, const int32_t* corr_idx, int32_t S, float softmax_scale, float lambda,
                          float sigma, int32_t max_keys, int32_t key_parts, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return paged_chunk_attention_strided(q, q_row, cache_k, cache_v, scale_k, scale_v, o, lse, dtype, n_tokens, cu_tokens, B, kv_len, visible,
                                         page_table, n_pages, page, max_pages, Hq, Hk, D, h, w, kv_frame_slot, max_frames, corr_uv, corr_idx, S,
                                         softmax_scale, lambda, sigma, max_keys, key_parts, workspace, workspace_bytes, nullptr, stream);
}

}  // extern "C"
