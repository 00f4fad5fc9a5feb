// Log probabilities of given tokens, entropy and top alternatives of rows of logits, and their gradient (rtopk_logprobs, rtopk_logprobs_backward).
//
//   logprob_t = (x_t - M) / T - ln S,   S = sum exp((x_j - M) / T),   M = max x
//   H         = ln S - sum p_j (x_j - M) / T
#include "rtopk_softmax.h"

namespace rtopk {

struct LogprobsParams {
    const char* logits;
    long long row_bytes, row0, m, k;
    u32 n, parts, part_vecs;
    float c, inv_t;
    const long long* tokens;   // [batch][m]
    const char* top_values;    // [batch][k], in the logits' type
    float4* partial;           // [batch][parts]
    float *logprobs, *entropy, *top_logprobs, *row_stats;
    // the gradient
    const float *grad_logprobs, *grad_entropy;
    char* grad;
    long long grad_bytes;
};

// ln p of a logit; -inf in a row without anything but -inf, NaN for a token that is none.
__device__ __forceinline__ float logprob_of(float x, float m, float s, float ln_s, float inv_t) {
    return s == 0.0f ? -__builtin_inff() : (x - m) * inv_t - ln_s;
}

constexpr int kStatsBlock = 256, kStatsVecs = 4;

template <int DT, bool W>
__global__ void __launch_bounds__(kStatsBlock) k_logprobs_part(LogprobsParams P) {
    __shared__ float4 sm[kStatsBlock / 64];
    const u32 part = blockIdx.x % P.parts;
    const long long row = P.row0 + blockIdx.x / P.parts;
    const RowView<DT> r(P.logits, row, P.row_bytes, P.n);
    const u32 v0 = part * P.part_vecs, v1 = part_end(v0, P.part_vecs, r.nvec);
    SoftSum a;
    sweep_vectors<DT, kStatsBlock, kStatsVecs, false>(r, v0, v1, [&](const u32x4 (&q)[kStatsVecs], u32) {
        constexpr int E = RowElem<DT>::E;
        float x[kStatsVecs * E];
#pragma unroll
        for (int i = 0; i < kStatsVecs; ++i) {
            float y[E];
            RowElem<DT>::unpack(q[i], y);
#pragma unroll
            for (int j = 0; j < E; ++j) x[i * E + j] = y[j];
        }
        soft_add<W>(a, x, P.c);
    });
    a = soft_block<kStatsBlock, W>(a, P.c, sm);
    if (threadIdx.x == 0) P.partial[row * P.parts + part] = packed(a);
}

constexpr int kFinishBlock = 64;

template <int DT, bool W>
__global__ void __launch_bounds__(kFinishBlock) k_logprobs_finish(LogprobsParams P) {
    const long long row = P.row0 + blockIdx.x;
    const RowView<DT> r(P.logits, row, P.row_bytes, P.n);
    SoftSum a;
    for (u32 i = threadIdx.x; i < P.parts; i += kFinishBlock) a = soft_join<W>(a, unpacked(P.partial[row * P.parts + i]), P.c);
    a = soft_block<kFinishBlock, W>(a, P.c, nullptr);
    const float ln_s = kLn2 * log2_fast(a.s);
    for (long long i = threadIdx.x; i < P.m; i += kFinishBlock) {
        const long long t = P.tokens[row * P.m + i];
        float v = 0.0f;
        if (t >= (long long)P.n) v = __builtin_nanf("");
        else if (t >= 0) v = logprob_of(RowElem<DT>::load(r.x, (u32)t), a.m, a.s, ln_s, P.inv_t);
        P.logprobs[row * P.m + i] = v;
    }
    for (long long i = threadIdx.x; i < P.k; i += kFinishBlock)
        P.top_logprobs[row * P.k + i] = logprob_of(RowElem<DT>::load(P.top_values + (size_t)(row * P.k) * RowElem<DT>::kBytes, (u32)i), a.m, a.s, ln_s, P.inv_t);
    if (threadIdx.x == 0) {
        if (W) P.entropy[row] = a.s == 0.0f ? 0.0f : ln_s - kLn2 * (a.w / a.s);
        if (P.row_stats) {
            P.row_stats[2 * row] = a.m;
            P.row_stats[2 * row + 1] = a.s;
        }
    }
}

// dx_j = (1/T) [ sum_i g_i (1[t_i = j] - p_j) - gH p_j (ln p_j + H) ]
constexpr int kGradBlock = 256, kGradVecs = 4;

template <int DT, bool W>
__global__ void __launch_bounds__(kGradBlock) k_logprobs_grad(LogprobsParams P) {
    extern __shared__ __align__(16) u32 lds[];
    __shared__ u32 twice;
    __shared__ float sums[kGradBlock / 64];
    const u32 part = blockIdx.x % P.parts;
    const long long row = P.row0 + blockIdx.x / P.parts;
    const RowView<DT> r(P.logits, row, P.row_bytes, P.n);
    char* out = P.grad + row * P.grad_bytes;
    const long long* tokens = P.tokens + row * P.m;
    const float* g = P.grad_logprobs + row * P.m;
    auto counts = [&](long long i) { const long long t = tokens[i]; return t >= 0 && t < (long long)P.n; };
    float sum = 0.0f;
    for (long long i = threadIdx.x; i < P.m; i += kGradBlock) sum += counts(i) ? g[i] : 0.0f;
    sum = sum_block<kGradBlock>(sum, sums);
    const float gh = W ? P.grad_entropy[row] : 0.0f;
    const u32 v0 = part * P.part_vecs, v1 = part_end(v0, P.part_vecs, r.nvec);
    const float m = P.row_stats[2 * row], s = P.row_stats[2 * row + 1], ref = finite_or_zero(m);
    const float inv_s = s == 0.0f ? 0.0f : 1.0f / s, log2_s = s == 0.0f ? 0.0f : log2_fast(s);
    const float a = -sum * P.inv_t * inv_s, b = -gh * P.inv_t * kLn2 * inv_s, h2 = W ? P.entropy[row] * (1.0f / kLn2) - log2_s : 0.0f;
    const ScaledExp<DT> dense(a, ref, P.c);
    write_gradient<DT, kGradBlock, kGradVecs, 1, false>(
        r, out, (((uintptr_t)out ^ (uintptr_t)r.x) & 15) == 0, v0, v1, P.m, lds, &twice, [&](long long i) { return tokens[i]; },
        [&](long long i) { return g[i]; },
        [&](float (&x)[RowElem<DT>::E]) {
            if (!W) {
                dense.of(x);
                return;
            }
#pragma unroll
            for (int j = 0; j < RowElem<DT>::E; ++j) {
                const float y = (x[j] - ref) * P.c;
                x[j] = exp2_fast(y) * (a + b * (fmaxf(y, kNothing) + h2));
            }
        },
        [&](float x, float gi) {
            const float y = (x - ref) * P.c, e = exp2_fast(y);
            return (W ? e * (a + b * (fmaxf(y, kNothing) + h2)) : e * a) + gi * P.inv_t;
        });
}

constexpr int64_t kLogprobsMostVecs = (int64_t)1 << 15;  // (the gradient's bitmap: a byte each)

static RowParts stats_parts(int64_t batch, int64_t n, int eb) {
    return deal_row(batch, n, eb, kStatsBlock * kStatsVecs, 2048, (int64_t)1 << 28);
}
static size_t partial_bytes(int64_t batch, int64_t n, int eb) { return up256((size_t)batch * stats_parts(batch, n, eb).parts * sizeof(float4)); }

}  // namespace rtopk

using namespace rtopk;

extern "C" {

rtopk_status rtopk_logprobs_workspace_bytes(int64_t batch, int64_t n, int64_t m, int64_t k, rtopk_dtype dt, size_t* bytes_out) {
    if (!bytes_out || batch < 1 || batch > 0x7fffffff || n < 1 || n > RTOPK_MAX_N || m < 0 || k < 0 || k > n) return RTOPK_ERR_INVALID_ARG;
    if (dt != RTOPK_F32 && dt != RTOPK_F16 && dt != RTOPK_BF16) return RTOPK_ERR_INVALID_ARG;
    const int eb = dt == RTOPK_F32 ? 4 : 2;
    size_t select = 0;
    if (k > 0) {
        const rtopk_status s = rtopk_workspace_bytes(batch, n, k, dt, RTOPK_FLAG_SORTED, &select);
        if (s != RTOPK_OK) return s;
        size_t one = 0;  // (rows that do not follow one another are selected from one by one)
        (void)rtopk_workspace_bytes(1, n, k, dt, RTOPK_FLAG_SORTED, &one);
        if (one > select) select = one;
        select += up256((size_t)batch * k * eb);
    }
    *bytes_out = partial_bytes(batch, n, eb) + select;
    return RTOPK_OK;
}

rtopk_status rtopk_logprobs(const void* logits, int64_t batch, int64_t n, int64_t row_stride, rtopk_dtype dt, float inv_temperature,
                            const int64_t* tokens, int64_t m, int64_t k, float* out_logprobs, float* out_entropy, float* out_row_stats,
                            float* out_top_logprobs, int64_t* out_top_indices, void* workspace, size_t workspace_bytes, void* hip_stream) {
    rtopk_status s = check_rows(logits, batch, n, row_stride, dt);
    if (s != RTOPK_OK) return s;
    if (!usable_temperature(inv_temperature) || m < 0 || m > 0x7fffffff || k < 0 || k > n || !workspace) return RTOPK_ERR_INVALID_ARG;
    if (m > 0 && (!tokens || !out_logprobs)) return RTOPK_ERR_INVALID_ARG;
    if (k > 0 && (!out_top_logprobs || !out_top_indices)) return RTOPK_ERR_INVALID_ARG;
    if (((uintptr_t)tokens | (uintptr_t)out_top_indices) % 8 || ((uintptr_t)out_logprobs | (uintptr_t)out_entropy | (uintptr_t)out_row_stats | (uintptr_t)out_top_logprobs) % 4 ||
        (uintptr_t)workspace % 256)
        return RTOPK_ERR_UNSUPPORTED;
    size_t need = 0;
    s = rtopk_logprobs_workspace_bytes(batch, n, m, k, dt, &need);
    if (s != RTOPK_OK) return s;
    if (workspace_bytes < need) return RTOPK_ERR_WORKSPACE_TOO_SMALL;
    const int eb = dt == RTOPK_F32 ? 4 : 2;
    const hipStream_t st = (hipStream_t)hip_stream;
    char* ws = (char*)workspace;
    char* top_values = ws + partial_bytes(batch, n, eb);
    if (k > 0) {
        char* select = top_values + up256((size_t)batch * k * eb);
        // rows that do not follow one another are selected from one by one
        const int64_t at_once = batch == 1 || row_stride == n ? batch : 1;
        for (int64_t row = 0; row < batch; row += at_once) {
            s = rtopk_select((const char*)logits + row * row_stride * eb, at_once, n, k, dt, 1, RTOPK_FLAG_SORTED, 0, top_values + row * k * eb,
                             out_top_indices + row * k, select, workspace_bytes - (size_t)(select - ws), hip_stream);
            if (s != RTOPK_OK) return s;
        }
    }
    const RowParts d = stats_parts(batch, n, eb);
    LogprobsParams P = {};
    P.logits = (const char*)logits;
    P.row_bytes = row_stride * eb;
    P.n = (u32)n;
    P.m = m;
    P.k = k;
    P.parts = d.parts;
    P.part_vecs = d.vecs;
    P.c = inv_temperature * kLog2e;
    P.inv_t = inv_temperature;
    P.tokens = (const long long*)tokens;
    P.top_values = top_values;
    P.partial = (float4*)ws;
    P.logprobs = out_logprobs;
    P.entropy = out_entropy;
    P.top_logprobs = out_top_logprobs;
    P.row_stats = out_row_stats;
    (void)hipGetLastError();  // an error left by earlier HIP calls of the process is not this call's
    return by_type(dt, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        const int64_t rows = kMostWorkgroups / d.parts > 0 ? kMostWorkgroups / d.parts : 1;
        for (P.row0 = 0; P.row0 < batch; P.row0 += rows) {
            const unsigned now = (unsigned)(batch - P.row0 < rows ? batch - P.row0 : rows);
            if (out_entropy) {
                hipLaunchKernelGGL((k_logprobs_part<DT, true>), dim3(now * d.parts), dim3(kStatsBlock), 0, st, P);
                hipLaunchKernelGGL((k_logprobs_finish<DT, true>), dim3(now), dim3(kFinishBlock), 0, st, P);
            } else {
                hipLaunchKernelGGL((k_logprobs_part<DT, false>), dim3(now * d.parts), dim3(kStatsBlock), 0, st, P);
                hipLaunchKernelGGL((k_logprobs_finish<DT, false>), dim3(now), dim3(kFinishBlock), 0, st, P);
            }
        }
        return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_ERR_HIP;
    });
}

rtopk_status rtopk_logprobs_backward(const void* logits, int64_t batch, int64_t n, int64_t row_stride, rtopk_dtype dt, float inv_temperature,
                                     const int64_t* tokens, int64_t m, const float* row_stats, const float* grad_logprobs, const float* entropy,
                                     const float* grad_entropy, void* out_grad, int64_t grad_stride, void* hip_stream) {
    rtopk_status s = check_rows(logits, batch, n, row_stride, dt);
    if (s == RTOPK_OK) s = check_rows(out_grad, batch, n, grad_stride, dt);
    if (s != RTOPK_OK) return s;
    const int eb = dt == RTOPK_F32 ? 4 : 2;
    if (!usable_temperature(inv_temperature) || m < 0 || m > 0x7fffffff || !row_stats || (m > 0 && (!tokens || !grad_logprobs)) || (grad_entropy && !entropy))
        return RTOPK_ERR_INVALID_ARG;
    if (rows_overlap(logits, row_stride, out_grad, grad_stride, batch, n, eb)) return RTOPK_ERR_INVALID_ARG;
    if ((uintptr_t)tokens % 8 || ((uintptr_t)row_stats | (uintptr_t)grad_logprobs | (uintptr_t)entropy | (uintptr_t)grad_entropy) % 4) return RTOPK_ERR_UNSUPPORTED;
    const RowParts d = deal_row(batch, n, eb, kGradBlock * kGradVecs, 4096, kLogprobsMostVecs);
    LogprobsParams P = {};
    P.logits = (const char*)logits;
    P.row_bytes = row_stride * eb;
    P.n = (u32)n;
    P.m = m;
    P.parts = d.parts;
    P.part_vecs = d.vecs;
    P.c = inv_temperature * kLog2e;
    P.inv_t = inv_temperature;
    P.tokens = (const long long*)tokens;
    P.entropy = (float*)entropy;
    P.row_stats = (float*)row_stats;
    P.grad_logprobs = grad_logprobs;
    P.grad_entropy = grad_entropy;
    P.grad = (char*)out_grad;
    P.grad_bytes = grad_stride * eb;
    (void)hipGetLastError();
    return by_type(dt, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        const int64_t rows = kMostWorkgroups / d.parts > 0 ? kMostWorkgroups / d.parts : 1;
        const size_t lds = m > 0 ? gradient_lds<DT, kGradBlock, kGradVecs>(d.vecs) : 0;
        for (P.row0 = 0; P.row0 < batch; P.row0 += rows) {
            const unsigned now = (unsigned)(batch - P.row0 < rows ? batch - P.row0 : rows);
            if (grad_entropy) hipLaunchKernelGGL((k_logprobs_grad<DT, true>), dim3(now * d.parts), dim3(kGradBlock), lds, (hipStream_t)hip_stream, P);
            else hipLaunchKernelGGL((k_logprobs_grad<DT, false>), dim3(now * d.parts), dim3(kGradBlock), lds, (hipStream_t)hip_stream, P);
        }
        return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_ERR_HIP;
    });
}

}  // extern "C"
