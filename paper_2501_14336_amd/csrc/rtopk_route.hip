// Routing to experts: the k best of a short row of scores, with a bias for balance, groups and renormalised weights, and its gradient
// (rtopk_route, rtopk_route_backward).
//
//   s_e = softmax or sigmoid of the logits;  c_e chooses: s_e + bias_e, or the logit itself where there is neither a bias nor a sum over a group
//   groups: the largest c of a group, or the sum of its two largest; experts of the best groups are chosen from
//   w_i = scale s_{e_i} [ / sum_l s_{e_l} ]
#include "rtopk_softmax.h"

namespace rtopk {

struct RouteParams {
    const char* logits;
    long long row_bytes, row0, tokens;
    u32 experts, groups, group_size, topk_groups, k;
    u32 flags;
    float scale;
    const float* bias;
    float* weights;            // [tokens][k]
    long long* chosen;         // [tokens][k]
    unsigned long long* counts;  // [experts], added to
    // the gradient
    const float* grad_weights;
    char* grad;
    long long grad_bytes;
};

constexpr int kRouteBlock = 256;  // a wave per token

// 1 / (1 + e^-x) in the steps that a 32-bit program takes, each rounded: what is chosen by it is chosen alike everywhere.
__device__ __forceinline__ float sigmoid_of(float x) { return 1.0f / (1.0f + expf(-x)); }

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ u32 wave_max_u32(u32 v) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = max(v, (u32)__shfl_xor((int)v, d));
    return v;
}

__device__ __forceinline__ float number_of_f32_key(u32 o) { return __uint_as_float((o & 0x80000000u) ? (o ^ 0x80000000u) : ~o); }

// What the wave's lanes wrote to LDS is there for all of them.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Scores of a lane's experts; all zero in a row without anything but -inf.
template <int N>
__device__ __forceinline__ void scores_of(const float (&x)[N], float (&s)[N], bool sigmoid) {
    if (sigmoid) {
#pragma unroll
        for (int j = 0; j < N; ++j) s[j] = sigmoid_of(x[j]);
        return;
    }
    float m = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) m = fmaxf(m, x[j]);
    m = finite_or_zero(wave_max(m));
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < N; ++j) sum += s[j] = expf(x[j] - m);
    sum = wave_sum(sum);
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = sum == 0.0f ? 0.0f : s[j] / sum;
}

// A wave per token; lane l holds experts l N to l N + N - 1.
template <int DT, int N>
__global__ void __launch_bounds__(kRouteBlock) k_route(RouteParams P) {
    __shared__ float stage[kRouteBlock / 64][64 * N];
    const u32 lane = lane_id(), wave = threadIdx.x >> 6;
    const long long row = P.row0 + (long long)blockIdx.x * (kRouteBlock / 64) + wave;
    if (row >= P.tokens) return;  // (no barrier below: a wave works by itself)
    const char* x_row = P.logits + row * P.row_bytes;
    const bool sigmoid = (P.flags & RTOPK_ROUTE_SIGMOID) != 0, top2 = (P.flags & RTOPK_ROUTE_GROUP_TOP2) != 0;
    float x[N], s[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const u32 e = lane * N + j;
        x[j] = e < P.experts ? RowElem<DT>::load(x_row, e) : -__builtin_inff();
    }
    scores_of(x, s, sigmoid);
    u32 key[N];  // orders the choice; 0 for what may not be chosen
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const u32 e = lane * N + j;
        float c = x[j];
        if (x[j] != -__builtin_inff()) {
            if (P.bias) c = s[j] + (e < P.experts ? P.bias[e] : 0.0f);
            else if (top2) c = s[j];
        }
        key[j] = e < P.experts ? KeyOf<RTOPK_F32>::key(__float_as_uint(c)) : 0u;
        if (P.groups > 1 && e < P.experts) stage[wave][e] = c;
    }
    if (P.groups > 1) {
        wave_sync();
        u32 gkey = 0;
        if (lane < P.groups) {
            u32 a = 0, b = 0;  // the keys of the two best
            for (u32 i = 0; i < P.group_size; ++i) {
                const u32 v = KeyOf<RTOPK_F32>::key(__float_as_uint(stage[wave][lane * P.group_size + i]));
                b = max(b, min(a, v));
                a = max(a, v);
            }
            const float best = number_of_f32_key(a), second = number_of_f32_key(b);
            gkey = !top2 || b == 0 ? a : KeyOf<RTOPK_F32>::key(__float_as_uint(best + second));
        }
        u32 better = 0;
        for (u32 g = 0; g < P.groups; ++g) {
            const u32 o = (u32)__shfl((int)gkey, (int)g);
            better += o > gkey || (o == gkey && g < lane);
        }
        const u64 stays = ballot64(lane < P.groups && better < P.topk_groups);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const u32 e = lane * N + j;
            if (e < P.experts && !((stays >> (e / P.group_size)) & 1)) key[j] = 0;
        }
    }
    float mine_s = 0.0f;
    u32 mine_e = 0;
    for (u32 r = 0; r < P.k; ++r) {
        u32 best = key[0], at = 0;
#pragma unroll
        for (int j = 1; j < N; ++j)
            if (key[j] > best) {
                best = key[j];
                at = j;
            }
        float score = s[0];
#pragma unroll
        for (int j = 1; j < N; ++j) score = at == (u32)j ? s[j] : score;
        const u32 top = wave_max_u32(best);
        const u32 from = (u32)__builtin_ctzll(ballot64(best == top));
        const u32 e = (u32)__shfl((int)(lane * N + at), (int)from);
        const float se = __shfl(score, (int)from);
        if (lane == r) {
            mine_e = e;
            mine_s = se;
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (lane == from && at == (u32)j) key[j] = 0;
    }
    float w = mine_s;
    if (P.flags & RTOPK_ROUTE_RENORMALIZE) {
        const float sum = wave_sum(lane < P.k ? mine_s : 0.0f);
        w = sum == 0.0f ? 0.0f : w / sum;
    }
    if (lane < P.k) {
        P.weights[row * P.k + lane] = P.scale * w;
        P.chosen[row * P.k + lane] = (long long)mine_e;
        if (P.counts) atomicAdd(&P.counts[mine_e], 1ull);
    }
}

// softmax:  dx_j = s_j (G_j - sum_l G_l s_l), or, renormalised, over the chosen alone with their shares in the place of s
// sigmoid:  dx_j = G_j s_j (1 - s_j), with G = (g - sum_l g_l share_l) / sum s where it is renormalised
template <int DT, int N>
__global__ void __launch_bounds__(kRouteBlock) k_route_grad(RouteParams P) {
    __shared__ float stage[kRouteBlock / 64][64 * N];
    const u32 lane = lane_id(), wave = threadIdx.x >> 6;
    const long long row = P.row0 + (long long)blockIdx.x * (kRouteBlock / 64) + wave;
    if (row >= P.tokens) return;
    const char* x_row = P.logits + row * P.row_bytes;
    char* out = P.grad + row * P.grad_bytes;
    const bool sigmoid = (P.flags & RTOPK_ROUTE_SIGMOID) != 0, renormalize = (P.flags & RTOPK_ROUTE_RENORMALIZE) != 0;
    float x[N], s[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const u32 e = lane * N + j;
        x[j] = e < P.experts ? RowElem<DT>::load(x_row, e) : -__builtin_inff();
    }
    scores_of(x, s, sigmoid);
#pragma unroll
    for (int j = 0; j < N; ++j) stage[wave][lane * N + j] = s[j];
    wave_sync();
    const long long e = lane < P.k ? P.chosen[row * P.k + lane] : -1;
    const bool there = e >= 0 && e < (long long)P.experts;
    const float se = there ? stage[wave][e] : 0.0f;
    float g = there ? P.scale * P.grad_weights[row * P.k + lane] : 0.0f;
    if (renormalize) {
        const float sum = wave_sum(se), inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const float mean = wave_sum(g * se * inv);
        g = (g - mean) * inv;
    }
    float dense = 0.0f;
    if (!sigmoid && !renormalize) dense = wave_sum(g * se);  // (renormalised, this sum is zero)
    const float d = there ? g * (sigmoid ? se * (1.0f - se) : se) : 0.0f;
    wave_sync();
#pragma unroll
    for (int j = 0; j < N; ++j) stage[wave][lane * N + j] = sigmoid ? 0.0f : -s[j] * dense;
    wave_sync();
    if (there) atomicAdd(&stage[wave][e], d);
    wave_sync();
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const u32 i = lane * N + j;
        if (i < P.experts) RowElem<DT>::store(out, i, stage[wave][i]);
    }
}

static rtopk_status check_route(const void* logits, int64_t tokens, int64_t experts, int64_t stride, rtopk_dtype dt, int64_t k, uint32_t flags, float scale) {
    const rtopk_status s = check_rows(logits, tokens, experts, stride, dt);
    if (s != RTOPK_OK) return s;
    if (experts > RTOPK_ROUTE_MAX_EXPERTS || k < 1 || k > experts || k > RTOPK_ROUTE_MAX_K || scale != scale) return RTOPK_ERR_INVALID_ARG;
    if (flags & ~(uint32_t)(RTOPK_ROUTE_SIGMOID | RTOPK_ROUTE_RENORMALIZE | RTOPK_ROUTE_GROUP_TOP2)) return RTOPK_ERR_INVALID_ARG;
    return RTOPK_OK;
}
// f(experts per lane)
template <class F>
static rtopk_status by_experts(int64_t experts, F&& f) {
    if (experts <= 64) return f(std::integral_constant<int, 1>{});
    if (experts <= 128) return f(std::integral_constant<int, 2>{});
    if (experts <= 256) return f(std::integral_constant<int, 4>{});
    if (experts <= 512) return f(std::integral_constant<int, 8>{});
    return f(std::integral_constant<int, 16>{});
}

}  // namespace rtopk

using namespace rtopk;

extern "C" {

rtopk_status rtopk_route(const void* logits, int64_t tokens, int64_t experts, int64_t row_stride, rtopk_dtype dt, const float* bias, int64_t groups,
                         int64_t topk_groups, int64_t k, uint32_t flags, float scale, float* out_weights, int64_t* out_experts, int64_t* counts,
                         void* hip_stream) {
    const rtopk_status s = check_route(logits, tokens, experts, row_stride, dt, k, flags, scale);
    if (s != RTOPK_OK) return s;
    if (!out_weights || !out_experts || groups < 1 || groups > RTOPK_ROUTE_MAX_GROUPS || experts % groups || topk_groups < 1 || topk_groups > groups ||
        k > experts / groups * topk_groups)
        return RTOPK_ERR_INVALID_ARG;
    if (((uintptr_t)bias | (uintptr_t)out_weights) % 4 || ((uintptr_t)out_experts | (uintptr_t)counts) % 8) return RTOPK_ERR_UNSUPPORTED;
    RouteParams P = {};
    P.logits = (const char*)logits;
    P.row_bytes = row_stride * (dt == RTOPK_F32 ? 4 : 2);
    P.tokens = tokens;
    P.experts = (u32)experts;
    P.groups = topk_groups < groups ? (u32)groups : 1u;  // (all groups stay: as if there were none)
    P.group_size = (u32)(experts / groups);
    P.topk_groups = (u32)topk_groups;
    P.k = (u32)k;
    P.flags = flags;
    P.scale = scale;
    P.bias = bias;
    P.weights = out_weights;
    P.chosen = (long long*)out_experts;
    P.counts = (unsigned long long*)counts;
    (void)hipGetLastError();  // an error left by earlier HIP calls of the process is not this call's
    return by_type(dt, [&](auto t) {
        return by_experts(experts, [&](auto per_lane) {
            constexpr int64_t kRows = kRouteBlock / 64;
            for (; P.row0 < tokens; P.row0 += kMostWorkgroups * kRows) {
                const int64_t wgs = (tokens - P.row0 + kRows - 1) / kRows;
                hipLaunchKernelGGL((k_route<decltype(t)::value, decltype(per_lane)::value>), dim3((unsigned)(wgs < kMostWorkgroups ? wgs : kMostWorkgroups)), dim3(kRouteBlock),
                                   0, (hipStream_t)hip_stream, P);
            }
            return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_ERR_HIP;
        });
    });
}

rtopk_status rtopk_route_backward(const void* logits, int64_t tokens, int64_t experts, int64_t row_stride, rtopk_dtype dt, const int64_t* chosen, int64_t k,
                                  uint32_t flags, float scale, const float* grad_weights, void* out_grad, int64_t grad_stride, void* hip_stream) {
    rtopk_status s = check_route(logits, tokens, experts, row_stride, dt, k, flags, scale);
    if (s == RTOPK_OK) s = check_rows(out_grad, tokens, experts, grad_stride, dt);
    if (s != RTOPK_OK) return s;
    if (!chosen || !grad_weights || rows_overlap(logits, row_stride, out_grad, grad_stride, tokens, experts, dt == RTOPK_F32 ? 4 : 2)) return RTOPK_ERR_INVALID_ARG;
    if ((uintptr_t)chosen % 8 || (uintptr_t)grad_weights % 4) return RTOPK_ERR_UNSUPPORTED;
    RouteParams P = {};
    P.logits = (const char*)logits;
    P.row_bytes = row_stride * (dt == RTOPK_F32 ? 4 : 2);
    P.tokens = tokens;
    P.experts = (u32)experts;
    P.k = (u32)k;
    P.flags = flags;
    P.scale = scale;
    P.chosen = (long long*)chosen;
    P.grad_weights = grad_weights;
    P.grad = (char*)out_grad;
    P.grad_bytes = grad_stride * (dt == RTOPK_F32 ? 4 : 2);
    (void)hipGetLastError();
    return by_type(dt, [&](auto t) {
        return by_experts(experts, [&](auto per_lane) {
            constexpr int64_t kRows = kRouteBlock / 64;
            for (; P.row0 < tokens; P.row0 += kMostWorkgroups * kRows) {
                const int64_t wgs = (tokens - P.row0 + kRows - 1) / kRows;
                hipLaunchKernelGGL((k_route_grad<decltype(t)::value, decltype(per_lane)::value>), dim3((unsigned)(wgs < kMostWorkgroups ? wgs : kMostWorkgroups)),
                                   dim3(kRouteBlock), 0, (hipStream_t)hip_stream, P);
            }
            return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_ERR_HIP;
        });
    });
}

}  // extern "C"
