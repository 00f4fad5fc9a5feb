// Distillation from a teacher's top logits: the divergence of a student's row from a teacher's list of (column, logit), and its gradient
// (rtopk_distill, rtopk_distill_backward, rtopk_distill_step).
//
//   q_i = exp(z_i / T) / sum exp(z_l / T), or exp(z_i / T - lse) with the teacher's own log-sum; then r = max(0, 1 - sum q) is the rest's share
//   L   = sum q_i (ln q_i - ln p_{t_i}) [ + r (ln r - ln P),  P = sum of p over the columns that are not listed ]
//   dL/dx_j = (1/T) [ (sum q + r) p_j - sum_{t_i = j} q_i - [j not listed] r p_j / P ]
//
// P is added up from the columns that are not listed, not taken as what the listed ones leave of 1: a trained student leaves 1e-6 and less.
#include "rtopk_distill.h"

namespace rtopk {

// A row's list; the thread's first entry is fetched when the kernel begins, three trips that the row's hide.
template <int DT>
struct RowList {
    struct Entry {
        long long t;
        float z, x;  // the teacher's and the student's logit
    };
    const DistillParams& P;
    const RowView<DT>& r;
    long long from;
    Entry first;
    __device__ __forceinline__ RowList(const DistillParams& P, long long row, const RowView<DT>& r) : P(P), r(r), from(row * P.k) {
        first = {-1, 0.0f, 0.0f};
        if ((long long)threadIdx.x < P.k) first = entry(threadIdx.x);
    }
    __device__ __forceinline__ Entry entry(long long i) const {
        Entry e = {P.columns[from + i], load_as_float(P.values, P.value_dt, (size_t)(from + i)), 0.0f};
        if (e.t >= 0 && e.t < (long long)P.n) e.x = RowElem<DT>::load(r.x, (u32)e.t);
        return e;
    }
    // f(entry, its number) for the thread's ones
    template <int B, class F>
    __device__ __forceinline__ void each(F&& f) const {
        if ((long long)threadIdx.x < P.k) f(first, (long long)threadIdx.x);
        for (long long i = (long long)threadIdx.x + B; i < P.k; i += B) f(entry(i), i);
    }
};

// The loss of a row, and what its gradient needs of it, from the sums of its columns (TAIL: of those that are not listed, and of those that are).
template <int DT, bool TAIL, int B>
__device__ __forceinline__ void loss_of_row(const DistillParams& P, long long row, const RowList<DT>& list, SoftSum a, const SoftSum& listed, float4* sm, double* sums) {
    const SoftSum others = a;
    if (TAIL) a = soft_join<false>(a, listed, P.c);
    DistillRow d;
    float ln_zmul = 0.0f, zs = 1.0f;
    if (TAIL) {
        d.zref = P.teacher_lse[row];
        d.zmul = 1.0f;
    } else {
        SoftSum z;
        list.template each<B>([&](auto e, long long) {
            if (e.t >= 0) {
                const float v[1] = {e.z};
                soft_add<false>(z, v, P.c);
            }
        });
        z = soft_block<B, false>(z, P.c, sm);
        zs = z.s;
        d.zref = finite_or_zero(z.m);
        d.zmul = zs == 0.0f ? 0.0f : 1.0f / zs;
        ln_zmul = zs == 0.0f ? 0.0f : -kLn2 * log2_fast(zs);
    }
    const float ln_s = kLn2 * log2_fast(a.s);
    float loss = 0.0f;
    double share = 0.0;
    list.template each<B>([&](auto e, long long) {
        if (e.t < 0) return;
        const float lq = ln_share(e.z, d, TAIL, ln_zmul, P.inv_t), qi = expf(lq);
        if (TAIL) share += exact_share(e.z, d.zref, P.inv_t);
        if (e.t >= (long long)P.n) loss += __builtin_nanf("");
        else if (qi != 0.0f) loss += qi * (lq - (a.s == 0.0f ? -__builtin_inff() : (e.x - a.m) * P.inv_t - ln_s));
    });
    loss = sum_block<B>(loss, (float*)sums);
    if (TAIL) share = sum_block<B>(share, sums + B / 64);
    loss += finish_row<TAIL>(d, a, others, share, zs, P);
    if (threadIdx.x == 0) {
        P.loss[row] = loss;
        if (P.rows) P.rows[row] = d;
    }
}

constexpr int kDistillVecs = 4;

// Statistics of a row, or of a part of one; TAIL: apart for columns that are listed and for the others.  WHOLE: of the row, and its loss.  One reading of the row: 200 rows of 50257 fp32 with
// the rest, lists of 50: 12.6 us, 3.2 TB/s from 200 compute units, one row each.  8 rows of 30011 fp16 with lists of 100:
// 6.1 us, the way of one workgroup.
template <int DT, bool NT, bool TAIL, int B, bool WHOLE>
__global__ void __launch_bounds__(B) k_distill_part(DistillParams P) {
    extern __shared__ u32 marks[];  // TAIL: a byte per vector of the part, a bit per column
    __shared__ float4 sm[3][B / 64];
    __shared__ double sums[2 * B / 64];
    __shared__ u32 twice;
    constexpr int E = RowElem<DT>::E, V = kDistillVecs;
    const u32 part = WHOLE ? 0u : blockIdx.x % P.parts;
    const long long row = P.row0 + (WHOLE ? blockIdx.x : blockIdx.x / P.parts);
    const RowView<DT> r(P.student, row, P.row_bytes, P.n);
    const u32 v0 = part * P.part_vecs, v1 = part_end(v0, P.part_vecs, r.nvec);
    const RowList<DT> list(P, row, r);
    SoftSum a, listed;
    bool first_counts = false;
    if (TAIL) {
        for (u32 i = threadIdx.x; i < (P.part_vecs + 3) / 4; i += B) marks[i] = 0;
        if (threadIdx.x == 0) twice = 0;
    }
    sweep_vectors<DT, B, V, NT>(r, v0, v1, [&](const u32x4 (&q)[V], u32 first) {
        if (TAIL && first == v0) {  // (with the first two tiles on their way)
            __syncthreads();
            auto add_listed = [&](auto&& counts) {
                list.template each<B>([&](auto e, long long i) {
                    const u64 p = (u64)e.t + r.lead - (u64)v0 * E;  // (wraps below the part)
                    if (e.t < 0 || e.t >= (long long)P.n || p >= (u64)(v1 - v0) * E || !counts((u32)p, i)) return;
                    if (i == (long long)threadIdx.x) {
                        first_counts = true;
                    } else {
                        const float x[1] = {e.x};
                        soft_add<false>(listed, x, P.c);
                    }
                });
            };
            add_listed([&](u32 p, long long) {
                const u32 bit = 1u << ((p / E & 3) * 8 + p % E);
                const bool again = (atomicOr(&marks[p / E >> 2], bit) & bit) != 0;
                if (again) twice = 1;
                return !again;
            });
            __syncthreads();
            if (twice) {  // a column listed twice counts once, whichever thread came first: by its first entry
                listed = SoftSum();
                first_counts = false;
                add_listed([&](u32, long long i) { return is_first_of_column(P.columns + list.from, i); });
            }
        }
        float x[V * E];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            u32 bits = 0;
            if (TAIL) {
                const u32 v = first + i * B + threadIdx.x;
                if (v < v1) bits = ((const uint8_t*)marks)[v - v0];
            }
            float y[E];
            RowElem<DT>::unpack(TAIL ? RowElem<DT>::without(q[i], bits) : q[i], y);
#pragma unroll
            for (int j = 0; j < E; ++j) x[i * E + j] = y[j];
        }
        soft_add<false>(a, x, P.c);
    });
    if (first_counts) {
        const float x[1] = {list.first.x};
        soft_add<false>(listed, x, P.c);
    }
    a = soft_block<B, false>(a, P.c, sm[0]);
    if (TAIL) listed = soft_block<B, false>(listed, P.c, sm[1]);
    if (WHOLE) {
        loss_of_row<DT, TAIL, B>(P, row, list, a, listed, sm[2], sums);
    } else if (threadIdx.x == 0) {
        P.partial[(row * P.parts + part) * 2] = packed(a);
        if (TAIL) P.partial[(row * P.parts + part) * 2 + 1] = packed(listed);
    }
}

constexpr int kDistillFinish = 256;

// The parts of a row put together, and its loss: where there are too few rows to fill the compute units with one each.
template <int DT, bool TAIL>
__global__ void __launch_bounds__(kDistillFinish) k_distill_finish(DistillParams P) {
    __shared__ float4 sm[3][kDistillFinish / 64];
    __shared__ double sums[2 * kDistillFinish / 64];
    const long long row = P.row0 + blockIdx.x;
    const RowView<DT> r(P.student, row, P.row_bytes, P.n);
    const RowList<DT> list(P, row, r);
    SoftSum a, listed;
    for (u32 i = threadIdx.x; i < P.parts; i += kDistillFinish) {
        a = soft_join<false>(a, unpacked(P.partial[(row * P.parts + i) * 2]), P.c);
        if (TAIL) listed = soft_join<false>(listed, unpacked(P.partial[(row * P.parts + i) * 2 + 1]), P.c);
    }
    a = soft_block<kDistillFinish, false>(a, P.c, sm[0]);
    if (TAIL) listed = soft_block<kDistillFinish, false>(listed, P.c, sm[1]);
    loss_of_row<DT, TAIL, kDistillFinish>(P, row, list, a, listed, sm[2], sums);
}

constexpr int kDistillGradBlock = 256, kDistillGradVecs = 2;

// One reading of the row and one writing of the gradient, bound by memory: 200 rows of 50257 fp32 with the rest 17.2 us, 4.7 TB/s.
template <int DT, bool NT>
__global__ void __launch_bounds__(kDistillGradBlock) k_distill_grad(DistillParams P) {
    extern __shared__ __align__(16) u32 lds[];
    __shared__ u32 twice;
    const u32 part = blockIdx.x % P.parts;
    const long long row = P.row0 + blockIdx.x / P.parts;
    const RowView<DT> r(P.student, row, P.row_bytes, P.n);
    char* out = P.grad + row * P.grad_bytes;
    const bool aligned = (((uintptr_t)out ^ (uintptr_t)r.x) & 15) == 0;
    const long long* columns = P.columns + row * P.k;
    const u32 v0 = part * P.part_vecs, v1 = part_end(v0, P.part_vecs, r.nvec);
    const DistillRow d = P.rows[row];
    const float g = P.grad_loss[row] * P.inv_t, a = g * d.dense, b = d.s == 0.0f ? 0.0f : d.q / d.s, m = finite_or_zero(d.m);
    const bool tail = P.teacher_lse != nullptr;
    if (g == 0.0f) {  // (padding: its logits may be anything)
        for (u32 v = v0 + threadIdx.x; v < v1; v += kDistillGradBlock) {
            const float none[RowElem<DT>::E] = {};
            store_vector<DT>(r, out, aligned, v, none);
        }
        return;
    }
    const ScaledExp<DT> dense(a, d.mu, P.c);
    write_gradient<DT, kDistillGradBlock, kDistillGradVecs, 4, NT>(
        r, out, aligned, v0, v1, P.k, lds, &twice, [&](long long i) { return columns[i]; },
        [&](long long i) {
            const float z = load_as_float(P.values, P.value_dt, (size_t)(row * P.k + i));
            return expf(ln_share(z, d, tail, 0.0f, P.inv_t)) * d.zmul;
        },
        [&](float (&x)[RowElem<DT>::E]) { dense.of(x); },
        [&](float x, float q) { return g * (b * exp2_fast((x - m) * P.c) - q); });
}

constexpr int64_t kDistillMostVecs = (int64_t)1 << 15;  // (the bitmaps: a byte each)

// One workgroup per row, which then has its loss too, or several, and a launch more.
constexpr int kPartBlock = 256;
static bool whole_rows(int64_t batch, int64_t n, int eb) { return (n + 14) * eb <= 16 * kDistillMostVecs && (batch >= 128 || n * eb <= 65536); }
static RowParts distill_parts(int64_t batch, int64_t n, int eb) {
    return deal_row(batch, n, eb, kPartBlock * kDistillVecs, 2048, kDistillMostVecs);
}

// 16-byte vectors that a row may take: one more than its bytes need where rows do not all start on a multiple of 16.
static int64_t vectors_of(const void* x, int64_t n, int64_t stride, rtopk_dtype dt) {
    const int64_t eb = dt == RTOPK_F32 ? 4 : 2, E = 16 / eb;
    const bool even = (uintptr_t)x % 16 == 0 && stride % E == 0;
    return (n + (even ? 0 : E - 1) + E - 1) / E;
}
// Whether workgroups keep their rows from the loss to the gradient.  Rows of more than 8192 vectors take a compute unit each, so a batch takes as long as the next multiple of 256: kept where
// it nearly is one (kept / in two launches, us, rows of 131072 bf16 with the rest: 257 rows 70 / 48, 400 71 / 66, 512 74 / 81, 600 103 / 95, 900 135 / 131, 1030 167 / 148).
// Of shorter ones several share a unit (rows of 65536: 130 rows 21 / 23, 257 30 / 32, 600 46 / 52).
static bool step_is_held(int64_t batch, int64_t vecs) {
    if (vecs <= 4096) return true;
    if (vecs <= 8192) return batch >= 128;
    return vecs <= kHeldVecs && batch * 10 >= (batch + 255) / 256 * 256 * 9;
}

}  // namespace rtopk

using namespace rtopk;

static rtopk_status check_lists(const void* student, int64_t batch, int64_t n, int64_t row_stride, rtopk_dtype dt, float inv_temperature,
                                const void* teacher_values, rtopk_dtype teacher_dt, const int64_t* teacher_columns, int64_t k, const float* teacher_lse) {
    const rtopk_status s = check_rows(student, batch, n, row_stride, dt);
    if (s != RTOPK_OK) return s;
    if (!usable_temperature(inv_temperature) || k < 1 || k > 0x7fffffff || !teacher_values || !teacher_columns) return RTOPK_ERR_INVALID_ARG;
    if (teacher_dt != RTOPK_F32 && teacher_dt != RTOPK_F16 && teacher_dt != RTOPK_BF16) return RTOPK_ERR_INVALID_ARG;
    if ((uintptr_t)teacher_columns % 8 || (uintptr_t)teacher_values % (teacher_dt == RTOPK_F32 ? 4 : 2) || (uintptr_t)teacher_lse % 4) return RTOPK_ERR_UNSUPPORTED;
    return RTOPK_OK;
}

static DistillParams distill_params(const void* student, int64_t n, int64_t row_stride, rtopk_dtype dt, float inv_temperature, const void* teacher_values,
                                    rtopk_dtype teacher_dt, const int64_t* teacher_columns, int64_t k, const float* teacher_lse) {
    DistillParams P = {};
    P.student = (const char*)student;
    P.row_bytes = row_stride * (dt == RTOPK_F32 ? 4 : 2);
    P.n = (u32)n;
    P.k = k;
    P.c = inv_temperature * kLog2e;
    P.inv_t = inv_temperature;
    P.values = teacher_values;
    P.value_dt = teacher_dt;
    P.columns = (const long long*)teacher_columns;
    P.teacher_lse = teacher_lse;
    return P;
}

extern "C" {

rtopk_status rtopk_distill_workspace_bytes(int64_t batch, int64_t n, int64_t k, rtopk_dtype dt, size_t* bytes_out) {
    if (!bytes_out || batch < 1 || batch > 0x7fffffff || n < 1 || n > RTOPK_MAX_N || k < 1 || k > 0x7fffffff) return RTOPK_ERR_INVALID_ARG;
    if (dt != RTOPK_F32 && dt != RTOPK_F16 && dt != RTOPK_BF16) return RTOPK_ERR_INVALID_ARG;
    const int eb = dt == RTOPK_F32 ? 4 : 2;
    *bytes_out = up256((size_t)batch * distill_parts(batch, n, eb).parts * 2 * sizeof(float4)) + up256((size_t)batch * sizeof(DistillRow));
    return RTOPK_OK;
}

rtopk_status rtopk_distill(const void* student, int64_t batch, int64_t n, int64_t row_stride, rtopk_dtype dt, float inv_temperature,
                           const void* teacher_values, rtopk_dtype teacher_dt, const int64_t* teacher_columns, int64_t k, const float* teacher_lse,
                           float* out_loss, float* out_row_stats, void* workspace, size_t workspace_bytes, void* hip_stream) {
    rtopk_status s = check_lists(student, batch, n, row_stride, dt, inv_temperature, teacher_values, teacher_dt, teacher_columns, k, teacher_lse);
    if (s != RTOPK_OK) return s;
    if (!out_loss || !workspace) return RTOPK_ERR_INVALID_ARG;
    if (((uintptr_t)out_loss | (uintptr_t)out_row_stats) % 4 || (uintptr_t)workspace % 256) return RTOPK_ERR_UNSUPPORTED;
    size_t need = 0;
    s = rtopk_distill_workspace_bytes(batch, n, k, dt, &need);
    if (s != RTOPK_OK) return s;
    if (workspace_bytes < need) return RTOPK_ERR_WORKSPACE_TOO_SMALL;
    DistillParams P = distill_params(student, n, row_stride, dt, inv_temperature, teacher_values, teacher_dt, teacher_columns, k, teacher_lse);
    const RowParts d = distill_parts(batch, n, dt == RTOPK_F32 ? 4 : 2);
    P.parts = d.parts;
    P.part_vecs = d.vecs;
    P.partial = (float4*)workspace;
    P.loss = out_loss;
    P.rows = (DistillRow*)out_row_stats;
    const hipStream_t st = (hipStream_t)hip_stream;
    (void)hipGetLastError();  // an error left by earlier HIP calls of the process is not this call's
    return by_type(dt, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        if (whole_rows(batch, n, dt == RTOPK_F32 ? 4 : 2)) {
            P.part_vecs = (u32)((n + 2 * (RowElem<DT>::E - 1)) / RowElem<DT>::E);
            auto of = [&](auto is_tail, auto block) {
                constexpr bool TAIL = decltype(is_tail)::value;
                constexpr int B = decltype(block)::value;
                for (P.row0 = 0; P.row0 < batch; P.row0 += kMostWorkgroups) {
                    const unsigned now = (unsigned)(batch - P.row0 < kMostWorkgroups ? batch - P.row0 : kMostWorkgroups);
                    const size_t lds = TAIL ? P.part_vecs + 3 : 0;
                    if (past_caches(batch, n, RowElem<DT>::kBytes)) hipLaunchKernelGGL((k_distill_part<DT, true, TAIL, B, true>), dim3(now), dim3(B), lds, st, P);
                    else hipLaunchKernelGGL((k_distill_part<DT, false, TAIL, B, true>), dim3(now), dim3(B), lds, st, P);
                }
            };
            auto by_block = [&](auto is_tail) {
                if (batch <= 256) of(is_tail, std::integral_constant<int, 1024>{});
                else if (batch <= 512) of(is_tail, std::integral_constant<int, 512>{});
                else of(is_tail, std::integral_constant<int, 256>{});
            };
            teacher_lse ? by_block(std::true_type{}) : by_block(std::false_type{});
            return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_ERR_HIP;
        }
        const int64_t rows = kMostWorkgroups / d.parts > 0 ? kMostWorkgroups / d.parts : 1;
        for (P.row0 = 0; P.row0 < batch; P.row0 += rows) {
            const unsigned now = (unsigned)(batch - P.row0 < rows ? batch - P.row0 : rows);
            auto of = [&](auto is_tail) {
                constexpr bool TAIL = decltype(is_tail)::value;
                hipLaunchKernelGGL((k_distill_part<DT, false, TAIL, kPartBlock, false>), dim3(now * d.parts), dim3(kPartBlock), TAIL ? d.vecs : 0, st, P);
                hipLaunchKernelGGL((k_distill_finish<DT, TAIL>), dim3(now), dim3(kDistillFinish), 0, st, P);
            };
            teacher_lse ? of(std::true_type{}) : of(std::false_type{});
        }
        return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_ERR_HIP;
    });
}

rtopk_status rtopk_distill_backward(const void* student, int64_t batch, int64_t n, int64_t row_stride, rtopk_dtype dt, float inv_temperature,
                                    const void* teacher_values, rtopk_dtype teacher_dt, const int64_t* teacher_columns, int64_t k,
                                    const float* teacher_lse, const float* row_stats, const float* grad_loss, void* out_grad, int64_t grad_stride,
                                    void* hip_stream) {
    rtopk_status s = check_lists(student, batch, n, row_stride, dt, inv_temperature, teacher_values, teacher_dt, teacher_columns, k, teacher_lse);
    if (s == RTOPK_OK) s = check_rows(out_grad, batch, n, grad_stride, dt);
    if (s != RTOPK_OK) return s;
    const int eb = dt == RTOPK_F32 ? 4 : 2;
    if (!row_stats || !grad_loss || rows_overlap(student, row_stride, out_grad, grad_stride, batch, n, eb)) return RTOPK_ERR_INVALID_ARG;
    if (((uintptr_t)row_stats | (uintptr_t)grad_loss) % 4) return RTOPK_ERR_UNSUPPORTED;
    DistillParams P = distill_params(student, n, row_stride, dt, inv_temperature, teacher_values, teacher_dt, teacher_columns, k, teacher_lse);
    const RowParts d = deal_row(batch, n, eb, kDistillGradBlock * kDistillGradVecs, 4096, kDistillMostVecs);
    P.parts = d.parts;
    P.part_vecs = d.vecs;
    P.rows = (DistillRow*)row_stats;
    P.grad_loss = grad_loss;
    P.grad = (char*)out_grad;
    P.grad_bytes = grad_stride * eb;
    (void)hipGetLastError();
    return by_type(dt, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        const int64_t rows = kMostWorkgroups / d.parts > 0 ? kMostWorkgroups / d.parts : 1;
        const size_t lds = gradient_lds<DT, kDistillGradBlock, kDistillGradVecs>(d.vecs);
        for (P.row0 = 0; P.row0 < batch; P.row0 += rows) {
            const unsigned now = (unsigned)(batch - P.row0 < rows ? batch - P.row0 : rows);
            if (past_caches(batch, n, eb)) hipLaunchKernelGGL((k_distill_grad<DT, true>), dim3(now * d.parts), dim3(kDistillGradBlock), lds, (hipStream_t)hip_stream, P);
            else hipLaunchKernelGGL((k_distill_grad<DT, false>), dim3(now * d.parts), dim3(kDistillGradBlock), lds, (hipStream_t)hip_stream, P);
        }
        return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_ERR_HIP;
    });
}

rtopk_status rtopk_distill_step(const void* student, int64_t batch, int64_t n, int64_t row_stride, rtopk_dtype dt, float inv_temperature,
                                const void* teacher_values, rtopk_dtype teacher_dt, const int64_t* teacher_columns, int64_t k,
                                const float* teacher_lse, const float* row_weights, float* out_loss, void* out_grad, int64_t grad_stride,
                                void* workspace, size_t workspace_bytes, void* hip_stream) {
    size_t need = 0;
    rtopk_status s = rtopk_distill_workspace_bytes(batch, n, k, dt, &need);
    if (s != RTOPK_OK) return s;
    if (!workspace || !out_grad || !row_weights) return RTOPK_ERR_INVALID_ARG;
    if (workspace_bytes < need) return RTOPK_ERR_WORKSPACE_TOO_SMALL;
    // what can be refused is, before anything is launched
    s = check_rows(out_grad, batch, n, grad_stride, dt);
    if (s != RTOPK_OK) return s;
    if ((uintptr_t)row_weights % 4) return RTOPK_ERR_UNSUPPORTED;
    if (rows_overlap(student, row_stride, out_grad, grad_stride, batch, n, dt == RTOPK_F32 ? 4 : 2)) return RTOPK_ERR_INVALID_ARG;
    if (step_is_held(batch, vectors_of(student, n, row_stride, dt))) {
        if (!student || !out_loss) return RTOPK_ERR_INVALID_ARG;
        s = check_lists(student, batch, n, row_stride, dt, inv_temperature, teacher_values, teacher_dt, teacher_columns, k, teacher_lse);
        if (s != RTOPK_OK) return s;
        if ((uintptr_t)out_loss % 4 || (uintptr_t)workspace % 256) return RTOPK_ERR_UNSUPPORTED;
        DistillParams P = distill_params(student, n, row_stride, dt, inv_temperature, teacher_values, teacher_dt, teacher_columns, k, teacher_lse);
        P.batch = batch;
        P.loss = out_loss;
        P.grad_loss = row_weights;
        P.grad = (char*)out_grad;
        P.grad_bytes = grad_stride * (dt == RTOPK_F32 ? 4 : 2);
        const int64_t vecs = vectors_of(student, n, row_stride, dt);
        (void)hipGetLastError();  // an error left by earlier HIP calls of the process is not this call's
        switch (dt) {
            case RTOPK_F32: return launch_distill_step_f32(P, vecs, (hipStream_t)hip_stream);
            case RTOPK_F16: return launch_distill_step_f16(P, vecs, (hipStream_t)hip_stream);
            case RTOPK_BF16: return launch_distill_step_bf16(P, vecs, (hipStream_t)hip_stream);
        }
        return RTOPK_ERR_INVALID_ARG;
    }
    float* rows = (float*)((char*)workspace + need - up256((size_t)batch * sizeof(DistillRow)));
    s = rtopk_distill(student, batch, n, row_stride, dt, inv_temperature, teacher_values, teacher_dt, teacher_columns, k, teacher_lse, out_loss, rows, workspace,
                      workspace_bytes, hip_stream);
    if (s != RTOPK_OK) return s;
    return rtopk_distill_backward(student, batch, n, row_stride, dt, inv_temperature, teacher_values, teacher_dt, teacher_columns, k, teacher_lse, rows, row_weights,
                                  out_grad, grad_stride, hip_stream);
}

}  // extern "C"
