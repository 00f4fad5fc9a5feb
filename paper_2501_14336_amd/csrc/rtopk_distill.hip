// Distillation from a teacher's top logits: the divergence of a student's row from a teacher's list of (column, logit), and its gradient
// (rtopk_distill, rtopk_distill_backward, rtopk_distill_step).
//
//   q_i = exp(z_i / T) / sum exp(z_l / T), or exp(z_i / T - lse) with the teacher's own log-sum; then r = max(0, 1 - sum q) is the rest's share
//   L   = sum q_i (ln q_i - ln p_{t_i}) [ + r (ln r - ln P),  P = sum of p over the columns that are not listed ]
//   dL/dx_j = (1/T) [ (sum q + r) p_j - sum_{t_i = j} q_i - [j not listed] r p_j / P ]
//
// P is added up from the columns that are not listed, not taken as what the listed ones leave of 1: a trained student leaves 1e-6 and less.
#include "rtopk_softmax.h"

namespace rtopk {

// What a row's forward pass leaves for its gradient.  p_j = exp((x_j - m) / T) / s.
struct DistillRow {
    float m, s;        // the student's maximum and sum
    float zref, zmul;  // q_i = exp((z_i - zref) / T) * zmul, or exp(z_i / T - zref) with the teacher's log-sum
    float mu, dense;   // columns not listed: dx = (g / T) exp((x - mu) / T) dense
    float q, spare;    // sum q + r
};
static_assert(sizeof(DistillRow) == RTOPK_DISTILL_ROW_STATS * sizeof(float), "as declared");

struct DistillParams {
    const char* student;
    long long row_bytes, row0, batch, k;
    u32 n, parts, part_vecs;
    float c, inv_t;
    const void* values;         // [batch][k], type value_dt
    int value_dt;
    const long long* columns;   // [batch][k]
    const float* teacher_lse;   // [batch], or null
    float4* partial;            // [batch][parts][2]: columns not listed, listed columns
    float* loss;
    DistillRow* rows;
    // the gradient
    const float* grad_loss;
    char* grad;
    long long grad_bytes;
};

constexpr int kDistillBlock = 256, kDistillVecs = 4;

// Statistics of a part of a row; TAIL: apart for columns that are listed and for the others.
template <int DT, bool TAIL>
__global__ void __launch_bounds__(kDistillBlock) k_distill_part(DistillParams P) {
    extern __shared__ u32 marks[];  // TAIL: a byte per vector of the part, a bit per column
    __shared__ float4 sm[kDistillBlock / 64];
    constexpr int E = RowElem<DT>::E;
    const u32 part = blockIdx.x % P.parts;
    const long long row = P.row0 + blockIdx.x / P.parts;
    const RowView<DT> r(P.student, row, P.row_bytes, P.n);
    const u32 v0 = part * P.part_vecs, v1 = part_end(v0, P.part_vecs, r.nvec);
    SoftSum a, listed;
    if (TAIL) {
        const long long* columns = P.columns + row * P.k;
        for (u32 i = threadIdx.x; i < (P.part_vecs + 3) / 4; i += kDistillBlock) marks[i] = 0;
        __syncthreads();
        for (long long i = threadIdx.x; i < P.k; i += kDistillBlock) {
            const long long t = columns[i];
            const u64 p = (u64)(t + r.lead) - (u64)v0 * E;  // (wraps below the part)
            if (t >= 0 && t < (long long)P.n && p < (u64)(v1 - v0) * E) {
                const u32 v = (u32)p / E, bit = 1u << ((v & 3) * 8 + (u32)p % E);
                if (!(atomicOr(&marks[v >> 2], bit) & bit)) {  // a column listed twice counts once
                    const float x[1] = {RowElem<DT>::load(r.x, (u32)t)};
                    soft_add<false>(listed, x, P.c);
                }
            }
        }
        __syncthreads();
    }
    sweep_vectors<DT, kDistillBlock, kDistillVecs, false>(r, v0, v1, [&](const u32x4 (&q)[kDistillVecs], u32 first) {
        float x[kDistillVecs * E];
#pragma unroll
        for (int i = 0; i < kDistillVecs; ++i) {
            u32 bits = 0;
            if (TAIL) {
                const u32 v = first + i * kDistillBlock + threadIdx.x;
                if (v < v1) bits = ((const uint8_t*)marks)[v - v0];
            }
            float y[E];
            RowElem<DT>::unpack(TAIL ? RowElem<DT>::without(q[i], bits) : q[i], y);
#pragma unroll
            for (int j = 0; j < E; ++j) x[i * E + j] = y[j];
        }
        soft_add<false>(a, x, P.c);
    });
    a = soft_block<kDistillBlock, false>(a, P.c, sm);
    if (threadIdx.x == 0) P.partial[(row * P.parts + part) * 2] = packed(a);
    if (TAIL) {
        __syncthreads();
        listed = soft_block<kDistillBlock, false>(listed, P.c, sm);
        if (threadIdx.x == 0) P.partial[(row * P.parts + part) * 2 + 1] = packed(listed);
    }
}

// ln of an entry's share.
__device__ __forceinline__ float ln_share(float z, const DistillRow& d, bool tail, float ln_zmul, float inv_t) {
    return tail ? z * inv_t - d.zref : (z - d.zref) * inv_t + ln_zmul;
}

// A row's statistics from the sums of all its columns (a), of those that are not listed (others), of the teacher's list (zs), and of its shares (share): fills d, whose zref and zmul
// are there, and returns the rest's part of the loss.
template <bool TAIL>
__device__ __forceinline__ float finish_row(DistillRow& d, const SoftSum& a, const SoftSum& others, double share, float zs, const DistillParams& P) {
    d.m = a.m;
    d.s = a.s;
    d.spare = 0.0f;
    if (!TAIL) {
        d.q = zs == 0.0f ? 0.0f : zs != zs ? zs : 1.0f;
        d.mu = finite_or_zero(a.m);
        d.dense = a.s == 0.0f ? 0.0f : d.q / a.s;
        return 0.0f;
    }
    const float rest = share < 1.0 ? (float)(1.0 - share) : share != share ? (float)share : 0.0f;
    const float ln_other = others.s == 0.0f ? -__builtin_inff() : (others.m - a.m) * P.inv_t + kLn2 * (log2_fast(others.s) - log2_fast(a.s));
    d.q = share < 1.0 ? 1.0f : (float)share;
    d.mu = finite_or_zero(others.m);
    d.dense = others.s == 0.0f ? 0.0f : d.q * exp2_fast((d.mu - finite_or_zero(a.m)) * P.c) / a.s - rest / others.s;
    return rest != 0.0f ? rest * (kLn2 * log2_fast(rest) - ln_other) : 0.0f;
}

// An entry's share under the teacher's log-sum, without the rounding of its logarithm: what all of them leave of 1 may be a millionth.
__device__ __forceinline__ double exact_share(float z, float lse, float inv_t) {
    const float p = z * inv_t, low = __builtin_fmaf(z, inv_t, -p), hi = p - lse, back = hi - p;  // p + low is z inv_t exactly; hi + rest is p - lse exactly
    const float rest = (p - (hi - back)) + (-lse - back);
    const double e = (double)expf(hi);
    return fabsf(hi) < 1e30f ? e * (1.0 + (double)(low + rest)) : e;  // (a masked entry has none to add)
}

constexpr int kDistillFinish = 256;

template <int DT>
__global__ void __launch_bounds__(kDistillFinish) k_distill_finish(DistillParams P) {
    __shared__ float4 sm[3][kDistillFinish / 64];
    __shared__ double sums[2][kDistillFinish / 64];
    const long long row = P.row0 + blockIdx.x;
    const bool tail = P.teacher_lse != nullptr;
    const RowView<DT> r(P.student, row, P.row_bytes, P.n);
    const long long* columns = P.columns + row * P.k;
    SoftSum a, listed, z;
    for (u32 i = threadIdx.x; i < P.parts; i += kDistillFinish) {
        a = soft_join<false>(a, unpacked(P.partial[(row * P.parts + i) * 2]), P.c);
        if (tail) listed = soft_join<false>(listed, unpacked(P.partial[(row * P.parts + i) * 2 + 1]), P.c);
    }
    a = soft_block<kDistillFinish, false>(a, P.c, sm[0]);
    const SoftSum others = a;
    if (tail) a = soft_join<false>(a, soft_block<kDistillFinish, false>(listed, P.c, sm[1]), P.c);
    DistillRow d;
    float ln_zmul = 0.0f;
    if (tail) {
        d.zref = P.teacher_lse[row];
        d.zmul = 1.0f;
    } else {
        for (long long i = threadIdx.x; i < P.k; i += kDistillFinish)
            if (columns[i] >= 0) {
                const float v[1] = {load_as_float(P.values, P.value_dt, (size_t)(row * P.k + i))};
                soft_add<false>(z, v, P.c);
            }
        z = soft_block<kDistillFinish, false>(z, P.c, sm[2]);
        d.zref = finite_or_zero(z.m);
        d.zmul = z.s == 0.0f ? 0.0f : 1.0f / z.s;
        ln_zmul = z.s == 0.0f ? 0.0f : -kLn2 * log2_fast(z.s);
    }
    const float ln_s = kLn2 * log2_fast(a.s);
    float loss = 0.0f;
    double q = 0.0;
    for (long long i = threadIdx.x; i < P.k; i += kDistillFinish) {
        const long long t = columns[i];
        if (t < 0) continue;
        const float z = load_as_float(P.values, P.value_dt, (size_t)(row * P.k + i)), lq = ln_share(z, d, tail, ln_zmul, P.inv_t), qi = expf(lq);
        if (tail) q += exact_share(z, d.zref, P.inv_t);
        if (t >= (long long)P.n) {
            loss += __builtin_nanf("");
        } else if (qi != 0.0f) {
            const float x = RowElem<DT>::load(r.x, (u32)t);
            loss += qi * (lq - (a.s == 0.0f ? -__builtin_inff() : (x - a.m) * P.inv_t - ln_s));
        }
    }
    loss = sum_block<kDistillFinish>(loss, (float*)sums[0]);
    if (tail) q = sum_block<kDistillFinish>(q, sums[1]);
    loss += tail ? finish_row<true>(d, a, others, q, z.s, P) : finish_row<false>(d, a, others, q, z.s, P);
    if (threadIdx.x == 0) {
        P.loss[row] = loss;
        if (P.rows) P.rows[row] = d;
    }
}

constexpr int kDistillGradBlock = 256, kDistillGradVecs = 4;

template <int DT>
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
    write_gradient<DT, kDistillGradBlock, kDistillGradVecs, 4, false>(
        r, out, aligned, v0, v1, P.k, lds, &twice, [&](long long i) { return columns[i]; },
        [&](long long i) {
            const float z = load_as_float(P.values, P.value_dt, (size_t)(row * P.k + i));
            return expf(ln_share(z, d, tail, 0.0f, P.inv_t)) * d.zmul;
        },
        [&](float (&x)[RowElem<DT>::E]) { dense.of(x); },
        [&](float x, float q) { return g * (b * exp2_fast((x - m) * P.c) - q); });
}

// Loss and gradient in one launch: a workgroup holds its row in registers between the two, so that the row is read once, and written once.  A vector's registers are free once its gradient is
// on its way, and take the vector of the workgroup's next row: that row comes in while this one goes out.  (A workgroup of 1024 threads has a compute unit to itself; with a
// launch of a workgroup per row the unit read, computed and wrote one after the other, 152 us for 1024 rows of 131072 bf16 with 50 entries each.)
// EVEN: rows start and end on multiples of 16 bytes.
template <int DT, int B, int NV, bool TAIL, bool EVEN>
__global__ void __launch_bounds__(B, 4) k_distill_step(DistillParams P) {
    extern __shared__ __align__(16) u32 lds[];
    __shared__ u32 twice;
    __shared__ float4 sm[3][B / 64];
    __shared__ double sums[2][B / 64];
    constexpr int E = RowElem<DT>::E, R = B >= 1024 ? 1 : B >= 512 ? 2 : 4, kChunk = E / 2;
    const u32x4 none = {RowElem<DT>::kMinusInf, RowElem<DT>::kMinusInf, RowElem<DT>::kMinusInf, RowElem<DT>::kMinusInf};
    long long row = blockIdx.x;
    // the thread's entries
    long long col[R];
    float z[R];
    auto fetch_entries = [&](long long of, long long (&c)[R], float (&v)[R]) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const long long i = threadIdx.x + (long long)k * B;
            c[k] = -1;
            v[k] = 0.0f;
            if (i < P.k) {
                c[k] = P.columns[of * P.k + i];
                v[k] = load_as_float(P.values, P.value_dt, (size_t)(of * P.k + i));
            }
        }
    };
    fetch_entries(row, col, z);
    // a vector of a row; EVEN: by a descriptor of the row's bytes, beyond which there is nothing
    auto descriptor = [&](const char* p, bool there) { return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, there ? (int)(P.n * RowElem<DT>::kBytes) : 0, 0x00027000); };
    auto fetch = [&](const RowView<DT>& r, __amdgpu_buffer_rsrc_t from, bool there, u32 v) {
        if constexpr (EVEN) {
            return __builtin_amdgcn_raw_buffer_load_b128(from, v * 16, 0, 2);
        } else {
            u32x4 q = none;
            if (there && v < r.nvec) q = r.trimmed(r.template load<true>(v), v);
            return q;
        }
    };
    u32x4 q[NV];
    {
        const RowView<DT> r(P.student, row, P.row_bytes, P.n);
        const auto from = descriptor(r.x, true);
#pragma unroll
        for (int i = 0; i < NV; ++i) q[i] = fetch(r, from, true, i * B + threadIdx.x);
    }
    for (;;) {
        u32 thread = threadIdx.x;
        asm volatile("" : "+v"(thread));  // (what depends on the thread alone is made anew for every row: kept, it takes the registers that hold the row)
        const long long next = row + gridDim.x;
        const bool more = next < P.batch;
        const RowView<DT> r(P.student, row, P.row_bytes, P.n), r_next(P.student, more ? next : row, P.row_bytes, P.n);
        const auto from_next = descriptor(r_next.x, more);
        char* out = P.grad + row * P.grad_bytes;
        const auto to = descriptor(out, true);
        const bool aligned = EVEN || (((uintptr_t)out ^ (uintptr_t)r.x) & 15) == 0;
        const long long* columns = P.columns + row * P.k;
        const float g = P.grad_loss[row] * P.inv_t;
        const auto at = [&](long long i) { return columns[i]; };
        DistillRow d;
        d.zref = TAIL ? P.teacher_lse[row] : 0.0f;
        float ln_zmul = 0.0f, zs = 1.0f;
        const auto unused = [](long long) { return 0.0f; };
        ListedColumns<DT, B, 1, R, decltype(at), decltype(unused)>::clear(r.nvec, lds, &twice);
        if (TAIL) __syncthreads();
        if (!TAIL) {
            SoftSum a;
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float v[1] = {col[k] >= 0 ? z[k] : -__builtin_inff()};
                soft_add<false>(a, v, P.c);
            }
            for (long long i = thread + (long long)R * B; i < P.k; i += B)
                if (columns[i] >= 0) {
                    const float v[1] = {load_as_float(P.values, P.value_dt, (size_t)(row * P.k + i))};
                    soft_add<false>(a, v, P.c);
                }
            a = soft_block<B, false>(a, P.c, sm[0]);
            d.zref = uniform(finite_or_zero(a.m));
            zs = uniform(a.s);
            ln_zmul = uniform(zs == 0.0f ? 0.0f : -kLn2 * log2_fast(zs));
        }
        auto ln_q = [&](float v) { return ln_share(v, d, TAIL, ln_zmul, P.inv_t); };
        float loss = 0.0f;
        double share = 0.0;  // TAIL: of all that is listed
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (col[k] >= (long long)P.n) loss = __builtin_nanf("");
            if (TAIL && col[k] >= 0) share += exact_share(z[k], d.zref, P.inv_t);
            z[k] = ln_q(z[k]);
        }
        for (long long i = thread + (long long)R * B; i < P.k; i += B) {
            const long long t = columns[i];
            if (t >= (long long)P.n) loss = __builtin_nanf("");
            if (TAIL && t >= 0) share += exact_share(load_as_float(P.values, P.value_dt, (size_t)(row * P.k + i)), d.zref, P.inv_t);
        }
        SoftSum listed;
        const auto ln_value = [&](long long i) { return ln_q(load_as_float(P.values, P.value_dt, (size_t)(row * P.k + i))); };
        const auto value = [&](long long i) { return expf(ln_value(i)); };
        ListedColumns<DT, B, 1, R, decltype(at), decltype(value)> list(
            std::true_type{}, r, 0, r.nvec, P.k, lds, &twice, at, value,
            [&](int k, long long& t, float& v) {
                t = col[k];
                v = expf(z[k]);
            },
            [&](u32 p) {
                if (TAIL) {
                    const float x[1] = {RowElem<DT>::load(r.x, p - r.lead)};
                    soft_add<false>(listed, x, P.c);
                }
            });
        // first pass: the softmax; TAIL: of what is not listed.  Listed columns' logits go to the threads that have their entries, by way of the tiles.  (Fetched by their columns they are a
        // line each: for 1024 of a row half as much again as the row.)
        SoftSum a;
        float x_of[R];
#pragma unroll
        for (int k = 0; k < R; ++k) x_of[k] = 0.0f;
        u32x4* const raw = (u32x4*)list.tile;
        static_assert(kChunk * B * 16 <= 2 * B * E * 4, "a chunk's vectors fit both tiles");
#pragma unroll
        for (int i0 = 0; i0 < NV; i0 += kChunk) {
            float x[kChunk * E];
#pragma unroll
            for (int i = 0; i < kChunk; ++i) {
                const u32 v = (i0 + i) * B + thread;
                if (EVEN && (u32)(i0 + i + 1) * B > r.nvec) q[i0 + i] = v < r.nvec ? q[i0 + i] : none;
                const u32 bits = v < r.nvec ? list.listed_of(v) : 0;
                if (bits) raw[i * B + thread] = q[i0 + i];
                float y[E];
                // (without a branch: with one, the compiler keeps both sides' registers)
                RowElem<DT>::unpack(TAIL ? RowElem<DT>::without(q[i0 + i], bits) : q[i0 + i], y);
#pragma unroll
                for (int j = 0; j < E; ++j) x[i * E + j] = y[j];
            }
            soft_add<false>(a, x, P.c);
            __syncthreads();
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const u32 p = list.place[k] - i0 * B * E;
                if (list.place[k] != list.kNone && p < kChunk * B * E) x_of[k] = RowElem<DT>::load((const char*)raw, p);
            }
            if (i0 + kChunk < NV) __syncthreads();
            __builtin_amdgcn_sched_barrier(0);  // (a chunk at a time: registers)
        }
        // (the second pass converts the row anew: kept as 32-bit numbers, it would not fit)
#pragma unroll
        for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(q[i]));
        if (TAIL) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float x[1] = {list.fresh[k] ? x_of[k] : -__builtin_inff()};
                soft_add<false>(listed, x, P.c);
            }
        }
        a = soft_block<B, false>(a, P.c, sm[1]);
        const SoftSum others = a;
        if (TAIL) a = soft_join<false>(a, soft_block<B, false>(listed, P.c, sm[2]), P.c);
        if (TAIL) share = sum_block<B>(share, sums[0]);
        const float of_rest = finish_row<TAIL>(d, a, others, share, zs, P);
        if (thread == 0) loss += of_rest;
        // the entries: their part of the loss, and their columns' gradients
        d.m = uniform(d.m), d.s = uniform(d.s), d.mu = uniform(d.mu), d.dense = uniform(d.dense), d.q = uniform(d.q);
        const float b = uniform(d.s == 0.0f ? 0.0f : d.q / d.s), m = finite_or_zero(d.m), ln_s = uniform(kLn2 * log2_fast(d.s));
        auto loss_of = [&](float lq, float x) {
            const float qi = expf(lq);
            return qi != 0.0f ? qi * (lq - (d.s == 0.0f ? -__builtin_inff() : (x - d.m) * P.inv_t - ln_s)) : 0.0f;
        };
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (col[k] >= 0 && col[k] < (long long)P.n) loss += loss_of(z[k], x_of[k]);
        for (long long i = thread + (long long)R * B; i < P.k; i += B) {
            const long long t = columns[i];
            if (t >= 0 && t < (long long)P.n) loss += loss_of(ln_value(i), RowElem<DT>::load(r.x, (u32)t));
        }
        loss = sum_block<B>(loss, (float*)sums[1]);
        if (thread == 0) P.loss[row] = loss;
        auto of_column = [&](int k, u32 p, float sum) {
            float x = 0.0f;
            if (k < 0) x = RowElem<DT>::load(r.x, p - r.lead);
#pragma unroll
            for (int l = 0; l < R; ++l) x = k == l ? x_of[l] : x;
            return g * (b * exp2_fast((x - m) * P.c) - sum);
        };
        list.work_out(of_column);
        // second pass: the gradient out, the next row in
        if (more) fetch_entries(next, col, z);
        if (g == 0.0f) {  // (padding: its logits may be anything)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const u32 v = i * B + thread;
                const float x[E] = {};
                if constexpr (EVEN) __builtin_amdgcn_raw_buffer_store_b128(RowElem<DT>::pack(x), to, v * 16, 0, 0);
                else if (v < r.nvec) store_vector<DT>(r, out, aligned, v, x);
                q[i] = fetch(r_next, from_next, more, v);
            }
        } else {
            const ScaledExp<DT> dense(g * d.dense, d.mu, P.c);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const u32 v = i * B + thread;
                float* const tile = list.tile + (i & 1) * B * E;
                if ((u32)i * B < r.nvec) {
                    list.put(i * B * E, tile, of_column);
                    __syncthreads();  // (the other tile is free then, too)
                }
                float x[E];
                RowElem<DT>::unpack(q[i], x);
                dense.of(x);
                listed_gradients<DT>(x, v < r.nvec ? list.listed_of(v) : 0, tile + thread * E);
                if constexpr (EVEN) __builtin_amdgcn_raw_buffer_store_b128(RowElem<DT>::pack(x), to, v * 16, 0, 0);
                else if (v < r.nvec) store_vector<DT>(r, out, aligned, v, x);
                q[i] = fetch(r_next, from_next, more, v);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (!more) break;
        row = next;
        __syncthreads();  // (the list's marks have been read)
    }
}

constexpr int64_t kDistillMostVecs = (int64_t)1 << 15;  // (the bitmaps: a byte each)

static RowParts distill_parts(int64_t batch, int64_t n, int eb) {
    return deal_row(batch, n, eb, kDistillBlock * kDistillVecs, 2048, kDistillMostVecs);
}

// 16-byte vectors that a row may take: one more than its bytes need where rows do not all start on a multiple of 16.
static int64_t vectors_of(const void* x, int64_t n, int64_t stride, rtopk_dtype dt) {
    const int64_t eb = dt == RTOPK_F32 ? 4 : 2, E = 16 / eb;
    const bool even = (uintptr_t)x % 16 == 0 && stride % E == 0;
    return (n + (even ? 0 : E - 1) + E - 1) / E;
}
static constexpr int64_t kHeldVecs = 1024 * 20;
static bool step_is_held(int64_t batch, int64_t vecs) { return vecs <= kHeldVecs && (batch >= 128 || vecs <= 4096); }

template <int DT, int B, int NV>
static void launch_step(const DistillParams& P, hipStream_t st) {
    const size_t lds = gradient_lds<DT, B, 2>(B * NV);  // (two tiles of a vector per thread)
    const bool even = (((uintptr_t)P.student | (uintptr_t)P.grad | (uintptr_t)P.row_bytes | (uintptr_t)P.grad_bytes) & 15) == 0 && P.n % RowElem<DT>::E == 0;
    const dim3 grid((unsigned)(P.batch < 256 * (1024 / B) ? P.batch : 256 * (1024 / B)));  // 1024 threads to a compute unit: the registers of more would not hold their rows
    auto go = [&](auto tail, auto is_even) { hipLaunchKernelGGL((k_distill_step<DT, B, NV, decltype(tail)::value, decltype(is_even)::value>), grid, dim3(B), lds, st, P); };
    if (P.teacher_lse) even ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
    else even ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
}
static rtopk_status launch_held_step(const DistillParams& P, rtopk_dtype dt, int64_t vecs, hipStream_t st) {
    (void)hipGetLastError();  // an error left by earlier HIP calls of the process is not this call's
    return by_type(dt, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        if (vecs <= 256 * 4) launch_step<DT, 256, 4>(P, st);
        else if (vecs <= 256 * 8) launch_step<DT, 256, 8>(P, st);
        else if (vecs <= 512 * 8) launch_step<DT, 512, 8>(P, st);
        else if (vecs <= 512 * 16) launch_step<DT, 512, 16>(P, st);
        else if (vecs <= 1024 * 16) launch_step<DT, 1024, 16>(P, st);
        else launch_step<DT, 1024, 20>(P, st);
        return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_ERR_HIP;
    });
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
        const int64_t rows = kMostWorkgroups / d.parts > 0 ? kMostWorkgroups / d.parts : 1;
        for (P.row0 = 0; P.row0 < batch; P.row0 += rows) {
            const unsigned now = (unsigned)(batch - P.row0 < rows ? batch - P.row0 : rows);
            if (teacher_lse) hipLaunchKernelGGL((k_distill_part<DT, true>), dim3(now * d.parts), dim3(kDistillBlock), d.vecs, st, P);
            else hipLaunchKernelGGL((k_distill_part<DT, false>), dim3(now * d.parts), dim3(kDistillBlock), 0, st, P);
            hipLaunchKernelGGL((k_distill_finish<DT>), dim3(now), dim3(kDistillFinish), 0, st, P);
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
            hipLaunchKernelGGL((k_distill_grad<DT>), dim3(now * d.parts), dim3(kDistillGradBlock), lds, (hipStream_t)hip_stream, P);
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
        return launch_held_step(P, dt, vectors_of(student, n, row_stride, dt), (hipStream_t)hip_stream);
    }
    float* rows = (float*)((char*)workspace + need - up256((size_t)batch * sizeof(DistillRow)));
    s = rtopk_distill(student, batch, n, row_stride, dt, inv_temperature, teacher_values, teacher_dt, teacher_columns, k, teacher_lse, out_loss, rows, workspace,
                      workspace_bytes, hip_stream);
    if (s != RTOPK_OK) return s;
    return rtopk_distill_backward(student, batch, n, row_stride, dt, inv_temperature, teacher_values, teacher_dt, teacher_columns, k, teacher_lse, rows, row_weights,
                                  out_grad, grad_stride, hip_stream);
}

}  // extern "C"
