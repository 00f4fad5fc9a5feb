// Distillation in one launch (rtopk_distill_step): the kernel and its launches for one type of logits.
#include "rtopk_distill.h"

namespace rtopk {

// Loss and gradient in one launch: a workgroup holds its row in registers between the two, so that the row is read once, and written once.  A vector's registers are free once its gradient is
// on its way, and take the vector of the workgroup's next row: that row comes in while this one goes out.  (A workgroup of 1024 threads has a compute unit to itself; with a
// launch of a workgroup per row the unit read, computed and wrote one after the other, 152 us for 1024 rows of 131072 bf16 with 50 entries each: 117 so.)  Bound by memory: with 1024
// entries each 132 us, 4.1 TB/s (125 in shorter runs), where a copy of as much takes 115; rows come in one after the other, so a unit's first has nothing to hide behind.
// EVEN: rows start and end on multiples of 16 bytes.
template <int DT, int B, int NV, bool TAIL, bool EVEN, bool LOOP>
__global__ void __launch_bounds__(B, 4) k_distill_step(DistillParams P) {
    extern __shared__ __align__(16) u32 lds[];
    __shared__ u32 twice;
    __shared__ float4 sm[3][B / 64];
    __shared__ double sums[2][B / 64];
    constexpr int E = RowElem<DT>::E, R = B >= 1024 ? 1 : B >= 512 ? 2 : 4, kChunk = E / 2;
    const u32x4 none = {RowElem<DT>::kMinusInf, RowElem<DT>::kMinusInf, RowElem<DT>::kMinusInf, RowElem<DT>::kMinusInf};
    long long row = P.row0 + blockIdx.x;
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
            const u32 first = v - threadIdx.x;
            if (there && first + B <= r.nvec && r.whole(first) && r.whole(first + B - 1)) return r.template load<true>(v);
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
        if (LOOP) asm volatile("" : "+v"(thread));  // (what depends on the thread alone is made anew for every row: kept, it takes the registers that hold the row)
        const long long next = row + gridDim.x;
        const bool more = LOOP && next < P.batch;
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
        if (TAIL && list.repeated) {  // a column listed twice counts once, whichever thread came first: by its first entry
            listed = SoftSum();
#pragma unroll
            for (int k = 0; k < R; ++k) list.fresh[k] = list.place[k] != list.kNone && is_first_of_column(columns, thread + (long long)k * B);
#pragma clang loop unroll(disable)
            for (long long i = thread + (long long)R * B; i < P.k; i += B) {
                const long long t = columns[i];
                if (t < 0 || t >= (long long)P.n || !is_first_of_column(columns, i)) continue;
                const float x[1] = {RowElem<DT>::load(r.x, (u32)t)};
                soft_add<false>(listed, x, P.c);
            }
        }
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
                if (LOOP) q[i] = fetch(r_next, from_next, more, v);
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
                if (LOOP) q[i] = fetch(r_next, from_next, more, v);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (!more) break;
        row = next;
        __syncthreads();  // (the list's marks have been read)
    }
}

template <int DT, int B, int NV>
static void launch_step(DistillParams P, hipStream_t st) {
    const size_t lds = gradient_lds<DT, B, 2>(B * NV);  // (two tiles of a vector per thread)
    const bool even = (((uintptr_t)P.student | (uintptr_t)P.grad | (uintptr_t)P.row_bytes | (uintptr_t)P.grad_bytes) & 15) == 0 && P.n % RowElem<DT>::E == 0;
    // A workgroup of 1024 threads stays for all rows of its compute unit; of smaller ones several share a unit, and are in different steps by themselves.
    constexpr bool kStays = B == 1024;
    const bool stays = kStays && even;
    auto go = [&](auto tail, auto is_even, int64_t wgs) {
        hipLaunchKernelGGL((k_distill_step<DT, B, NV, decltype(tail)::value, decltype(is_even)::value, decltype(is_even)::value && kStays>), dim3((unsigned)wgs), dim3(B), lds, st, P);
    };
    const int64_t most = stays ? (int64_t)1 << 40 : kMostWorkgroups;  // rows of a launch
    for (P.row0 = 0; P.row0 < P.batch; P.row0 += most) {
        const int64_t rows = P.batch - P.row0 < most ? P.batch - P.row0 : most, wgs = stays && rows > 256 ? 256 : rows;
        if (P.teacher_lse) even ? go(std::true_type{}, std::true_type{}, wgs) : go(std::true_type{}, std::false_type{}, wgs);
        else even ? go(std::false_type{}, std::true_type{}, wgs) : go(std::false_type{}, std::false_type{}, wgs);
    }
}
template <int DT>
static rtopk_status launch_step_of(const DistillParams& P, int64_t vecs, hipStream_t st) {
    if (vecs <= 256 * 4) launch_step<DT, 256, 4>(P, st);
    else if (vecs <= 256 * 8) launch_step<DT, 256, 8>(P, st);
    else if (vecs <= 512 * 8) launch_step<DT, 512, 8>(P, st);
    else if (vecs <= 512 * 16) launch_step<DT, 512, 16>(P, st);
    else if (vecs <= 1024 * 16) launch_step<DT, 1024, 16>(P, st);
    else launch_step<DT, 1024, 20>(P, st);
    return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_ERR_HIP;
}

}  // namespace rtopk
