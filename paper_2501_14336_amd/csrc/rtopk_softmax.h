// What the operators on whole rows of logits share (rtopk_logprobs.hip, rtopk_distill.hip): reading a row by 16-byte vectors
// from wherever it starts, the running maximum and sums of a softmax, and how a row is dealt to workgroups.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "rtopk.h"
#include "rtopk_device.h"

namespace rtopk {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
// Below this many powers of two a term is zero in 32 bits, and so is its product with its own logarithm.  (Where a masked logit makes the logarithm infinite the product would be NaN.)
constexpr float kNothing = -200.0f;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// ------------------------------------------------------------------------------------------------
// elements
// ------------------------------------------------------------------------------------------------
template <int DT>
struct RowElem {
    static constexpr int kBytes = DT == RTOPK_F32 ? 4 : 2;
    static constexpr int E = 16 / kBytes;  // elements of a 16-byte vector
    static constexpr u32 kMinusInf = DT == RTOPK_F32 ? 0xff800000u : DT == RTOPK_F16 ? 0xfc00fc00u : 0xff80ff80u;

    __device__ static __forceinline__ float from_bits(u32 b) {
        if (DT == RTOPK_F32) return __uint_as_float(b);
        if (DT == RTOPK_F16) return (float)__builtin_bit_cast(_Float16, (uint16_t)b);
        return __uint_as_float(b << 16);
    }
    __device__ static __forceinline__ float load(const char* row, u32 i) {
        return DT == RTOPK_F32 ? *(const float*)(row + (size_t)i * 4) : from_bits(*(const uint16_t*)(row + (size_t)i * 2));
    }
    __device__ static __forceinline__ void unpack(const u32x4& q, float (&x)[E]) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (DT == RTOPK_F32) {
                x[w] = __uint_as_float(q[w]);
            } else if constexpr (DT == RTOPK_BF16) {
                x[2 * w] = __uint_as_float(q[w] << 16);
                x[2 * w + 1] = __uint_as_float(q[w] & 0xffff0000u);
            } else {
                x[2 * w] = from_bits(q[w] & 0xffffu);
                x[2 * w + 1] = from_bits(q[w] >> 16);
            }
        }
    }
    // To the nearest, ties to even; a NaN stays one.
    __device__ static __forceinline__ u32 to_bits(float x) {
        if (DT == RTOPK_F32) return __float_as_uint(x);
        if (DT == RTOPK_F16) return __builtin_bit_cast(uint16_t, (_Float16)x);
        const u32 b = __float_as_uint(x);
        return x != x ? 0x7fc0u : (b + 0x7fffu + ((b >> 16) & 1u)) >> 16;
    }
    __device__ static __forceinline__ void store(char* row, u32 i, float x) {
        if (DT == RTOPK_F32) *(float*)(row + (size_t)i * 4) = x;
        else *(uint16_t*)(row + (size_t)i * 2) = (uint16_t)to_bits(x);
    }
    __device__ static __forceinline__ u32x4 pack(const float (&x)[E]) {
        u32x4 q;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if constexpr (DT == RTOPK_F32) q[w] = __float_as_uint(x[w]);
            else q[w] = to_bits(x[2 * w]) | (to_bits(x[2 * w + 1]) << 16);
        }
        return q;
    }
};

// An element of an array whose type is known at run time only (a teacher's logits).
__device__ __forceinline__ float load_as_float(const void* a, int dt, size_t i) {
    if (dt == RTOPK_F32) return ((const float*)a)[i];
    const u32 b = ((const uint16_t*)a)[i];
    return dt == RTOPK_F16 ? RowElem<RTOPK_F16>::from_bits(b) : RowElem<RTOPK_BF16>::from_bits(b);
}

// ------------------------------------------------------------------------------------------------
// rows
// ------------------------------------------------------------------------------------------------
// A row as vectors of 16 bytes from the 16-byte boundary at or before its first element; column j is element lead + j of them.
template <int DT>
struct RowView {
    static constexpr int E = RowElem<DT>::E;
    const char* x;      // the first element
    const char* base;   // ... and the boundary
    u32 lead, n, nvec;

    __device__ __forceinline__ RowView(const void* rows, long long row, long long row_bytes, u32 n_) {
        x = (const char*)rows + row * row_bytes;
        base = (const char*)((uintptr_t)x & ~(uintptr_t)15);
        lead = (u32)(x - base) / RowElem<DT>::kBytes;
        n = n_;
        nvec = (lead + n + E - 1) / E;  // (n is at most 2^31)
    }
    template <bool NT>
    __device__ __forceinline__ u32x4 load(u32 v) const {
        const global_vec_ptr p = (global_vec_ptr)(base + (size_t)v * 16);
        return NT ? __builtin_nontemporal_load(p) : *p;
    }
    // Is vector v's every element one of the row's?
    __device__ __forceinline__ bool whole(u32 v) const { return (v != 0 || lead == 0) && (u64)(v + 1) * E <= (u64)lead + n; }
    // ... those that are not: -inf, which adds nothing to a softmax.
    __device__ __forceinline__ u32x4 trimmed(u32x4 q, u32 v) const {
        u32x4 r = q;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const u32 col = v * E + j - lead;  // (wraps below the row's start)
            if (col >= n) {
                if constexpr (E == 4) r[j] = RowElem<DT>::kMinusInf;
                else r[j / 2] = (j & 1) ? (r[j / 2] & 0xffffu) | (RowElem<DT>::kMinusInf & 0xffff0000u)
                                        : (r[j / 2] & 0xffff0000u) | (RowElem<DT>::kMinusInf & 0xffffu);
            }
        }
        return r;
    }
};

// The end of a workgroup's vectors, which begin at v0 (there are none where the row, by where it starts, has fewer than it could have).
__device__ __forceinline__ u32 part_end(u32 v0, u32 vecs, u32 nvec) { return max(v0, min(v0 + vecs, nvec)); }

// f(vectors, first) for every tile of vectors [v0, v1): lane t of the workgroup holds vectors first + t, first + t + B, ...; what lies outside
// the row or the range is -inf.
template <int DT, int B, int V, bool NT, class F>
__device__ __forceinline__ void sweep_vectors(const RowView<DT>& r, u32 v0, u32 v1, F&& f) {
    const u32x4 none = {RowElem<DT>::kMinusInf, RowElem<DT>::kMinusInf, RowElem<DT>::kMinusInf, RowElem<DT>::kMinusInf};
    for (u32 t = v0; t < v1; t += B * V) {
        u32x4 q[V];
        if (t + B * V <= v1 && r.whole(t) && r.whole(t + B * V - 1)) {
#pragma unroll
            for (int i = 0; i < V; ++i) q[i] = r.template load<NT>(t + i * B + threadIdx.x);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const u32 v = t + i * B + threadIdx.x;
                q[i] = none;
                if (v < v1) q[i] = r.trimmed(r.template load<NT>(v), v);
            }
        }
        f(q, t);
    }
}

// ------------------------------------------------------------------------------------------------
// softmax statistics: m the largest logit, s = sum 2^((x - m) c), w = sum of those terms times their exponents, with c = log2(e) / temperature.
// m is -inf and s 0 where there is nothing but -inf; a NaN or +inf anywhere makes s NaN, and with it all that is made from it.  (The maximum
// itself passes over NaNs.)  Everything is kept in 32 bits; a lane adds up a few hundred terms, lanes and waves are joined in a fixed order.
// ------------------------------------------------------------------------------------------------
struct SoftSum {
    float m = -__builtin_inff(), s = 0.0f, w = 0.0f;
};
__device__ __forceinline__ float4 packed(const SoftSum& a) { return make_float4(a.m, a.s, a.w, 0.0f); }
__device__ __forceinline__ SoftSum unpacked(const float4& p) {
    SoftSum a;
    a.m = p.x;
    a.s = p.y;
    a.w = p.z;
    return a;
}
__device__ __forceinline__ float finite_or_zero(float m) { return m == -__builtin_inff() ? 0.0f : m; }

template <bool W>
__device__ __forceinline__ void soft_rescale(SoftSum& a, float m, float ref, float c) {  // to the larger maximum m (ref: m, or 0 for -inf)
    const float d = fmaxf((a.m - ref) * c, kNothing * 4.0f);  // (a.m = -inf has s = 0; a factor of 2^-800 is zero)
    const float f = exp2_fast(d);
    if (W) a.w = f * (a.w + a.s * d);
    a.s *= f;
    a.m = m;
}
template <bool W, int N>
__device__ __forceinline__ void soft_add(SoftSum& a, const float (&x)[N], float c) {
    float t = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) t = fmaxf(t, x[j]);
    t = fmaxf(t, a.m);
    const float ref = finite_or_zero(t);
    soft_rescale<W>(a, t, ref, c);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const float y = (x[j] - ref) * c, e = exp2_fast(y);
        a.s += e;
        if (W) a.w += e * fmaxf(y, kNothing);
    }
}
template <bool W>
__device__ __forceinline__ SoftSum soft_join(SoftSum a, SoftSum b, float c) {
    const float m = fmaxf(a.m, b.m), ref = finite_or_zero(m);
    soft_rescale<W>(a, m, ref, c);
    soft_rescale<W>(b, m, ref, c);
    a.s += b.s;
    if (W) a.w += b.w;
    return a;
}
template <bool W>
__device__ __forceinline__ SoftSum soft_wave(SoftSum a, float c) {  // the same in every lane
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        SoftSum b;
        b.m = __shfl_xor(a.m, d);
        b.s = __shfl_xor(a.s, d);
        if (W) b.w = __shfl_xor(a.w, d);
        a = soft_join<W>(a, b, c);
    }
    return a;
}
// Over the workgroup, the same in every thread.  `sm` has an entry per wave; it may be used again after the next barrier.
template <int B, bool W>
__device__ __forceinline__ SoftSum soft_block(SoftSum a, float c, float4* sm) {
    a = soft_wave<W>(a, c);
    if constexpr (B == 64) return a;
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = packed(a);
    __syncthreads();
    a = unpacked(sm[0]);
#pragma unroll
    for (int i = 1; i < B / 64; ++i) a = soft_join<W>(a, unpacked(sm[i]), c);
    return a;
}
template <int B, class T>
__device__ __forceinline__ T sum_block(T v, T* sm) {  // likewise
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    if constexpr (B == 64) return v;
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sm[0];
#pragma unroll
    for (int i = 1; i < B / 64; ++i) v += sm[i];
    return v;
}

// ------------------------------------------------------------------------------------------------
// gradients: dense(x) for every element, then the listed columns anew, listed(x, sum of its entries' values).
// ------------------------------------------------------------------------------------------------
// Columns are listed in no order and may be listed more than once.  The workgroup marks its own in an LDS bitmap, a byte per vector; where
// a mark is found set, the whole list is gone through for every entry, lowest entry first, so that sums have one order.
//   at(i)     the column of entry i, or negative
//   value(i)  what it adds
template <int DT, int B, int V, bool NT, class At, class Value, class Dense, class Listed>
__device__ __forceinline__ void write_gradient(const RowView<DT>& r, char* out, bool aligned, u32 v0, u32 v1, long long entries, u32* marks, u32* twice,
                                               At&& at, Value&& value, Dense&& dense, Listed&& listed) {
    constexpr int E = RowElem<DT>::E;
    auto mine = [&](long long t) {
        const u64 p = (u64)(t + r.lead) - (u64)v0 * E;  // (wraps below the range)
        return t >= 0 && t < (long long)r.n && p < (u64)(v1 - v0) * E;
    };
    const bool many = entries > 1;
    if (many) {
        for (u32 i = threadIdx.x; i < (v1 - v0 + 3) / 4; i += B) marks[i] = 0;
        if (threadIdx.x == 0) *twice = 0;
        __syncthreads();
        for (long long i = threadIdx.x; i < entries; i += B) {
            const long long t = at(i);
            if (mine(t)) {
                const u32 p = (u32)(t + r.lead - (long long)v0 * E), v = p / E, bit = 1u << ((v & 3) * 8 + p % E);
                if (atomicOr(&marks[v >> 2], bit) & bit) *twice = 1;
            }
        }
    }
    sweep_vectors<DT, B, V, NT>(r, v0, v1, [&](const u32x4 (&q)[V], u32 first) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const u32 v = first + i * B + threadIdx.x;
            if (v < v1) {
                float x[E];
                RowElem<DT>::unpack(q[i], x);
#pragma unroll
                for (int j = 0; j < E; ++j) x[j] = dense(x[j]);
                if (aligned && r.whole(v)) {
                    typedef __attribute__((address_space(1))) u32x4* vec_out;
                    *(vec_out)(out + ((long long)v * E - r.lead) * RowElem<DT>::kBytes) = RowElem<DT>::pack(x);
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const u32 col = v * E + j - r.lead;
                        if (col < r.n) RowElem<DT>::store(out, col, x[j]);
                    }
                }
            }
        }
    });
    __syncthreads();  // (and what was stored is there: a listed column is written after the dense one)
    const bool repeated = many && *twice != 0;
    for (long long i = threadIdx.x; i < entries; i += B) {
        const long long t = at(i);
        if (!mine(t)) continue;
        float sum = value(i);
        bool first = true;
        if (repeated) {
            sum = 0.0f;
            for (long long l = 0; l < entries; ++l)
                if (at(l) == t) {
                    if (l < i) first = false;
                    sum += value(l);
                }
        }
        if (first) RowElem<DT>::store(out, (u32)t, listed(RowElem<DT>::load(r.x, (u32)t), sum));
    }
}

// ------------------------------------------------------------------------------------------------
// host: how many workgroups a row is dealt to
// ------------------------------------------------------------------------------------------------
struct RowParts {
    u32 parts, vecs;  // workgroups per row, and vectors of each
};
static inline RowParts deal_row(int64_t batch, int64_t n, int elem_bytes, int64_t tile_vecs, int64_t want_wgs, int64_t most_vecs) {
    const int64_t E = 16 / elem_bytes, nvec = (n + 2 * (E - 1)) / E, tiles = (nvec + tile_vecs - 1) / tile_vecs;  // (wherever it starts)
    int64_t parts = want_wgs / batch;
    if (parts < 1) parts = 1;
    if (parts > tiles) parts = tiles;
    int64_t per = (tiles + parts - 1) / parts;
    if (per * tile_vecs > most_vecs) per = most_vecs / tile_vecs;
    parts = (tiles + per - 1) / per;
    return RowParts{(u32)parts, (u32)(per * tile_vecs)};
}
static inline size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
// Workgroups of one launch (a grid has less than 2^32 threads); larger batches take several.
constexpr int64_t kMostWorkgroups = (int64_t)1 << 21;

template <class F>
static inline rtopk_status by_type(rtopk_dtype dt, F&& f) {
    switch (dt) {
        case RTOPK_F32: return f(std::integral_constant<int, RTOPK_F32>{});
        case RTOPK_F16: return f(std::integral_constant<int, RTOPK_F16>{});
        case RTOPK_BF16: return f(std::integral_constant<int, RTOPK_BF16>{});
    }
    return RTOPK_ERR_INVALID_ARG;
}

// Arguments that every operator on rows has.
static inline rtopk_status check_rows(const void* x, int64_t batch, int64_t n, int64_t stride, rtopk_dtype dt) {
    if (!x || batch < 1 || batch > 0x7fffffff || n < 1 || n > RTOPK_MAX_N) return RTOPK_ERR_INVALID_ARG;
    if (dt != RTOPK_F32 && dt != RTOPK_F16 && dt != RTOPK_BF16) return RTOPK_ERR_INVALID_ARG;
    if (batch > 1 && (stride < n || stride > (int64_t)1 << 40)) return RTOPK_ERR_INVALID_ARG;
    if ((uintptr_t)x % (dt == RTOPK_F32 ? 4 : 2)) return RTOPK_ERR_UNSUPPORTED;
    return RTOPK_OK;
}
static inline bool usable_temperature(float inv) {
    const float c = inv * kLog2e;
    return inv >= 1.1754944e-38f && c <= 3.0e38f;
}
// Do the rows of two arrays of one shape and type share memory?
static inline bool rows_overlap(const void* a, int64_t sa, const void* b, int64_t sb, int64_t batch, int64_t n, int elem_bytes) {
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    const uintptr_t a1 = a0 + (uintptr_t)(((batch - 1) * sa + n) * elem_bytes), b1 = b0 + (uintptr_t)(((batch - 1) * sb + n) * elem_bytes);
    return a0 < b1 && b0 < a1;
}

}  // namespace rtopk
