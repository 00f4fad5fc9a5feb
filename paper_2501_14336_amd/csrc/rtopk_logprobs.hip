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
    u64* part_top;             // [batch][parts][k]: the parts' best entries, best first; 0 where a part has fewer
    long long* top_indices;
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

// ------------------------------------------------------------------------------------------------
// The k best of a sweep (k up to 64), on the way.  Elements are entries: the key of the number, NaN above all, above the complement of the column, so that all differ and the
// larger is the better one.
//
// A lane keeps its running maximum for the softmax anyway.  Of the lane maxima of groups of lanes, the r-th largest of each group has r elements that are not below it, and the (k / r)-th best of those has k: a
// bound of the k-th best.  One is taken after the first tile; from then on a lane notes the vectors whose maximum is not below it, a bit each.  Another, from
// all the lanes have seen, is taken at the end, and only what was noted by lanes whose maximum is not below that is fetched again: of data in no order about twice k vectors, of which about
// as many elements are listed and ranked by comparing each with all others.  A list too long for LDS (equal elements, or the best in few lanes) leads to a radix selection of the
// part, whose cost does not depend on the data.
// ------------------------------------------------------------------------------------------------
constexpr int kMostTop = 64;
constexpr u32 kListRoom = 1024;
constexpr u32 kNotedVecs = 64;     // vectors of a lane: bits of its note
constexpr u32 kMostEntries = 4096;  // of a row's parts together
static_assert(kMostEntries / 256 * kMostTop <= kListRoom, "what k_logprobs_finish lists");

__device__ __forceinline__ u32 key_of(float x) { return KeyOf<RTOPK_F32>::key(__float_as_uint(x)); }
__device__ __forceinline__ float number_of(u32 key) { return __uint_as_float((key & 0x80000000u) ? (key ^ 0x80000000u) : ~key); }  // (the key of all NaNs gives one)
__device__ __forceinline__ u64 entry_of(u32 key, u32 col) { return ((u64)key << 32) | (u32)~col; }

constexpr int kBoundGroups = 16;  // of a workgroup's threads

// The largest of a group of GL lanes, in all of them.
template <int GL>
__device__ __forceinline__ u32 group_largest(u32 v) {
    auto turned = [](auto ctrl, u32 v) { return (u32)__builtin_amdgcn_update_dpp((int)v, (int)v, decltype(ctrl)::value, 0xf, 0xf, false); };
    v = max(v, turned(std::integral_constant<int, 0x128>{}, v));
    v = max(v, turned(std::integral_constant<int, 0x124>{}, v));
    v = max(v, turned(std::integral_constant<int, 0x122>{}, v));
    v = max(v, turned(std::integral_constant<int, 0x121>{}, v));
    if constexpr (GL >= 32) {
        const auto rows = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max(rows[0], rows[1]);
    }
    if constexpr (GL >= 64) {
        const auto halves = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = max(halves[0], halves[1]);
    }
    return v;
}

// A bound that at least `want` of the workgroup's threads' keys are not below; 0 where it finds none.  `threads`: the first so many that have one.  `sm` has an entry per group and is free after
// the next barrier.
template <int B>
__device__ __forceinline__ u32 bound_of_threads(u32 v, u32 threads, u32 want, u32* sm) {
    constexpr u32 kLanes = B / kBoundGroups;
    const u32 groups = max(min(threads, (u32)B) / kLanes, 1u);  // full ones: the rest may hold anything
    const u32 least = (want + groups - 1) / groups, each = least + (least > 1 ? 1u : 0u);
    // (a round more than it takes, and fewer groups: 32 of 2853 rows of 5808 bf16 21.1 us, without 23.8)
    u32 best = 0;
    for (u32 i = 0; i < each; ++i) {  // what at least so many of the group's lanes are not below
        best = group_largest<kLanes>(v);
        v = v == best ? 0u : v;
    }
    if (threadIdx.x % kLanes == 0) sm[threadIdx.x / kLanes] = threads < kLanes ? 0u : best;
    __syncthreads();
    const u32 g = lane_id() % kBoundGroups, mine = g < groups ? sm[g] : 0u, enough = (want + each - 1) / each;
    u32 not_below = 0;  // of so many groups as it takes, the best ones
#pragma unroll
    for (int i = 0; i < kBoundGroups; ++i) not_below += (u32)__builtin_amdgcn_readlane((int)mine, i) >= mine;
    return group_largest<kBoundGroups>(not_below >= enough ? mine : 0u);
}

template <int B>
struct TopShared {
    u64 list[kListRoom];
    u32 hist[256];
    u64 bound64;
    u32 bound[2][kBoundGroups];
    u32 count, digit, above, scan[B / 64];
};

// list[0, count) in order to out(rank, entry), the best `want` of them.
template <int B, class Out>
__device__ __forceinline__ void rank_list(const u64* list, u32 count, u32 want, Out&& out) {
    for (u32 i = threadIdx.x; i < count; i += B) {
        const u64 e = list[i];
        u32 rank = 0;
#pragma unroll 8  // (a trip to LDS for eight at a time)
        for (u32 j = 0; j < count; ++j) rank += list[j] > e;
        if (rank < want) out(rank, e);
    }
}

// The `want` best entries of the part's columns into sm.list, in no order; they are there after the next barrier.
template <int DT, int B>
__device__ __noinline__ void select_radix(const RowView<DT> r, u32 v0, u32 v1, u32 want, TopShared<B>& sm) {
    constexpr int E = RowElem<DT>::E;
    auto each = [&](u32 v, auto&& f) {  // f(key, column) for the elements of a vector
        float x[E];
        RowElem<DT>::unpack(r.template load<false>(v), x);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const u32 col = v * E + j - r.lead;
            if (col < r.n) f(key_of(x[j]), col);
        }
    };
    u32 prefix = 0, rank = want;  // the key's digits so far; its rank among those that have them
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (u32 i = threadIdx.x; i < 256; i += B) sm.hist[i] = 0;
        __syncthreads();
        for (u32 v = v0 + threadIdx.x; v < v1; v += B)
            each(v, [&](u32 key, u32) {
                if (shift == 24 || (key >> ((shift + 8) & 31)) == prefix) {
                    const u32 digit = (key >> shift) & 255u, first = __builtin_amdgcn_readfirstlane(digit);
                    const u64 alike = ballot64(digit == first), all = ballot64(true);
                    if (alike == all) {  // (a crowd: one add for the wave)
                        if (lane_id() == (u32)__builtin_ctzll(all)) atomicAdd(&sm.hist[first], (u32)__builtin_popcountll(all));
                    } else {
                        atomicAdd(&sm.hist[digit], 1u);
                    }
                }
            });
        __syncthreads();
        if (threadIdx.x == 0) {
            u32 d = 255, above = 0;
            while (d > 0 && above + sm.hist[d] < rank) above += sm.hist[d--];
            sm.digit = d;
            sm.above = above;
        }
        __syncthreads();
        rank -= sm.above;
        prefix = (prefix << 8) | sm.digit;
    }
    // what is better, and the first `rank` of what is equal
    if (threadIdx.x == 0) sm.count = 0;
    __syncthreads();
    for (u32 v = v0 + threadIdx.x; v < v1; v += B)
        each(v, [&](u32 key, u32 col) {
            if (key > prefix) sm.list[atomicAdd(&sm.count, 1u)] = entry_of(key, col);
        });
    __syncthreads();
    u32 found = 0;
    for (u32 t = v0; t < v1 && found < rank; t += B) {
        const u32 v = t + threadIdx.x;
        u32 mine = 0;
        if (v < v1) each(v, [&](u32 key, u32) { mine += key == prefix; });
        u32 before = mine;  // inclusive sums over the wave, then over the waves
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const u32 o = (u32)__shfl_up((int)before, d);
            before += lane_id() >= (u32)d ? o : 0u;
        }
        if (lane_id() == 63) sm.scan[threadIdx.x >> 6] = before;
        __syncthreads();
        u32 total = 0;
        for (u32 w = 0; w < B / 64; ++w) {
            if (w == threadIdx.x >> 6) before += total;
            total += sm.scan[w];
        }
        u32 at = found + before - mine;
        if (v < v1)
            each(v, [&](u32 key, u32 col) {
                if (key == prefix && at++ < rank) sm.list[want - rank + at - 1] = entry_of(key, col);
            });
        found += total;
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------
// The sweep of a row or a part of one.
// ------------------------------------------------------------------------------------------------
template <int DT>
__device__ __forceinline__ void write_logprob(const LogprobsParams& P, long long row, long long i, float x, long long t, const SoftSum& a, float ln_s) {
    float v = 0.0f;
    if (t >= (long long)P.n) v = __builtin_nanf("");
    else if (t >= 0) v = logprob_of(x, a.m, a.s, ln_s, P.inv_t);
    P.logprobs[row * P.m + i] = v;
}
template <bool W>
__device__ __forceinline__ void write_stats(const LogprobsParams& P, long long row, const SoftSum& a, float ln_s) {
    if (W) P.entropy[row] = a.s == 0.0f ? 0.0f : ln_s - kLn2 * (a.w / a.s);
    if (P.row_stats) {
        P.row_stats[2 * row] = a.m;
        P.row_stats[2 * row + 1] = a.s;
    }
}
__device__ __forceinline__ void write_top(const LogprobsParams& P, long long row, u32 rank, u64 e, const SoftSum& a, float ln_s) {
    P.top_logprobs[row * P.k + rank] = logprob_of(number_of((u32)(e >> 32)), a.m, a.s, ln_s, P.inv_t);
    P.top_indices[row * P.k + rank] = (long long)(u32)~(u32)e;
}

struct NoTop {};

// The one pass over a row, by a workgroup that then has its results, or, where there are few rows, by several that leave their parts to k_logprobs_finish.  Bound by memory where there is
// much of it: 1024 rows of 131072 bf16, scored with their entropy, 48 us or 5.6 TB/s; 512 rows of 100003 fp16 24 us, 4.3 TB/s; 300 rows of 50257 fp32 with 5 alternatives 16.6 us,
// 3.6 TB/s (each compute unit has a row or two: the second does not fill them).  One row of 131072 bf16 with 20 alternatives: 6.0 us, as long as 16 of them, a wave's way from its
// loads to what it lists.  16-bit logits come within a fifth of the rate of 2^x, a quarter of that of sums.
template <int DT, int B, int V, bool NT, bool W, bool TOP, bool WHOLE>
__global__ void __launch_bounds__(B) k_logprobs_sweep(LogprobsParams P) {
    constexpr int E = RowElem<DT>::E;
    __shared__ float4 sm[B / 64];
    __shared__ std::conditional_t<TOP, TopShared<B>, NoTop> top;
    const u32 part = WHOLE ? 0u : blockIdx.x % P.parts;
    const long long row = P.row0 + (WHOLE ? blockIdx.x : blockIdx.x / P.parts);
    const RowView<DT> r(P.logits, row, P.row_bytes, P.n);
    const u32 v0 = part * P.part_vecs, v1 = part_end(v0, P.part_vecs, r.nvec);
    const bool one_tile = v1 - v0 <= B * V;  // what is listed is listed from the registers
    long long token = -1;  // the thread's first
    float x_of = 0.0f;
    if (WHOLE && (long long)threadIdx.x < P.m) {
        token = P.tokens[row * P.m + threadIdx.x];
        if (token >= 0 && token < (long long)P.n) x_of = RowElem<DT>::load(r.x, (u32)token);
    }
    SoftSum a;
    u64 noted = 0;
    u32 bound = 0, tiles = 0;
    float bound_number = -__builtin_inff();
    if constexpr (TOP) {
        if (threadIdx.x == 0) top.count = 0;
    }
    auto list_vector = [&](u32 v, const float (&x)[E]) {
        if constexpr (TOP) {
            u32 which = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) which |= !(x[j] < bound_number) ? 1u << j : 0u;
            while (which) {  // (one, mostly)
                const u32 j = (u32)__builtin_ctz(which), col = v * E + j - r.lead;
                which &= which - 1;
                float y = x[0];
#pragma unroll
                for (int i = 1; i < E; ++i) y = j == (u32)i ? x[i] : y;
                if (col < r.n && key_of(y) >= bound) {
                    const u32 place = atomicAdd(&top.count, 1u);
                    if (place < kListRoom) top.list[place] = entry_of(key_of(y), col);
                }
            }
        }
    };
    sweep_vectors<DT, B, V, NT>(r, v0, v1, [&](const u32x4 (&q)[V], u32 first) {
        float x[V * E], most[V], t = a.m;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float y[E];
            RowElem<DT>::unpack(q[i], y);
            most[i] = largest(-__builtin_inff(), y);
            t = __builtin_elementwise_maximum(t, most[i]);
#pragma unroll
            for (int j = 0; j < E; ++j) x[i * E + j] = y[j];
        }
        soft_add_to<W>(a, x, t, P.c);
        if constexpr (TOP) {
            if (first == v0) {
                bound = bound_of_threads<B>(key_of(a.m), v1 - v0, (u32)P.k, top.bound[0]);
                bound_number = bound == 0 ? -__builtin_inff() : number_of(bound);
            }
            u32 hits = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) hits |= !(most[i] < bound_number) ? 1u << i : 0u;
            if (one_tile) {
                if (hits) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float y[E];
#pragma unroll
                        for (int j = 0; j < E; ++j) y[j] = x[i * E + j];
                        if ((hits >> i) & 1) list_vector(first + i * B + threadIdx.x, y);
                    }
                }
            } else {
                noted |= (u64)hits << (tiles * V);
                ++tiles;
            }
        }
    });
    const float mine = a.m;
    a = soft_block<B, W>(a, P.c, sm);
    const float ln_s = kLn2 * log2_fast(a.s);
    if constexpr (TOP) {
        const long long here = (long long)min((u64)v1 * E, (u64)r.lead + r.n) - (long long)max((u64)v0 * E, (u64)r.lead);  // columns
        const u32 want = here < P.k ? (here < 0 ? 0u : (u32)here) : (u32)P.k;
        if (!one_tile) {
            bound = max(bound, bound_of_threads<B>(key_of(mine), B, (u32)P.k, top.bound[1]));
            bound_number = bound == 0 ? -__builtin_inff() : number_of(bound);
            if (!(mine < bound_number)) {
                while (noted) {
                    // (four vectors on their way at a time)
                    u32 at[4];
                    u32x4 q[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        at[i] = noted ? v0 + (u32)__builtin_ctzll(noted) * B + threadIdx.x : v1;
                        noted &= noted - 1;
                        if (at[i] < v1) q[i] = r.template load<false>(at[i]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (at[i] < v1) {
                            float x[E];
                            RowElem<DT>::unpack(q[i], x);
                            list_vector(at[i], x);
                        }
                }
            }
        }
        __syncthreads();
        u32 count = top.count;
        if (count > kListRoom || count < want) {
            select_radix<DT, B>(r, v0, v1, want, top);
            __syncthreads();
            count = want;
        }
        if (WHOLE) {
            rank_list<B>(top.list, count, want, [&](u32 rank, u64 e) { write_top(P, row, rank, e, a, ln_s); });
        } else {
            u64* out = P.part_top + (row * P.parts + part) * P.k;
            rank_list<B>(top.list, count, want, [&](u32 rank, u64 e) { out[rank] = e; });
            for (u32 i = want + threadIdx.x; i < (u32)P.k; i += B) out[i] = 0;
        }
    }
    if (!WHOLE) {
        if (threadIdx.x == 0) P.partial[row * P.parts + part] = packed(a);
        return;
    }
    if (!TOP)
        for (long long i = threadIdx.x; i < P.k; i += B)
            P.top_logprobs[row * P.k + i] = logprob_of(RowElem<DT>::load(P.top_values + (size_t)(row * P.k) * RowElem<DT>::kBytes, (u32)i), a.m, a.s, ln_s, P.inv_t);
    for (long long i = threadIdx.x; i < P.m; i += B) {
        if (i >= B) {
            token = P.tokens[row * P.m + i];
            x_of = token >= 0 && token < (long long)P.n ? RowElem<DT>::load(r.x, (u32)token) : 0.0f;
        }
        write_logprob<DT>(P, row, i, x_of, token, a, ln_s);
    }
    if (threadIdx.x == 0) write_stats<W>(P, row, a, ln_s);
}

// A row's parts put together.  TOP: their lists too; otherwise the alternatives' values are there already (P.top_values).  4.4 us for 33 parts with 20 entries each (a launch that does
// nothing takes 2): one trip to what other units wrote, then ranks by comparisons in LDS.
constexpr int kFinishBlock = 256;

template <int DT, bool W, bool TOP>
__global__ void __launch_bounds__(kFinishBlock) k_logprobs_finish(LogprobsParams P) {
    __shared__ float4 sm[kFinishBlock / 64];
    __shared__ std::conditional_t<TOP, TopShared<kFinishBlock>, NoTop> top;
    const long long row = P.row0 + blockIdx.x;
    const RowView<DT> r(P.logits, row, P.row_bytes, P.n);
    // everything that has to be fetched at once: what other compute units wrote is far away
    long long token = -1;  // the thread's first
    if ((long long)threadIdx.x < P.m) token = P.tokens[row * P.m + threadIdx.x];
    const u64* lists = P.part_top + row * P.parts * P.k;
    const u32 entries = TOP ? P.parts * (u32)P.k : 0u;
    constexpr int kEach = TOP ? kMostEntries / kFinishBlock : 1;
    u64 e[kEach], best = 0;
    const u64 head = TOP && threadIdx.x < P.parts ? lists[threadIdx.x * (u32)P.k] : 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const u32 i = j * kFinishBlock + threadIdx.x;
        e[j] = 0;
        if (j * kFinishBlock < entries) e[j] = i < entries ? lists[i] : 0;
    }
    SoftSum a;
    for (u32 i = threadIdx.x; i < P.parts; i += kFinishBlock) a = soft_join<W>(a, unpacked(P.partial[row * P.parts + i]), P.c);
    float x_of = token >= 0 && token < (long long)P.n ? RowElem<DT>::load(r.x, (u32)token) : 0.0f;
    a = soft_block<kFinishBlock, W>(a, P.c, sm);
    const float ln_s = kLn2 * log2_fast(a.s);
    if constexpr (TOP) {
        if (threadIdx.x == 0) top.count = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) best = max(best, e[j]);
        // A bound: where there are parts enough and k is small, the k-th best of the parts' first entries (k parts have any that are not below it, at most k each); else the k-th best
        // of the threads' best ones (k threads have any, at most kMostEntries / 256 each).  The list has room for either.  (Entries are all different, but for the zeros of parts and
        // threads that have none.)
        const bool by_heads = P.parts >= (u32)P.k && P.parts <= kFinishBlock && (u32)(P.k * P.k) <= kListRoom;
        const u64 mine = by_heads ? head : best;
        const u32 others = by_heads ? P.parts : kFinishBlock;
        top.list[threadIdx.x] = mine;
        if (threadIdx.x == 0) top.bound64 = 0;
        __syncthreads();
        u32 rank = 0;
#pragma unroll 16
        for (u32 j = 0; j < others; ++j) rank += top.list[j] > mine;
        if (rank == (u32)P.k - 1 && mine != 0 && threadIdx.x < others) top.bound64 = mine;
        __syncthreads();
        const u64 bound = top.bound64;
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (j * kFinishBlock < entries && e[j] >= bound && e[j] != 0) {
                const u32 place = atomicAdd(&top.count, 1u);
                if (place < kListRoom) top.list[place] = e[j];
            }
        __syncthreads();
        rank_list<kFinishBlock>(top.list, min(top.count, kListRoom), (u32)P.k, [&](u32 rank, u64 x) { write_top(P, row, rank, x, a, ln_s); });
    } else {
        for (long long i = threadIdx.x; i < P.k; i += kFinishBlock)
            P.top_logprobs[row * P.k + i] = logprob_of(RowElem<DT>::load(P.top_values + (size_t)(row * P.k) * RowElem<DT>::kBytes, (u32)i), a.m, a.s, ln_s, P.inv_t);
    }
    for (long long i = threadIdx.x; i < P.m; i += kFinishBlock) {
        if (i >= kFinishBlock) {
            token = P.tokens[row * P.m + i];
            x_of = token >= 0 && token < (long long)P.n ? RowElem<DT>::load(r.x, (u32)token) : 0.0f;
        }
        write_logprob<DT>(P, row, i, x_of, token, a, ln_s);
    }
    if (threadIdx.x == 0) write_stats<W>(P, row, a, ln_s);
}

// dx_j = (1/T) [ sum_i g_i (1[t_i = j] - p_j) - gH p_j (ln p_j + H) ]
// One reading and one writing of the row, bound by memory: 512 rows of 100003 fp16 with the entropy's gradient 38.8 us, 5.3 TB/s.
constexpr int kGradBlock = 256, kGradVecs = 2;

template <int DT, bool NT, bool W>
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
    write_gradient<DT, kGradBlock, kGradVecs, 1, NT>(
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

// How a call goes.
struct LogprobsPlan {
    bool top;    // alternatives by the sweep itself (otherwise rtopk_select finds them first)
    int block;   // a workgroup of so many threads takes a row; 0: several share one, and a second launch puts their parts together
    bool past_caches;  // rows are read past the caches
    u32 parts, part_vecs;
    size_t partial_bytes, top_bytes, select_bytes;
    size_t bytes() const { return partial_bytes + top_bytes + select_bytes; }
};
constexpr int kPartBlock = 256, kPartVecs = 2, kWholeVecs = 4;

static rtopk_status make_plan(int64_t batch, int64_t n, int64_t m, int64_t k, rtopk_dtype dt, LogprobsPlan* L) {
    if (batch < 1 || batch > 0x7fffffff || n < 1 || n > RTOPK_MAX_N || m < 0 || m > 0x7fffffff || k < 0 || k > n) return RTOPK_ERR_INVALID_ARG;
    if (dt != RTOPK_F32 && dt != RTOPK_F16 && dt != RTOPK_BF16) return RTOPK_ERR_INVALID_ARG;
    const int eb = dt == RTOPK_F32 ? 4 : 2, E = 16 / eb;
    const int64_t vecs = (n + 2 * (E - 1)) / E;  // (wherever a row starts)
    *L = LogprobsPlan{};
    L->top = k > 0 && k <= kMostTop;
    if ((batch >= 128 && vecs <= (int64_t)kNotedVecs * 1024) || vecs <= 4096) {
        L->block = vecs <= 256 * kWholeVecs || (batch > 512 && vecs <= (int64_t)kNotedVecs * 256) ? 256 : batch > 256 && vecs <= (int64_t)kNotedVecs * 512 ? 512 : 1024;
        L->past_caches = past_caches(batch, n, eb);
        L->parts = 1;
        L->part_vecs = (u32)vecs;
    } else {
        const int64_t tile = kPartBlock * kPartVecs, most = L->top ? kMostEntries / k : (int64_t)1 << 20;
        int64_t want = 1024 / batch < 1 ? 1 : 1024 / batch;
        if (want > most) want = most;
        const int64_t longest = L->top ? (int64_t)kNotedVecs * kPartBlock : (int64_t)1 << 28;
        RowParts d = deal_row(batch, n, eb, tile, want * batch, longest);
        if (d.parts > most) {  // a row too long for so many parts: its alternatives are selected apart
            L->top = false;
            d = deal_row(batch, n, eb, tile, 1024, (int64_t)1 << 28);
        }
        L->parts = d.parts;
        L->part_vecs = d.vecs;
        L->partial_bytes = up256((size_t)batch * d.parts * sizeof(float4));
        if (L->top) L->top_bytes = up256((size_t)batch * d.parts * k * 8);
    }
    if (k > 0 && !L->top) {
        size_t all = 0, one = 0;  // (rows that do not follow one another are selected from one by one)
        const rtopk_status s = rtopk_workspace_bytes(batch, n, k, dt, RTOPK_FLAG_SORTED, &all);
        if (s != RTOPK_OK) return s;
        (void)rtopk_workspace_bytes(1, n, k, dt, RTOPK_FLAG_SORTED, &one);
        L->top_bytes = up256((size_t)batch * k * eb);
        L->select_bytes = all > one ? all : one;
    }
    return RTOPK_OK;
}

template <int DT, bool W, bool TOP>
static void launch_logprobs(LogprobsParams P, const LogprobsPlan& L, int64_t batch, hipStream_t st) {
    const int64_t rows = kMostWorkgroups / L.parts > 0 ? kMostWorkgroups / L.parts : 1;
    for (P.row0 = 0; P.row0 < batch; P.row0 += rows) {
        const unsigned now = (unsigned)(batch - P.row0 < rows ? batch - P.row0 : rows);
        auto whole = [&](auto block) {
            constexpr int B = decltype(block)::value;
            if (L.past_caches) hipLaunchKernelGGL((k_logprobs_sweep<DT, B, kWholeVecs, true, W, TOP, true>), dim3(now), dim3(B), 0, st, P);
            else hipLaunchKernelGGL((k_logprobs_sweep<DT, B, kWholeVecs, false, W, TOP, true>), dim3(now), dim3(B), 0, st, P);
        };
        if (L.block == 256) whole(std::integral_constant<int, 256>{});
        else if (L.block == 512) whole(std::integral_constant<int, 512>{});
        else if (L.block == 1024) whole(std::integral_constant<int, 1024>{});
        else {
            hipLaunchKernelGGL((k_logprobs_sweep<DT, kPartBlock, kPartVecs, false, W, TOP, false>), dim3(now * L.parts), dim3(kPartBlock), 0, st, P);
            hipLaunchKernelGGL((k_logprobs_finish<DT, W, TOP>), dim3(now), dim3(kFinishBlock), 0, st, P);
        }
    }
}

}  // namespace rtopk

using namespace rtopk;

extern "C" {

rtopk_status rtopk_logprobs_workspace_bytes(int64_t batch, int64_t n, int64_t m, int64_t k, rtopk_dtype dt, size_t* bytes_out) {
    if (!bytes_out) return RTOPK_ERR_INVALID_ARG;
    LogprobsPlan L;
    const rtopk_status s = make_plan(batch, n, m, k, dt, &L);
    if (s == RTOPK_OK) *bytes_out = L.bytes() > 256 ? L.bytes() : 256;
    return s;
}

rtopk_status rtopk_logprobs(const void* logits, int64_t batch, int64_t n, int64_t row_stride, rtopk_dtype dt, float inv_temperature,
                            const int64_t* tokens, int64_t m, int64_t k, float* out_logprobs, float* out_entropy, float* out_row_stats,
                            float* out_top_logprobs, int64_t* out_top_indices, void* workspace, size_t workspace_bytes, void* hip_stream) {
    rtopk_status s = check_rows(logits, batch, n, row_stride, dt);
    if (s != RTOPK_OK) return s;
    if (!usable_temperature(inv_temperature) || !workspace) return RTOPK_ERR_INVALID_ARG;
    LogprobsPlan L;
    s = make_plan(batch, n, m, k, dt, &L);
    if (s != RTOPK_OK) return s;
    if (m > 0 && (!tokens || !out_logprobs)) return RTOPK_ERR_INVALID_ARG;
    if (k > 0 && (!out_top_logprobs || !out_top_indices)) return RTOPK_ERR_INVALID_ARG;
    if (((uintptr_t)tokens | (uintptr_t)out_top_indices) % 8 || ((uintptr_t)out_logprobs | (uintptr_t)out_entropy | (uintptr_t)out_row_stats | (uintptr_t)out_top_logprobs) % 4 ||
        (uintptr_t)workspace % 256)
        return RTOPK_ERR_UNSUPPORTED;
    if (workspace_bytes < L.bytes() || workspace_bytes < 256) return RTOPK_ERR_WORKSPACE_TOO_SMALL;
    const int eb = dt == RTOPK_F32 ? 4 : 2;
    char* ws = (char*)workspace;
    char* top = ws + L.partial_bytes;
    if (L.select_bytes) {
        // (rows that do not follow one another one by one)
        const int64_t at_once = batch == 1 || row_stride == n ? batch : 1;
        for (int64_t row = 0; row < batch; row += at_once) {
            s = rtopk_select((const char*)logits + row * row_stride * eb, at_once, n, k, dt, 1, RTOPK_FLAG_SORTED, 0, top + row * k * eb,
                             out_top_indices + row * k, top + L.top_bytes, L.select_bytes, hip_stream);
            if (s != RTOPK_OK) return s;
        }
    }
    LogprobsParams P = {};
    P.logits = (const char*)logits;
    P.row_bytes = row_stride * eb;
    P.n = (u32)n;
    P.m = m;
    P.k = k;
    P.parts = L.parts;
    P.part_vecs = L.part_vecs;
    P.c = inv_temperature * kLog2e;
    P.inv_t = inv_temperature;
    P.tokens = (const long long*)tokens;
    P.top_values = top;
    P.part_top = (u64*)top;
    P.top_indices = (long long*)out_top_indices;
    P.partial = (float4*)ws;
    P.logprobs = out_logprobs;
    P.entropy = out_entropy;
    P.top_logprobs = out_top_logprobs;
    P.row_stats = out_row_stats;
    const hipStream_t st = (hipStream_t)hip_stream;
    (void)hipGetLastError();  // an error left by earlier HIP calls of the process is not this call's
    return by_type(dt, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        if (out_entropy) L.top ? launch_logprobs<DT, true, true>(P, L, batch, st) : launch_logprobs<DT, true, false>(P, L, batch, st);
        else L.top ? launch_logprobs<DT, false, true>(P, L, batch, st) : launch_logprobs<DT, false, false>(P, L, batch, st);
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
            auto go = [&](auto nt, auto w) {
                hipLaunchKernelGGL((k_logprobs_grad<DT, decltype(nt)::value, decltype(w)::value>), dim3(now * d.parts), dim3(kGradBlock), lds, (hipStream_t)hip_stream, P);
            };
            if (past_caches(batch, n, eb)) grad_entropy ? go(std::true_type{}, std::true_type{}) : go(std::true_type{}, std::false_type{});
            else grad_entropy ? go(std::false_type{}, std::true_type{}) : go(std::false_type{}, std::false_type{});
        }
        return hipGetLastError() == hipSuccess ? RTOPK_OK : RTOPK_ERR_HIP;
    });
}

}  // extern "C"
