// libcce, router of a mixture-of-experts layer: top-k experts, their weights and counts, balance and z loss, and the gradient of the
// logits.  C ABI declared in include/cce_router.h.
//
// A row belongs to L lanes of a wavefront, each with VALUES logits in registers, 16 bytes of neighbours at a time (Columns); a wavefront
// takes 64 / L rows at a time and walks the rows with a grid stride.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <type_traits>

#include "../../include/cce.h"
#include "../../include/cce_router.h"
#include "host_util.h"
#include "vec_util.h"

namespace cce {

constexpr int kRouterBlocks = 256;                     // workgroups of the forward pass, each with one set of partial sums: one a CU
// Wavefronts of a workgroup: as many of 128 registers as a CU holds, half of them where the sums of each would fill the LDS or where lanes
// have more values (with_wide_shape).
constexpr bool wide_lanes(int lanes, int values) { return values >= 2 * lanes; }
constexpr int router_waves(int lanes, int values) { return lanes == 64 || wide_lanes(lanes, values) ? 8 : 16; }
constexpr int kGradBlocks = 512;                       // workgroups of the backward pass: two a CU, several trips each
constexpr int kJoinExperts = 8, kJoinParts = 256 / kJoinExperts;      // experts of a workgroup that joins them, threads of an expert

struct RouterArgs {
    const void* logits;
    const int32_t* labels;
    int32_t* indices;
    float* weights;
    float* lse;
    int32_t* counts;
    float* prob_sums;
    float* losses;
    // workspace, one entry (row of E) for each workgroup
    float* part_sums;
    int32_t* part_counts;
    double* part_z;
    int32_t* part_rows;
    int32_t* ticket;
    int64_t N;
    int32_t E, k, renormalize, ignore_index, blocks;
};

struct RouterGradArgs {
    const void* logits;
    const int32_t* indices;
    const float* lse;
    const int32_t* counts;
    const float* d_weights;
    const float* d_losses;
    void* d_logits;
    int64_t N;
    int32_t E, k, renormalize;
};

// A step of a reduction over lanes: lane ^ 1, ^ 2, then mirrored halves and rows of 16 (equal to ^ 4 and ^ 8 once smaller groups agree), ^ 16, ^ 32.
template <int STEP>
__device__ __forceinline__ uint32_t other_lane(uint32_t x) {
    if (STEP == 1) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xb1, 0xf, 0xf, false);
    if (STEP == 2) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4e, 0xf, 0xf, false);
    if (STEP == 4) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xf, 0xf, false);
    if (STEP == 8) return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xf, 0xf, false);
    if (STEP == 16) return (uint32_t)__builtin_amdgcn_ds_swizzle((int)x, 0x401f);
    return (uint32_t)__shfl_xor((int)x, 32);
}
// Of the lane in front, of the same 16.
__device__ __forceinline__ uint32_t lane_before(uint32_t x) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false); }

template <int L, int STEP = 1, class Op>
__device__ __forceinline__ uint32_t over_lanes(uint32_t x, Op op) {
    if constexpr (STEP < L) return over_lanes<L, STEP * 2>(op(x, other_lane<STEP>(x)), op);
    else return x;
}
template <int L>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
    return over_lanes<L>(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int L>
__device__ __forceinline__ uint32_t lanes_min(uint32_t x) {
    return over_lanes<L>(x, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
template <int L>
__device__ __forceinline__ float lanes_fmax(float x) {
    return __uint_as_float(over_lanes<L>(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
    return __uint_as_float(over_lanes<L>(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// The columns of a lane: value j of lane `sub` of a row.
template <bool BF16, int L, int VALUES>
struct Columns {
    static constexpr int kVec = VALUES < (BF16 ? 8 : 4) ? VALUES : (BF16 ? 8 : 4), kGroups = VALUES / kVec;
    static constexpr int of(int sub, int j) { return (j / kVec * L + sub) * kVec + j % kVec; }
};

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
    union { __bf16 h[2]; uint32_t u; } cv;
    cv.h[0] = (__bf16)lo;
    cv.h[1] = (__bf16)hi;
    return cv.u;
}

// A lane's logits of a row at `from` as they lie in memory, two bf16 values a word; -inf behind the row's end, and everywhere if not
// read.  whole: the row's start and length allow 16-byte accesses.
template <bool BF16, int L, int VALUES>
struct RawLogits {
    using C = Columns<BF16, L, VALUES>;
    static constexpr int kWords = BF16 ? (VALUES + 1) / 2 : VALUES;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const void* from, int64_t row, int E, int sub, bool whole, bool read) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = BF16 ? 0xff80ff80u : 0xff800000u;
        if (!read) return;
        if (C::kVec == (BF16 ? 8 : 4) && whole) {
            const char* const p = (const char*)from + row * E * (BF16 ? 2 : 4);
#pragma unroll
            for (int g = 0; g < C::kGroups; ++g) {
                const int at = C::of(sub, g * C::kVec);
                if (at >= E) continue;
                const au32x4 v = *(const au32x4*)(p + at * (BF16 ? 2 : 4));
#pragma unroll
                for (int e = 0; e < 4; ++e) w[(4 * g + e) % kWords] = v[e];
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < VALUES; ++j) {
            const int at = C::of(sub, j);
            if (at >= E) continue;
            if (!BF16) w[j % kWords] = ((const uint32_t*)from)[row * E + at];
            else {
                const uint32_t u = ((const uint16_t*)from)[row * E + at];
                w[j / 2] = j & 1 ? (w[j / 2] & 0xffffu) | u << 16 : (w[j / 2] & 0xffff0000u) | u;
            }
        }
    }
    __device__ __forceinline__ float value(int j) const {
        if (!BF16) return __uint_as_float(w[j % kWords]);
        return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    }
    // bf16: the values as 16-bit numbers around 2^15 in the same order, -0 as 0, two a word.
    __device__ __forceinline__ uint32_t ordered(int i) const {
        typedef __attribute__((ext_vector_type(2))) short s16x2;
        const s16x2 u = __builtin_bit_cast(s16x2, w[i]), sign = u >> 15, m = u & (short)0x7fff;
        return __builtin_bit_cast(uint32_t, (m ^ sign) - sign) ^ 0x80008000u;
    }
};

template <bool BF16, int L, int VALUES>
__device__ __forceinline__ void store_values(void* to, int64_t row, int E, int sub, bool whole, const float (&x)[VALUES]) {
    using C = Columns<BF16, L, VALUES>;
    if (C::kVec == (BF16 ? 8 : 4) && whole) {
        char* const p = (char*)to + row * E * (BF16 ? 2 : 4);
#pragma unroll
        for (int g = 0; g < C::kGroups; ++g) {
            const int at = C::of(sub, g * C::kVec);
            if (at >= E) continue;
            au32x4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = BF16 ? bf16_pair(x[(g * C::kVec + 2 * e) % VALUES], x[(g * C::kVec + 2 * e + 1) % VALUES])
                            : __float_as_uint(x[(g * C::kVec + e) % VALUES]);
            *(au32x4*)(p + at * (BF16 ? 2 : 4)) = v;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < VALUES; ++j) {
        const int at = C::of(sub, j);
        if (at >= E) continue;
        if (BF16) ((uint16_t*)to)[row * E + at] = (uint16_t)bf16_pair(x[j], 0.f);
        else ((float*)to)[row * E + at] = x[j];
    }
}

// Unsigned numbers in the order of the values that are numbers; -0 as 0.
__device__ __forceinline__ uint32_t ordered_bits(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
// Unsigned numbers in the order of the values; NaN above all, 0 for -inf.
__device__ __forceinline__ uint32_t rank_of(float x) {
    const uint32_t u = __float_as_uint(x);
    if (x != x) return 0xffffffffu;
    if (u == 0xff800000u) return 0u;
    // -0 and 0 are equal
    return u == 0x80000000u ? 0x80000000u : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t rank) {
    if (rank == 0xffffffffu) return __uint_as_float(0x7fc00000u);
    if (rank == 0u) return -INFINITY;
    return __uint_as_float(rank >> 31 ? rank ^ 0x80000000u : ~rank);
}

// ------------------------------------------------------------------------------------------
// Forward.
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ void write_losses(const RouterArgs& a, double balance, double z, int n) {
    const double rows = n > 0 ? (double)n : 1.0;
    a.losses[0] = (float)(balance * ((double)a.E / (double)a.k) / (rows * rows));
    a.losses[1] = (float)(z / rows);
}

// Sorting networks: x[0] the largest.  Of x whose first half falls and whose second half rises (or any rotation of that) the
// last log2 N steps are enough.
template <int N, bool MERGE>
__device__ __forceinline__ void sort_falling(uint32_t* x) {
#pragma unroll
    for (int size = MERGE ? N : 2; size <= N; size *= 2)
#pragma unroll
        for (int step = size / 2; step >= 1; step /= 2)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int k = i ^ step;
                if (k < i) continue;
                const uint32_t a = x[i], b = x[k], most = a > b ? a : b, least = a > b ? b : a;
                const bool falls = size == N || (i & size) == 0;
                x[i] = falls ? most : least;
                x[k] = falls ? least : most;
            }
}

// The K largest of a row's keys, falling, in every lane of the row: each lane's own, then lists merged with other lanes'.  The
// larger of a falling list and another one read backwards are the K largest of both.
template <int K, int L, int STEP = 1>
__device__ __forceinline__ void merge_lanes(uint32_t (&list)[K]) {
    if constexpr (STEP < L) {
        uint32_t other[K];
#pragma unroll
        for (int i = 0; i < K; ++i) other[i] = other_lane<STEP>(list[i]);
#pragma unroll
        for (int i = 0; i < K; ++i) list[i] = list[i] > other[K - 1 - i] ? list[i] : other[K - 1 - i];
        sort_falling<K, true>(list);
        merge_lanes<K, L, STEP * 2>(list);
    }
}
template <int K, int VALUES>
__device__ __forceinline__ void own_largest(const uint32_t (&key)[VALUES], uint32_t (&list)[K]) {
#pragma unroll
    for (int g = 0; g < VALUES; g += K) {
        uint32_t part[K];
#pragma unroll
        for (int i = 0; i < K; ++i) part[i] = g + i < VALUES ? key[(g + i) % VALUES] : 0u;
        sort_falling<K, false>(part);
        if (g == 0) {
#pragma unroll
            for (int i = 0; i < K; ++i) list[i] = part[i];
        } else {
#pragma unroll
            for (int i = 0; i < K; ++i) list[i] = list[i] > part[K - 1 - i] ? list[i] : part[K - 1 - i];
            sort_falling<K, true>(list);
        }
    }
}

// TOP > 0 (k <= TOP): a logit and its column make one 32-bit key, and the TOP largest of a row come out of sorting networks.  Of fp32 logits the
// column takes the place of the last bits, so that the outcome is checked against the whole values.  0, and rows that hold a NaN or +inf or fail
// the check: k rounds of a maximum over the row.  The launch alone, 65536 x 256, k = 8, bf16: rounds 53 us, networks 26, with_wide_shape 23; the
// whole call in fp32: rounds 52.5, networks 43.7.
template <bool BF16, int L, int VALUES, int TOP>
__global__ __launch_bounds__(64 * router_waves(L, VALUES), wide_lanes(L, VALUES) ? 2 : 4) void router_forward_kernel(const RouterArgs a) {
    using C = Columns<BF16, L, VALUES>;
    constexpr int kRows = 64 / L;                                     // of a wavefront
    constexpr int kRouterWaves = router_waves(L, VALUES), kRouterThreads = 64 * kRouterWaves;
    constexpr int kSlots = TOP ? 1 : (CCE_ROUTER_MAX_TOP_K + L - 1) / L;      // chosen experts a lane keeps
    constexpr int kColumns = L * VALUES;
    static_assert(TOP <= L, "a lane for each chosen expert");
    __shared__ int32_t count[kColumns];
    __shared__ float sums[kRouterWaves][kColumns];
    __shared__ double zs[kRouterWaves];
    __shared__ int32_t ns[kRouterWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane & (L - 1);
    for (int e = threadIdx.x; e < kColumns; e += kRouterThreads) count[e] = 0;
    __syncthreads();
    const bool whole = a.E % C::kVec == 0 && ((uintptr_t)a.logits & 15) == 0;
    float total_p[VALUES];
#pragma unroll
    for (int j = 0; j < VALUES; ++j) total_p[j] = 0.f;
    double z = 0.0;
    int rows = 0;
    const int64_t step = (int64_t)gridDim.x * kRouterWaves * kRows;
    // the labels two trips ahead, the logits one: nothing of a trip waits for memory
    auto taken_row = [&](int64_t row) { return row < a.N && !(a.labels && a.labels[row] == a.ignore_index); };
    const int64_t begin = ((int64_t)blockIdx.x * kRouterWaves + wave) * kRows;
    RawLogits<BF16, L, VALUES> ahead;
    ahead.load(a.logits, begin + lane / L, a.E, sub, whole, taken_row(begin + lane / L));
    bool read_next = taken_row(begin + step + lane / L);
    for (int64_t first = begin; first < a.N; first += step) {
        const int64_t row = first + lane / L;
        const bool there = row < a.N;
        const RawLogits<BF16, L, VALUES> raw = ahead;
        float x[VALUES];
#pragma unroll
        for (int j = 0; j < VALUES; ++j) x[j] = raw.value(j);
        ahead.load(a.logits, row + step, a.E, sub, whole, read_next);
        read_next = taken_row(row + 2 * step);
        float most_x = x[0];
#pragma unroll
        for (int j = 1; j < VALUES; ++j) most_x = fmaxf(most_x, x[j]);
        most_x = lanes_fmax<L>(most_x);
        bool live = most_x > -INFINITY;
        float top = live ? most_x : 0.f;
        float p[VALUES], part = 0.f;
#pragma unroll
        for (int j = 0; j < VALUES; ++j) {
            p[j] = __expf(x[j] - top);
            part += p[j];
        }
        float total = lanes_sum<L>(part);
        int index[kSlots];
        float weight[kSlots], chosen = 0.f;
        bool rounds = TOP == 0;
        if constexpr (TOP != 0) rounds = __ballot(total != total) != 0;          // a NaN, or +inf less itself, in one of the rows
        if constexpr (TOP != 0) {
            if (!rounds) {
                uint32_t key[VALUES], list[TOP];
#pragma unroll
                for (int j = 0; j < VALUES; ++j) {
                    if constexpr (BF16) {
                        const uint32_t pair = raw.ordered(j / 2);
                        key[j] = (j & 1 ? pair & 0xffff0000u : pair << 16) | (uint32_t)(0xffff - C::of(sub, j));
                    } else {
                        key[j] = (ordered_bits(x[j]) & ~(uint32_t)(kColumns - 1)) | (uint32_t)(kColumns - 1 - C::of(sub, j));
                    }
                }
                own_largest<TOP, VALUES>(key, list);
                merge_lanes<TOP, L>(list);
                uint32_t mine = 0u;
#pragma unroll
                for (int i = 0; i < TOP; ++i) mine = sub == i ? list[i] : mine;
                float value;
                bool taken;
                if constexpr (BF16) {
                    // 0x8000 - 0x7f80: -inf
                    taken = sub < a.k && (mine >> 16) > 0x80u;
                    const int32_t v = (int32_t)(mine >> 16) - 0x8000, magnitude = v < 0 ? -v : v;
                    value = __uint_as_float((uint32_t)magnitude << 16 | (v < 0 ? 0x80000000u : 0u));
                    index[0] = taken ? (int)(0xffffu - (mine & 0xffffu)) : -1;
                } else {
                    taken = sub < a.k && mine >= 0x00800000u;         // -inf: 0x007fffff
                    index[0] = taken ? kColumns - 1 - (int)(mine & (uint32_t)(kColumns - 1)) : -1;
                    value = taken ? ((const float*)a.logits)[row * a.E + index[0]] : -INFINITY;
                    // The chosen ones are right if they fall in their whole values, and as many of the row's are not below the last one as there are
                    // chosen ones (which equal values at the border are not).
                    const float before = __uint_as_float(lane_before(__float_as_uint(value)));
                    const int index_before = (int)lane_before((uint32_t)index[0]);
                    const float last = __shfl(value, (lane & ~(L - 1)) + a.k - 1);
                    uint32_t above = 0u;
#pragma unroll
                    for (int j = 0; j < VALUES; ++j) above += x[j] >= last ? 1u : 0u;
                    above = over_lanes<L>(above, [](uint32_t p, uint32_t q) { return p + q; });
                    const bool order = !taken || sub == 0 || before > value || (before == value && index_before < index[0]);
                    rounds = __ballot(!order || (last > -INFINITY && above != (uint32_t)a.k)) != 0;
                }
                weight[0] = taken ? __expf(value - top) : 0.f;
                chosen = lanes_sum<L>(weight[0]);
            }
        }
        if (rounds) {
            uint32_t rank[VALUES], best = 0u;
#pragma unroll
            for (int j = 0; j < VALUES; ++j) {
                rank[j] = rank_of(x[j]);
                best = rank[j] > best ? rank[j] : best;
            }
            uint32_t most = lanes_max<L>(best);
            live = most != 0u;                                        // (also of a row of NaN)
            chosen = 0.f;
            if (live) top = value_of(most);
            if (total != total) total = __uint_as_float(0x7fc00000u);
#pragma unroll
            for (int q = 0; q < kSlots; ++q) {
                index[q] = -1;
                weight[q] = 0.f;
                for (int s = 0; s < L && q * L + s < a.k; ++s) {
                    // the largest rank left, its first column, and both out of the running
                    uint32_t mine = (uint32_t)kColumns;
#pragma unroll
                    for (int j = VALUES - 1; j >= 0; --j) mine = rank[j] == most ? (uint32_t)C::of(sub, j) : mine;
                    const uint32_t column = lanes_min<L>(mine);
                    const bool taken = most != 0u;
                    const float w = taken ? __expf(value_of(most) - top) : 0.f;
                    if (TOP == 0) chosen += w;
                    if (sub == s) {
                        index[q] = taken ? (int)column : -1;
                        weight[q] = w;
                    }
                    best = 0u;
#pragma unroll
                    for (int j = 0; j < VALUES; ++j) {
                        rank[j] = column == (uint32_t)C::of(sub, j) ? 0u : rank[j];
                        best = rank[j] > best ? rank[j] : best;
                    }
                    most = lanes_max<L>(best);
                }
            }
            if constexpr (TOP != 0) chosen = lanes_sum<L>(weight[0]);  // (in the networks' order: a row's bits do not depend on its neighbours)
        }
        const float inv = live ? __builtin_amdgcn_rcpf(total) : 0.f;              // (a row that takes no part: p is 0)
        const float lse = live ? top + __logf(total) : 0.f;
#pragma unroll
        for (int j = 0; j < VALUES; ++j) total_p[j] = fmaf(p[j], inv, total_p[j]);
        const float norm = a.renormalize ? (live ? __builtin_amdgcn_rcpf(chosen) : 0.f) : inv;
#pragma unroll
        for (int q = 0; q < kSlots; ++q) {
            const int s = q * L + sub;
            if (s >= a.k || !there) continue;
            a.indices[row * a.k + s] = index[q];
            a.weights[row * a.k + s] = index[q] >= 0 ? weight[q] * norm : 0.f;
            if (index[q] >= 0) atomicAdd(&count[index[q]], 1);
        }
        if (sub == 0 && there) {
            a.lse[row] = lse;
            z = fma((double)lse, (double)lse, z);
            rows += live ? 1 : 0;
        }
    }
    // the wavefront's rows, then the workgroup's
#pragma unroll
    for (int j = 0; j < VALUES; ++j) {
#pragma unroll
        for (int o = L; o < 64; o *= 2) total_p[j] += __shfl_xor(total_p[j], o);
        if (lane < L) sums[wave][C::of(sub, j)] = total_p[j];
    }
#pragma unroll
    for (int o = L; o < 64; o *= 2) {
        z += __shfl_xor(z, o);
        rows += __shfl_xor(rows, o);
    }
    if (lane == 0) {
        zs[wave] = z;
        ns[wave] = rows;
    }
    __syncthreads();
    double group_z = 0.0;
    int group_rows = 0;
#pragma unroll
    for (int w = 0; w < kRouterWaves; ++w) {
        group_z += zs[w];
        group_rows += ns[w];
    }
    const bool alone = a.blocks == 1;
    double balance = 0.0;
    for (int e = threadIdx.x; e < a.E; e += kRouterThreads) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kRouterWaves; ++w) sum += sums[w][e];
        if (alone) {
            a.prob_sums[e] = sum;
            a.counts[e] = count[e];
            balance += (double)count[e] * (double)sum;
        } else {
            a.part_sums[(int64_t)blockIdx.x * a.E + e] = sum;
            a.part_counts[(int64_t)blockIdx.x * a.E + e] = count[e];
        }
    }
    if (!alone) {
        if (threadIdx.x == 0) {
            a.part_z[blockIdx.x] = group_z;
            a.part_rows[blockIdx.x] = group_rows;
            if (blockIdx.x == 0) a.ticket[0] = 0;
        }
        return;
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) balance += __shfl_xor(balance, o);
    __syncthreads();
    if (lane == 0) zs[wave] = balance;
    __syncthreads();
    if (threadIdx.x == 0) {
        balance = 0.0;
#pragma unroll
        for (int w = 0; w < kRouterWaves; ++w) balance += zs[w];
        a.counts[a.E] = group_rows;
        write_losses(a, balance, group_z, group_rows);
    }
}

// Joins the workgroups' sums: kJoinExperts experts a workgroup, kJoinParts threads an expert, all loads in flight; the last
// workgroup to end forms the losses.
__global__ __launch_bounds__(256) void router_join_kernel(const RouterArgs a) {
    __shared__ double red[256];
    __shared__ int32_t redn[256];
    __shared__ int32_t last;
    const int of = (int)threadIdx.x % kJoinExperts, part = (int)threadIdx.x / kJoinExperts, e = (int)blockIdx.x * kJoinExperts + of;
    constexpr int kLoads = kRouterBlocks / kJoinParts;
    static_assert(kRouterBlocks == 256, "a thread for each workgroup's z");
    float x[kLoads];
    int n[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
        const int at = part + u * kJoinParts;
        const bool there = at < a.blocks && e < a.E;
        x[u] = there ? a.part_sums[(int64_t)at * a.E + e] : 0.f;
        n[u] = there ? a.part_counts[(int64_t)at * a.E + e] : 0;
    }
    double z = (int)threadIdx.x < a.blocks ? a.part_z[threadIdx.x] : 0.0;
    int rows = (int)threadIdx.x < a.blocks ? a.part_rows[threadIdx.x] : 0;
    double sum = 0.0;
    int count = 0;
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
        sum += (double)x[u];
        count += n[u];
    }
    red[threadIdx.x] = sum;
    redn[threadIdx.x] = count;
    __syncthreads();
    for (int half = 128; half >= kJoinExperts; half >>= 1) {
        if ((int)threadIdx.x < half) {
            red[threadIdx.x] += red[threadIdx.x + half];
            redn[threadIdx.x] += redn[threadIdx.x + half];
        }
        __syncthreads();
    }
    if (threadIdx.x < kJoinExperts && e < a.E) {
        __hip_atomic_store(a.prob_sums + e, (float)red[threadIdx.x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(a.counts + e, redn[threadIdx.x], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(a.ticket, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    double balance = 0.0;
    for (int i = threadIdx.x; i < a.E; i += 256)
        balance += (double)__hip_atomic_load(a.counts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) *
                   (double)__hip_atomic_load(a.prob_sums + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        balance += __shfl_xor(balance, o);
        z += __shfl_xor(z, o);
        rows += __shfl_xor(rows, o);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        red[threadIdx.x >> 6] = balance;
        red[4 + (threadIdx.x >> 6)] = z;
        redn[threadIdx.x >> 6] = rows;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        rows = (redn[0] + redn[1]) + (redn[2] + redn[3]);
        a.counts[a.E] = rows;
        write_losses(a, (red[0] + red[1]) + (red[2] + red[3]), (red[4] + red[5]) + (red[6] + red[7]), rows);
    }
}

// ------------------------------------------------------------------------------------------
// Backward.  With d_e the gradient of p_e,  d logit_e = p_e (d_e - sum p d + 2 dz lse / n); d_e has the balance loss's part,
// beta c_e, and for a chosen expert that of its weight: dw, or with renormalized weights (dw - T / S) / S, where S is the sum of the
// row's chosen p and T that of p dw; the latter parts' share of sum p d is T, or 0 (T / S - S T / S^2).
// ------------------------------------------------------------------------------------------
template <bool BF16, int L, int VALUES>
__global__ __launch_bounds__(512, 4) void router_backward_kernel(const RouterGradArgs a) {
    using C = Columns<BF16, L, VALUES>;
    constexpr int kRows = 64 / L, kRouterWaves = 8;
    constexpr int kSlots = (CCE_ROUTER_MAX_TOP_K + L - 1) / L;
    constexpr int kColumns = L * VALUES;
    __shared__ float chosen_d[kRouterWaves * kRows][kColumns];      // 16 to 32 KB
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane & (L - 1);
    float* const mine = chosen_d[wave * kRows + lane / L];
    const bool whole = a.E % C::kVec == 0 && (((uintptr_t)a.logits | (uintptr_t)a.d_logits) & 15) == 0;
    float share[VALUES];                                              // beta c_e
    const int n = a.counts[a.E];
    const double rows = n > 0 ? (double)n : 1.0;
    const float beta = a.d_losses ? (float)((double)a.d_losses[0] * a.E / (a.k * rows * rows)) : 0.f;
    const float gamma = a.d_losses ? (float)(2.0 * (double)a.d_losses[1] / rows) : 0.f;
#pragma unroll
    for (int j = 0; j < VALUES; ++j) {
        share[j] = C::of(sub, j) < a.E ? beta * (float)a.counts[C::of(sub, j)] : 0.f;
        mine[C::of(sub, j)] = 0.f;
    }
    wave_lds_order();
    const int64_t step = (int64_t)gridDim.x * kRouterWaves * kRows;
    const int64_t begin = ((int64_t)blockIdx.x * kRouterWaves + wave) * kRows;
    // a trip's first index, by which its loads go, one trip ahead
    auto first_index = [&](int64_t row) { return row < a.N ? a.indices[row * a.k] : -1; };
    int next = first_index(begin + lane / L);
    for (int64_t first = begin; first < a.N; first += step) {
        const int64_t row = first + lane / L;
        const bool there = row < a.N, live = next >= 0;
        next = first_index(row + step);
        const float lse = live ? a.lse[row] : 0.f;
        RawLogits<BF16, L, VALUES> x;
        x.load(a.logits, row, a.E, sub, whole, live);
        int index[kSlots];
        float ps[kSlots], dw[kSlots], S = 0.f, T = 0.f;
#pragma unroll
        for (int q = 0; q < kSlots; ++q) {
            const int s = q * L + sub;
            index[q] = live && s < a.k && a.d_weights ? a.indices[row * a.k + s] : -1;
            if (index[q] >= a.E) index[q] = -1;
            ps[q] = dw[q] = 0.f;
            if (index[q] < 0) continue;
            const float logit = BF16 ? __uint_as_float((uint32_t)((const uint16_t*)a.logits)[row * a.E + index[q]] << 16)
                                     : ((const float*)a.logits)[row * a.E + index[q]];
            ps[q] = __expf(logit - lse);
            dw[q] = a.d_weights[row * a.k + s];
            S += ps[q];
            T += ps[q] * dw[q];
        }
        S = lanes_sum<L>(S);
        T = lanes_sum<L>(T);
        const float inv = a.renormalize ? (S > 0.f ? 1.f / S : 0.f) : 1.f, mean = a.renormalize ? T * inv : 0.f;
        float p[VALUES], dot = 0.f;
#pragma unroll
        for (int j = 0; j < VALUES; ++j) {
            p[j] = __expf(x.value(j) - lse);
            dot += p[j] * share[j];
        }
        dot = lanes_sum<L>(dot) + (a.renormalize ? 0.f : T) - gamma * lse;
#pragma unroll
        for (int q = 0; q < kSlots; ++q)
            if (index[q] >= 0) mine[index[q]] = (dw[q] - mean) * inv;
        wave_lds_order();                                             // a row's lanes are of one wavefront
        float d[VALUES];
#pragma unroll
        for (int j = 0; j < VALUES; ++j) d[j] = live ? p[j] * (share[j] + mine[C::of(sub, j)] - dot) : 0.f;
        wave_lds_order();
#pragma unroll
        for (int q = 0; q < kSlots; ++q)
            if (index[q] >= 0) mine[index[q]] = 0.f;
        wave_lds_order();
        if (there) store_values<BF16, L, VALUES>(a.d_logits, row, a.E, sub, whole, d);
    }
}

// ------------------------------------------------------------------------------------------
// Host side.
// ------------------------------------------------------------------------------------------
static bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

static int check_sizes(int64_t N, int64_t E) {
    if (N <= 0 || E <= 0) return CCE_ERR_INVALID;
    if (N > 0x7fffffffLL || E > CCE_ROUTER_MAX_EXPERTS) return CCE_ERR_UNSUPPORTED;
    return CCE_OK;
}

// Rows that a workgroup of so many wavefronts takes at a time.
static int64_t rows_of_group(int64_t E, int waves) { return waves * (E <= 64 ? 8 : E <= 256 ? 4 : E <= 512 ? 2 : 1); }

// Workgroups.  One takes two or three trips rather than leaving a join to a second launch, us of the launches without / with it: 256 x 64, k = 4
// 8.1 / 11.2, 384 x 64 9.9 / 11.1, 512 x 64 11.8 / 11.0, 128 x 128, k = 8 8.7 / 12.1, 192 x 128 10.6 / 12.2 (fp32 13.2 / 12.2), 128 x 256 12.9 / 15.8.
static int64_t forward_blocks(int64_t N, int64_t E) {
    const int64_t rows = rows_of_group(E, router_waves(E > 512 ? 64 : 8, 1)), want = (N + rows - 1) / rows;
    if (want <= (E <= 64 ? 3 : 2)) return 1;
    return want < kRouterBlocks ? want : kRouterBlocks;
}

// launch(BF16, L, VALUES as integral constants) for E columns
template <class Launch>
static void with_shape(bool bf16, int64_t E, Launch launch) {
#define CCE_ROUTER_SHAPE(L, VALUES) \
    (bf16 ? launch(std::true_type{}, std::integral_constant<int, L>{}, std::integral_constant<int, VALUES>{}) \
          : launch(std::false_type{}, std::integral_constant<int, L>{}, std::integral_constant<int, VALUES>{}))
    if (E <= 8) CCE_ROUTER_SHAPE(8, 1);
    else if (E <= 16) CCE_ROUTER_SHAPE(8, 2);
    else if (E <= 32) CCE_ROUTER_SHAPE(8, 4);
    else if (E <= 64) CCE_ROUTER_SHAPE(8, 8);
    else if (E <= 128) CCE_ROUTER_SHAPE(16, 8);
    else if (E <= 256) CCE_ROUTER_SHAPE(16, 16);
    else if (E <= 512) CCE_ROUTER_SHAPE(32, 16);
    else CCE_ROUTER_SHAPE(64, 16);
#undef CCE_ROUTER_SHAPE
}

// Half as many lanes a row, each with twice the values: fewer operations, most of them saved in merging the lanes' lists, but fewer
// wavefronts and longer gathers.  For lists of 8 of bf16 keys and whole 16-byte loads (fp32: 43.8 / 42.5, 4096 rows 19.3 / 23.4); narrow / wide, us: 65536 x 256, k = 8: 34.3 / 31.4, 65536 x 128, k = 8:
// 23.7 / 22.0, 32768 x 512, k = 8: 35.5 / 32.0; 65536 x 160, k = 4: 25.6 / 26.2, 32768 x 511, k = 8: 45.4 / 56.8.
static bool takes_wide(const RouterArgs& a) { return a.k > 4 && a.E > 64 && a.E <= 512 && a.E % 8 == 0 && ((uintptr_t)a.logits & 15) == 0; }
template <class Launch>
static void with_wide_shape(int64_t E, Launch launch) {
    if (E <= 128) launch(std::integral_constant<int, 8>{}, std::integral_constant<int, 16>{});
    else if (E <= 256) launch(std::integral_constant<int, 8>{}, std::integral_constant<int, 32>{});
    else launch(std::integral_constant<int, 16>{}, std::integral_constant<int, 32>{});
}

}  // namespace cce

using namespace cce;

extern "C" {

size_t cce_router_workspace_bytes(int64_t N, int64_t E) {
    if (check_sizes(N, E) != CCE_OK) return 0;
    const int64_t blocks = forward_blocks(N, E);
    return (size_t)round_up(blocks * (E * 8 + 8 + 4) + 4, 256);
}

int cce_router_forward(const void* logits, int32_t logits_bf16, const int32_t* labels, int64_t N, int64_t E, int32_t top_k,
                       int32_t renormalize, int32_t ignore_index, int32_t* indices, float* weights, float* lse, int32_t* counts,
                       float* prob_sums, float* losses, void* workspace, size_t workspace_bytes, void* stream_) {
    const int rc = check_sizes(N, E);
    if (rc != CCE_OK) return rc;
    if (top_k < 1 || top_k > E || (logits_bf16 != 0 && logits_bf16 != 1) || (renormalize != 0 && renormalize != 1)) return CCE_ERR_INVALID;
    if (top_k > CCE_ROUTER_MAX_TOP_K) return CCE_ERR_UNSUPPORTED;
    if (!logits || !indices || !weights || !lse || !counts || !prob_sums || !losses || !workspace) return CCE_ERR_INVALID;
    if (misaligned(logits, logits_bf16 ? 2 : 4) || misaligned(labels, 4) || misaligned(indices, 4) || misaligned(weights, 4) || misaligned(lse, 4) ||
        misaligned(counts, 4) || misaligned(prob_sums, 4) || misaligned(losses, 4) || misaligned(workspace, 256)) return CCE_ERR_INVALID;
    if (workspace_bytes < cce_router_workspace_bytes(N, E)) return CCE_ERR_INVALID;
    hipStream_t stream = (hipStream_t)stream_;
    (void)hipGetLastError();
    RouterArgs a;
    const int64_t blocks = forward_blocks(N, E);
    a.logits = logits; a.labels = labels; a.indices = indices; a.weights = weights; a.lse = lse; a.counts = counts;
    a.prob_sums = prob_sums; a.losses = losses;
    char* p = (char*)workspace;
    a.part_z = (double*)p; p += blocks * 8;
    a.part_sums = (float*)p; p += blocks * E * 4;
    a.part_counts = (int32_t*)p; p += blocks * E * 4;
    a.part_rows = (int32_t*)p; p += blocks * 4;
    a.ticket = (int32_t*)p;
    a.N = N; a.E = (int32_t)E; a.k = top_k; a.renormalize = renormalize; a.ignore_index = ignore_index; a.blocks = (int32_t)blocks;
    auto run = [&](auto bf16, auto l, auto values, auto top) {
        constexpr int L = decltype(l)::value, VALUES = decltype(values)::value;
        hipLaunchKernelGGL((router_forward_kernel<decltype(bf16)::value, L, VALUES, decltype(top)::value>), dim3((unsigned)blocks),
                           dim3(64 * router_waves(L, VALUES)), 0, stream, a);
    };
    if (logits_bf16 != 0 && top_k <= 8 && takes_wide(a)) {
        with_wide_shape(E, [&](auto l, auto values) { run(std::true_type{}, l, values, std::integral_constant<int, 8>{}); });
    } else {
        with_shape(logits_bf16 != 0, E, [&](auto bf16, auto l, auto values) {
            if (top_k <= 2) return run(bf16, l, values, std::integral_constant<int, 2>{});
            if (top_k <= 4) return run(bf16, l, values, std::integral_constant<int, 4>{});
            if (top_k <= 8) return run(bf16, l, values, std::integral_constant<int, 8>{});
            run(bf16, l, values, std::integral_constant<int, 0>{});
        });
    }
    if (blocks > 1)
        hipLaunchKernelGGL(router_join_kernel, dim3((unsigned)((E + kJoinExperts - 1) / kJoinExperts)), dim3(256), 0, stream, a);
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

int cce_router_backward(const void* logits, int32_t logits_bf16, const int32_t* indices, const float* lse, const int32_t* counts,
                        const float* d_weights, const float* d_losses, int64_t N, int64_t E, int32_t top_k, int32_t renormalize,
                        void* d_logits, void* stream_) {
    const int rc = check_sizes(N, E);
    if (rc != CCE_OK) return rc;
    if (top_k < 1 || top_k > E || (logits_bf16 != 0 && logits_bf16 != 1) || (renormalize != 0 && renormalize != 1)) return CCE_ERR_INVALID;
    if (top_k > CCE_ROUTER_MAX_TOP_K) return CCE_ERR_UNSUPPORTED;
    if (!logits || !indices || !lse || !counts || !d_logits) return CCE_ERR_INVALID;
    if (misaligned(logits, logits_bf16 ? 2 : 4) || misaligned(d_logits, logits_bf16 ? 2 : 4) || misaligned(indices, 4) || misaligned(lse, 4) ||
        misaligned(counts, 4) || misaligned(d_weights, 4) || misaligned(d_losses, 4)) return CCE_ERR_INVALID;
    hipStream_t stream = (hipStream_t)stream_;
    (void)hipGetLastError();
    RouterGradArgs a;
    a.logits = logits; a.indices = indices; a.lse = lse; a.counts = counts; a.d_weights = d_weights; a.d_losses = d_losses;
    a.d_logits = d_logits; a.N = N; a.E = (int32_t)E; a.k = top_k; a.renormalize = renormalize;
    const int64_t rows = rows_of_group(E, 8), want = (N + rows - 1) / rows, blocks = want < kGradBlocks ? want : kGradBlocks;
    with_shape(logits_bf16 != 0, E, [&](auto bf16, auto l, auto values) {
        hipLaunchKernelGGL((router_backward_kernel<decltype(bf16)::value, decltype(l)::value, decltype(values)::value>),
                           dim3((unsigned)blocks), dim3(512), 0, stream, a);
    });
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

}  // extern "C"
