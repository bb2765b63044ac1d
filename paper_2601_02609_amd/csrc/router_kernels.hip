// libcce, router of a mixture-of-experts layer: top-k experts, their weights and counts, balance and z loss, and the gradient of the
// logits.  C ABI declared in include/cce_router.h.
//
// A row belongs to L lanes of a wavefront, each with VALUES neighbouring logits in registers; a wavefront takes 64 / L rows at a time
// and walks the rows with a grid stride.
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

constexpr int kRouterThreads = 256;
constexpr int kRouterWaves = kRouterThreads / 64;
constexpr int kRouterBlocks = 512;                     // workgroups of the forward pass, each with one set of partial sums
constexpr int kJoinExperts = 16;                       // experts of a workgroup that joins them

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
__device__ __forceinline__ float lanes_sum(float x) {
    return __uint_as_float(over_lanes<L>(__float_as_uint(x), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// VALUES logits from column `at` on of a row at `from`; -inf behind the row's end.  whole: the row's start and length allow
// loads of as many bytes as a lane has.
template <bool BF16, int VALUES>
__device__ __forceinline__ void load_logits(const void* from, int64_t row, int E, int at, bool whole, float (&x)[VALUES]) {
    constexpr int kBytes = VALUES * (BF16 ? 2 : 4);
    if (kBytes >= 8 && whole && at < E) {
        const char* p = (const char*)from + (row * E + at) * (BF16 ? 2 : 4);
        if constexpr (BF16 && kBytes >= 8) {
#pragma unroll
            for (int j = 0; j < VALUES; j += 4) {
                const uint2 v = *(const uint2*)(p + 2 * j);
                x[j] = __uint_as_float(v.x << 16);
                x[j + 1] = __uint_as_float(v.x & 0xffff0000u);
                x[j + 2] = __uint_as_float(v.y << 16);
                x[j + 3] = __uint_as_float(v.y & 0xffff0000u);
            }
        } else if constexpr (!BF16 && kBytes >= 8) {
#pragma unroll
            for (int j = 0; j < VALUES; j += 2) {
                const float2 v = *(const float2*)(p + 4 * j);
                x[j] = v.x;
                x[j + 1] = v.y;
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < VALUES; ++j) {
        if (at + j >= E) x[j] = -INFINITY;
        else if (BF16) x[j] = __uint_as_float((uint32_t)((const uint16_t*)from)[row * E + at + j] << 16);
        else x[j] = ((const float*)from)[row * E + at + j];
    }
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

template <bool BF16, int L, int VALUES>
__global__ __launch_bounds__(kRouterThreads) void router_forward_kernel(const RouterArgs a) {
    constexpr int kRows = 64 / L;                                     // of a wavefront
    constexpr int kSlots = (CCE_ROUTER_MAX_TOP_K + L - 1) / L;        // chosen experts a lane keeps
    constexpr int kColumns = L * VALUES;
    __shared__ int32_t count[kColumns];
    __shared__ float sums[kRouterWaves][kColumns];
    __shared__ double zs[kRouterWaves];
    __shared__ int32_t ns[kRouterWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane & (L - 1), at = sub * VALUES;
    for (int e = threadIdx.x; e < kColumns; e += kRouterThreads) count[e] = 0;
    __syncthreads();
    const bool whole = a.E % VALUES == 0 && ((uintptr_t)a.logits & 15) == 0;
    float total_p[VALUES];
#pragma unroll
    for (int j = 0; j < VALUES; ++j) total_p[j] = 0.f;
    double z = 0.0;
    int rows = 0;
    const int64_t step = (int64_t)gridDim.x * kRouterWaves * kRows;
    for (int64_t first = ((int64_t)blockIdx.x * kRouterWaves + wave) * kRows; first < a.N; first += step) {
        const int64_t row = first + lane / L;
        const bool there = row < a.N, read = there && !(a.labels && a.labels[row] == a.ignore_index);
        float x[VALUES];
        if (read) load_logits<BF16, VALUES>(a.logits, row, a.E, at, whole, x);
        else {
#pragma unroll
            for (int j = 0; j < VALUES; ++j) x[j] = -INFINITY;
        }
        uint32_t rank[VALUES], best = 0u;
#pragma unroll
        for (int j = 0; j < VALUES; ++j) {
            rank[j] = rank_of(x[j]);
            best = rank[j] > best ? rank[j] : best;
        }
        uint32_t most = lanes_max<L>(best);
        const bool live = most != 0u;
        const float top = live ? value_of(most) : 0.f;
        float p[VALUES], part = 0.f;
#pragma unroll
        for (int j = 0; j < VALUES; ++j) {
            p[j] = __expf(x[j] - top);
            part += p[j];
        }
        const float total = lanes_sum<L>(part), inv = live ? 1.f / total : 0.f;
        const float lse = live ? top + __logf(total) : 0.f;
#pragma unroll
        for (int j = 0; j < VALUES; ++j) total_p[j] += live ? p[j] * inv : 0.f;
        int index[kSlots];
        float weight[kSlots], chosen = 0.f;
#pragma unroll
        for (int q = 0; q < kSlots; ++q) {
            index[q] = -1;
            weight[q] = 0.f;
            for (int s = 0; s < L && q * L + s < a.k; ++s) {
                // the largest rank left, its first column, and both out of the running
                uint32_t mine = (uint32_t)kColumns;
#pragma unroll
                for (int j = VALUES - 1; j >= 0; --j) mine = rank[j] == most ? (uint32_t)(at + j) : mine;
                const uint32_t column = lanes_min<L>(mine);
                const bool taken = most != 0u;
                const float w = taken ? __expf(value_of(most) - top) : 0.f;
                chosen += w;
                if (sub == s) {
                    index[q] = taken ? (int)column : -1;
                    weight[q] = w;
                }
                best = 0u;
#pragma unroll
                for (int j = 0; j < VALUES; ++j) {
                    rank[j] = column == (uint32_t)(at + j) ? 0u : rank[j];
                    best = rank[j] > best ? rank[j] : best;
                }
                most = lanes_max<L>(best);
            }
        }
        const float norm = a.renormalize ? (live ? 1.f / chosen : 0.f) : inv;
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
        if (lane < L) sums[wave][at + j] = total_p[j];
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
        a.counts[a.E] = group_rows;
        write_losses(a, (zs[0] + zs[1]) + (zs[2] + zs[3]), group_z, group_rows);
    }
}

// Joins the workgroups' sums: kJoinExperts experts a workgroup, 16 threads an expert; the last workgroup to end forms the losses.
__global__ __launch_bounds__(256) void router_join_kernel(const RouterArgs a) {
    __shared__ double red[256];
    __shared__ int32_t redn[256];
    __shared__ int32_t last;
    const int e = (int)blockIdx.x * kJoinExperts + (int)(threadIdx.x & 15), part = (int)(threadIdx.x >> 4);
    double sum = 0.0;
    int count = 0;
    if (e < a.E) {
        for (int b = part; b < a.blocks; b += 16) {
            sum += (double)a.part_sums[(int64_t)b * a.E + e];
            count += a.part_counts[(int64_t)b * a.E + e];
        }
    }
    red[threadIdx.x] = sum;
    redn[threadIdx.x] = count;
    __syncthreads();
    if (threadIdx.x < 16 && e < a.E) {
        for (int p = 1; p < 16; ++p) {
            sum += red[16 * p + threadIdx.x];
            count += redn[16 * p + threadIdx.x];
        }
        __hip_atomic_store(a.prob_sums + e, (float)sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(a.counts + e, count, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(a.ticket, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    double balance = 0.0, z = 0.0;
    int rows = 0;
    for (int i = threadIdx.x; i < a.E; i += 256)
        balance += (double)__hip_atomic_load(a.counts + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) *
                   (double)__hip_atomic_load(a.prob_sums + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    for (int b = threadIdx.x; b < a.blocks; b += 256) {
        z += a.part_z[b];
        rows += a.part_rows[b];
    }
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
__global__ __launch_bounds__(kRouterThreads) void router_backward_kernel(const RouterGradArgs a) {
    constexpr int kRows = 64 / L;
    constexpr int kSlots = (CCE_ROUTER_MAX_TOP_K + L - 1) / L;
    constexpr int kColumns = L * VALUES;
    __shared__ float chosen_d[kRouterWaves * kRows][kColumns];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane & (L - 1), at = sub * VALUES;
    float* const mine = chosen_d[wave * kRows + lane / L];
    const bool whole = a.E % VALUES == 0 && (((uintptr_t)a.logits | (uintptr_t)a.d_logits) & 15) == 0;
    float share[VALUES];                                              // beta c_e
    const int n = a.counts[a.E];
    const double rows = n > 0 ? (double)n : 1.0;
    const float beta = a.d_losses ? (float)((double)a.d_losses[0] * a.E / (a.k * rows * rows)) : 0.f;
    const float gamma = a.d_losses ? (float)(2.0 * (double)a.d_losses[1] / rows) : 0.f;
#pragma unroll
    for (int j = 0; j < VALUES; ++j) {
        share[j] = at + j < a.E ? beta * (float)a.counts[at + j] : 0.f;
        mine[at + j] = 0.f;
    }
    const int64_t step = (int64_t)gridDim.x * kRouterWaves * kRows;
    for (int64_t first = ((int64_t)blockIdx.x * kRouterWaves + wave) * kRows; first < a.N; first += step) {
        const int64_t row = first + lane / L;
        const bool there = row < a.N, live = there && a.indices[row * a.k] >= 0;
        const float lse = live ? a.lse[row] : 0.f;
        float x[VALUES];
        if (live) load_logits<BF16, VALUES>(a.logits, row, a.E, at, whole, x);
        else {
#pragma unroll
            for (int j = 0; j < VALUES; ++j) x[j] = -INFINITY;
        }
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
            p[j] = __expf(x[j] - lse);
            dot += p[j] * share[j];
        }
        dot = lanes_sum<L>(dot) + (a.renormalize ? 0.f : T) - gamma * lse;
#pragma unroll
        for (int q = 0; q < kSlots; ++q)
            if (index[q] >= 0) mine[index[q]] = (dw[q] - mean) * inv;
        __builtin_amdgcn_wave_barrier();                              // a row's lanes are of one wavefront, whose LDS accesses keep their order
        float d[VALUES];
#pragma unroll
        for (int j = 0; j < VALUES; ++j) d[j] = live ? p[j] * (share[j] + mine[at + j] - dot) : 0.f;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int q = 0; q < kSlots; ++q)
            if (index[q] >= 0) mine[index[q]] = 0.f;
        __builtin_amdgcn_wave_barrier();
        if (!there) continue;
        if (BF16) {
            uint16_t* const to = (uint16_t*)a.d_logits + row * a.E + at;
#pragma unroll
            for (int j = 0; j < VALUES; ++j) {
                union { __bf16 h; uint16_t u; } cv;
                cv.h = (__bf16)d[j];
                if (at + j < a.E) to[j] = cv.u;
            }
        } else {
            float* const to = (float*)a.d_logits + row * a.E + at;
#pragma unroll
            for (int j = 0; j < VALUES; ++j)
                if (at + j < a.E) to[j] = d[j];
        }
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

static int rows_of_group(int64_t E) { return kRouterWaves * (E <= 64 ? 8 : E <= 256 ? 4 : E <= 512 ? 2 : 1); }

static int64_t forward_blocks(int64_t N, int64_t E) {
    const int64_t rows = rows_of_group(E), want = (N + rows - 1) / rows;
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
    with_shape(logits_bf16 != 0, E, [&](auto bf16, auto l, auto values) {
        hipLaunchKernelGGL((router_forward_kernel<decltype(bf16)::value, decltype(l)::value, decltype(values)::value>),
                           dim3((unsigned)blocks), dim3(kRouterThreads), 0, stream, a);
    });
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
    const int64_t rows = rows_of_group(E), want = (N + rows - 1) / rows, blocks = want < 2048 ? want : 2048;
    with_shape(logits_bf16 != 0, E, [&](auto bf16, auto l, auto values) {
        hipLaunchKernelGGL((router_backward_kernel<decltype(bf16)::value, decltype(l)::value, decltype(values)::value>),
                           dim3((unsigned)blocks), dim3(kRouterThreads), 0, stream, a);
    });
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

}  // extern "C"
