// libcce, embedding kernels: lookup of rows of the bf16 matrix with scaling, and its gradient.
// C ABI declared in include/cce_embed.h.
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/cce.h"
#include "../../include/cce_embed.h"
#include "host_util.h"
#include "vec_util.h"

namespace cce {

constexpr int64_t kEmbedMaxRows = (int64_t)1 << 24;      // V
constexpr int64_t kEmbedMaxDim = 65536;                  // D
constexpr int64_t kMaxBlocks = (1 << 24) - 1;            // of 256 threads: a launch has fewer than 2^32 threads

// Whether a token names a row; a bad one that is not ignore_index is reported.
__device__ __forceinline__ bool token_takes_part(int token, int V, int ignore_index, int32_t* status) {
    if (token == ignore_index) return false;
    if ((unsigned)token < (unsigned)V) return true;
    if (status) atomicOr(status, CCE_STATUS_BAD_TOKEN);
    return false;
}

// y_i = scale * W[t_i]: a thread per 16 bytes of y.
__global__ __launch_bounds__(256) void embedding_forward_kernel(
        const int32_t* __restrict__ tokens, const uint16_t* __restrict__ weight, int64_t chunks, int row_chunks, int V,
        int ignore_index, float scale, uint16_t* __restrict__ out, int32_t* status) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / row_chunks;
        const int c = (int)(i - row * row_chunks);
        const int token = tokens[row];
        float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (token_takes_part(token, V, ignore_index, c == 0 ? status : nullptr)) {
            unpack8(((const au32x4*)weight)[(size_t)token * row_chunks + c], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= scale;
        }
        ((au32x4*)out)[i] = pack8(f);
    }
}

// One wavefront per row of dW: it looks through the tokens 64 at a time and adds the rows of d_out whose
// token is its own, in order.
__global__ __launch_bounds__(256) void embedding_backward_kernel(
        const int32_t* __restrict__ tokens, const uint16_t* __restrict__ d_out, int N, int row_chunks, int V,
        int ignore_index, float scale, float* __restrict__ dW, int accumulate, int32_t* status) {
    const int lane = threadIdx.x & 63;
    const int v = blockIdx.x * 4 + (int)(threadIdx.x >> 6);
    if (v >= V) return;
    for (int c0 = 0; c0 < row_chunks; c0 += 64) {
        const int c = c0 + lane;
        float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        bool any = false;
        for (int64_t base = 0; base < N; base += 64) {
            const int token = base + lane < N ? tokens[base + lane] : ignore_index;
            const bool ok = token_takes_part(token, V, ignore_index, v == 0 ? status : nullptr);
            unsigned long long hits = __ballot(ok && token == v);
            while (hits) {
                const int64_t row = base + __ffsll(hits) - 1;
                hits &= hits - 1;
                any = true;
                if (c < row_chunks) {
                    float f[8];
                    unpack8(((const au32x4*)d_out)[(size_t)row * row_chunks + c], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += f[e];
                }
            }
        }
        if (c >= row_chunks || (accumulate && !any)) continue;
        af32x4* to = (af32x4*)dW + ((size_t)v * row_chunks + c) * 2;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            af32x4 r = {scale * sum[4 * h], scale * sum[4 * h + 1], scale * sum[4 * h + 2], scale * sum[4 * h + 3]};
            to[h] = accumulate ? to[h] + r : r;
        }
    }
}

static int embed_shape(int64_t N, int64_t D, int64_t V) {
    if (N <= 0 || D <= 0 || V <= 0) return CCE_ERR_INVALID;
    if (N > 0x7fffffff || D % 8 != 0 || D > kEmbedMaxDim || V > kEmbedMaxRows) return CCE_ERR_UNSUPPORTED;
    return CCE_OK;
}

}  // namespace cce

using namespace cce;

extern "C" {

int cce_embedding_forward(const int32_t* tokens, const void* weight, int64_t N, int64_t D, int64_t V,
                          int32_t ignore_index, float scale, void* out, int32_t* status, void* stream_) {
    if (!tokens || !weight || !out) return CCE_ERR_INVALID;
    const int rc = embed_shape(N, D, V);
    if (rc != CCE_OK) return rc;
    if ((((uintptr_t)weight | (uintptr_t)out) & 15) || (((uintptr_t)tokens | (uintptr_t)status) & 3)) return CCE_ERR_INVALID;
    const int64_t chunks = N * (D / 8), want = (chunks + 255) / 256;
    (void)hipGetLastError();
    hipLaunchKernelGGL(embedding_forward_kernel, dim3((unsigned)(want < kMaxBlocks ? want : kMaxBlocks)), dim3(256), 0, (hipStream_t)stream_,
                       tokens, (const uint16_t*)weight, chunks, (int)(D / 8), (int)V, ignore_index, scale, (uint16_t*)out, status);
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

size_t cce_embedding_workspace_bytes(int64_t N, int64_t D, int64_t V) {
    return embed_shape(N, D, V) == CCE_OK ? 256 : 0;
}

int cce_embedding_backward(const int32_t* tokens, const void* d_out, int64_t N, int64_t D, int64_t V,
                           int32_t ignore_index, float scale, float* dW, int accumulate_dW, int32_t* status,
                           void* workspace, size_t workspace_bytes, void* stream_) {
    if (!tokens || !d_out || !dW || !workspace) return CCE_ERR_INVALID;
    const int rc = embed_shape(N, D, V);
    if (rc != CCE_OK) return rc;
    if ((((uintptr_t)d_out | (uintptr_t)dW) & 15) || (((uintptr_t)tokens | (uintptr_t)status) & 3)) return CCE_ERR_INVALID;
    if (((uintptr_t)workspace & 255) || workspace_bytes < cce_embedding_workspace_bytes(N, D, V)) return CCE_ERR_INVALID;
    (void)hipGetLastError();
    hipLaunchKernelGGL(embedding_backward_kernel, dim3((unsigned)((V + 3) / 4)), dim3(256), 0, (hipStream_t)stream_,
                       tokens, (const uint16_t*)d_out, (int)N, (int)(D / 8), (int)V, ignore_index, scale, dW,
                       accumulate_dW ? 1 : 0, status);
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

}  // extern "C"
