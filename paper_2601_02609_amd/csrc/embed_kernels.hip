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
constexpr int64_t kEmbedMaxValues = (int64_t)1 << 37;    // V * D: half a terabyte of dW
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

// ------------------------------------------------------------------------------------------
// Gradient by sorted tokens, in three launches without atomics on results:
//   order   positions grouped by token, ascending inside a token, and where each token's group begins
//   sum     the groups' rows in pieces of the same number of rows, whatever the tokens are (a few tokens have most
//           of the rows): a group inside a piece goes straight to dW, the part of one that crosses a piece's end to
//           a partial row; beside it, zeros for the rows of dW that no token names
//   join    the partial rows of the groups that cross, in order
// The order of all sums follows from the tokens and the sizes.
// ------------------------------------------------------------------------------------------
constexpr int kSliceKeys = 768;                 // rows of the matrix that an order workgroup counts: 48 KB of LDS
constexpr int kOrderWaves = 16;
constexpr int kJoinWaves = 8;
constexpr int kMinPiece = 16;                   // rows of a piece, more where that makes over kMaxPieces
constexpr int kMaxPieces = 2048;

// Slices of the vocabulary: token t is key t / slices of slice t % slices (a power of two).  The frequent tokens, which
// tokenizers number first, are spread over the slices.
static int slice_bits(int64_t V) {
    int bits = 8;
    while ((V + (1 << bits) - 1) >> bits > kSliceKeys) ++bits;
    return bits;
}

struct EmbedBackward {
    const int32_t* tokens;
    const uint16_t* d_out;
    float* dW;
    int32_t* status;
    int32_t* starts;          // [slices][keys + 1]: where a key's group begins in `order`
    int32_t* order;           // [N] positions
    int32_t* sorted;          // [N] their tokens
    float* partial;           // [pieces][2][D]: of the group a piece begins within, of the one that it begins and does not end
    int N, V, ignore_index, bits, keys, row_chunks, piece, strips, accumulate;
    float scale;
};

// A workgroup per slice looks through all tokens twice (they stay in the L2s): its wavefronts, each with a range of
// positions, count their keys in LDS; after a scan over keys and wavefronts they go through their ranges again, 64
// positions at a time, and give the positions of one key consecutive places.
__global__ __launch_bounds__(64 * kOrderWaves) void embedding_order_kernel(const EmbedBackward a) {
    __shared__ uint32_t count[kOrderWaves * kSliceKeys];
    __shared__ uint32_t wave_total[kOrderWaves], wave_below[kOrderWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int slice = blockIdx.x, mask = (1 << a.bits) - 1;
    uint32_t* own = count + w * a.keys;
    for (int i = threadIdx.x; i < kOrderWaves * a.keys; i += 64 * kOrderWaves) count[i] = 0u;
    __syncthreads();

    const int64_t range = ((int64_t)a.N + 64 * kOrderWaves - 1) / (64 * kOrderWaves) * 64;
    const int64_t begin = w * range, end = begin + range < a.N ? begin + range : a.N;
    uint32_t below = 0u;
    for (int64_t i = begin; i < end; i += 256) {
        int token[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) token[u] = i + 64 * u + lane < end ? a.tokens[i + 64 * u + lane] : a.ignore_index;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (!token_takes_part(token[u], a.V, a.ignore_index, slice == 0 ? a.status : nullptr)) continue;
            const int s = token[u] & mask;
            below += s < slice ? 1u : 0u;
            if (s == slice) atomicAdd(&own[token[u] >> a.bits], 1u);
        }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) below += (uint32_t)__shfl_xor((int)below, o);
    if (lane == 0) wave_below[w] = below;
    __syncthreads();

    // exclusive scan over the keys of this slice, behind everything in the slices below
    uint32_t base = 0u;
#pragma unroll
    for (int i = 0; i < kOrderWaves; ++i) base += wave_below[i];
    const int key = threadIdx.x;
    uint32_t total = 0u;
    if (key < a.keys)
        for (int i = 0; i < kOrderWaves; ++i) total += count[i * a.keys + key];
    uint32_t scan = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = (uint32_t)__shfl_up((int)scan, o);
        if (lane >= o) scan += x;
    }
    if (lane == 63) wave_total[w] = scan;
    __syncthreads();
    for (int i = 0; i < w; ++i) base += wave_total[i];
    uint32_t at = base + scan - total;
    if (key <= a.keys) a.starts[(size_t)slice * (a.keys + 1) + key] = (int32_t)at;
    if (key < a.keys)
        for (int i = 0; i < kOrderWaves; ++i) {
            const uint32_t n = count[i * a.keys + key];
            count[i * a.keys + key] = at;
            at += n;
        }
    __syncthreads();

    for (int64_t i = begin; i < end; i += 256) {
        int token[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) token[u] = i + 64 * u + lane < end ? a.tokens[i + 64 * u + lane] : a.ignore_index;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const bool mine = token_takes_part(token[u], a.V, a.ignore_index, nullptr) && (token[u] & mask) == slice;
            unsigned long long left = __ballot(mine);
            while (left) {                                   // a trip per key among the 64
                const int leader = __ffsll(left) - 1;
                const int t = __builtin_amdgcn_readlane(token[u], leader);
                const unsigned long long same = __ballot(mine && token[u] == t);
                int place = 0;
                if (lane == leader) place = (int)atomicAdd(&own[t >> a.bits], (uint32_t)__popcll(same));
                place = __builtin_amdgcn_readlane(place, leader);
                if (mine && token[u] == t) {
                    place += __popcll(same & ((1ull << lane) - 1ull));
                    a.order[place] = (int32_t)(i + 64 * u + lane);
                    a.sorted[place] = t;
                }
                left &= ~same;
            }
        }
    }
}

// A value of lane j of each group of eight lanes.  Wavefronts that work on one row have it in a scalar register.
template <int LPR>
__device__ __forceinline__ int of_lane(int x, int j) {
    if constexpr (LPR == 64) return __builtin_amdgcn_readlane(x, j);
    else return __shfl(x, j, 8);
}

// LPR lanes share a row (a strip of 512 columns of it if D > 512), 16 bytes each, and take one piece.  Eight rows, and
// the rows of dW that they end at, are in flight.
template <int LPR>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const EmbedBackward a, int sum_blocks) {
    const int slices = 1 << a.bits;
    if ((int)blockIdx.x >= sum_blocks) {                     // zeros: 64 keys of a slice for each workgroup
        const int slice = ((int)blockIdx.x - sum_blocks) & (slices - 1);
        const int first = (((int)blockIdx.x - sum_blocks) >> a.bits) * 64;
        const int32_t* starts = a.starts + (size_t)slice * (a.keys + 1);
        const int key = first + (int)(threadIdx.x & 63);
        const int64_t row = ((int64_t)key << a.bits) + slice;
        unsigned long long none = __ballot(key < a.keys && row < a.V && starts[key < a.keys ? key : 0] == starts[key < a.keys ? key + 1 : 0]);
        const int width = a.row_chunks * 2;
        while (none) {
            const int64_t v = ((int64_t)(first + __ffsll(none) - 1) << a.bits) + slice;
            none &= none - 1;
            af32x4* to = (af32x4*)a.dW + (size_t)v * width;
            for (int i = threadIdx.x; i < width; i += 256) to[i] = af32x4{0.f, 0.f, 0.f, 0.f};
        }
        return;
    }
    const int M = a.starts[(size_t)slices * (a.keys + 1) - 1];
    const int64_t item = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPR;
    int64_t piece = item / a.strips;
    int c = (int)(item - piece * a.strips) * LPR + (int)(threadIdx.x % LPR);
    if constexpr (LPR == 64) piece = __builtin_amdgcn_readfirstlane((int)piece);
    const bool live = c < a.row_chunks;
    if (!live) c = 0;                                        // reads along with the first chunk's lane, stores nothing
    const int64_t first = piece * a.piece;
    if (first >= M) return;
    const int64_t last = first + a.piece < M ? first + a.piece : M;
    const int before = first > 0 ? a.sorted[first - 1] : -1;
    bool begun = before == a.sorted[first];                  // the present group began in front of the piece
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    float* partial = a.partial + ((size_t)piece * 2 * a.row_chunks + c) * 8;
    auto store_partial = [&](int which) {
        if (!live) return;
        af32x4* to = (af32x4*)(partial + (size_t)which * a.row_chunks * 8);
        to[0] = af32x4{sum[0], sum[1], sum[2], sum[3]};
        to[1] = af32x4{sum[4], sum[5], sum[6], sum[7]};
    };
    for (int64_t b = first; b < last; b += 8) {
        const int j0 = threadIdx.x & 7;
        const int rows = last - b < 8 ? (int)(last - b) : 8;
        int pos = 0, token = -1, next = -1;
        if (j0 < rows) {
            pos = a.order[b + j0];
            token = a.sorted[b + j0];
            if (b + j0 + 1 < M) next = a.sorted[b + j0 + 1];
        }
        au32x4 x[8];
        af32x4 w[8][2];
        bool inside = begun;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < rows) x[j] = ((const au32x4*)a.d_out)[(size_t)of_lane<LPR>(pos, j) * a.row_chunks + c];
        if (a.accumulate) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int t = of_lane<LPR>(token, j);
                if (j < rows && t != of_lane<LPR>(next, j)) {
                    if (!inside) {
                        const af32x4* from = (const af32x4*)a.dW + ((size_t)t * a.row_chunks + c) * 2;
                        w[j][0] = from[0];
                        w[j][1] = from[1];
                    }
                    inside = false;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (j >= rows) continue;
            float f[8];
            unpack8(x[j], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += f[e];
            const int t = of_lane<LPR>(token, j);
            if (t == of_lane<LPR>(next, j)) continue;
            if (begun) {
                store_partial(0);
            } else if (live) {
                af32x4* to = (af32x4*)a.dW + ((size_t)t * a.row_chunks + c) * 2;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    af32x4 r = {a.scale * sum[4 * h], a.scale * sum[4 * h + 1], a.scale * sum[4 * h + 2], a.scale * sum[4 * h + 3]};
                    to[h] = a.accumulate ? w[j][h] + r : r;
                }
            }
            begun = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = 0.f;
        }
    }
    if (last < M && a.sorted[last - 1] == a.sorted[last]) store_partial(begun ? 0 : 1);
}

// A workgroup per slice and 256 columns: of its slice's keys it takes those whose group crosses a piece's end, and its
// wavefronts share the group's partial rows: the last one of the piece where it begins, the first ones of the others.
__global__ __launch_bounds__(64 * kJoinWaves) void embedding_join_kernel(const EmbedBackward a, int strips) {
    __shared__ af32x4 red[kJoinWaves][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int slice = blockIdx.x / strips;
    const int quads = a.row_chunks * 2, c = ((int)blockIdx.x - slice * strips) * 64 + lane;
    const int32_t* starts = a.starts + (size_t)slice * (a.keys + 1);
    const af32x4* partial = (const af32x4*)a.partial;
    for (int first = 0; first < a.keys; first += 64) {
        const int key = first + lane;
        const int from = key < a.keys ? starts[key] : 0, to = key < a.keys ? starts[key + 1] : 0;
        unsigned long long crossing = __ballot(to > from && from / a.piece != (to - 1) / a.piece);
        while (crossing) {                                   // the same for all wavefronts of the workgroup
            const int k = __ffsll(crossing) - 1;
            crossing &= crossing - 1;
            const int p = __builtin_amdgcn_readlane(from, k) / a.piece, q = (__builtin_amdgcn_readlane(to, k) - 1) / a.piece;
            af32x4 sum = {0.f, 0.f, 0.f, 0.f};
            if (c < quads) {
                for (int i = p + w; i <= q; i += kJoinWaves) sum += partial[((size_t)i * 2 + (i == p ? 1 : 0)) * quads + c];
            }
            red[w][lane] = sum;
            __syncthreads();
            if (w == 0 && c < quads) {
#pragma unroll
                for (int i = 1; i < kJoinWaves; ++i) sum += red[i][lane];
                af32x4* at = (af32x4*)a.dW + (size_t)(((int64_t)(first + k) << a.bits) + slice) * quads + c;
                const af32x4 r = a.scale * sum;
                at[0] = a.accumulate ? at[0] + r : r;
            }
            __syncthreads();
        }
    }
}

// Rows of a piece.
static int embed_piece(int64_t N) {
    const int64_t rows = (N + kMaxPieces - 1) / kMaxPieces;
    return (int)(rows <= kMinPiece ? kMinPiece : (rows + 7) / 8 * 8);
}

// At most this many pieces for N rows or fewer.
static int64_t embed_pieces(int64_t N) {
    const int64_t n = (N + kMinPiece - 1) / kMinPiece;
    return n < kMaxPieces ? n : kMaxPieces;
}

static int embed_shape(int64_t N, int64_t D, int64_t V) {
    if (N <= 0 || D <= 0 || V <= 0) return CCE_ERR_INVALID;
    if (N > 0x7fffffff || D % 8 != 0 || D > kEmbedMaxDim || V > kEmbedMaxRows || V * D > kEmbedMaxValues) return CCE_ERR_UNSUPPORTED;
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
    if (embed_shape(N, D, V) != CCE_OK) return 0;
    const int bits = slice_bits(V);
    const int64_t starts = (((V + (1 << bits) - 1) >> bits) + 1) << bits;
    return (size_t)(round_up(starts * 4, 256) + 2 * round_up(N * 4, 256) + embed_pieces(N) * 2 * D * 4);
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
    hipStream_t stream = (hipStream_t)stream_;
    EmbedBackward a;
    a.tokens = tokens;
    a.d_out = (const uint16_t*)d_out;
    a.dW = dW;
    a.status = status;
    a.N = (int)N; a.V = (int)V; a.ignore_index = ignore_index;
    a.bits = slice_bits(V);
    a.keys = (int)((V + (1 << a.bits) - 1) >> a.bits);
    a.row_chunks = (int)(D / 8);
    a.piece = embed_piece(N);
    a.accumulate = accumulate_dW ? 1 : 0;
    a.scale = scale;
    const int slices = 1 << a.bits;
    char* at = (char*)workspace;
    a.starts = (int32_t*)at; at += round_up((int64_t)(a.keys + 1) * slices * 4, 256);
    a.order = (int32_t*)at; at += round_up(N * 4, 256);
    a.sorted = (int32_t*)at; at += round_up(N * 4, 256);
    a.partial = (float*)at;
    hipLaunchKernelGGL(embedding_order_kernel, dim3((unsigned)slices), dim3(64 * kOrderWaves), 0, stream, a);

    const int lanes = D <= 64 ? 8 : D <= 128 ? 16 : D <= 256 ? 32 : 64;
    a.strips = (a.row_chunks + lanes - 1) / lanes;
    const int64_t pieces = (N + a.piece - 1) / a.piece;
    const int sum_blocks = (int)((pieces * a.strips * lanes + 255) / 256);
    const int zero_blocks = a.accumulate ? 0 : (a.keys + 63) / 64 * slices;
    const dim3 grid((unsigned)(sum_blocks + zero_blocks));
    if (lanes == 8) hipLaunchKernelGGL(embedding_sum_kernel<8>, grid, dim3(256), 0, stream, a, sum_blocks);
    else if (lanes == 16) hipLaunchKernelGGL(embedding_sum_kernel<16>, grid, dim3(256), 0, stream, a, sum_blocks);
    else if (lanes == 32) hipLaunchKernelGGL(embedding_sum_kernel<32>, grid, dim3(256), 0, stream, a, sum_blocks);
    else hipLaunchKernelGGL(embedding_sum_kernel<64>, grid, dim3(256), 0, stream, a, sum_blocks);

    if (pieces > 1) {
        const int strips = (int)((D + 255) / 256);
        hipLaunchKernelGGL(embedding_join_kernel, dim3((unsigned)(slices * strips)), dim3(64 * kJoinWaves), 0, stream, a, strips);
    }
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

}  // extern "C"
