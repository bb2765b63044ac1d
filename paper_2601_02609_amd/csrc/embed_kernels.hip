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
constexpr int64_t kStreamOut = (int64_t)192 << 20;        // bytes of an output that the last-level cache (256 MB) cannot keep
constexpr int64_t kMaxBlocks = (1 << 24) - 1;            // of 256 threads: a launch has fewer than 2^32 threads

// Whether a token names a row; a bad one that is not ignore_index is reported.
__device__ __forceinline__ bool token_takes_part(int token, int V, int ignore_index, int32_t* status) {
    if (token == ignore_index) return false;
    if ((unsigned)token < (unsigned)V) return true;
    if (status) atomicOr(status, CCE_STATUS_BAD_TOKEN);
    return false;
}

// y_i = scale * W[t_i]: two chunks of 16 bytes of y a thread, 4 KB of the workgroup apart, whose tokens, rows and stores are
// in flight together (four: 3.0 -> 3.3 us for one token, 3 % longer for large outputs; one, a division each: 86 us at 32768 x
// 3584 against 69).  A chunk's row within the workgroup's 8 KB by multiplication: `inverse` is ceil(2^32 / row_chunks),
// exact for the numbers below 2^17 that occur.
// STREAM: y of kStreamOut or more is written past the caches, which could not keep it for the kernel that reads it and do keep
// rows of W then: 32768 x 3584 (224 MiB) 69 -> 48 us, with the final norm behind it 175 -> 170; smaller ones, that kernel finds in
// the caches: 32768 x 2048 (128 MiB) with the norm 87 against 92 us.
constexpr int kLookupChunks = 512;

template <bool STREAM>
__global__ __launch_bounds__(256) void embedding_forward_kernel(
        const int32_t* __restrict__ tokens, const uint16_t* __restrict__ weight, int64_t chunks, int row_chunks, uint64_t inverse,
        int V, int ignore_index, float scale, uint16_t* __restrict__ out, int32_t* status) {
    for (int64_t first = (int64_t)blockIdx.x * kLookupChunks; first < chunks; first += (int64_t)gridDim.x * kLookupChunks) {
        const int64_t row0 = first / row_chunks;
        const int c0 = (int)(first - row0 * row_chunks);
        const int live = chunks - first < kLookupChunks ? (int)(chunks - first) : kLookupChunks;
        int token[2], c[2];
        bool ok[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = u * 256 + (int)threadIdx.x;
            const uint32_t o = (uint32_t)(c0 + (i < live ? i : 0));
            const int row = (int)(((uint64_t)o * inverse) >> 32);
            c[u] = (int)o - row * row_chunks;
            token[u] = tokens[row0 + row];
        }
        au32x4 v[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            ok[u] = token_takes_part(token[u], V, ignore_index, c[u] == 0 ? status : nullptr);
            if (ok[u]) v[u] = ((const au32x4*)weight)[(size_t)token[u] * row_chunks + c[u]];
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int i = u * 256 + (int)threadIdx.x;
            float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (ok[u]) unpack8(v[u], f);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] *= scale;
            const au32x4 y = ok[u] ? pack8(f) : au32x4{0u, 0u, 0u, 0u};
            if (i >= live) continue;
            if (STREAM) __builtin_nontemporal_store(y, (au32x4*)out + first + i); else ((au32x4*)out)[first + i] = y;
        }
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
constexpr int kSliceKeys = 640;                 // rows of the matrix that an order workgroup counts: 40 KB of LDS
constexpr int kKeyBits = 10;
static_assert(kSliceKeys <= 1 << kKeyBits, "bits of a key");
constexpr int kOrderWaves = 16;
constexpr int kOrderLoads = 8;                  // loads of tokens in flight, and as many ahead
constexpr int kFound = 1024;                    // positions that a wavefront notes: 32 KB of LDS
constexpr int kSmallTokens = 1024;              // one launch takes: a thread each
constexpr int kSmallRows = 2048, kSmallRowsAdd = 4096;    // and rows of strips, which one workgroup may have all of
constexpr int kSmallShare = 16;                 // rows of a key that one wavefront adds up
constexpr int kJoinShort = 16;                  // pieces of a group that one wavefront joins, and one more
// Wavefronts that the sum is cut into, if there are rows for them.  Added to dW, the pieces take unequal times (rows of dW are read
// where groups end) and more of them even out: 32768 x 3584 124 -> 118 us, 32768 x 1024 of uniform tokens 72 -> 67; overwriting,
// they cost: 16384 x 2048 101 -> 108.
constexpr int64_t kSumWaves = 4096, kSumWavesAdd = 8192;
constexpr int64_t kMaxPieces = 4096;            // more make the join of a frequent token's partial rows long
constexpr int64_t kStreamBytes = (int64_t)128 << 20;      // half of the last-level cache
// A dW of this size or more gets its zeros past the caches in the three launches: 500 MiB with 16384 x 4096 rows 149 -> 133 us;
// smaller ones what reads dW next finds there: the sum of squares of 219 MiB with the gradient in front of it 85 against 102 us.
// The one launch for few tokens writes all zeros through the caches.
constexpr int64_t kStreamZeros = (int64_t)256 << 20;

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
    int N, V, ignore_index, bits, keys, row_chunks, piece, strips, accumulate, stream_zeros;
    float scale;
};

// How many of the lanes in front of this one are in `mask`.
__device__ __forceinline__ uint32_t lanes_in_front(unsigned long long mask) {
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// Of the lanes `among`, those that have this lane's key: they find each other bit by bit.
__device__ __forceinline__ unsigned long long lanes_of_key(unsigned long long among, uint32_t key) {
    unsigned long long same = among;
#pragma unroll
    for (int b = 0; b < kKeyBits; ++b) {
        const uint32_t bit = 0u - (key >> b & 1u);
        const unsigned long long ones = __ballot(bit != 0u);
        same &= ~(ones ^ ((unsigned long long)bit << 32 | bit));
    }
    return same;
}

// A workgroup per slice looks through all tokens (which stay in the L2s): its wavefronts, each with a range of positions,
// count their keys in LDS and note what they found there; after a scan over keys and wavefronts they give the positions
// of one key consecutive places.  64 tokens that none is in the slice of cost a handful of instructions, most of them
// scalar: all slices together do that slices * N / 64 times, which is what bounds the kernel, and above 32768 tokens the slice of
// the most frequent one: 7.7 us for 8192 tokens under Zipf's law, 16 for 32768, 25 for 65536 (16 if all are as frequent).
// That is for 256 slices, up to 163840 rows of the matrix.  A CU's registers (65 a thread here) hold one workgroup, so that 512
// slices take two rounds: the whole call with rows of 256 values added to dW takes 19.2, 33.6 and 50.0 us for 8192, 32768 and
// 65536 tokens of 163840 rows, and 22.5, 40.0 and 60.8 us of 163841 (262144: 23.4, 41.4, 61.5).
__global__ __launch_bounds__(64 * kOrderWaves) void embedding_order_kernel(const EmbedBackward a) {
    __shared__ uint32_t count[kOrderWaves * kSliceKeys];
    __shared__ uint16_t found[kOrderWaves][kFound];          // places in the wavefront's range
    __shared__ uint32_t wave_total[kOrderWaves], wave_below[kOrderWaves];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int slice = blockIdx.x, mask = (1 << a.bits) - 1;
    uint32_t* own = count + w * a.keys;
    const int64_t range = ((int64_t)a.N + 64 * kOrderWaves - 1) / (64 * kOrderWaves) * 64;
    const int64_t begin = w * range, end = begin + range < a.N ? begin + range : a.N;
    const bool report = slice == 0 && a.status != nullptr;
    unsigned long long bad = 0ull;
    auto load = [&](int64_t i, int (&token)[kOrderLoads]) {  // -1 behind the end; every load is made, none waits for another
        const int64_t from = i < a.N ? i : 0;
        const int left = i < end ? (end - i < 64 * kOrderLoads ? (int)(end - i) : 64 * kOrderLoads) : 0;
#pragma unroll
        for (int u = 0; u < kOrderLoads; ++u) token[u] = a.tokens[from + (64 * u + lane < left ? 64 * u + lane : 0)];
#pragma unroll
        for (int u = 0; u < kOrderLoads; ++u) token[u] = 64 * u + lane < left ? token[u] : -1;
    };
    auto valid = [&](int token) { return (unsigned)token < (unsigned)a.V && token != a.ignore_index; };
    uint32_t below = 0u, n = 0u;                             // tokens of slices below and of this one, in scalar registers
    int token[kOrderLoads], next[kOrderLoads];
    load(begin, token);
    for (int i = threadIdx.x; i < kOrderWaves * a.keys; i += 64 * kOrderWaves) count[i] = 0u;
    __syncthreads();
    for (int64_t i = begin; i < end; i += 64 * kOrderLoads) {
        load(i + 64 * kOrderLoads, next);
#pragma unroll
        for (int u = 0; u < kOrderLoads; ++u) {
            const int s = token[u] & mask;
            const unsigned long long ok = __ballot(valid(token[u]));
            if (report) bad |= __ballot(token[u] != a.ignore_index && i + 64 * u + lane < end) & ~ok;
            below += (uint32_t)__popcll(__ballot(s < slice) & ok);
            const unsigned long long mine = __ballot(s == slice) & ok;
            if (mine != 0ull) {
                if (s == slice && valid(token[u])) {
                    const uint32_t place = n + lanes_in_front(mine);
                    atomicAdd(&own[(uint32_t)token[u] >> a.bits], 1u);
                    if (place < (uint32_t)kFound) found[w][place] = (uint16_t)((i - begin) + 64 * u + lane);
                }
                n += (uint32_t)__popcll(mine);
            }
            token[u] = next[u];
        }
    }
    if (bad != 0ull && lane == 0) atomicOr(a.status, CCE_STATUS_BAD_TOKEN);
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
            const uint32_t here = count[i * a.keys + key];
            count[i * a.keys + key] = at;
            at += here;
        }
    __syncthreads();

    // 64 positions, those of `mine` in ascending order with keys of this slice
    auto place_them = [&](unsigned long long mine, uint32_t k, int64_t position) {
        const unsigned long long same = lanes_of_key(mine, k);
        if (mine >> lane & 1ull) {
            const int leader = __ffsll(same) - 1;
            uint32_t to = 0u;
            if (lane == leader) to = atomicAdd(&own[k], (uint32_t)__popcll(same));
            to = (uint32_t)__shfl((int)to, leader) + lanes_in_front(same);
            a.order[to] = (int32_t)position;
            a.sorted[to] = (int32_t)(k << a.bits) + slice;
        }
    };
    auto place_found = [&](uint32_t many, int64_t from) {    // what found[w] holds, as places behind `from`
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        for (uint32_t i = 0; i < many; i += 256) {
            int64_t position[4];
            int t[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t j = i + 64 * u + lane;
                position[u] = from + (j < many ? found[w][j] : 0);
                t[u] = a.tokens[position[u]];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + 64 * u < many) place_them(__ballot(i + 64 * u + lane < many), (uint32_t)t[u] >> a.bits, position[u]);
        }
    };
    if (n <= (uint32_t)kFound && range <= 65536) {
        place_found(n, begin);
        return;
    }
    // more than was noted: through the range again, noting as many as fit
    uint32_t many = 0u;
    int64_t from = begin;                                    // what the noted places are counted from
    load(begin, token);
    for (int64_t i = begin; i < end; i += 64 * kOrderLoads) {
        load(i + 64 * kOrderLoads, next);
#pragma unroll
        for (int u = 0; u < kOrderLoads; ++u) {
            const bool is_mine = valid(token[u]) && (token[u] & mask) == slice;
            const unsigned long long mine = __ballot(is_mine);
            if (mine != 0ull) {
                if (is_mine) found[w][many + lanes_in_front(mine)] = (uint16_t)((i - from) + 64 * u + lane);
                many += (uint32_t)__popcll(mine);
                if (many > (uint32_t)kFound - 64u) {
                    place_found(many, from);
                    many = 0u;
                }
            }
            token[u] = next[u];
        }
        if (i + 2 * 64 * kOrderLoads - from > 65536) {       // the next ones' places would pass 16 bits
            place_found(many, from);
            many = 0u;
            from = i + 64 * kOrderLoads;
        }
    }
    place_found(many, from);
}

// A value of lane j of each group of eight lanes.  Wavefronts that work on one row have it in a scalar register.
template <int LPR>
__device__ __forceinline__ int of_lane(int x, int j) {
    if constexpr (LPR == 64) return __builtin_amdgcn_readlane(x, j);
    else return __shfl(x, j, 8);
}

// LPR lanes share a row (a strip of 512 columns of it if D > 512), 16 bytes each, and take one piece.  Eight rows, and
// the rows of dW that they end at, are in flight.
// STREAM: d_out of kStreamBytes or more, read past the caches, which keep more of dW then: 140 -> 123 us for 32768 x 3584 added to
// dW, 93 -> 85 for 32768 x 2048 (128 MiB); below, rows that the launch before left there are worth more (16384 x 2048 45 -> 50).
// Only where a wavefront has a row: narrower ones lose 1 to 4 % (262144 x 256 179 -> 185, 524288 x 128 318 -> 323, 1048576 x 64
// 621 -> 630, into a new dW 603 -> 617).
// 137 registers (147 with fewer lanes a row), three wavefronts a SIMD: what is in flight fills them.
template <int LPR, bool STREAM>
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
            if (a.stream_zeros) {
                for (int i = threadIdx.x; i < width; i += 256) __builtin_nontemporal_store(af32x4{0.f, 0.f, 0.f, 0.f}, to + i);
            } else {
                for (int i = threadIdx.x; i < width; i += 256) to[i] = af32x4{0.f, 0.f, 0.f, 0.f};
            }
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
    if (first >= a.N) return;
    // positions and tokens of eight rows, and the token behind each; entries from M on say nothing, but may be loaded with it
    const int j0 = threadIdx.x & 7;
    int pos = 0, token = -1, next = -1;
    auto load_rows = [&](int64_t b) {
        if (b + j0 < a.N) {
            pos = a.order[b + j0];
            token = a.sorted[b + j0];
        }
        if (b + j0 + 1 < a.N) next = a.sorted[b + j0 + 1];
    };
    load_rows(first);
    const int before = first > 0 ? a.sorted[first - 1] : -1, at_first = a.sorted[first];
    if (first >= M) return;
    const int64_t last = first + a.piece < M ? first + a.piece : M;
    bool begun = before == at_first;                         // the present group began in front of the piece
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    float* partial = a.partial + ((size_t)piece * 2 * a.row_chunks + c) * 8;
    auto store_partial = [&](int which) {
        if (!live) return;
        af32x4* to = (af32x4*)(partial + (size_t)which * a.row_chunks * 8);
        to[0] = af32x4{sum[0], sum[1], sum[2], sum[3]};
        to[1] = af32x4{sum[4], sum[5], sum[6], sum[7]};
    };
    for (int64_t b = first; b < last; b += 8) {
        const int rows = last - b < 8 ? (int)(last - b) : 8;
        const int row = pos, of = token, behind = b + j0 + 1 < M ? next : -1;
        if (b + 8 < last) load_rows(b + 8);
        au32x4 x[8];
        af32x4 w[8][2];
        bool inside = begun;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < rows) {
                const au32x4* from = (const au32x4*)a.d_out + (size_t)of_lane<LPR>(row, j) * a.row_chunks + c;
                x[j] = STREAM ? __builtin_nontemporal_load(from) : *from;
            }
        if (a.accumulate) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int t = of_lane<LPR>(of, j);
                if (j < rows && t != of_lane<LPR>(behind, j)) {
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
            const int t = of_lane<LPR>(of, j);
            if (t == of_lane<LPR>(behind, j)) continue;
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
// WAVES of a workgroup: four where more workgroups are than fit the card at a time (32768 x 3584 117.9 -> 115.1 us in all, 2048 x
// 4096 24.8 -> 22.9), sixteen for one strip, where a frequent token's partial rows are the time (65536 x 64 45.2 -> 42.8),
// eight between (8192 x 896 with four 22.1 -> 23.8).
template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void embedding_join_kernel(const EmbedBackward a, int strips) {
    __shared__ af32x4 red[WAVES][64];
    __shared__ int crossing[kSliceKeys][3];                  // key, first and last piece
    __shared__ int groups;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int slice = blockIdx.x / strips;
    const int quads = a.row_chunks * 2, c = ((int)blockIdx.x - slice * strips) * 64 + lane;
    const int32_t* starts = a.starts + (size_t)slice * (a.keys + 1);
    const af32x4* partial = (const af32x4*)a.partial;
    if (threadIdx.x == 0) groups = 0;
    __syncthreads();
    for (int key = threadIdx.x; key < a.keys; key += 64 * WAVES) {
        const int from = starts[key], to = starts[key + 1];
        const int p = from / a.piece, q = (to - 1) / a.piece;
        if (to > from && p != q) {                           // in whatever order: no sum is over two groups
            const int g = atomicAdd(&groups, 1);
            crossing[g][0] = key;
            crossing[g][1] = p;
            crossing[g][2] = q;
        }
    }
    __syncthreads();
    // short groups: a wavefront each; long ones: the wavefronts share the partial rows
    const int n = groups;
    auto rows_of = [&](int p, int q, int step, int from) {
        af32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int first = p + from; first <= q; first += 8 * step) {
            af32x4 x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = first + u * step;
                x[u] = af32x4{0.f, 0.f, 0.f, 0.f};
                if (i <= q) x[u] = partial[((size_t)i * 2 + (i == p ? 1 : 0)) * quads + c];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) sum += x[u];
        }
        return sum;
    };
    auto row_at = [&](int key) { return (af32x4*)a.dW + (size_t)(((int64_t)key << a.bits) + slice) * quads + c; };
    for (int g = w; g < n; g += WAVES) {
        const int p = crossing[g][1], q = crossing[g][2];
        if (q - p >= kJoinShort || c >= quads) continue;
        af32x4* at = row_at(crossing[g][0]);
        af32x4 old = {0.f, 0.f, 0.f, 0.f};
        if (a.accumulate) old = at[0];
        at[0] = old + a.scale * rows_of(p, q, 1, 0);
    }
    for (int g = 0; g < n; ++g) {
        const int p = crossing[g][1], q = crossing[g][2];
        if (q - p < kJoinShort) continue;                    // the same for all
        af32x4* at = row_at(crossing[g][0]);
        af32x4 sum = {0.f, 0.f, 0.f, 0.f}, old = sum;
        if (c < quads) {
            if (w == 0 && a.accumulate) old = at[0];
            sum = rows_of(p, q, WAVES, w);
        }
        red[w][lane] = sum;
        __syncthreads();
        if (w == 0 && c < quads) {
#pragma unroll
            for (int i = 1; i < WAVES; ++i) sum += red[i][lane];
            at[0] = old + a.scale * sum;
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------
// Few tokens: one launch.  A workgroup per slice finds its positions among all N <= kSmallTokens in order, then a wavefront
// sums a key's rows (a strip of 512 columns of them) by itself, or all of them share the rows of a key that has many.
// Bound by latency, launches above all.  Against the three launches: 257 x 64 into a new dW 13.1 -> 4.9 us; added to dW, 512 x 896
// 15.9 -> 6.1, 1024 x 896 16.9 -> 7.5, 1024 x 2048 17.6 -> 10.5, 512 x 3584 19.1 -> 9.8.  kSmallRowsAdd bounds what one workgroup
// may have to sum if all tokens are the same, which no rule on sizes can see and where the one launch loses: added to dW, 1024 x 896
// 15.0 -> 25.2 us then, 1024 x 2048 15.2 -> 46.2, 512 x 3584 13.7 -> 40.2.
// Into a new dW the launches saved count for as much with large matrices, whose zeros are the time: 512 x 2048 into 151936 rows
// 238 -> 218 us, 1 x 896 into as many 108 -> 93, 256 x 4096 into 32000 105 -> 89, 1024 x 1024 into 32000 31 -> 21.  kSmallRows is where
// a frequent token's workgroup begins to outlast the others' zeros: 1024 x 2048 into 32000 rows would take 53.2 us against 45.8
// under Zipf's law (uniform tokens 38.3 against 44.5); if all tokens are the same, 1024 x 896 takes 37.8 against 27.0.
// ------------------------------------------------------------------------------------------
__global__ __launch_bounds__(64 * kOrderWaves) void embedding_small_kernel(const EmbedBackward a) {
    __shared__ uint32_t mine[kSmallTokens];                  // this slice's positions, ascending, and their keys in the upper 16 bits
    __shared__ uint16_t rows[kSmallTokens];                  // the positions, those of a key together
    __shared__ uint32_t first[kSliceKeys], many[kSliceKeys]; // of each key: its first place in `mine`, how many it has
    __shared__ uint32_t begin[kSliceKeys];                   // where its rows begin, then where the next one goes
    __shared__ uint32_t keys_here[kSmallTokens];
    __shared__ uint32_t wave_count[kOrderWaves], keys_found, rows_given;
    __shared__ float red[kOrderWaves][512];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int slice = blockIdx.x, mask = (1 << a.bits) - 1;
    const int token = (int)threadIdx.x < a.N ? a.tokens[threadIdx.x] : a.ignore_index;
    const bool ok = token_takes_part(token, a.V, a.ignore_index, slice == 0 ? a.status : nullptr);
    const unsigned long long hits = __ballot(ok && (token & mask) == slice);
    if (lane == 0) wave_count[w] = (uint32_t)__popcll(hits);
    if ((int)threadIdx.x < a.keys) { first[threadIdx.x] = 0xffffffffu; many[threadIdx.x] = 0u; }
    if (threadIdx.x == 0) keys_found = rows_given = 0u;
    __syncthreads();
    uint32_t at = 0u, n = 0u;
#pragma unroll
    for (int i = 0; i < kOrderWaves; ++i) {
        at += i < w ? wave_count[i] : 0u;
        n += wave_count[i];
    }
    if (hits >> lane & 1ull) {
        const uint32_t key = (uint32_t)token >> a.bits;
        at += lanes_in_front(hits);
        mine[at] = key << 16 | threadIdx.x;
        atomicMin(&first[key], at);
        atomicAdd(&many[key], 1u);
    }
    __syncthreads();
    const uint32_t own = threadIdx.x < n ? mine[threadIdx.x] : 0u, key = own >> 16;
    if (threadIdx.x < n && first[key] == threadIdx.x) {      // keys in whatever order: no sum is over two of them
        keys_here[atomicAdd(&keys_found, 1u)] = key;
        begin[key] = atomicAdd(&rows_given, many[key]);
    }
    __syncthreads();
    const unsigned long long live = __ballot(threadIdx.x < n);
    const unsigned long long same = lanes_of_key(live, key);
    const int leader = live >> lane & 1ull ? __ffsll(same) - 1 : lane;
    for (uint32_t turn = 0; turn * 64u < n; ++turn) {        // one wavefront after the other, so that positions stay in order
        if (w == (int)turn) {
            uint32_t to = 0u;
            if (lane == leader && threadIdx.x < n) to = atomicAdd(&begin[key], (uint32_t)__popcll(same));
            to = (uint32_t)__shfl((int)to, leader) + lanes_in_front(same);
            if (threadIdx.x < n) rows[to] = (uint16_t)own;
        }
        __syncthreads();
    }
    const int found = (int)keys_found;                       // and begin is where a key's rows end now

    // the rows `from` up to `to` of this slice's, one chunk a lane, eight rows in flight
    auto sum_rows = [&](uint32_t from, uint32_t to, int c, float (&sum)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = 0.f;
        for (uint32_t i = from; i < to; i += 8) {
            au32x4 x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const size_t row = rows[i + j < to ? i + j : i];
                x[j] = ((const au32x4*)a.d_out)[row * a.row_chunks + c];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (i + j >= to) continue;
                float f[8];
                unpack8(x[j], f);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += f[e];
            }
        }
    };
    auto row_at = [&](uint32_t k, int c) { return (af32x4*)a.dW + ((((size_t)k << a.bits) + slice) * a.row_chunks + c) * 2; };
    auto add_to_row = [&](af32x4* to, const af32x4 (&old)[2], const float (&sum)[8]) {
        to[0] = old[0] + af32x4{a.scale * sum[0], a.scale * sum[1], a.scale * sum[2], a.scale * sum[3]};
        to[1] = old[1] + af32x4{a.scale * sum[4], a.scale * sum[5], a.scale * sum[6], a.scale * sum[7]};
    };
    for (int item = w; item < found * a.strips; item += kOrderWaves) {
        const uint32_t k = keys_here[item / a.strips], to = begin[k], from = to - many[k];
        const int c = item % a.strips * 64 + lane;
        if (to - from > (uint32_t)kSmallShare || c >= a.row_chunks) continue;
        af32x4* at_row = row_at(k, c);
        af32x4 old[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        if (a.accumulate) { old[0] = at_row[0]; old[1] = at_row[1]; }
        float sum[8];
        sum_rows(from, to, c, sum);
        add_to_row(at_row, old, sum);
    }
    // a key with many rows: the wavefronts take `side` strips side by side and `parts` parts of the rows
    int side = 1;
    while (side < a.strips && side < kOrderWaves) side <<= 1;
    const int parts = kOrderWaves / side;
    for (int g = 0; g < found; ++g) {
        const uint32_t k = keys_here[g], to = begin[k], from = to - many[k];
        if (to - from <= (uint32_t)kSmallShare) continue;    // the same for all
        const uint32_t part = (to - from + parts - 1) / parts;
        for (int strip = 0; strip < a.strips; strip += side) {
            const int c = (strip + w % side) * 64 + lane;
            const uint32_t low = from + (w / side) * part, high = low + part < to ? low + part : to;
            float sum[8];
            sum_rows(low, c < a.row_chunks ? high : low, c, sum);
#pragma unroll
            for (int e = 0; e < 8; ++e) red[w][lane * 8 + e] = sum[e];
            __syncthreads();
            if (w < side && c < a.row_chunks) {
                af32x4* at_row = row_at(k, c);
                af32x4 old[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
                if (a.accumulate) { old[0] = at_row[0]; old[1] = at_row[1]; }
                for (int i = 1; i < parts; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += red[i * side + w][lane * 8 + e];
                add_to_row(at_row, old, sum);
            }
            __syncthreads();
        }
    }
    if (a.accumulate) return;
    const int width = a.row_chunks * 2;
    for (int k = w; k < a.keys; k += kOrderWaves) {
        const int64_t v = ((int64_t)k << a.bits) + slice;
        if (many[k] != 0u || v >= a.V) continue;
        af32x4* to = (af32x4*)a.dW + (size_t)v * width;
        for (int i = lane; i < width; i += 64) to[i] = af32x4{0.f, 0.f, 0.f, 0.f};
    }
}

// Lanes that share a row, and the rest of a row's chunks in further strips.
static int embed_lanes(int64_t D) { return D <= 64 ? 8 : D <= 128 ? 16 : D <= 256 ? 32 : 64; }

// Rows of a piece, a multiple of eight (what a wavefront has in flight): as many as leave `waves` wavefronts and kMaxPieces pieces.
static int64_t embed_piece(int64_t N, int64_t D, int64_t waves) {
    const int64_t lanes = embed_lanes(D), strips = (D / 8 + lanes - 1) / lanes;
    const int64_t by_waves = (N * strips * lanes / 64 + waves - 1) / waves, by_pieces = (N + kMaxPieces - 1) / kMaxPieces;
    const int64_t rows = by_waves > by_pieces ? by_waves : by_pieces;
    return rows <= 8 ? 8 : (rows + 7) / 8 * 8;
}

// No N' <= N rows have more pieces.
static int64_t embed_pieces(int64_t N, int64_t D) {
    const int64_t lanes = embed_lanes(D), strips = (D / 8 + lanes - 1) / lanes, short_ones = (N + 7) / 8;
    const int64_t by_waves = kSumWavesAdd * 64 / (strips * lanes) + 1, most = by_waves < kMaxPieces ? by_waves : kMaxPieces;
    return short_ones < most ? short_ones : most;
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
    const int64_t row_chunks = D / 8, chunks = N * row_chunks, want = (chunks + kLookupChunks - 1) / kLookupChunks;
    (void)hipGetLastError();
    const dim3 grid((unsigned)(want < kMaxBlocks ? want : kMaxBlocks));
    const uint64_t inverse = (((uint64_t)1 << 32) + row_chunks - 1) / row_chunks;
    hipStream_t stream = (hipStream_t)stream_;
#define CCE_EMBED_LOOKUP(STREAM) hipLaunchKernelGGL(embedding_forward_kernel<STREAM>, grid, dim3(256), 0, stream, tokens, \
        (const uint16_t*)weight, chunks, (int)row_chunks, inverse, (int)V, ignore_index, scale, (uint16_t*)out, status)
    if (N * D * 2 >= kStreamOut) CCE_EMBED_LOOKUP(true); else CCE_EMBED_LOOKUP(false);
#undef CCE_EMBED_LOOKUP
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

size_t cce_embedding_workspace_bytes(int64_t N, int64_t D, int64_t V) {
    if (embed_shape(N, D, V) != CCE_OK) return 0;
    const int bits = slice_bits(V);
    const int64_t starts = (((V + (1 << bits) - 1) >> bits) + 1) << bits;
    return (size_t)(round_up(starts * 4, 256) + 2 * round_up(N * 4, 256) + embed_pieces(N, D) * 2 * D * 4);
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
    a.accumulate = accumulate_dW ? 1 : 0;
    a.piece = (int)embed_piece(N, D, a.accumulate ? kSumWavesAdd : kSumWaves);
    a.stream_zeros = V * D * 4 >= kStreamZeros ? 1 : 0;
    a.scale = scale;
    const int slices = 1 << a.bits;
    char* at = (char*)workspace;
    a.starts = (int32_t*)at; at += round_up((int64_t)(a.keys + 1) * slices * 4, 256);
    a.order = (int32_t*)at; at += round_up(N * 4, 256);
    a.sorted = (int32_t*)at; at += round_up(N * 4, 256);
    a.partial = (float*)at;
    const int64_t pieces = (N + a.piece - 1) / a.piece;
    if ((size_t)(at - (char*)workspace) + (size_t)pieces * 2 * D * 4 > workspace_bytes) return CCE_ERR_INVALID;
    if (N <= kSmallTokens && N * ((a.row_chunks + 63) / 64) <= (a.accumulate ? kSmallRowsAdd : kSmallRows)) {
        a.strips = (a.row_chunks + 63) / 64;
        hipLaunchKernelGGL(embedding_small_kernel, dim3((unsigned)slices), dim3(64 * kOrderWaves), 0, stream, a);
        return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
    }
    hipLaunchKernelGGL(embedding_order_kernel, dim3((unsigned)slices), dim3(64 * kOrderWaves), 0, stream, a);

    const int lanes = embed_lanes(D);
    a.strips = (a.row_chunks + lanes - 1) / lanes;
    const int sum_blocks = (int)((pieces * a.strips * lanes + 255) / 256);
    const int zero_blocks = a.accumulate ? 0 : (a.keys + 63) / 64 * slices;
    const dim3 grid((unsigned)(sum_blocks + zero_blocks));
    const bool stream_rows = N * D * 2 >= kStreamBytes;
#define CCE_EMBED_SUM(LPR, STREAM) hipLaunchKernelGGL((embedding_sum_kernel<LPR, STREAM>), grid, dim3(256), 0, stream, a, sum_blocks)
    if (lanes == 8) CCE_EMBED_SUM(8, false); else if (lanes == 16) CCE_EMBED_SUM(16, false); else if (lanes == 32) CCE_EMBED_SUM(32, false);
    else if (stream_rows) CCE_EMBED_SUM(64, true); else CCE_EMBED_SUM(64, false);
#undef CCE_EMBED_SUM

    if (pieces > 1) {
        const int strips = (int)((D + 255) / 256), groups = slices * strips;
#define CCE_EMBED_JOIN(WAVES) hipLaunchKernelGGL(embedding_join_kernel<WAVES>, dim3((unsigned)groups), dim3(64 * WAVES), 0, stream, a, strips)
        if (groups > 2048) CCE_EMBED_JOIN(4); else if (strips > 1) CCE_EMBED_JOIN(8); else CCE_EMBED_JOIN(16);
#undef CCE_EMBED_JOIN
    }
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

}  // extern "C"
