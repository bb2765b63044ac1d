// libcce, optimizer kernels for matrices: momentum, Newton-Schulz products, update.  C ABI declared in include/cce_muon.h.
//
// A matrix is worked on as X of r x c, r <= c (transposed on the way in and out where it is taller than wide).  Small ones are
// taken by a workgroup each in one launch, thin ones in three (see both below), all others in the workspace, rows and columns padded with zeros
// to multiples of 64.  Per step three launches over all matrices of a group (the first two steps of matrices much wider than high are taken as one,
// see pairs_steps):
//
//   gram    A = X X^T             half of the tiles, the other half mirrored
//   poly    M = b A + c A A       the same
//   apply   X = (a + M) X
//
// Rounding.  Products take fp16 operands (11 bits) and add in fp32.  Rounding all of X, A and M to them would leave an error of
// 2 % (6e-3 of matrices with a few large directions), because the diagonals of A and M are much larger than what lies beside them, and the
// linear part a X carries small directions next to large ones.  So the diagonals of A and M are kept in fp32 and taken out of the
// 16-bit operands (M's in the later steps alone, see apart_steps), and the linear part is taken from X as h + l, a 16-bit and an 8-bit value.
// Largest error (2-norm, of the result's) over matrices of rank 1 to 64, with noise and without, of noise, and with singular values down to 1e-4:
// 1.4e-3 (512 x 1280 of rank 1; others 0.7 to 1.2), of noise 0.6 to 1.2e-3; bf16's rounding of a result adds 1.7e-3.  Of ones, or blocks
// of ones, where all values round alike: up to 8e-3.  Of few directions on a few large rows and columns, where few roundings count: 1.3e-3 in the
// middle, 3.6e-3 at most (4.8e-3 of 33 to 64 rows); with two steps as one, whose M is four times as large and multiplies h's rounding, 2.1e-3 and 6.2e-3.
//
// Scales, powers of two: X 2^13, A 2^13, M 2^10; l see split1.  Singular values stay below 2.5 (checked for the coefficients),
// values of X too; A's are below 6.25 and M's below 60: within fp16's 65504.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>
#include <type_traits>

#include "../../include/cce.h"
#include "../../include/cce_muon.h"
#include "gemm_core.h"
#include "host_util.h"
#include "vec_util.h"
#include "wg_map.h"

namespace cce {

typedef __attribute__((ext_vector_type(4))) _Float16 f16x4;

constexpr int kGroup = 240;                            // matrices whose products share their launches
constexpr int64_t kGroupBytes = (int64_t)3 << 30;      // workspace of a group of more than one matrix
constexpr int64_t kPartialBytes = (int64_t)256 * 256 * 256 * 4;      // of a part of a tile's sum for each CU
constexpr int64_t kLargeRows = 1024, kLongColumns = 2048;      // from so many (padded) rows or columns on a group may have them
constexpr uint32_t kMaxSplits = 8;                     // parts of a sum: 16 cost the join more than they save (14336 x 100 347 us / 357, 4 x 4096 x 256 331 / 383)
constexpr int kPairRows = 512;                         // from so many (padded) rows on two steps may be taken as one
constexpr int kEnds = 56;                              // matrices of a launch that reads or writes the caller's: kernel arguments hold 4 KB
constexpr int64_t kMaxMatrix = (int64_t)1 << 30;       // values of a padded matrix: byte offsets of 16-bit values stay below 2^32
constexpr int64_t kMaxSide = 16384;                    // smaller side
constexpr int kNormParts = 256;                        // partial sums of a matrix
constexpr int kNormValues = 8192;                      // values of a part, more where that gives too many parts
constexpr float kScaleX = 0x1p13f, kScaleA = 0x1p13f, kScaleM = 0x1p10f;
constexpr double kMaxSigma = 2.5, kMaxM = 60.0;

struct NsMatrix {
    const void* grad;
    float* momentum;
    float* param;              // null: only out is written
    uint16_t* out;
    uint64_t base;             // byte offset in the workspace
    int32_t rows, cols;        // of the caller's matrix
    float lr, decay;           // decay: 1 - lr * weight_decay
};

struct NsArgs {
    NsMatrix t[kEnds];
    uint32_t first[kEnds];     // twice a matrix's first workgroup, plus 1 if its gradient is bf16
    char* ws;
    const float* clip_coef;
    float mu, a, b, c, eps;
    int32_t nesterov;
    uint32_t count, flip;      // flip: which of the two copies of h is read
};

struct NsShape {
    uint32_t base;             // in units of 256 bytes
    int32_t rows, cols;
};

struct NsProductArgs {
    NsShape t[kGroup];
    uint32_t first[kGroup];    // twice a matrix's first workgroup
    char* ws;
    float a, b, c;
    uint32_t count, flip;
    uint32_t tiles, split_tiles, splits;      // tiles of 256 x 256: how many, the last of them in parts of their sums, parts each
    uint32_t partials;         // the parts' place, in units of 256 bytes
    uint32_t kind;             // of a symmetric product
    uint32_t apart;            // whether M acts on h alone (apart_steps)
    float on_x;                // what of its diagonal does not
};
static_assert(sizeof(NsArgs) <= 4096 && sizeof(NsProductArgs) <= 4096, "kernel arguments hold 4 KB");

__device__ __forceinline__ char* workspace_of(const NsArgs& a, int i) { return a.ws + a.t[i].base; }
__device__ __forceinline__ char* workspace_of(const NsProductArgs& a, int i) { return a.ws + (uint64_t)a.t[i].base * 256; }

// Where a matrix's operands lie, in bytes behind its base.
struct NsLayout {
    int r, c, rp, cp;                 // sides and padded sides
    uint64_t h1, l, a, m, da, dm, partials, bytes;      // the first copy of h: 0
    uint64_t s, t, ds, dt;            // of two steps taken as one, in the copy of h that is not read then
    __host__ __device__ __forceinline__ NsLayout(int rows, int cols) {
        r = rows < cols ? rows : cols;
        c = rows < cols ? cols : rows;
        rp = (r + 63) & ~63;
        cp = (c + 63) & ~63;
        const uint64_t x = (uint64_t)rp * cp * 2, square = (uint64_t)rp * rp * 2, p = (uint64_t)rp * panel_rows() * 2, d = (uint64_t)rp * 4;
        h1 = x;
        s = h1;
        t = s + square;
        ds = t + square;
        dt = ds + d;
        l = 2 * x;
        a = l + x / 2;
        m = a + square;
        da = m + p;
        dm = da + d;
        partials = dm + d;
        bytes = partials + kNormParts * 8;
    }
    __device__ __forceinline__ uint64_t h(uint32_t flip) const { return flip ? h1 : 0; }
    // M lies in panels of 32 columns, whose rows are padded to whole tiles
    __host__ __device__ __forceinline__ int panel_rows() const { return (r + 255) & ~255; }
    __device__ __forceinline__ uint32_t panel(int row, int col) const {
        return (uint32_t)(col >> 5) * (uint32_t)panel_rows() * 32u + (uint32_t)row * 32u + (uint32_t)(col & 31);
    }
};

// Which matrix workgroup w belongs to, b = 2 w + 1: the last one that begins at or before it.
__device__ __forceinline__ int matrix_of(const uint32_t* first, int count, uint32_t b) {
    int n = 0;
    for (int base = 0; base < count; base += 64) {
        const int i = base + (int)(threadIdx.x & 63);
        n += (int)__popcll(__ballot(i < count && first[i] <= b));
    }
    return __builtin_amdgcn_readfirstlane(n - 1);
}

__device__ __forceinline__ float grad_value(const void* grad, bool bf16, int64_t i) {
    return bf16 ? __uint_as_float((uint32_t)((const uint16_t*)grad)[i] << 16) : ((const float*)grad)[i];
}
__device__ __forceinline__ af32x4 grad_values(const void* grad, bool bf16, int64_t i) {
    if (!bf16) return *(const af32x4*)((const float*)grad + i);
    const u32x2 p = *(const u32x2*)((const uint16_t*)grad + i);
    return af32x4{__uint_as_float(p[0] << 16), __uint_as_float(p[0] & 0xffff0000u), __uint_as_float(p[1] << 16), __uint_as_float(p[1] & 0xffff0000u)};
}
__device__ __forceinline__ bool aligned(const void* p, unsigned to) { return ((uintptr_t)p & (to - 1)) == 0; }

// A pointer that is the same in every lane, in scalar registers: base of the loads into LDS.
template <class T>
__device__ __forceinline__ T* uniform(T* p) {
    const uint64_t x = (uint64_t)(uintptr_t)p;
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x), hi = (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32));
    return (T*)(uintptr_t)((uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ float new_momentum(float m, float g, float mu) { return mu * m + (1.f - mu) * g; }
__device__ __forceinline__ float direction(float m, float g, float mu, int nesterov) { return nesterov ? mu * m + (1.f - mu) * g : m; }

// Sum of a double over a workgroup of four wavefronts, for all of its threads.
__device__ __forceinline__ double group_sum(double x, double* red) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ int norm_parts(int64_t n) {
    const int64_t parts = (n + kNormValues - 1) / kNormValues;
    return parts < kNormParts ? (int)parts : kNormParts;
}

// ------------------------------------------------------------------------------------------
// Momentum, and partial sums of squares of what is orthogonalised, in fp64: 1e-20 and 1e20 have squares in no fp32.
// ------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void ns_norm_kernel(const NsArgs a) {
    __shared__ double red[4];
    const int i = matrix_of(a.first, (int)a.count, 2 * blockIdx.x + 1);
    const NsMatrix& t = a.t[i];
    const bool bf16 = (a.first[i] & 1u) != 0u;
    const int64_t n = (int64_t)t.rows * t.cols;
    const int part = (int)(blockIdx.x - (a.first[i] >> 1)), parts = norm_parts(n);
    const float clip = a.clip_coef ? a.clip_coef[0] : 1.f;
    const bool vec = aligned(t.grad, bf16 ? 8 : 16) && aligned(t.momentum, 16);
    double sum = 0.0;
    for (int64_t at = ((int64_t)part * 256 + threadIdx.x) * 4; at < n; at += (int64_t)parts * 1024) {
        const int left = n - at < 4 ? (int)(n - at) : 4;
        af32x4 u = {0.f, 0.f, 0.f, 0.f};
        if (vec && left == 4) {
            u = grad_values(t.grad, bf16, at);
            if (t.momentum) {
                af32x4 m = *(const af32x4*)(t.momentum + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float g = u[e] * clip;
                    m[e] = new_momentum(m[e], g, a.mu);
                    u[e] = direction(m[e], g, a.mu, a.nesterov);
                }
                *(af32x4*)(t.momentum + at) = m;
            }
        } else {
            for (int e = 0; e < left; ++e) {
                float g = grad_value(t.grad, bf16, at + e);
                if (t.momentum) {
                    g *= clip;
                    const float m = new_momentum(t.momentum[at + e], g, a.mu);
                    t.momentum[at + e] = m;
                    g = direction(m, g, a.mu, a.nesterov);
                }
                u[e] = g;
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) sum = fma((double)u[e], (double)u[e], sum);
    }
    sum = group_sum(sum, red);
    if (threadIdx.x == 0) ((double*)(a.ws + t.base + NsLayout(t.rows, t.cols).partials))[part] = sum;
}

// x as h + l: h has x's first 11 bits, l the next eight, as a whole number of 2^-8 of h's last place, 128 more so that it is positive.  (Four bits
// in E4M3 left 4e-3 of the results of matrices of rank 1, X's first rounding amplified by the steps; these leave 0.7 to 1.4e-3, and cost a
// tiled call next to nothing.)
__device__ __forceinline__ uint32_t exponent_bits(_Float16 h) {          // 2^e for h of [2^e, 2^(e + 1)); 2^-14 for less, as h's last place is
    const uint32_t u = __float_as_uint((float)h) & 0x7f800000u;
    return u > 0x38800000u ? u : 0x38800000u;
}
__device__ __forceinline__ float split1(float x, _Float16& h) {
    const float s = x * kScaleX;
    h = (_Float16)s;
    return fmaf(s - (float)h, __uint_as_float(0x88000000u - exponent_bits(h)), 128.f);      // 2^18 / 2^e
}
// What l stands for, 2^18 kScaleX times of it.
__device__ __forceinline__ float rest_of(_Float16 h, uint32_t l) { return ((float)(l & 0xffu) - 128.f) * __uint_as_float(exponent_bits(h)); }
// Rounded to the nearest whole number from 0 to 255.
__device__ __forceinline__ uint32_t pack_u8(float a, float b, float c, float d) {
    return __builtin_amdgcn_cvt_pk_u8_f32(d, 3, __builtin_amdgcn_cvt_pk_u8_f32(c, 2, __builtin_amdgcn_cvt_pk_u8_f32(b, 1, __builtin_amdgcn_cvt_pk_u8_f32(a, 0, 0u))));
}
__device__ __forceinline__ void split8(const float (&x)[8], f16x8& h, u32x2& l) {
    float r[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        _Float16 v;
        r[e] = split1(x[e], v);
        h[e] = v;
    }
    l = u32x2{pack_u8(r[0], r[1], r[2], r[3]), pack_u8(r[4], r[5], r[6], r[7])};
}
__device__ __forceinline__ void split4(const af32x4& x, f16x4& h, uint32_t& l) {
    float r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        _Float16 v;
        r[e] = split1(x[e], v);
        h[e] = v;
    }
    l = pack_u8(r[0], r[1], r[2], r[3]);
}

// ------------------------------------------------------------------------------------------
// X = G / (|G| + eps), 64 x 64 values a workgroup, transposed through LDS where G is taller than wide.
// ------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void ns_prep_kernel(const NsArgs a) {
    __shared__ double red[4];
    __shared__ float tile[64][65];
    const int i = matrix_of(a.first, (int)a.count, 2 * blockIdx.x + 1);
    const NsMatrix& t = a.t[i];
    const bool bf16 = (a.first[i] & 1u) != 0u;
    const NsLayout at(t.rows, t.cols);
    char* const base = a.ws + t.base;
    const int64_t n = (int64_t)t.rows * t.cols;
    const int w = (int)(blockIdx.x - (a.first[i] >> 1)), tiles = at.cp / 64;
    const int row0 = w / tiles * 64, col0 = w % tiles * 64;
    const double sum = group_sum((int)threadIdx.x < norm_parts(n) ? ((const double*)(base + at.partials))[threadIdx.x] : 0.0, red);
    const double inv = sum <= 0x1.fffffffffffffp1023 ? 1.0 / (sqrt(sum) + (double)a.eps) : (double)NAN;
    const float clip = a.clip_coef ? a.clip_coef[0] : 1.f;
    const bool tall = t.rows > t.cols;
    const bool vec = (t.cols & 3) == 0 && aligned(t.grad, bf16 ? 8 : 16) && aligned(t.momentum, 16);
    const int r0 = tall ? col0 : row0, c0 = tall ? row0 : col0;                // in the caller's matrix
    const int q = (threadIdx.x & 15) * 4;
    _Float16* const H = (_Float16*)(base + at.h(0));
    uint8_t* const L = (uint8_t*)(base + at.l);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int y = (int)(threadIdx.x >> 4) + 16 * k, row = r0 + y, col = c0 + q;
        const int left = row < t.rows ? t.cols - col : 0;
        const int64_t j = (int64_t)row * t.cols + col;
        af32x4 x = {0.f, 0.f, 0.f, 0.f};
        if (vec && left >= 4) {
            x = grad_values(t.grad, bf16, j);
            if (t.momentum) {
                const af32x4 m = *(const af32x4*)(t.momentum + j);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = direction(m[e], x[e] * clip, a.mu, a.nesterov);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = (float)((double)x[e] * inv);
        } else {
            for (int e = 0; e < 4; ++e) {
                if (e >= left) continue;
                float u = grad_value(t.grad, bf16, j + e);
                if (t.momentum) u = direction(t.momentum[j + e], u * clip, a.mu, a.nesterov);
                x[e] = (float)((double)u * inv);
            }
        }
        if (tall) {
#pragma unroll
            for (int e = 0; e < 4; ++e) tile[y][q + e] = x[e];
        } else {
            f16x4 h;
            uint32_t l;
            split4(x, h, l);
            const uint32_t to = (uint32_t)(row0 + y) * (uint32_t)at.cp + (uint32_t)(col0 + q);
            *(f16x4*)(H + to) = h;
            *(uint32_t*)(L + to) = l;
        }
    }
    if (!tall) return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int y = (int)(threadIdx.x >> 4) + 16 * k;
        f16x4 h;
        uint32_t l;
        split4(af32x4{tile[q][y], tile[q + 1][y], tile[q + 2][y], tile[q + 3][y]}, h, l);
        const uint32_t to = (uint32_t)(row0 + y) * (uint32_t)at.cp + (uint32_t)(col0 + q);
        *(f16x4*)(H + to) = h;
        *(uint32_t*)(L + to) = l;
    }
}

// ------------------------------------------------------------------------------------------
// The products.  A wavefront's results go through LDS, 32 rows at a time, from the matrix instruction's layout (four rows of a
// column a lane) to whole lines of rows: eight neighbouring values a lane.
// ------------------------------------------------------------------------------------------
typedef TileCfg<2, 2, 2, 2, 2> SymTile;                // 128 x 128 by four wavefronts of 64 x 64, 2 x 32 KB stages: two workgroups a CU
constexpr int kSymPitch = 64 + 4;                      // floats of a staged row
constexpr int kSymMirror = 64 + 8;                     // 16-bit values of a staged row of the mirrored tile
constexpr int kSymWave = 32 * kSymPitch * 4 + 64 * kSymMirror * 2;
constexpr int kSymLds = 4 * kSymWave > SymTile::kLdsBytes ? 4 * kSymWave : SymTile::kLdsBytes;
typedef TileDuo ApplyTile;                             // 256 columns of X x 128 rows
constexpr int kApplyPitch = 128 + 4;
constexpr int kApplyWave = 32 * kApplyPitch * 4;
constexpr int kResident = 512;                         // workgroups on the card at a time
static_assert(4 * kApplyWave <= ApplyTile::kLdsBytes && 2 * kSymLds <= 160 * 1024 && 2 * ApplyTile::kLdsBytes <= 160 * 1024, "two workgroups a CU");

// Tile w of the lower triangle, by rows.
__device__ __forceinline__ void triangle(int w, int& i, int& j) {
    i = (int)((sqrtf(8.f * (float)w + 1.f) - 1.f) * 0.5f);
    while ((i + 1) * (i + 2) / 2 <= w) ++i;
    while (i * (i + 1) / 2 > w) --i;
    j = w - i * (i + 1) / 2;
}

__device__ __forceinline__ void read8(const CCE_LDS float* p, float (&x)[8]) {
    const f32x4 lo = *(const CCE_LDS f32x4*)p, hi = *(const CCE_LDS f32x4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = lo[e];
        x[4 + e] = hi[e];
    }
}

// The symmetric products.  All matrices but X are polynomials of one A: they are symmetric, and any two of them commute, up to their rounding.
// The last product of two steps taken as one is computed in full, T S: a tile's mirror image would be of S T, in which S = 3.4 along the smaller
// directions multiplies what T's rounding turns the large ones to, where T S has its 0.7 (rank 1, 512 x 1280 0.7e-3 instead of 1.4, with a few large rows
// and columns 3e-3 instead of 7).
enum : int { kGram, kPoly, kProduct, kWholeProduct };
enum SymKind : uint32_t {
    kOfX,                      // A = X X^T
    kOfA,                      // M = b A + c A A
    // of two steps taken as one
    kFirst,                    // S = a + b A + c A A
    kBetween,                  // T = S A
    kNextA,                    // A = S T
    kSecond,                   // T = a + b A + c A A
    kBoth                      // a + M = T S
};

// Operands X, Y and the result Y X with the diagonals that are held beside them.
struct SymBuffers {
    const _Float16* x;
    const _Float16* y;
    const float* dx;
    const float* dy;
    _Float16* out;
    float* dout;
    float of_x;                // 1 / scale of x; y's is M's in a product
    float add, scale;          // what the result's diagonal has more, and the result's scale
    bool panel;                // the result lies in panels, as M does
    template <int MODE>
    __device__ __forceinline__ void init(const NsProductArgs& a, const NsLayout& at, char* base) {
        if (MODE == kGram) {
            x = y = (const _Float16*)(base + at.h(a.flip));
            dx = dy = nullptr;
            out = (_Float16*)(base + at.a);
            dout = (float*)(base + at.da);
            panel = false;
            return;
        }
        const bool last = a.kind == kOfA || a.kind == kBoth, to_t = a.kind == kBetween || a.kind == kSecond;
        if (MODE == kPoly) {
            x = y = (const _Float16*)(base + at.a);
            dx = dy = (const float*)(base + at.da);
            out = (_Float16*)(base + (last ? at.m : to_t ? at.t : at.s));
            dout = (float*)(base + (last ? at.dm : to_t ? at.dt : at.ds));
            add = last ? 0.f : a.a;
        } else if (MODE == kProduct) {
            x = (const _Float16*)(base + (to_t ? at.a : at.t));
            y = (const _Float16*)(base + at.s);
            dx = (const float*)(base + (to_t ? at.da : at.dt));
            dy = (const float*)(base + at.ds);
            out = (_Float16*)(base + (to_t ? at.t : at.a));
            dout = (float*)(base + (to_t ? at.dt : at.da));
            of_x = 1.f / kScaleA;
            add = 0.f;
            scale = kScaleA;
        } else {
            x = (const _Float16*)(base + at.s);
            y = (const _Float16*)(base + at.t);
            dx = (const float*)(base + at.ds);
            dy = (const float*)(base + at.dt);
            out = (_Float16*)(base + at.m);
            dout = (float*)(base + at.dm);
            of_x = 1.f / kScaleM;
            add = -a.a;
            scale = kScaleM;
        }
        panel = last;
    }
    __device__ __forceinline__ _Float16* at_place(const NsLayout& at, int row, int col) const {
        return out + (panel ? at.panel(row, col) : (uint32_t)row * (uint32_t)at.rp + col);
    }
};

// A value of a result (row n, column m) from the product's p: what lies beside the diagonal, scaled, and what the diagonal would be.
template <int MODE>
__device__ __forceinline__ float symmetric_value(const NsProductArgs& a, const SymBuffers& of, float p, _Float16 x, _Float16 y, float dn, float dm, float& diagonal) {
    if (MODE == kGram) {
        diagonal = p * (1.f / (kScaleX * kScaleX));
        return diagonal * kScaleA;
    }
    if (MODE == kPoly) {
        p *= a.c / (kScaleA * kScaleA);
        diagonal = a.b * dn + (a.c * dn * dn + p) + of.add;
        return ((a.b + a.c * (dn + dm)) * ((float)x * (1.f / kScaleA)) + p) * kScaleM;
    }
    p *= of.of_x * (1.f / kScaleM);
    diagonal = dn * dm + p + of.add;
    return (dn * ((float)x * of.of_x) + (dm * ((float)y * (1.f / kScaleM)) + p)) * of.scale;
}

// Value n of the diagonal: what of it is held beside the operand, and the operand's where it is not 0.
// Behind the store of the lane's eight values, which has a 0 in its place: a rounding for each of the
// eight, where it is needed once a row, took 11 us more of 256 x 256 (179) and 70 of 4 x 4096 x 4096 (5320).
template <int MODE>
__device__ __forceinline__ void give_diagonal(const NsProductArgs& a, const SymBuffers& of, const NsLayout& at, int n, float diagonal) {
    if (MODE != kGram && a.apart) {
        // (what is beyond fp16's range stays beside it: S2 S1 less both a may be up to 120)
        const _Float16 value = (_Float16)__builtin_amdgcn_fmed3f((diagonal - a.on_x) * kScaleM, -61440.f, 61440.f);
        diagonal -= (float)value * (1.f / kScaleM);
        *of.at_place(at, n, n) = value;
    }
    of.dout[n] = diagonal;
}

// Tile w of a matrix of `side` x `side` tiles.
template <int MODE>
__device__ __forceinline__ void tile_of(int w, int side, int& i, int& j) {
    if (MODE != kWholeProduct) return triangle(w, i, j);
    i = w / side;
    j = w - i * side;
}

// A tile and its mirror image.
template <int MODE>
__global__ __launch_bounds__(SymTile::kThreads, 2) void ns_symmetric_kernel(const NsProductArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    CCE_LDS char* const smem = (CCE_LDS char*)smem_generic;
    const uint32_t id = (uint32_t)xcd_round_id((int)blockIdx.x, (int)gridDim.x, kResident);
    const int i = matrix_of(a.first, (int)a.count, 2 * id + 1);
    const NsLayout at(a.t[i].rows, a.t[i].cols);
    char* const base = workspace_of(a, i);
    SymBuffers of;
    of.init<MODE>(a, at, base);
    int ti, tj;
    tile_of<MODE>((int)(id - (a.first[i] >> 1)), (at.rp + SymTile::BM - 1) / SymTile::BM, ti, tj);
    const int m0 = __builtin_amdgcn_readfirstlane(ti * SymTile::BM), n0 = __builtin_amdgcn_readfirstlane(tj * SymTile::BN);
    f32x16 acc[SymTile::TM][SymTile::TN];
#pragma unroll
    for (int bm = 0; bm < SymTile::TM; ++bm)
#pragma unroll
        for (int bn = 0; bn < SymTile::TN; ++bn) acc[bm][bn] = f32x16{};
    {
        const int k = MODE == kGram ? at.cp : at.rp;
        OperandTile<true, SymTile::BM, 0, SymTile::NW, SymTile::BK> x, y;
        x.init(uniform(of.x), k, m0, at.rp, k);
        y.init(uniform(of.y), k, n0, at.rp, k);
        gemm_mainloop<SymTile, true, true, true, true>(acc, x, y, k, smem);
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    CCE_LDS float* const rows = (CCE_LDS float*)(smem + wave * kSymWave);
    CCE_LDS _Float16* const mirror = (CCE_LDS _Float16*)(smem + wave * kSymWave + 32 * kSymPitch * 4);
    const int wm = m0 + wave_m<SymTile>() * 64, wn = n0 + wave_n<SymTile>() * 64;      // this wavefront's corner
    const int q = (lane & 7) * 8;                                                      // this lane's columns
    const int m = wm + q;
    const bool inside_m = m < at.rp, mirrored = MODE != kWholeProduct && m0 != n0;
    f32x4 dc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    if (MODE != kGram && inside_m) {
        dc[0] = *(const f32x4*)(of.dx + m);
        dc[1] = *(const f32x4*)(of.dx + m + 4);
    }
#pragma unroll
    for (int bn = 0; bn < SymTile::TN; ++bn) {
        // all loads of 32 rows together, from rows that are there
        f16x8 ox[4], oy[4];
        float dn[4];
        if (MODE != kGram) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int n = wn + bn * 32 + 8 * k + (lane >> 3);
                const bool there = inside_m && n < at.rp;
                const uint32_t place = there ? (uint32_t)n * (uint32_t)at.rp + m : 0u;
                ox[k] = *(const f16x8*)(of.x + place);
                if (MODE >= kProduct) oy[k] = *(const f16x8*)(of.y + place);
                dn[k] = of.dy[there ? n : 0];
            }
        }
#pragma unroll
        for (int bm = 0; bm < SymTile::TM; ++bm)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(CCE_LDS f32x4*)(rows + (lane & 31) * kSymPitch + bm * 32 + 8 * g + 4 * (lane >> 5)) =
                    f32x4{acc[bm][bn][4 * g], acc[bm][bn][4 * g + 1], acc[bm][bn][4 * g + 2], acc[bm][bn][4 * g + 3]};
        wave_lds_order();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int y = 8 * k + (lane >> 3), n = wn + bn * 32 + y;
            const bool inside = inside_m && n < at.rp;
            float x[8];
            read8(rows + y * kSymPitch + q, x);
            f16x8 v;
            float own = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float diagonal;
                const float beside = symmetric_value<MODE>(a, of, x[e], ox[k][e], oy[k][e], dn[k], dc[e >> 2][e & 3], diagonal);
                const bool here = m + e == n;
                own = here ? diagonal : own;
                v[e] = here ? (_Float16)0.f : (_Float16)beside;
            }
            if (inside) *(f16x8*)of.at_place(at, n, m) = v;
            if (inside && (uint32_t)(n - m) < 8u) give_diagonal<MODE>(a, of, at, n, own);
            if (mirrored)
#pragma unroll
                for (int e = 0; e < 8; ++e) mirror[(q + e) * kSymMirror + bn * 32 + y] = v[e];
        }
        wave_lds_order();
    }
    if (!mirrored) return;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int y = 8 * k + (lane >> 3), row = wm + y, col = wn + q;                 // of the mirrored tile
        const f16x8 v = *(const CCE_LDS f16x8*)(mirror + y * kSymMirror + q);
        if (row < at.rp && col < at.rp) *(f16x8*)of.at_place(at, row, col) = v;
    }
}

// The same on 256 x 256 tiles of two groups of wavefronts that take turns (see PingTile), one workgroup a CU.
typedef TileSquare SymPing;
constexpr int kPingPitch = 32 + 4;                     // floats of a staged row: 32 columns of 64 rows
constexpr int kPingMirror = 128 + 8;
constexpr int kPingWave = 64 * kPingPitch * 4 + 32 * kPingMirror * 2;
constexpr int kPingLds = 8 * kPingWave > SymPing::kLdsBytes ? 8 * kPingWave : SymPing::kLdsBytes;
static_assert(kPingLds <= 160 * 1024, "160 KB LDS");

// A wavefront's part of tile (ti, tj) and of its mirror image.
template <int MODE>
__device__ __forceinline__ void symmetric_ping_rows(const NsProductArgs& a, const NsLayout& at, const SymBuffers& of, f32x4 (&acc)[SymPing::NA][SymPing::NB],
                                                    int ti, int tj, int wave, CCE_LDS char* smem) {
    const int lane = threadIdx.x & 63, wm = wave / SymPing::WN, wn = wave % SymPing::WN, m0 = ti * SymPing::BM, n0 = tj * SymPing::BN;
    CCE_LDS float* const rows = (CCE_LDS float*)smem;
    CCE_LDS _Float16* const mirror = (CCE_LDS _Float16*)(smem + 64 * kPingPitch * 4);
    const int q = (lane & 3) * 8, nw = n0 + wn * SymPing::TNR;
    const bool mirrored = MODE != kWholeProduct && ti != tj;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
        const int mw = m0 + part * (SymPing::BM / 2) + wm * 32, m = mw + q;            // 32 columns of the result
        if (mw >= at.rp) continue;
        f32x4 dc[2];
        if (MODE != kGram) {
            dc[0] = *(const f32x4*)(of.dx + m);
            dc[1] = *(const f32x4*)(of.dx + m + 4);
        }
#pragma unroll
        for (int side = 0; side < 2; ++side) {
            f16x8 ox[4], oy[4];
            float dn[4];
            if (MODE != kGram) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int n = nw + 64 * side + 16 * k + (lane >> 2);
                    const uint32_t place = n < at.rp ? (uint32_t)n * (uint32_t)at.rp + m : 0u;
                    ox[k] = *(const f16x8*)(of.x + place);
                    if (MODE >= kProduct) oy[k] = *(const f16x8*)(of.y + place);
                    dn[k] = of.dy[n < at.rp ? n : 0];
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int b = 0; b < SymPing::QA; ++b)
                    *(CCE_LDS f32x4*)(rows + (16 * j + (lane & 15)) * kPingPitch + 16 * b + 4 * (lane >> 4)) = acc[part * SymPing::QA + b][4 * side + j];
            wave_lds_order();
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int y = 16 * k + (lane >> 2), n = nw + 64 * side + y;
                float x[8];
                read8(rows + y * kPingPitch + q, x);
                f16x8 v;
                float own = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float diagonal;
                    const float beside = symmetric_value<MODE>(a, of, x[e], ox[k][e], oy[k][e], dn[k], dc[e >> 2][e & 3], diagonal);
                    const bool here = m + e == n;
                    own = here ? diagonal : own;
                    v[e] = here ? (_Float16)0.f : (_Float16)beside;
                }
                if (n < at.rp) *(f16x8*)of.at_place(at, n, m) = v;
                if (n < at.rp && (uint32_t)(n - m) < 8u) give_diagonal<MODE>(a, of, at, n, own);
                if (mirrored)
#pragma unroll
                    for (int e = 0; e < 8; ++e) mirror[(q + e) * kPingMirror + 64 * side + y] = v[e];
            }
            wave_lds_order();
        }
        if (mirrored) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int y = 4 * k + (lane >> 4), row = mw + y, col = nw + (lane & 15) * 8;     // of the mirrored tile
                const f16x8 v = *(const CCE_LDS f16x8*)(mirror + y * kPingMirror + (lane & 15) * 8);
                *(f16x8*)of.at_place(at, row, col) = v;
            }
            wave_lds_order();
        }
    }
}

// The last a.split_tiles tiles, where they would leave most CUs without one, are computed in a.splits parts of the sum each, which
// ns_symmetric_join_kernel adds in their order.
template <int MODE>
__global__ __launch_bounds__(SymPing::kThreads, 2) void ns_symmetric_ping_kernel(const NsProductArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    CCE_LDS char* const smem = (CCE_LDS char*)smem_generic;
    const uint32_t id = (uint32_t)xcd_round_id((int)blockIdx.x, (int)gridDim.x, kResident / 2), whole = gridDim.x - a.split_tiles * a.splits;
    const bool part = id >= whole;
    const uint32_t tile = part ? whole + (id - whole) / a.splits : id;
    const int i = matrix_of(a.first, (int)a.count, 2 * tile + 1);
    const NsLayout at(a.t[i].rows, a.t[i].cols);
    SymBuffers of;
    of.init<MODE>(a, at, workspace_of(a, i));
    int ti, tj;
    tile_of<MODE>((int)(tile - (a.first[i] >> 1)), (at.rp + SymPing::BM - 1) / SymPing::BM, ti, tj);
    ti = __builtin_amdgcn_readfirstlane(ti);
    tj = __builtin_amdgcn_readfirstlane(tj);
    const int m0 = ti * SymPing::BM, n0 = tj * SymPing::BN;
    const int m_rows = at.rp - m0 < SymPing::BM ? at.rp - m0 : SymPing::BM, parts = m_rows > SymPing::BM / 2 ? 2 : 1;
    f32x4 acc[SymPing::NA][SymPing::NB];
#pragma unroll
    for (int x = 0; x < SymPing::NA; ++x)
#pragma unroll
        for (int y = 0; y < SymPing::NB; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
    {
        const uint32_t ld = (uint32_t)(MODE == kGram ? at.cp : at.rp) * 2u;
        const int slices = (MODE == kGram ? at.cp : at.rp) / SymPing::BK;
        int first = 0, KT = slices;
        if (part) {
            const int split = (int)((id - whole) % a.splits), splits = (int)a.splits;
            first = slices * split / splits;
            KT = slices * (split + 1) / splits - first;
        }
        const char* const from_x = uniform((const char*)of.x + (size_t)first * (2 * SymPing::BK));
        const char* const from_y = uniform((const char*)of.y + (size_t)first * (2 * SymPing::BK));
        PingPong<SymPing, ARows::kHalves, true> turns;
        PingLoads<SymPing, ARows::kHalves> loads;
        turns.init(smem);
        loads.init(smem, ld);
#pragma unroll
        for (int x = 0; x < SymPing::kBLoads; ++x) {
            const int row = n0 + loads.row(x);
            loads.set_b_row(x, row < at.rp ? row : at.rp - 1, ld);
        }
        loads.on = true;
        loads.tile(uniform(from_x + (size_t)m0 * ld), m_rows, from_y, ld);
        __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0): what the compiler has loaded so far, which cannot see the loads of the slices
        loads.issue(0, 0);
        loads.issue(0, 1);
        turns.start();
        auto request = [&](int stage, int half) {
            if (loads.on) loads.issue(stage, half);
        };
#pragma nounroll
        for (int kt = 0;;) {
            if (kt + 1 < KT) {
                loads.a += 2 * SymPing::BK;
                loads.b += 2 * SymPing::BK;
            } else {
                loads.on = false;
            }
            turns.slice(acc, parts, request);
            if (++kt == KT) break;
            turns.barrier();
        }
        turns.tile_done();                             // every wavefront has its last fragments
    }
    const int wave = threadIdx.x >> 6;
    if (part) {
        f32x4* const to = (f32x4*)(a.ws + (uint64_t)a.partials * 256) + ((size_t)(id - whole) * 8 + wave) * (SymPing::NA * SymPing::NB * 64) + (threadIdx.x & 63);
#pragma unroll
        for (int x = 0; x < SymPing::NA; ++x)
#pragma unroll
            for (int y = 0; y < SymPing::NB; ++y) to[(x * SymPing::NB + y) * 64] = acc[x][y];
        return;
    }
    symmetric_ping_rows<MODE>(a, at, of, acc, ti, tj, wave, smem + wave * kPingWave);
}

// A wavefront of a split tile a workgroup.
template <int MODE>
__global__ __launch_bounds__(64) void ns_symmetric_join_kernel(const NsProductArgs a) {
    __shared__ __attribute__((aligned(1024))) char smem_generic[kPingWave];
    const uint32_t split = blockIdx.x >> 3, tile = a.tiles - a.split_tiles + split;
    const int wave = (int)(blockIdx.x & 7u);
    const int i = matrix_of(a.first, (int)a.count, 2 * tile + 1);
    const NsLayout at(a.t[i].rows, a.t[i].cols);
    SymBuffers of;
    of.init<MODE>(a, at, workspace_of(a, i));
    int ti, tj;
    tile_of<MODE>((int)(tile - (a.first[i] >> 1)), (at.rp + SymPing::BM - 1) / SymPing::BM, ti, tj);
    const f32x4* from = (const f32x4*)(a.ws + (uint64_t)a.partials * 256) + ((size_t)split * a.splits * 8 + wave) * (SymPing::NA * SymPing::NB * 64) + threadIdx.x;
    f32x4 acc[SymPing::NA][SymPing::NB];
#pragma unroll
    for (int x = 0; x < SymPing::NA; ++x)
#pragma unroll
        for (int y = 0; y < SymPing::NB; ++y) acc[x][y] = from[(x * SymPing::NB + y) * 64];
    for (uint32_t k = 1; k < a.splits; ++k) {
        from += 8 * SymPing::NA * SymPing::NB * 64;
#pragma unroll
        for (int x = 0; x < SymPing::NA; ++x)
#pragma unroll
            for (int y = 0; y < SymPing::NB; ++y) acc[x][y] += from[(x * SymPing::NB + y) * 64];
    }
    symmetric_ping_rows<MODE>(a, at, of, acc, ti, tj, wave, (CCE_LDS char*)smem_generic);
}

__device__ __forceinline__ uint16_t bf16_bits(float x) {
    union { __bf16 h; uint16_t u; } cv;
    cv.h = (__bf16)x;
    return cv.u;
}

// Four values of the result for the caller: into the parameters and their copy, or into the copy alone.  vec: all four are
// there and lie where 16-byte (8-byte) accesses may be made.  The parameters are loaded in front, those of several calls together: the
// compiler moves no load before a store that might write the same memory.
__device__ __forceinline__ f32x4 param4(const NsMatrix& t, int64_t at, int count, bool vec) {
    f32x4 p = {0.f, 0.f, 0.f, 0.f};
    if (!t.param) return p;
    if (vec) return *(const f32x4*)(t.param + at);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < count) p[e] = t.param[at + e];
    return p;
}
__device__ __forceinline__ void give4(const NsMatrix& t, int64_t to, const f32x4& p, f32x4 x, int count, bool vec) {
    if (t.param) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = p[e] * t.decay - t.lr * x[e];
    }
    if (vec) {
        if (t.param) *(f32x4*)(t.param + to) = x;
        if (t.out) {
            union { __bf16 h[4]; u32x2 u; } cv;
#pragma unroll
            for (int e = 0; e < 4; ++e) cv.h[e] = (__bf16)x[e];
            *(u32x2*)(t.out + to) = cv.u;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (e >= count) continue;
        if (t.param) t.param[to + e] = x[e];
        if (t.out) t.out[to + e] = bf16_bits(x[e]);
    }
}

// X = (a + M) X of 32 rows and 128 columns of X a wavefront, from (n0, m0) on: what is loaded, in front of the products' way through
// LDS, and what is made of them.
struct ApplyRows {
    f16x8 h[8];
    u32x2 l[8];
    float keep[8];
    __device__ __forceinline__ void load(const NsLayout& at, const char* base, int flip, int n0, int m0) {
        const _Float16* const H = (const _Float16*)(base + at.h((uint32_t)flip));
        const uint8_t* const L = (const uint8_t*)(base + at.l);
        const float* const dm = (const float*)(base + at.dm);
        const int lane = threadIdx.x & 63, m = m0 + (lane & 15) * 8;
        // all loads together, from rows that are there
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int n = n0 + 4 * k + (lane >> 4);
            const bool there = n < at.rp && m < at.cp;
            const uint32_t j = there ? (uint32_t)n * (uint32_t)at.cp + m : 0u;
            h[k] = *(const f16x8*)(H + j);
            l[k] = *(const u32x2*)(L + j);
            keep[k] = dm[there ? n : 0];
        }
    }
    // rows: 32 rows of 128 products in LDS, kApplyPitch apart
    template <bool LAST, class Args, class Matrix>
    __device__ __forceinline__ void finish(const Args& a, const Matrix& t, const NsLayout& at, char* base, int n0, int m0, CCE_LDS float* rows) const {
        _Float16* const H1 = (_Float16*)(base + at.h(a.flip ^ 1));
        uint8_t* const L = (uint8_t*)(base + at.l);
        const int lane = threadIdx.x & 63, q = (lane & 15) * 8, m = m0 + q;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int y = 4 * k + (lane >> 4), n = n0 + y;
            const uint32_t j = (uint32_t)n * (uint32_t)at.cp + m;
            const float of_h = (a.a + keep[k]) * (1.f / kScaleX), of_l = of_h * 0x1p-18f;
            float x[8];
            read8(rows + y * kApplyPitch + q, x);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = fmaf(of_h, (float)h[k][e], fmaf(of_l, rest_of(h[k][e], l[k][e >> 2] >> 8 * (e & 3)), x[e] * (1.f / (kScaleX * kScaleM))));
            if (!LAST) {
                f16x8 h1;
                u32x2 l1;
                split8(x, h1, l1);
                if (n < at.rp && m < at.cp) {
                    *(f16x8*)(H1 + j) = h1;
                    *(u32x2*)(L + j) = l1;
                }
            } else {
                *(CCE_LDS f32x4*)(rows + y * kApplyPitch + q) = f32x4{x[0], x[1], x[2], x[3]};
                *(CCE_LDS f32x4*)(rows + y * kApplyPitch + q + 4) = f32x4{x[4], x[5], x[6], x[7]};
            }
        }
        wave_lds_order();
        if constexpr (LAST) {
            // to the caller, four values in a row of their matrix a lane: rows of X, or columns
            const bool tall = t.rows > t.cols, vec = (t.cols & 3) == 0 && aligned(t.param, 16) && aligned(t.out, 8);
            const int z = tall ? (lane & 7) * 4 : (lane & 31) * 4;
            auto value = [&](int y, int e) { return tall ? rows[(z + e) * kApplyPitch + y] : rows[y * kApplyPitch + z + e]; };
#pragma unroll 1
            for (int k0 = 0; k0 < 16; k0 += 8) {
                const int y0 = tall ? 8 * k0 + (lane >> 3) : 2 * k0 + (lane >> 5), step = tall ? 8 : 2;
                const int line = (tall ? m0 : n0) + y0, in_line = (tall ? n0 : m0) + z;
                const int lines = tall ? at.c : at.r, length = tall ? at.r : at.c;
                if (vec) {
                    f32x4 p[8];
                    if (t.param) {
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            p[k] = *(const f32x4*)(t.param + (line + step * k < lines && in_line < length ? (int64_t)(line + step * k) * t.cols + in_line : 0));
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        f32x4 x;
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            x[e] = value(y0 + step * k, e);
                            if (t.param) x[e] = p[k][e] * t.decay - t.lr * x[e];
                        }
                        if (line + step * k < lines && in_line < length) {
                            const int64_t to = (int64_t)(line + step * k) * t.cols + in_line;
                            if (t.param) *(f32x4*)(t.param + to) = x;
                            if (t.out) {
                                union { __bf16 h[4]; u32x2 u; } cv;
#pragma unroll
                                for (int e = 0; e < 4; ++e) cv.h[e] = (__bf16)x[e];
                                *(u32x2*)(t.out + to) = cv.u;
                            }
                        }
                    }
                } else {
#pragma unroll 1
                    for (int k = 0; k < 8; ++k)
#pragma unroll 1
                        for (int e = 0; e < 4; ++e) {
                            if (line + step * k >= lines || in_line + e >= length) continue;
                            const int64_t to = (int64_t)(line + step * k) * t.cols + in_line + e;
                            float y = value(y0 + step * k, e);
                            if (t.param) {
                                y = t.param[to] * t.decay - t.lr * y;
                                t.param[to] = y;
                            }
                            if (t.out) t.out[to] = bf16_bits(y);
                        }
                }
            }
            wave_lds_order();
        }
    }
};

template <bool LAST> using ApplyArgs = std::conditional_t<LAST, NsArgs, NsProductArgs>;

// X = (a + M) X; LAST: to the caller.  256 columns x 128 rows, two workgroups a CU.
template <bool LAST>
__global__ __launch_bounds__(ApplyTile::kThreads, 2) void ns_apply_kernel(const ApplyArgs<LAST> a) {
    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    CCE_LDS char* const smem = (CCE_LDS char*)smem_generic;
    const uint32_t id = (uint32_t)xcd_round_id((int)blockIdx.x, (int)gridDim.x, kResident);
    const int i = matrix_of(a.first, (int)a.count, 2 * id + 1);
    const auto& t = a.t[i];
    const NsLayout at(t.rows, t.cols);
    char* const base = workspace_of(a, i);
    const int w = (int)(id - (a.first[i] >> 1)), row_tiles = (at.rp + ApplyTile::BN - 1) / ApplyTile::BN;
    const int m0 = __builtin_amdgcn_readfirstlane(w / row_tiles * ApplyTile::BM), n0 = __builtin_amdgcn_readfirstlane(w % row_tiles * ApplyTile::BN);
    f32x16 acc[ApplyTile::TM][ApplyTile::TN];
#pragma unroll
    for (int bm = 0; bm < ApplyTile::TM; ++bm)
#pragma unroll
        for (int bn = 0; bn < ApplyTile::TN; ++bn) acc[bm][bn] = f32x16{};
    {
        OperandTile<false, ApplyTile::BM, 0, ApplyTile::NW, ApplyTile::BK> x;
        PanelTile<true, ApplyTile::BN, ApplyTile::NW, ApplyTile::BK> y;
        x.init(uniform((const _Float16*)(base + at.h(a.flip))), at.cp, m0, at.cp, at.rp);
        y.init((const uint16_t*)uniform(base + at.m), (uint32_t)at.panel_rows() * 32u, n0, 0);
        y.base = uniform(y.base);
        gemm_mainloop<ApplyTile, false, true, true, true>(acc, x, y, at.rp, smem);
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    CCE_LDS float* const rows = (CCE_LDS float*)(smem + wave * kApplyWave);
    const int wm = m0 + wave_m<ApplyTile>() * 128, wn = n0 + wave_n<ApplyTile>() * 64;
#pragma unroll
    for (int bn = 0; bn < ApplyTile::TN; ++bn) {
        ApplyRows of;
        of.load(at, base, (int)a.flip, wn + bn * 32, wm);
#pragma unroll
        for (int bm = 0; bm < ApplyTile::TM; ++bm)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(CCE_LDS f32x4*)(rows + (lane & 31) * kApplyPitch + bm * 32 + 8 * g + 4 * (lane >> 5)) =
                    f32x4{acc[bm][bn][4 * g], acc[bm][bn][4 * g + 1], acc[bm][bn][4 * g + 2], acc[bm][bn][4 * g + 3]};
        wave_lds_order();
        of.finish<LAST>(a, t, at, base, wn + bn * 32, wm, rows);
    }
}

// The same on 256 x 256 tiles of two groups of wavefronts that take turns (see TurnTile), one workgroup a CU.
constexpr int kTurnLds = 8 * kApplyWave > TurnTile::kLdsBytes ? 8 * kApplyWave : TurnTile::kLdsBytes;
static_assert(kTurnLds <= 160 * 1024, "160 KB LDS");
constexpr int kTurnRows = 128;                         // fewest (padded) rows: its loop has four slices at least

template <bool LAST>
__global__ __launch_bounds__(TurnTile::kThreads, 2) void ns_apply_turn_kernel(const ApplyArgs<LAST> a) {
    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    CCE_LDS char* const smem = (CCE_LDS char*)smem_generic;
    const uint32_t id = (uint32_t)xcd_round_id((int)blockIdx.x, (int)gridDim.x, kResident / 2);
    const int i = matrix_of(a.first, (int)a.count, 2 * id + 1);
    const auto& t = a.t[i];
    const NsLayout at(t.rows, t.cols);
    char* const base = workspace_of(a, i);
    const int w = (int)(id - (a.first[i] >> 1)), row_tiles = (at.rp + TurnTile::BN - 1) / TurnTile::BN;
    const int m0 = __builtin_amdgcn_readfirstlane(w / row_tiles * TurnTile::BM), n0 = __builtin_amdgcn_readfirstlane(w % row_tiles * TurnTile::BN);
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    TurnLoop<true, 0, true> loop;
    loop.init(smem, wave, uniform(base + at.h(a.flip)), (uint32_t)at.cp * 2u, m0, at.cp, at.rp,
              (const uint16_t*)uniform(base + at.m), (uint32_t)at.panel_rows() * 32u, n0, 0);
    __builtin_amdgcn_s_waitcnt(0x0f70);                // vmcnt(0): what the compiler has loaded so far, which cannot see the loads of the slices
    const int KT = loop.slices(at.rp);
    const int wm = m0 + 128 * loop.group, wn = n0 + (wave & 3) * 64;
    if (wm >= at.cp) {                                 // (its columns lie behind the matrix: loads and barriers only)
        loop.idle(KT);
        return;
    }
    f32x4 acc[TurnTile::NA][TurnTile::NB];
#pragma unroll
    for (int x = 0; x < TurnTile::NA; ++x)
#pragma unroll
        for (int y = 0; y < TurnTile::NB; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
    loop.run(acc, KT);
    const int lane = threadIdx.x & 63;
    CCE_LDS float* const rows = (CCE_LDS float*)(smem + wave * kApplyWave);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (wn + half * 32 >= at.rp) continue;
        ApplyRows of;
        of.load(at, base, (int)a.flip, wn + half * 32, wm);
#pragma unroll
        for (int x = 0; x < TurnTile::NA; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y)
                *(CCE_LDS f32x4*)(rows + (16 * y + (lane & 15)) * kApplyPitch + 16 * x + 4 * (lane >> 4)) = acc[x][2 * half + y];
        wave_lds_order();
        of.finish<LAST>(a, t, at, base, wn + half * 32, wm, rows);
    }
}

// ------------------------------------------------------------------------------------------
// A matrix of few rows in one workgroup, all steps in one launch: X in fp32 in the accumulators (blocks of 16 x 16 by eight
// wavefronts, block column j of wavefront w being 8 j + w), its h in LDS for the products.
//
//   gram    up to 64 rows each wavefront sums over its own columns; of more rows wavefronts share the blocks of A, each over all columns of h
//   poly    wavefronts share the blocks
//   apply   each wavefront its own columns, which no other one reads: X stays in its registers
//
// Rounding.  The roundings of the operands of few rows even out little, and the steps amplify those that are not along a matrix's large
// directions by up to 485, so that it shows of matrices of low rank.  Up to 64 rows M is multiplied with the next 11 bits of X too, and up to 32
// all products have their operands' next 11 bits (kWhole).  Of more rows M acts on h alone in the steps behind which much is amplified (apart_steps):
// 65 x 200 6.9e-3 / 1.1e-3.  Largest error (2-norm, of the result's) over spectra of rank 1 to 64, noise and singular
// values down to 1e-4, without / with: 17 x 17 2.3e-2 / 3e-5, 33 x 33 1.6e-2 / 1.2e-3, 64 x 256 6.7e-3 / 9e-4; us 17 x 17 9.7 / 11.0,
// 32 x 512 14.5 / 19.2, 64 x 256 19.8 / 21.9, 64 x 1024 45 / 55.
//
// The 17 launches of the tiled path take 115 us for 64 x 256, mostly waiting for each other.  128 x 448 63 us.
// ------------------------------------------------------------------------------------------
constexpr int kSmallThreads = 512;
constexpr int kSmallMatrices = 48;

struct NsSmallArgs {
    NsMatrix t[kSmallMatrices];
    uint64_t bf16;                                     // bit i: matrix i has a bf16 gradient
    float coefficients[CCE_NS_MAX_STEPS][3];
    const float* clip_coef;
    float mu, eps;
    int32_t nesterov, steps;
    uint32_t apart;                                    // bit s: in step s M acts on h alone (apart_steps)
};
static_assert(sizeof(NsSmallArgs) <= 4096, "kernel arguments hold 4 KB");

// RB blocks of 16 rows, up to NB block columns a wavefront.
template <int RB_, int NB_>
struct SmallShape {
    static constexpr int RB = RB_, NB = NB_, kRows = 16 * RB_, kColumns = RB_ < 8 ? NB_ * 128 : 448;
    static constexpr int kPitchA = kRows + 8;
    static constexpr bool kOwnSums = RB_ <= 4;           // A from each wavefront's own columns
    static constexpr bool kWhole = RB_ == 2;             // remainders of X, A and M in all products
    static constexpr int kPairs = RB_ * (RB_ + 1) / 2;   // blocks of A, of each two that mirror each other one
    static constexpr int kSumBytes = kOwnSums ? 8 * kPairs * 1024 : 0, kSquares = kWhole ? 4 : kOwnSums ? 2 : 1;      // (M in A's place where it has no other)
    static constexpr int kStagePitch = 16 + 1, kStageBytes = kRows * kStagePitch * 4;      // a block column of a wavefront, on its way in or out
    static constexpr int pitch(int c) { return ((c + 63) & ~63) + 8; }
    static constexpr int h_bytes(int c) { return kRows * pitch(c) * 2; }
    static constexpr int kRest = 64 + kSquares * kRows * kPitchA * 2 + kRows * 8;
    // whether the wavefronts' sums have room of their own; else they lie over h, of which none is needed then
    static constexpr bool apart(int c) { return kRest + h_bytes(c) + kSumBytes <= 160 * 1024; }
    static constexpr int h_room(int c) { return apart(c) || h_bytes(c) > kSumBytes ? h_bytes(c) : kSumBytes; }
    static constexpr int lds(int c) {
        const int work = kRest + h_room(c) + (apart(c) ? kSumBytes : 0), stages = 64 + 8 * kStageBytes;
        return work > stages ? work : stages;
    }
};
typedef SmallShape<2, 6> Small32;
typedef SmallShape<4, 8> Small64;
typedef SmallShape<8, 4> Small128;
static_assert(Small32::lds(Small32::kColumns) <= 160 * 1024 && Small64::lds(Small64::kColumns) <= 160 * 1024 &&
              Small128::lds(Small128::kColumns) <= 160 * 1024, "160 KB LDS");
static_assert(Small32::apart(Small32::kColumns) && Small64::apart(448) && !Small64::apart(449), "either form is tested");
// Columns of the matrices that are taken so; from there on thin ones take three launches, us of a step on 48 matrices in one workgroup each /
// in three launches: 16 x 512 20 / 22, 16 x 896 27 / 23, 16 x 2048 46 / 26, 32 x 512 26 / 32, 32 x 768 35 / 34,
// 64 x 512 48 / 78, 64 x 1024 83 / 85.
__host__ __device__ constexpr int small_columns(int64_t rows) {
    return rows <= 16 ? 512 : rows <= 32 ? Small32::kColumns : rows <= 64 ? Small64::kColumns : rows <= 128 ? Small128::kColumns : 0;
}

__device__ __forceinline__ f16x4 half4(const f32x4& x) {
    f16x4 h;
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = (_Float16)x[e];
    return h;
}
// What x has beyond its h, of h's scale: the next 11 bits.
__device__ __forceinline__ f16x4 rest4(const f32x4& x, const f16x4& h) {
    f16x4 l;
#pragma unroll
    for (int e = 0; e < 4; ++e) l[e] = (_Float16)(x[e] - (float)h[e]);
    return l;
}

// How a wavefront's block columns go in and out.
enum : int {
    kVectors,                  // wide, four columns of a lane by one access
    kStaged,                   // wide, where lines of the caller's memory and a lane's four columns do not meet
    kColumns                   // tall: neighbouring lanes have neighbours in memory
};

template <class S, int WAY>
__device__ __forceinline__ void small_matrix(const NsSmallArgs& a, const NsMatrix& t, bool bf16, CCE_LDS char* smem) {
    constexpr int RB = S::RB, NB = S::NB;
    constexpr int BI = RB == 8 ? 2 : 1, BJ = RB == 8 ? 4 : RB == 4 ? 2 : 1;        // blocks of A a wavefront computes
    constexpr int kPerRow = RB / BJ;                                               // wavefronts beside each other
    const int r = t.rows < t.cols ? t.rows : t.cols, c = t.rows < t.cols ? t.cols : t.rows;
    const int columns = (c + 63) & ~63, block_columns = columns >> 4, pitch = columns + 8;
    CCE_LDS double* const red = (CCE_LDS double*)smem;
    CCE_LDS _Float16* const H = (CCE_LDS _Float16*)(smem + 64);
    CCE_LDS _Float16* const A = (CCE_LDS _Float16*)(smem + 64 + S::h_room(c));
    constexpr int kSquare = S::kRows * S::kPitchA;
    CCE_LDS _Float16* const M = A + (S::kSquares > 1 ? kSquare : 0);
    CCE_LDS _Float16* const A_rest = A + 2 * kSquare;                                 // (of kWhole)
    CCE_LDS _Float16* const M_rest = A + 3 * kSquare;
    CCE_LDS float* const da = (CCE_LDS float*)(A + S::kSquares * kSquare);
    CCE_LDS float* const dm = da + S::kRows;
    const bool apart = S::apart(c);
    CCE_LDS float* const sums = apart ? dm + S::kRows : (CCE_LDS float*)H;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int l16 = lane & 15, quad = lane >> 4;
    int mine = __builtin_amdgcn_readfirstlane((block_columns + 7 - wave) >> 3);       // this wavefront's block columns
    const float coefficient = a.coefficients[0][lane < 3 * CCE_NS_MAX_STEPS ? lane : 0];
    const float clip = a.clip_coef ? a.clip_coef[0] : 1.f;
    // kStaged: a block column goes through this wavefront's stage, element k of it is the k-th in the caller's order
    CCE_LDS float* const stage = (CCE_LDS float*)(smem + 64 + wave * S::kStageBytes);
    auto staged = [&](int j, auto element) {
#pragma nounroll
        for (int k = lane; k < S::kRows * 16; k += 64) {
            const int row = k >> 4, in = k & 15, col = 16 * (8 * j + wave) + in;
            if (row < r && col < c) element(row * t.cols + col, stage[row * S::kStagePitch + in]);
        }
    };
    // kColumns: element by element
    auto each = [&](auto element, int j) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = 16 * rb + l16, col = 16 * (8 * j + wave) + 4 * quad + e;
                if (row < r && col < c) element(rb, e, col * t.cols + row);
            }
    };
    // accumulator element e of block (rb, j): row 16 rb + l16, column 16 (8 j + wave) + 4 quad + e
    f32x4 x[NB][RB];
    double sum = 0.0;
#pragma unroll
    for (int j = 0; j < NB; ++j) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) x[j][rb] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (j >= mine) continue;
        const int col = 16 * (8 * j + wave) + 4 * quad;
        if constexpr (WAY == kVectors) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int row = 16 * rb + l16;
                if (row >= r || col >= c) continue;
                const int at = row * t.cols + col;
                f32x4 u = grad_values(t.grad, bf16, at);
                if (t.momentum) {
                    f32x4 m = *(const f32x4*)(t.momentum + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float g = u[e] * clip;
                        m[e] = new_momentum(m[e], g, a.mu);
                        u[e] = direction(m[e], g, a.mu, a.nesterov);
                    }
                    *(f32x4*)(t.momentum + at) = m;
                }
                x[j][rb] = u;
            }
        } else if constexpr (WAY == kColumns) {
            f32x4 grads[RB], moments[RB];
            each([&](int rb, int e, int at) {
                grads[rb][e] = grad_value(t.grad, bf16, at);
                moments[rb][e] = t.momentum ? t.momentum[at] : 0.f;
            }, j);
            each([&](int rb, int e, int at) {
                float g = grads[rb][e];
                if (t.momentum) {
                    g *= clip;
                    const float m = new_momentum(moments[rb][e], g, a.mu);
                    t.momentum[at] = m;
                    g = direction(m, g, a.mu, a.nesterov);
                }
                x[j][rb][e] = g;
            }, j);
        } else {
            wave_lds_order();
            staged(j, [&](int at, CCE_LDS float& to) {
                float g = grad_value(t.grad, bf16, at);
                if (t.momentum) {
                    g *= clip;
                    const float m = new_momentum(t.momentum[at], g, a.mu);
                    t.momentum[at] = m;
                    g = direction(m, g, a.mu, a.nesterov);
                }
                to = g;
            });
            wave_lds_order();
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int row = 16 * rb + l16;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (row < r && col + e < c) x[j][rb][e] = stage[row * S::kStagePitch + 4 * quad + e];
            }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fma((double)x[j][rb][e], (double)x[j][rb][e], sum);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) red[wave] = sum;
    __syncthreads();
    sum = ((red[0] + red[1]) + (red[2] + red[3])) + ((red[4] + red[5]) + (red[6] + red[7]));
    // X scaled as its h is; M, whose rows are few, needs no scale
    const double inv = sum <= 0x1.fffffffffffffp1023 ? (double)kScaleX / (sqrt(sum) + (double)a.eps) : (double)NAN;
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const bool inside = 16 * rb + l16 < r;
#pragma unroll
            for (int e = 0; e < 4; ++e)               // (zeros behind the edges also where inv is no number)
                x[j][rb][e] = inside && 16 * (8 * j + wave) + 4 * quad + e < c ? (float)((double)x[j][rb][e] * inv) : 0.f;
        }

    const int bi = wave / kPerRow * BI, bj = wave % kPerRow * BJ;     // this wavefront's blocks of A: from (bi, bj) on
    const bool has_blocks = bi < RB;
    const int frag = l16 * pitch + 8 * quad, frag_a = l16 * S::kPitchA + 8 * quad;
    // blocks (bi + y, bj + z) += P Q^T over columns k to k + 31, whose fragments lie at p and q
    auto blocks_product = [&](f32x4 (&g)[BI][BJ], const CCE_LDS _Float16* p, const CCE_LDS _Float16* q, int pitch_p, int k) {
        f16x8 m[BI];
#pragma unroll
        for (int y = 0; y < BI; ++y) m[y] = *(const CCE_LDS f16x8*)(p + 16 * (bi + y) * pitch_p + k);
#pragma unroll
        for (int z = 0; z < BJ; ++z) {
            const f16x8 n = *(const CCE_LDS f16x8*)(q + 16 * (bj + z) * pitch_p + k);
#pragma unroll
            for (int y = 0; y < BI; ++y) g[y][z] = __builtin_amdgcn_mfma_f32_16x16x32_f16(m[y], n, g[y][z], 0, 0, 0);
        }
    };
    for (int s = 0; s < a.steps; ++s) {
        auto of_lane = [&](int i) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(coefficient), i)); };
        const float ca = of_lane(3 * s), cb = of_lane(3 * s + 1), cc = of_lane(3 * s + 2);
        asm volatile("" : "+s"(mine));                // (comparisons with it are made where they are needed: kept over the loop they were spilled)
        auto write_h = [&]() {
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if (j >= mine) continue;
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    *(CCE_LDS f16x4*)(H + (16 * rb + l16) * pitch + 16 * (8 * j + wave) + 4 * quad) = half4(x[j][rb]);
            }
        };
        f32x4 g[BI][BJ];
        f16x4 o[BI][BJ];
#pragma unroll
        for (int y = 0; y < BI; ++y)
#pragma unroll
            for (int z = 0; z < BJ; ++z) g[y][z] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (S::kOwnSums) {
            // Two block columns of a wavefront are a fragment as they lie in its registers (which of its k an element is does not matter, it is
            // the same one in both operands): sums over its own columns of the blocks on and below the diagonal, without LDS.  Then the
            // eight sums of each block through LDS: 64 x 256 in 23 us, 48 matrices of 16 x 896 in 29 when every wavefront read all of h.
            f32x4 part[S::kPairs];
#pragma unroll
            for (int p = 0; p < S::kPairs; ++p) part[p] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < NB; j += 2) {
                if (j >= mine) continue;
                f16x8 h[RB], l[RB];
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    const f16x4 lo = half4(x[j][rb]), hi = half4(x[j + 1][rb]);
                    h[rb] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    if constexpr (S::kWhole) l[rb] = __builtin_shufflevector(rest4(x[j][rb], lo), rest4(x[j + 1][rb], hi), 0, 1, 2, 3, 4, 5, 6, 7);
                }
#pragma unroll
                for (int y = 0; y < RB; ++y)
#pragma unroll
                    for (int z = 0; z <= y; ++z) {
                        f32x4& to = part[y * (y + 1) / 2 + z];
                        if constexpr (S::kWhole) {
                            to = __builtin_amdgcn_mfma_f32_16x16x32_f16(h[y], l[z], to, 0, 0, 0);
                            to = __builtin_amdgcn_mfma_f32_16x16x32_f16(l[y], h[z], to, 0, 0, 0);
                        }
                        to = __builtin_amdgcn_mfma_f32_16x16x32_f16(h[y], h[z], to, 0, 0, 0);
                    }
            }
            if (!apart) __syncthreads();               // h is not needed any more
#pragma unroll
            for (int p = 0; p < S::kPairs; ++p) *(CCE_LDS f32x4*)(sums + (wave * S::kPairs + p) * 256 + 4 * lane) = part[p];
            __syncthreads();
        } else {
            write_h();
            __syncthreads();
        }
        if constexpr (S::kOwnSums) {
#pragma unroll
            for (int p0 = 0; p0 < S::kPairs; p0 += 8) {
                const int p = p0 + wave;
                if (p >= S::kPairs) continue;
                const int y = p >= 6 ? 3 : p >= 3 ? 2 : p >= 1 ? 1 : 0, z = p - y * (y + 1) / 2;
                f32x4 v[8];
#pragma unroll
                for (int w = 0; w < 8; ++w) v[w] = *(const CCE_LDS f32x4*)(sums + (w * S::kPairs + p) * 256 + 4 * lane);
                const f32x4 sum = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
                // element e: column 16 y + 4 quad + e of row 16 z + l16
                f32x4 beside;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float value = sum[e] * (1.f / (kScaleX * kScaleX));
                    const bool diagonal = y == z && 4 * quad + e == l16;
                    if (diagonal) da[16 * y + l16] = value;
                    beside[e] = diagonal ? 0.f : value * kScaleA;
                }
                auto place = [&](CCE_LDS _Float16* to, const f16x4& v) {
                    *(CCE_LDS f16x4*)(to + (16 * z + l16) * S::kPitchA + 16 * y + 4 * quad) = v;
                    if (y != z)
#pragma unroll
                        for (int e = 0; e < 4; ++e) to[(16 * y + 4 * quad + e) * S::kPitchA + 16 * z + l16] = v[e];
                };
                const f16x4 of_a = half4(beside);
                place(A, of_a);
                if constexpr (S::kWhole) place(A_rest, rest4(beside, of_a));
            }
        } else if (has_blocks) {
            for (int k = 0; k < columns; k += 64) {
                blocks_product(g, H + frag, H + frag, pitch, k);
                blocks_product(g, H + frag, H + frag, pitch, k + 32);
            }
            // element e of a block: column 16 (bi + y) + 4 quad + e of row 16 (bj + z) + l16
#pragma unroll
            for (int y = 0; y < BI; ++y)
#pragma unroll
                for (int z = 0; z < BJ; ++z) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = g[y][z][e] * (1.f / (kScaleX * kScaleX));
                        const bool diagonal = 16 * (bi + y) + 4 * quad + e == 16 * (bj + z) + l16;
                        if (diagonal) da[16 * (bi + y) + 4 * quad + e] = v;
                        o[y][z][e] = diagonal ? (_Float16)0.f : (_Float16)(v * kScaleA);
                        g[y][z][e] = 0.f;
                    }
                    *(CCE_LDS f16x4*)(A + (16 * (bj + z) + l16) * S::kPitchA + 16 * (bi + y) + 4 * quad) = o[y][z];
                }
        }
        __syncthreads();
        if (has_blocks) {
#pragma unroll
            for (int k = 0; k < S::kRows; k += 32) {
                blocks_product(g, A + frag_a, A + frag_a, S::kPitchA, k);
                if constexpr (S::kWhole) {
                    blocks_product(g, A + frag_a, A_rest + frag_a, S::kPitchA, k);
                    blocks_product(g, A_rest + frag_a, A + frag_a, S::kPitchA, k);
                }
            }
        }
        if constexpr (S::kOwnSums) write_h();
        else __syncthreads();                          // M takes A's place
        if (has_blocks) {
            if constexpr (S::kOwnSums) {
#pragma unroll
                for (int z = 0; z < BJ; ++z) o[0][z] = *(const CCE_LDS f16x4*)(A + (16 * (bj + z) + l16) * S::kPitchA + 16 * bi + 4 * quad);
            }
#pragma unroll
            for (int y = 0; y < BI; ++y) {
                const f32x4 dc = *(const CCE_LDS f32x4*)(da + 16 * (bi + y) + 4 * quad);
#pragma unroll
                for (int z = 0; z < BJ; ++z) {
                    const float dn = da[16 * (bj + z) + l16];
                    f32x4 beside;
                    f16x4 rest = {};
                    if constexpr (S::kWhole) rest = *(const CCE_LDS f16x4*)(A_rest + (16 * (bj + z) + l16) * S::kPitchA + 16 * (bi + y) + 4 * quad);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int col = 16 * (bi + y) + 4 * quad + e;
                        const bool diagonal = col == 16 * (bj + z) + l16;
                        const float p = g[y][z][e] * (cc / (kScaleA * kScaleA));
                        const float v = (cb + cc * (dn + dc[e])) * (((float)o[y][z][e] + (float)rest[e]) * (1.f / kScaleA)) + p;
                        float d = cb * dn + (cc * dn * dn + p), of_h = 0.f;
                        if (!S::kOwnSums && (a.apart >> s & 1u)) {
                            of_h = (float)(_Float16)d;
                            d -= of_h;
                        }
                        if (diagonal) dm[col] = d;
                        beside[e] = diagonal ? of_h : v;
                    }
                    const f16x4 m = half4(beside);
                    *(CCE_LDS f16x4*)(M + (16 * (bj + z) + l16) * S::kPitchA + 16 * (bi + y) + 4 * quad) = m;
                    if constexpr (S::kWhole)
                        *(CCE_LDS f16x4*)(M_rest + (16 * (bj + z) + l16) * S::kPitchA + 16 * (bi + y) + 4 * quad) = rest4(beside, m);
                }
            }
        }
        __syncthreads();
        asm volatile("" : "+s"(mine));
        float keep[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) keep[rb] = ca + dm[16 * rb + l16];
        // 8 rows of a column a lane, from k on, by transpose reads
        auto column_rows = [&](int j, int k) {
            const CCE_LDS _Float16* const p = H + (k + 8 * quad + (l16 >> 2)) * pitch + 16 * (8 * j + wave) + 4 * (l16 & 3);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((CCE_LDS s16x4*)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((CCE_LDS s16x4*)(p + 4 * pitch));
            return __builtin_bit_cast(f16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        if constexpr (S::kOwnSums) {
            // Products of M with h, and with what X has beyond it, which takes h's place: with h alone the diagonal of M, which acts on X itself, and
            // the rest of M would not act on the same matrix, and what M leaves of X's smallest directions is the small difference of both.
            constexpr int KB = S::kRows / 32;
            f16x8 m[KB][RB], m_rest[KB][RB];
#pragma unroll
            for (int k = 0; k < KB; ++k)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    m[k][rb] = *(const CCE_LDS f16x8*)(M + 16 * rb * S::kPitchA + frag_a + 32 * k);
                    if constexpr (S::kWhole) m_rest[k][rb] = *(const CCE_LDS f16x8*)(M_rest + 16 * rb * S::kPitchA + frag_a + 32 * k);
                }
#pragma unroll
            for (int j0 = 0; j0 < NB; j0 += 2) {
                if (j0 >= mine) continue;
                f16x8 h[2][KB];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int k = 0; k < KB; ++k) h[j][k] = column_rows(j0 + j < mine ? j0 + j : j0, 32 * k);
                wave_lds_order();
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (j0 + j >= mine) continue;
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) {
                        f32x4& v = x[j0 + j][rb];
                        *(CCE_LDS f16x4*)(H + (16 * rb + l16) * pitch + 16 * (8 * (j0 + j) + wave) + 4 * quad) = rest4(v, half4(v));
                        v *= keep[rb];
#pragma unroll
                        for (int k = 0; k < KB; ++k) {
                            v = __builtin_amdgcn_mfma_f32_16x16x32_f16(h[j][k], m[k][rb], v, 0, 0, 0);
                            if constexpr (S::kWhole) v = __builtin_amdgcn_mfma_f32_16x16x32_f16(h[j][k], m_rest[k][rb], v, 0, 0, 0);
                        }
                    }
                }
            }
            wave_lds_order();
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if (j >= mine) continue;
#pragma unroll
                for (int k = 0; k < KB; ++k) {
                    const f16x8 l = column_rows(j, 32 * k);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) x[j][rb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(l, m[k][rb], x[j][rb], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if (j >= mine) continue;
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) x[j][rb] *= keep[rb];
            }
#pragma unroll
            for (int k = 0; k < S::kRows; k += 32) {
                f16x8 m[RB];
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) m[rb] = *(const CCE_LDS f16x8*)(M + 16 * rb * S::kPitchA + frag_a + k);
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    if (j >= mine) continue;
                    const f16x8 h = column_rows(j, k);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) x[j][rb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, m[rb], x[j][rb], 0, 0, 0);
                }
            }
        }
    }
    if constexpr (WAY == kStaged) __syncthreads();     // the stages lie over other wavefronts' columns
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        if (j >= mine) continue;
        const int col = 16 * (8 * j + wave) + 4 * quad;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) x[j][rb] *= 1.f / kScaleX;
        if constexpr (WAY == kVectors) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int at = (16 * rb + l16) * t.cols + col;
                if (16 * rb + l16 < r && col < c) give4(t, at, param4(t, at, 4, true), x[j][rb], 4, true);
            }
        } else if constexpr (WAY == kColumns) {
            f32x4 p[RB];
            if (t.param) each([&](int rb, int e, int at) { p[rb][e] = t.param[at]; }, j);
            each([&](int rb, int e, int at) {
                float y = x[j][rb][e];
                if (t.param) {
                    y = p[rb][e] * t.decay - t.lr * y;
                    t.param[at] = y;
                }
                if (t.out) t.out[at] = bf16_bits(y);
            }, j);
        } else {
            wave_lds_order();
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int e = 0; e < 4; ++e) stage[(16 * rb + l16) * S::kStagePitch + 4 * quad + e] = x[j][rb][e];
            wave_lds_order();
            staged(j, [&](int at, CCE_LDS float& from) {
                float y = from;
                if (t.param) {
                    y = t.param[at] * t.decay - t.lr * y;
                    t.param[at] = y;
                }
                if (t.out) t.out[at] = bf16_bits(y);
            });
        }
    }
}

// ------------------------------------------------------------------------------------------
// Up to 64 rows, more columns than a workgroup takes.  Every step's polynomial is one of the first A = X X^T: with S = a + b A + c A A the
// next A is S A S, and the result Q X, where Q is the product of all S.  So X is read twice and written once, in three launches:
//
//   gram    momentum, and the sums of G G^T over a part of the columns each workgroup
//   steps   a workgroup a matrix: joins the sums, |G| from their diagonal, the steps on r x r matrices
//   apply   Q X, to the caller
//
// A direction that a step moves has its share of A amplified by up to the steps' square (2e5 for 3.4445^5), an error of A with
// it: 1e-7 of fp32 would show where |G|'s largest directions are 500 times the others'.  The r x r matrices are held and multiplied in 64
// bits, X and Q in 32.
// 16 x 4096 takes 23 us, 48 matrices of 16 x 14336 (66 MB in and out) 50 us on the GPU (17 + 11 + 22), 8 of 64 x 4096 76 (13 + 44 + 17: the steps
// are bound by the latency and rate of 64-bit products on a CU).  The tiled path, whose first product has one workgroup a matrix here, took
// 300, 1108 and 268 (of 48 rows) us.
// ------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(4))) double f64x4;
constexpr int64_t kThinRows = 64;
constexpr int kThinThreads = 256, kThinStepThreads = 512;
constexpr int kThinParts = 64;                         // workgroups that sum a matrix, at most
constexpr int kThinColumns = 256;                      // columns of one, more where that gives too many

struct NsThinArgs {
    NsArgs a;
    float coefficients[CCE_NS_MAX_STEPS][3];
    int32_t steps;
};
static_assert(sizeof(NsThinArgs) <= 4096, "kernel arguments hold 4 KB");

// Where a matrix's sums and Q lie, in bytes behind its base.
struct ThinLayout {
    int r, c, blocks, parts, columns;                  // blocks of 16 rows; columns of a part
    uint64_t q, inv, bytes;
    __host__ __device__ __forceinline__ ThinLayout(int rows, int cols) {
        r = rows < cols ? rows : cols;
        c = rows < cols ? cols : rows;
        blocks = r <= 16 ? 1 : r <= 32 ? 2 : 4;
        parts = c / kThinColumns < kThinParts ? (c + kThinColumns - 1) / kThinColumns : kThinParts;
        columns = ((c + parts - 1) / parts + 63) & ~63;
        parts = (c + columns - 1) / columns;
        q = (uint64_t)parts * (uint64_t)(blocks * (blocks + 1) / 2) * 2048;
        inv = q + (uint64_t)(blocks * blocks) * 1024;
        bytes = inv + 256;
    }
};

// Row of element e of a 64-bit matrix instruction's result.
__device__ __forceinline__ int f64_row(int quad, int e) { return 4 * e + quad; }

// Momentum, and the sums of G G^T over the columns of a wavefront: 16 from `begin` on, and every `step` columns, up to `end`.
template <int RB, class Args>
__device__ __forceinline__ void thin_sums(const Args& a, const NsMatrix& t, bool bf16, int begin, int step, int end, f64x4 (&sum)[RB * (RB + 1) / 2]) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4, r = t.rows < t.cols ? t.rows : t.cols;
    const bool tall = t.rows > t.cols, vec = !tall && (t.cols & 3) == 0 && aligned(t.grad, bf16 ? 8 : 16) && aligned(t.momentum, 16);
    const float clip = a.clip_coef ? a.clip_coef[0] : 1.f;
#pragma unroll
    for (int p = 0; p < RB * (RB + 1) / 2; ++p) sum[p] = f64x4{0.0, 0.0, 0.0, 0.0};
    // a trip's loads are in flight during the products of the trip before
    f32x4 g[RB], m[RB];
    auto place = [&](int row, int col) { return tall ? (int64_t)col * t.cols + row : (int64_t)row * t.cols + col; };
    auto load = [&](int col0) {
        const int col = col0 + 4 * quad;
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int row = 16 * rb + l16;
            g[rb] = m[rb] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (row >= r || col >= end) continue;
            if (vec) {
                g[rb] = grad_values(t.grad, bf16, place(row, col));
                if (t.momentum) m[rb] = *(const f32x4*)(t.momentum + place(row, col));
                continue;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int64_t i = place(row, col + e < end ? col + e : col);
                g[rb][e] = grad_value(t.grad, bf16, i);
                if (t.momentum) m[rb][e] = t.momentum[i];
            }
        }
    };
    load(begin);
    for (int col0 = begin; col0 < end; col0 += step) {
        const int col = col0 + 4 * quad;
        f32x4 x[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            const int row = 16 * rb + l16;
            x[rb] = g[rb];
            if (t.momentum) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float clipped = g[rb][e] * clip;
                    m[rb][e] = new_momentum(m[rb][e], clipped, a.mu);
                    x[rb][e] = direction(m[rb][e], clipped, a.mu, a.nesterov);
                }
                if (row < r && col < end) {
                    if (vec) *(f32x4*)(t.momentum + place(row, col)) = m[rb];
                    else
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (col + e < end) t.momentum[place(row, col + e)] = m[rb][e];
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) x[rb][e] = row < r && col + e < end ? x[rb][e] : 0.f;
        }
        load(col0 + step);
        // which column an instruction's k is does not matter, it is the same one in both operands
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            double v[RB];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) v[rb] = (double)x[rb][e];
#pragma unroll
            for (int y = 0; y < RB; ++y)
#pragma unroll
                for (int z = 0; z <= y; ++z)
                    sum[y * (y + 1) / 2 + z] = __builtin_amdgcn_mfma_f64_16x16x4f64(v[y], v[z], sum[y * (y + 1) / 2 + z], 0, 0, 0);
        }
    }
}

template <int RB>
__device__ __forceinline__ void thin_gram(const NsArgs& a, const NsMatrix& t, bool bf16, const ThinLayout& at, int part, CCE_LDS double* red) {
    constexpr int kPairs = RB * (RB + 1) / 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    f64x4 sum[kPairs];
    thin_sums<RB>(a, t, bf16, part * at.columns + 16 * wave, 64, (part + 1) * at.columns < at.c ? (part + 1) * at.columns : at.c, sum);
#pragma unroll
    for (int p = 0; p < kPairs; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) red[(wave * kPairs + p) * 256 + 64 * e + lane] = sum[p][e];
    __syncthreads();
    double* const to = (double*)(a.ws + t.base) + (size_t)part * (kPairs * 256);
    for (int i = threadIdx.x; i < kPairs * 256; i += kThinThreads)
        to[i] = (red[i] + red[kPairs * 256 + i]) + (red[2 * kPairs * 256 + i] + red[3 * kPairs * 256 + i]);
}
constexpr int kThinGramLds = 4 * 10 * 256 * 8;

__global__ __launch_bounds__(kThinThreads, 2) void ns_thin_gram_kernel(const NsArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    CCE_LDS double* const red = (CCE_LDS double*)smem_generic;
    const int i = matrix_of(a.first, (int)a.count, 2 * blockIdx.x + 1);
    const NsMatrix& t = a.t[i];
    const bool bf16 = (a.first[i] & 1u) != 0u;
    const ThinLayout at(t.rows, t.cols);
    const int part = (int)(blockIdx.x - (a.first[i] >> 1));
    if (at.blocks == 1) thin_gram<1>(a, t, bf16, at, part, red);
    else if (at.blocks == 2) thin_gram<2>(a, t, bf16, at, part, red);
    else thin_gram<4>(a, t, bf16, at, part, red);
}

// Q from G G^T in A, and what scales G to X.  The r x r matrices lie in LDS, symmetric up to their rounding, so that either operand's fragments are
// read along rows.  Of Q each wavefront has its blocks (thin_block), in registers.
template <int RB> constexpr int kThinPitch = 16 * RB + 8;
template <int RB> constexpr int kThinBlocks = RB == 4 ? 2 : 1;           // of a wavefront, beside each other
template <int RB>
__device__ __forceinline__ void thin_polynomial(const float (&coefficients)[CCE_NS_MAX_STEPS][3], int steps, float eps, int threads, CCE_LDS double* lds,
                                                f64x4 (&q)[kThinBlocks<RB>], double& inv) {
    constexpr int R = 16 * RB, P = kThinPitch<RB>, BZ = kThinBlocks<RB>;
    const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    CCE_LDS double* const A = lds;
    CCE_LDS double* const S = A + R * P;
    CCE_LDS double* const U = S + R * P;
    CCE_LDS double* const Q = U + R * P;
    CCE_LDS double* const trace = Q + R * P;
    __syncthreads();
    if (wave == 0) {
        double d = lane < R ? A[lane * P + lane] : 0.0;
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) d += __shfl_xor(d, o);
        if (lane == 0) trace[0] = d;
    }
    __syncthreads();
    const double sum = trace[0];
    inv = sum <= 0x1.fffffffffffffp1023 ? 1.0 / (sqrt(sum) + (double)eps) : (double)NAN;
    for (int i = threadIdx.x; i < R * R; i += threads) A[i / R * P + i % R] *= inv * inv;
    __syncthreads();
    const int by = wave * BZ / RB, bz = wave * BZ % RB;               // this wavefront's blocks: (by, bz), and the next
    const bool has = by < RB;
    auto product = [&](const CCE_LDS double* x, const CCE_LDS double* y, f64x4 (&g)[BZ]) {
#pragma unroll
        for (int b = 0; b < BZ; ++b) g[b] = f64x4{0.0, 0.0, 0.0, 0.0};
        if (!has) return;
#pragma unroll
        for (int k0 = 0; k0 < R; k0 += 4) {
            const int k = k0 + quad;
            const double v = x[k * P + 16 * by + l16];
#pragma unroll
            for (int b = 0; b < BZ; ++b) g[b] = __builtin_amdgcn_mfma_f64_16x16x4f64(v, y[k * P + 16 * (bz + b) + l16], g[b], 0, 0, 0);
        }
    };
    auto place = [&](int b, int e) { return (16 * by + f64_row(quad, e)) * P + 16 * (bz + b) + l16; };
    auto write = [&](CCE_LDS double* to, const f64x4 (&g)[BZ]) {
        if (!has) return;
#pragma unroll
        for (int b = 0; b < BZ; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) to[place(b, e)] = g[b][e];
    };
    for (int s = 0; s < steps; ++s) {
        const double ca = coefficients[s][0], cb = coefficients[s][1], cc = coefficients[s][2];
        f64x4 g[BZ];
        product(A, A, g);
        if (has) {
#pragma unroll
            for (int b = 0; b < BZ; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    g[b][e] = fma(cc, g[b][e], cb * A[place(b, e)]) + (by == bz + b && f64_row(quad, e) == l16 ? ca : 0.0);
        }
        write(S, g);
        __syncthreads();
        if (s == 0) {
#pragma unroll
            for (int b = 0; b < BZ; ++b) q[b] = g[b];
        } else {
            product(S, Q, q);
        }
        if (s + 1 == steps) break;
        product(S, A, g);
        write(U, g);
        __syncthreads();
        write(Q, q);
        product(S, U, g);
        write(A, g);
        __syncthreads();
    }
}

// q(row, column) of this wavefront's blocks
template <int RB, class Element>
__device__ __forceinline__ void thin_block(const f64x4 (&q)[kThinBlocks<RB>], Element element) {
    constexpr int BZ = kThinBlocks<RB>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (wave * BZ / RB >= RB) return;
#pragma unroll
    for (int b = 0; b < BZ; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) element(16 * (wave * BZ / RB) + f64_row(lane >> 4, e), 16 * (wave * BZ % RB + b) + (lane & 15), (float)q[b][e]);
}

template <int RB>
__device__ __forceinline__ void thin_steps(const NsThinArgs& args, const NsMatrix& t, const ThinLayout& at, CCE_LDS double* A) {
    constexpr int R = 16 * RB, P = kThinPitch<RB>, kPairs = RB * (RB + 1) / 2;
    char* const base = args.a.ws + t.base;
    for (int i = threadIdx.x; i < kPairs * 256; i += kThinStepThreads) {
        const double* from = (const double*)base + i;
        double sum = 0.0;
        for (int k0 = 0; k0 < at.parts; k0 += 8) {
            double v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = k0 + k < at.parts ? from[(size_t)(k0 + k) * (kPairs * 256)] : 0.0;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += v[k];
        }
        const int p = i >> 8, y = p >= 6 ? 3 : p >= 3 ? 2 : p >= 1 ? 1 : 0, z = p - y * (y + 1) / 2;
        const int row = 16 * y + f64_row((i & 63) >> 4, (i & 255) >> 6), col = 16 * z + (i & 15);
        A[row * P + col] = sum;
        if (y != z) A[col * P + row] = sum;
    }
    f64x4 q[kThinBlocks<RB>];
    double inv;
    thin_polynomial<RB>(args.coefficients, args.steps, args.a.eps, kThinStepThreads, A, q, inv);
    float* const out = (float*)(base + at.q);
    thin_block<RB>(q, [&](int row, int col, float x) { out[row * R + col] = x; });
    if (threadIdx.x == 0) *(double*)(base + at.inv) = inv;
}
constexpr int thin_step_lds(int blocks) { return (4 * 16 * blocks * (16 * blocks + 8) + 1) * 8; }
static_assert(thin_step_lds(4) <= 160 * 1024, "160 KB LDS");

__global__ __launch_bounds__(kThinStepThreads, 2) void ns_thin_steps_kernel(const NsThinArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    CCE_LDS double* const lds = (CCE_LDS double*)smem_generic;
    const NsMatrix& t = a.a.t[blockIdx.x];
    const ThinLayout at(t.rows, t.cols);
    if (at.blocks == 1) thin_steps<1>(a, t, at, lds);
    else if (at.blocks == 2) thin_steps<2>(a, t, at, lds);
    else thin_steps<4>(a, t, at, lds);
}

// 64 columns a wavefront, as four sets of 16: of a wide matrix set s is every fourth column from the s-th on, so that a lane has four
// neighbours of a row in memory; of a tall one 16 neighbouring columns, of which a lane has four neighbouring rows.
template <int RB, class Args, class Row>
__device__ __forceinline__ void thin_columns(const Args& a, const NsMatrix& t, bool bf16, double inv, Row q_of, int c0) {
    const int r = t.rows < t.cols ? t.rows : t.cols, c = t.rows < t.cols ? t.cols : t.rows;
    const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
    const bool tall = t.rows > t.cols, vec_in = (t.cols & 3) == 0 && aligned(t.grad, bf16 ? 8 : 16) && aligned(t.momentum, 16);
    const bool vec_out = (t.cols & 3) == 0 && aligned(t.param, 16) && aligned(t.out, 8);
    const float clip = a.clip_coef ? a.clip_coef[0] : 1.f;
    // four neighbours in memory: of line `line` of the caller's matrix from `in` on, `left` of them there
    auto four = [&](int line, int in, int left) {
        const int64_t i = (int64_t)line * t.cols + in;
        f32x4 u = {0.f, 0.f, 0.f, 0.f};
        if (vec_in && left >= 4) {
            u = grad_values(t.grad, bf16, i);
            if (t.momentum) {
                const f32x4 m = *(const f32x4*)(t.momentum + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) u[e] = direction(m[e], u[e] * clip, a.mu, a.nesterov);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (e >= left) continue;
                u[e] = grad_value(t.grad, bf16, i + e);
                if (t.momentum) u[e] = direction(t.momentum[i + e], u[e] * clip, a.mu, a.nesterov);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = e < left ? (float)((double)u[e] * inv) : 0.f;
        return u;
    };
    f32x4 x[RB][4];                                    // [t][e][s] wide, [t][s][e] tall: row 16 t + 4 quad + e, set s
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = 16 * b + 4 * quad + (tall ? 0 : k), col = c0 + (tall ? 16 * k + l16 : 4 * l16);
            const int left = row < r && col < c ? (tall ? r - row : c - col) : 0;
            x[b][k] = tall ? four(col, row, left) : four(row, col, left);
        }
    f32x4 q[RB];
#pragma unroll
    for (int ro = 0; ro < RB; ++ro) {
#pragma unroll
        for (int b = 0; b < RB; ++b) q[b] = q_of(16 * ro + l16, 16 * b + 4 * quad);
        f32x4 p[4];
        int left[4];
        int64_t to[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = 16 * ro + 4 * quad + (tall ? 0 : k), col = c0 + (tall ? 16 * k + l16 : 4 * l16);
            const bool there = row < r && col < c;
            left[k] = there ? (tall ? r - row : c - col) : 0;
            to[k] = !there ? 0 : tall ? (int64_t)col * t.cols + row : (int64_t)row * t.cols + col;
            p[k] = param4(t, to[k], left[k], vec_out);
        }
        f32x4 y[4];                                    // of each set: rows 16 ro + 4 quad + g of column l16
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            y[s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    y[s] = __builtin_amdgcn_mfma_f32_16x16x4f32(q[b][e], tall ? x[b][s][e] : x[b][e][s], y[s], 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (left[k] == 0) continue;
            give4(t, to[k], p[k], tall ? y[k] : f32x4{y[0][k], y[1][k], y[2][k], y[3][k]}, left[k], vec_out);
        }
    }
}

template <int RB>
__device__ __forceinline__ void thin_apply(const NsArgs& a, const NsMatrix& t, bool bf16, const ThinLayout& at, int c0) {
    const char* const base = a.ws + t.base;
    const float* const Q = (const float*)(base + at.q);
    thin_columns<RB>(a, t, bf16, *(const double*)(base + at.inv), [&](int row, int col) { return *(const f32x4*)(Q + row * (16 * RB) + col); }, c0);
}

__global__ __launch_bounds__(kThinThreads, 2) void ns_thin_apply_kernel(const NsArgs a) {
    const int i = matrix_of(a.first, (int)a.count, 2 * blockIdx.x + 1);
    const NsMatrix& t = a.t[i];
    const bool bf16 = (a.first[i] & 1u) != 0u;
    const ThinLayout at(t.rows, t.cols);
    const int c0 = ((int)(blockIdx.x - (a.first[i] >> 1)) * (kThinThreads / 64) + (int)(threadIdx.x >> 6)) * 64;
    if (c0 >= at.c) return;
    if (at.blocks == 1) thin_apply<1>(a, t, bf16, at, c0);
    else if (at.blocks == 2) thin_apply<2>(a, t, bf16, at, c0);
    else thin_apply<4>(a, t, bf16, at, c0);
}

// Code for the matrix's columns and its way in and out: as one piece of code for all it takes 3 us longer, a half of it 1 us.
template <int WAY>
__device__ __forceinline__ void small_matrix_of(const NsSmallArgs& a, const NsMatrix& t, bool bf16, CCE_LDS char* smem) {
    const int r = t.rows < t.cols ? t.rows : t.cols, c = t.rows < t.cols ? t.cols : t.rows;
    if (r <= 32) {
        if (c <= 256) small_matrix<SmallShape<2, 2>, WAY>(a, t, bf16, smem);
        else small_matrix<Small32, WAY>(a, t, bf16, smem);
    } else if (r <= 64) {
        if (c <= 256) small_matrix<SmallShape<4, 2>, WAY>(a, t, bf16, smem);
        else if (c <= 512) small_matrix<SmallShape<4, 4>, WAY>(a, t, bf16, smem);
        else small_matrix<Small64, WAY>(a, t, bf16, smem);
    } else {
        if (c <= 256) small_matrix<SmallShape<8, 2>, WAY>(a, t, bf16, smem);
        else small_matrix<Small128, WAY>(a, t, bf16, smem);
    }
}

// Up to 16 rows: as thin matrices are, in one launch.  With few values to a matrix the roundings of 16-bit operands need not even out: they left
// up to 3e-3 of a matrix of 5 x 7.  16 x 16 10 us with them, 11 here, 16 x 512 16 and 14.
__device__ __forceinline__ void tiny_matrix(const NsSmallArgs& a, const NsMatrix& t, bool bf16, CCE_LDS char* smem) {
    CCE_LDS double* const red = (CCE_LDS double*)smem;
    CCE_LDS double* const A = red + kSmallThreads / 64 * 256;
    CCE_LDS float* const Q = (CCE_LDS float*)red;
    const int c = t.rows < t.cols ? t.cols : t.rows, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    f64x4 sum[1], q[1];
    thin_sums<1>(a, t, bf16, 16 * wave, kSmallThreads / 4, c, sum);
#pragma unroll
    for (int e = 0; e < 4; ++e) red[wave * 256 + 64 * e + lane] = sum[0][e];
    __syncthreads();
    if (threadIdx.x < 256) {
        double x = red[threadIdx.x];
#pragma unroll
        for (int w = 1; w < kSmallThreads / 64; ++w) x += red[w * 256 + threadIdx.x];
        A[f64_row((int)(threadIdx.x & 63) >> 4, (int)threadIdx.x >> 6) * kThinPitch<1> + (int)(threadIdx.x & 15)] = x;
    }
    double inv;
    thin_polynomial<1>(a.coefficients, a.steps, a.eps, kSmallThreads, A, q, inv);
    thin_block<1>(q, [&](int row, int col, float x) { Q[row * 16 + col] = x; });
    __syncthreads();
    for (int c0 = 64 * wave; c0 < c; c0 += kSmallThreads)
        thin_columns<1>(a, t, bf16, inv, [&](int row, int col) { return *(const CCE_LDS f32x4*)(Q + row * 16 + col); }, c0);
}
constexpr int kTinyLds = (kSmallThreads / 64 * 256 + 4 * 16 * kThinPitch<1> + 1) * 8;

__global__ __launch_bounds__(kSmallThreads, 2) void ns_small_kernel(const NsSmallArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char smem_generic[];
    CCE_LDS char* const smem = (CCE_LDS char*)smem_generic;
    const NsMatrix& t = a.t[blockIdx.x];
    const bool bf16 = (a.bf16 >> blockIdx.x & 1u) != 0u;
    if (t.rows <= 16 || t.cols <= 16) tiny_matrix(a, t, bf16, smem);
    else if (t.rows > t.cols) small_matrix_of<kColumns>(a, t, bf16, smem);
    else if ((t.cols & 3) == 0 && aligned(t.grad, bf16 ? 8 : 16) && aligned(t.momentum, 16) && aligned(t.param, 16) && aligned(t.out, 8))
        small_matrix_of<kVectors>(a, t, bf16, smem);
    else small_matrix_of<kStaged>(a, t, bf16, smem);
}

// ------------------------------------------------------------------------------------------
// Host side.
// ------------------------------------------------------------------------------------------
static bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

static int check_sizes(const cce_matrix* matrices, int64_t count) {
    if (!matrices || count <= 0) return CCE_ERR_INVALID;
    for (int64_t i = 0; i < count; ++i) {
        const cce_matrix& t = matrices[i];
        if (t.rows < 0 || t.cols < 0) return CCE_ERR_INVALID;
        if (t.rows == 0 || t.cols == 0) continue;
        if (t.rows > kMaxMatrix || t.cols > kMaxMatrix || round_up(t.rows, 64) * round_up(t.cols, 64) > kMaxMatrix) return CCE_ERR_UNSUPPORTED;
        if (t.rows > kMaxSide && t.cols > kMaxSide) return CCE_ERR_UNSUPPORTED;
    }
    return CCE_OK;
}

static int check_gradients(const cce_matrix* matrices, int64_t count) {
    const int rc = check_sizes(matrices, count);
    if (rc != CCE_OK) return rc;
    for (int64_t i = 0; i < count; ++i) {
        const cce_matrix& t = matrices[i];
        if (t.rows == 0 || t.cols == 0) continue;
        if (t.reserved != 0 || (t.grad_bf16 != 0 && t.grad_bf16 != 1)) return CCE_ERR_INVALID;
        if (!t.grad || misaligned(t.grad, t.grad_bf16 ? 2 : 4)) return CCE_ERR_INVALID;
    }
    return CCE_OK;
}

// The largest |a x + b x^3 + c x^5| in [0, top]: at its end or where the derivative a + 3 b y + 5 c y^2, y = x^2, is 0.
static double largest_value(double a, double b, double c, double top) {
    double at[3] = {top, 0.0, 0.0};
    int n = 1;
    const double root = 9.0 * b * b - 20.0 * a * c;
    if (c != 0.0 && root >= 0.0) {
        const double y0 = (-3.0 * b - sqrt(root)) / (10.0 * c), y1 = (-3.0 * b + sqrt(root)) / (10.0 * c);
        if (y0 > 0.0 && y0 < top * top) at[n++] = sqrt(y0);
        if (y1 > 0.0 && y1 < top * top) at[n++] = sqrt(y1);
    } else if (c == 0.0 && b != 0.0) {
        const double y = -a / (3.0 * b);
        if (y > 0.0 && y < top * top) at[n++] = sqrt(y);
    }
    double next = 0.0;
    for (int k = 0; k < n; ++k) {
        const double x = at[k];
        next = fmax(next, fabs(a * x + b * x * x * x + c * x * x * x * x * x));
    }
    return next;
}

// Whether the steps keep singular values that begin at 1 or below within what the scales hold.
static int check_coefficients(const float* coefficients, int steps) {
    double top = 1.0;
    for (int s = 0; s < steps; ++s) {
        const double a = coefficients[3 * s], b = coefficients[3 * s + 1], c = coefficients[3 * s + 2];
        if (!(isfinite(a) && isfinite(b) && isfinite(c))) return CCE_ERR_INVALID;
        if (fabs(b) * top * top + fabs(c) * top * top * top * top > kMaxM) return CCE_ERR_UNSUPPORTED;
        const double next = largest_value(a, b, c, top);
        if (next > kMaxSigma) return CCE_ERR_UNSUPPORTED;
        top = fmax(next, 1e-6);
    }
    return CCE_OK;
}

// Whether S of the first two steps, and their product, stay within M's scale: singular values begin at 1 or below.
static bool may_pair(const float* coefficients, int steps) {
    if (steps < 2) return false;
    double top = 1.0, both = 1.0;
    for (int s = 0; s < 2; ++s) {
        const double a = coefficients[3 * s], b = coefficients[3 * s + 1], c = coefficients[3 * s + 2];
        const double vertex = c != 0.0 ? -b / (2.0 * c) : -1.0;
        double largest = fmax(fabs(a), fabs(a + b * top * top + c * top * top * top * top));
        if (vertex > 0.0 && vertex < top * top) largest = fmax(largest, fabs(a + b * vertex + c * vertex * vertex));
        both *= largest;
        if (largest > kMaxM || both > kMaxM) return false;
        top = largest_value(a, b, c, top);
    }
    return true;
}

// The steps in which all of M acts on h alone, and a on all of X.  What X has beyond h, l, then lacks M l, which has M's large directions and so is
// amplified by nothing.  Otherwise M's diagonal D acts on all of X, as it may in other steps: it lacks (M - D) l, which is less where M is mostly
// its diagonal, as of noise, but D l is along the smallest directions too, which the steps behind it amplify by the product of their a.
// Largest error of 130 x 130, from the oracle's rounded form, with D on X in all steps / from a factor of 41 on / 12 / in none apart: rank 1 5.0e-3 /
// 0.9 / 0.8, rank 32 2.4 / 2.0 / 1.1, noise 0.83 / 0.84 / 1.0 / 1.4: from 8 on.
constexpr double kAmplified = 8.0;
static uint32_t apart_steps(const float* coefficients, int steps) {
    uint32_t apart = 0;
    double behind = 1.0;
    for (int s = steps - 1; s >= 0; --s) {
        if (behind >= kAmplified) apart |= 1u << s;
        behind *= fabs((double)coefficients[3 * s]);
    }
    return apart;
}

static uint32_t sym_tiles(const NsLayout& at, bool large, bool whole) {
    const int side = large ? SymPing::BM : SymTile::BM;
    const uint32_t n = (uint32_t)((at.rp + side - 1) / side);
    return whole ? n * n : n * (n + 1) / 2;
}
static uint32_t apply_tiles(const NsLayout& at, bool large) {
    const int rows = large ? TurnTile::BN : ApplyTile::BN;
    return (uint32_t)((at.rp + rows - 1) / rows) * (uint32_t)((at.cp + ApplyTile::BM - 1) / ApplyTile::BM);
}
static_assert(ApplyTile::BM == TurnTile::BM, "either form of a launch covers as many columns");

template <class K>
static bool allow_lds(K kernel, int bytes) { return hip_ok(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes)); }

// LDS of a matrix that a workgroup takes alone; 0 of one for the tiled launches.
static int small_lds(const cce_matrix& t) {
    const int64_t r = t.rows < t.cols ? t.rows : t.cols, c = t.rows < t.cols ? t.cols : t.rows;
    if (c > small_columns(r)) return 0;
    return r <= 16 ? kTinyLds : r <= 32 ? Small32::lds((int)c) : r <= 64 ? Small64::lds((int)c) : Small128::lds((int)c);
}

static bool is_thin(const cce_matrix& t) { return (t.rows <= kThinRows || t.cols <= kThinRows) && small_lds(t) == 0; }

// The thin matrices from `i` on that share their launches; moves i behind them.  Returns their workspace.
template <class Take>
static int64_t next_thin_group(const cce_matrix* matrices, int64_t count, int64_t& i, Take take) {
    int64_t bytes = 0;
    int n = 0;
    for (; i < count && n < kEnds; ++i) {
        const cce_matrix& t = matrices[i];
        if (t.rows == 0 || t.cols == 0 || !is_thin(t)) continue;
        take(t, (uint64_t)bytes);
        ++n;
        bytes += (int64_t)ThinLayout((int)t.rows, (int)t.cols).bytes;
    }
    return bytes;
}

// Whether the first two steps of a matrix are taken as one, X = (S2 S1) X with A = S1 X X^T S1: a product of r c and one of 2 r c are
// saved for four of r r.  Not in later steps: the first A, whose trace is 1, takes its operands' rounding better than they do (2-norm of the
// error for 256 x 1024: of a matrix of noise 7.2e-4, 7.1 with the first two, 8.7 with the second and third; with a spectrum down to 1e-3 6.8,
// 6.8 and 9.1).  What they cost in accuracy is where few roundings count, see the head.  us without / with: 32 x 512 x 2048 655 / 627, 8 x 896 x 3584 730 / 683, 16 x 1024 x 4096 1768 / 1616, 4 x 1500 x 4096 975 / 936,
// 3584 x 14336 3385 / 3040, a 24-layer model 7657 / 7290; 512 x 1088 254 / 260, 1024 x 2176 375 / 379: nothing gained below 2.5 columns a row.
static bool pairs_steps(const cce_matrix& t) {
    const NsLayout at((int)t.rows, (int)t.cols);
    return at.rp >= kPairRows && 2 * at.cp >= 5 * at.rp;               // (S and T, and their diagonals, lie in a copy of h)
}

// The matrices from `i` on that share their launches; moves i behind them.  Returns their workspace.
template <class Take>
static int64_t next_group(const cce_matrix* matrices, int64_t count, bool pairs, int64_t& i, Take take) {
    int64_t bytes = 0;
    int n = 0;
    bool large = false;
    for (; i < count && n < kGroup; ++i) {
        const cce_matrix& t = matrices[i];
        if (t.rows == 0 || t.cols == 0 || small_lds(t) != 0 || is_thin(t) || pairs_steps(t) != pairs) continue;
        const NsLayout at((int)t.rows, (int)t.cols);
        if (n != 0 && bytes + (int64_t)at.bytes > kGroupBytes - kPartialBytes) break;
        take(t, (uint64_t)bytes);
        ++n;
        bytes += (int64_t)at.bytes;
        large = large || at.rp >= kLargeRows || at.cp >= kLongColumns;
    }
    return bytes + (large ? kPartialBytes : 0);
}

static NsMatrix table_entry(const cce_matrix& t, bool step, float lr, uint64_t base) {
    const float rate = lr * t.lr_scale;
    return NsMatrix{t.grad, step ? t.momentum : nullptr, step ? t.param : nullptr, (uint16_t*)t.out_bf16, base,
                    (int32_t)t.rows, (int32_t)t.cols, rate, 1.f - rate * t.weight_decay};
}

// The matrices that a workgroup takes alone.
static bool run_small(const cce_matrix* matrices, int64_t count, bool step, float lr, float mu, int nesterov, const float* coefficients,
                      int steps, float eps, const float* clip_coef, hipStream_t stream) {
    NsSmallArgs a;
    a.clip_coef = clip_coef;
    a.mu = mu;
    a.eps = eps;
    a.nesterov = nesterov;
    a.steps = steps;
    a.apart = apart_steps(coefficients, steps);
    for (int s = 0; s < 3 * steps; ++s) a.coefficients[s / 3][s % 3] = coefficients[s];
    for (int64_t i = 0; i < count;) {
        int n = 0, bytes = 0;
        a.bf16 = 0;
        for (; i < count && n < kSmallMatrices; ++i) {
            const cce_matrix& t = matrices[i];
            if (t.rows == 0 || t.cols == 0) continue;
            const int own = small_lds(t);
            if (own == 0) continue;
            bytes = own > bytes ? own : bytes;
            a.bf16 |= (uint64_t)t.grad_bf16 << n;
            a.t[n++] = table_entry(t, step, lr, 0);
        }
        if (n == 0) continue;
        if (!allow_lds(ns_small_kernel, 160 * 1024)) return false;
        hipLaunchKernelGGL(ns_small_kernel, dim3((unsigned)n), dim3(kSmallThreads), bytes, stream, a);
    }
    return true;
}

static bool run_thin(const cce_matrix* matrices, int64_t count, bool step, float lr, float mu, int nesterov, const float* coefficients,
                     int steps, float eps, const float* clip_coef, void* workspace, hipStream_t stream) {
    NsThinArgs args;
    NsArgs& a = args.a;
    a.ws = (char*)workspace;
    a.clip_coef = clip_coef;
    a.mu = mu;
    a.nesterov = nesterov;
    a.eps = eps;
    args.steps = steps;
    for (int s = 0; s < 3 * steps; ++s) args.coefficients[s / 3][s % 3] = coefficients[s];
    for (int64_t i = 0; i < count;) {
        a.count = 0;
        uint32_t blocks = 0, parts[kEnds], columns[kEnds], grads[kEnds];
        int most = 1;
        next_thin_group(matrices, count, i, [&](const cce_matrix& t, uint64_t base) {
            const ThinLayout at((int)t.rows, (int)t.cols);
            most = at.blocks > most ? at.blocks : most;
            a.t[a.count] = table_entry(t, step, lr, base);
            parts[a.count] = (uint32_t)at.parts;
            columns[a.count] = (uint32_t)(at.c + kThinThreads - 1) / kThinThreads;
            grads[a.count++] = (uint32_t)t.grad_bf16;
        });
        if (a.count == 0) continue;
        if (!allow_lds(ns_thin_gram_kernel, kThinGramLds) || !allow_lds(ns_thin_steps_kernel, thin_step_lds(4))) return false;
        auto place = [&](const uint32_t* per) {
            blocks = 0;
            for (uint32_t k = 0; k < a.count; ++k) {
                a.first[k] = 2 * blocks + grads[k];
                blocks += per[k];
            }
        };
        place(parts);
        hipLaunchKernelGGL(ns_thin_gram_kernel, dim3(blocks), dim3(kThinThreads), 4 * (most * (most + 1) / 2) * 2048, stream, a);
        hipLaunchKernelGGL(ns_thin_steps_kernel, dim3(a.count), dim3(kThinStepThreads), thin_step_lds(most), stream, args);
        place(columns);
        hipLaunchKernelGGL(ns_thin_apply_kernel, dim3(blocks), dim3(kThinThreads), 0, stream, a);
    }
    return true;
}

// Whether a launch takes tiles of 256 x 256, one workgroup a CU, or the smaller ones, two a CU: by the rounds of slices that either takes.
// A round of either does as many products a slice; smaller tiles that have a CU each take 0.6 of one.
// A and M: the last tiles of a round of 256 x 256 that is less than half full are split (p.splits), which costs a launch as long as 20 slices.
// X: an epilogue is as long as 12 slices, which only the smaller tiles put beside products; 256 x 256 from 2048 rows on.
// Few rows and many columns: the one or few tiles of gram split, 100 x 4096 319 -> 257 us, 100 x 14336 824 -> 347, 512 x 14336 841 -> 445.
// Smaller tiles / 256 x 256 in all launches of a kind, whole calls, us: gram of 4 x 4096 x 4096 6240 / 5930, of 3584 x 14336 3460 / 3350, of
// 1024 x 4096 470 / 423, of 2048 x 2048 498 / 558, of 64 x 640 x 640 923 / 931; apply of 4 x 4096 x 4096 5690 / 5280, of
// 12 x 2048 x 2048 2460 / 2310, of 2048 x 2048 498 / 542, of 6 x 1536 x 6144 1926 / 1948, of a 24-layer model's matrices 7520 / 7750.
template <class Length, class Tiles, class Layout>
static bool large_tiles(int op, int n, Length length, Tiles tiles, Layout layout, NsProductArgs& p) {
    constexpr uint32_t kCus = kResident / 2;
    double work[2] = {0.0, 0.0};
    uint32_t count[2] = {0, 0};
    int shortest = 1 << 30;
    bool any = false;
    p.split_tiles = 0;
    p.splits = 1;
    for (int k = 0; k < n; ++k) {
        if (op == 2 && layout(k).rp < kTurnRows) return false;
        any = any || layout(k).rp >= kLargeRows || (op == 0 && layout(k).cp >= kLongColumns);
        shortest = length(k) < shortest ? length(k) : shortest;
        for (int of_256 = 0; of_256 < 2; ++of_256) {
            const uint32_t t = tiles(k, of_256 != 0);
            work[of_256] += (double)t * length(k);
            count[of_256] += t;
        }
    }
    p.tiles = count[1];
    if (!any) return false;
    const double mean[2] = {work[0] / count[0], work[1] / count[1]};
    const double small_rounds = count[0] <= kCus ? 0.6 : ceil((double)count[0] / kResident);
    if (op == 2) return mean[1] >= 2048.0 && ceil((double)count[1] / kCus) <= small_rounds;
    const uint32_t left = count[1] % kCus, most = left ? kCus / left : 1, longest = (uint32_t)(shortest / SymPing::BK);
    uint32_t splits = most < longest ? most : longest;
    splits = splits < kMaxSplits ? splits : kMaxSplits;
    const double rounds = (double)(count[1] / kCus) + (left == 0 ? 0.0 : 1.0 / splits);
    if (rounds * mean[1] + (splits > 1 ? 20.0 * SymPing::BK : 0.0) >= small_rounds * mean[0]) return false;
    if (splits > 1) {
        p.split_tiles = left;
        p.splits = splits;
    }
    return true;
}

static int run_groups(const cce_matrix* matrices, int64_t count, bool step, float lr, float mu, int nesterov, const float* coefficients,
                      int steps, float eps, const float* clip_coef, void* workspace, hipStream_t stream) {
    bool any = false;
    for (int64_t i = 0; i < count; ++i) any = any || (matrices[i].rows != 0 && matrices[i].cols != 0);
    if (!any) return CCE_OK;                           // (nothing is asked of the device)
    if (!run_small(matrices, count, step, lr, mu, nesterov, coefficients, steps, eps, clip_coef, stream)) return CCE_ERR_HIP;
    if (!run_thin(matrices, count, step, lr, mu, nesterov, coefficients, steps, eps, clip_coef, workspace, stream)) return CCE_ERR_HIP;
    NsArgs a;
    NsProductArgs products[4];                         // gram, poly, apply, whole products
    a.ws = (char*)workspace;
    for (auto& p : products) p.ws = (char*)workspace;
    a.clip_coef = clip_coef;
    a.mu = mu;
    a.nesterov = nesterov;
    a.eps = eps;
    for (const bool pairs : {false, true})
    for (int64_t i = 0; i < count;) {
        int64_t index[kGroup];
        uint64_t base[kGroup];
        int n = 0;
        int64_t partials = 0;                          // behind the matrices
        next_group(matrices, count, pairs, i, [&](const cce_matrix& t, uint64_t at) {
            index[n] = &t - matrices;
            base[n++] = at;
            partials = (int64_t)at + (int64_t)NsLayout((int)t.rows, (int)t.cols).bytes;
        });
        if (n == 0) continue;
        if (!allow_lds(ns_symmetric_kernel<kGram>, kSymLds) || !allow_lds(ns_symmetric_kernel<kPoly>, kSymLds) ||
            !allow_lds(ns_symmetric_kernel<kProduct>, kSymLds) || !allow_lds(ns_symmetric_kernel<kWholeProduct>, kSymLds) ||
            !allow_lds(ns_symmetric_ping_kernel<kGram>, kPingLds) ||
            !allow_lds(ns_symmetric_ping_kernel<kPoly>, kPingLds) || !allow_lds(ns_symmetric_ping_kernel<kProduct>, kPingLds) ||
            !allow_lds(ns_symmetric_ping_kernel<kWholeProduct>, kPingLds) ||
            !allow_lds(ns_apply_kernel<false>, ApplyTile::kLdsBytes) || !allow_lds(ns_apply_kernel<true>, ApplyTile::kLdsBytes) ||
            !allow_lds(ns_apply_turn_kernel<false>, kTurnLds) || !allow_lds(ns_apply_turn_kernel<true>, kTurnLds))
            return CCE_ERR_HIP;
        auto layout = [&](int k) { return NsLayout((int)matrices[index[k]].rows, (int)matrices[index[k]].cols); };
        // launches over as many matrices as their arguments hold
        auto ends = [&](auto blocks_of, auto launch) {
            for (int k = 0; k < n;) {
                uint32_t blocks = 0;
                for (a.count = 0; k < n && a.count < (uint32_t)kEnds; ++k, ++a.count) {
                    const cce_matrix& t = matrices[index[k]];
                    a.t[a.count] = table_entry(t, step, lr, base[k]);
                    a.first[a.count] = 2 * blocks + (uint32_t)t.grad_bf16;
                    blocks += blocks_of(t, layout(k));
                }
                launch(blocks);
            }
        };
        // the matrices with the longest sums of a product first: the shorter ones fill what they leave
        uint32_t grid[4];
        bool large[4];
        for (int op = 0; op < (pairs ? 4 : 3); ++op) {
            NsProductArgs& p = products[op];
            int order[kGroup];
            auto length = [&](int x) { return op == 0 ? layout(x).cp : layout(x).rp; };
            auto tiles = [&](int x, bool of_256) { return op == 2 ? apply_tiles(layout(x), of_256) : sym_tiles(layout(x), of_256, op == 3); };
            for (int k = 0; k < n; ++k) {
                int to = k;
                for (; to > 0 && length(order[to - 1]) < length(k); --to) order[to] = order[to - 1];
                order[to] = k;
            }
            large[op] = large_tiles(op, n, length, tiles, layout, p);
            grid[op] = 0;
            p.count = (uint32_t)n;
            for (int k = 0; k < n; ++k) {
                const cce_matrix& t = matrices[index[order[k]]];
                p.t[k] = NsShape{(uint32_t)(base[order[k]] / 256), (int32_t)t.rows, (int32_t)t.cols};
                p.first[k] = 2 * grid[op];
                grid[op] += tiles(order[k], large[op]);
            }
            if (large[op]) grid[op] += p.split_tiles * (p.splits - 1);
            p.partials = (uint32_t)(partials / 256);
        }
        ends([](const cce_matrix& t, const NsLayout&) {
            const int64_t parts = (t.rows * t.cols + kNormValues - 1) / kNormValues;
            return (uint32_t)(parts < kNormParts ? parts : kNormParts);
        }, [&](uint32_t blocks) { hipLaunchKernelGGL(ns_norm_kernel, dim3(blocks), dim3(256), 0, stream, a); });
        ends([](const cce_matrix&, const NsLayout& at) { return (uint32_t)(at.rp / 64) * (uint32_t)(at.cp / 64); },
             [&](uint32_t blocks) { hipLaunchKernelGGL(ns_prep_kernel, dim3(blocks), dim3(256), 0, stream, a); });
        auto coefficients_of = [&](int s) {
            for (auto& p : products) {
                p.a = coefficients[3 * s];
                p.b = coefficients[3 * s + 1];
                p.c = coefficients[3 * s + 2];
            }
        };
        const uint32_t apart = apart_steps(coefficients, steps);
        int s = 0;
        auto symmetric = [&](auto mode, uint32_t kind) {
            constexpr int MODE = decltype(mode)::value;
            const int op = MODE == kGram ? 0 : MODE == kWholeProduct ? 3 : 1;
            NsProductArgs& p = products[op];
            p.kind = kind;
            p.apart = (kind == kOfA || kind == kBoth) ? apart >> s & 1u : 0u;
            p.on_x = kind == kBoth ? p.a * (coefficients[3 * (s - 1)] - 1.f) : 0.f;      // a of both steps, less what the apply has
            if (large[op]) hipLaunchKernelGGL(ns_symmetric_ping_kernel<MODE>, dim3(grid[op]), dim3(SymPing::kThreads), kPingLds, stream, p);
            else hipLaunchKernelGGL(ns_symmetric_kernel<MODE>, dim3(grid[op]), dim3(SymTile::kThreads), kSymLds, stream, p);
            if (large[op] && p.split_tiles) hipLaunchKernelGGL(ns_symmetric_join_kernel<MODE>, dim3(8 * p.split_tiles), dim3(64), 0, stream, p);
        };
        constexpr std::integral_constant<int, kGram> gram{};
        constexpr std::integral_constant<int, kPoly> poly{};
        constexpr std::integral_constant<int, kProduct> product{};
        constexpr std::integral_constant<int, kWholeProduct> whole{};
        uint32_t flip = 0;
        for (; s < steps; ++s) {
            for (auto& p : products) p.flip = flip;
            coefficients_of(s);
            symmetric(gram, kOfX);
            if (s == 0 && pairs && may_pair(coefficients, steps)) {
                symmetric(poly, kFirst);
                symmetric(product, kBetween);
                symmetric(product, kNextA);
                coefficients_of(++s);
                symmetric(poly, kSecond);
                symmetric(whole, kBoth);
            } else {
                symmetric(poly, kOfA);
            }
            if (s + 1 == steps) break;
            if (large[2]) hipLaunchKernelGGL(ns_apply_turn_kernel<false>, dim3(grid[2]), dim3(TurnTile::kThreads), kTurnLds, stream, products[2]);
            else hipLaunchKernelGGL(ns_apply_kernel<false>, dim3(grid[2]), dim3(ApplyTile::kThreads), ApplyTile::kLdsBytes, stream, products[2]);
            flip ^= 1;
        }
        a.flip = products[2].flip;
        a.a = products[2].a;
        a.b = products[2].b;
        a.c = products[2].c;
        ends([&](const cce_matrix&, const NsLayout& at) { return apply_tiles(at, large[2]); }, [&](uint32_t blocks) {
            if (large[2]) hipLaunchKernelGGL(ns_apply_turn_kernel<true>, dim3(blocks), dim3(TurnTile::kThreads), kTurnLds, stream, a);
            else hipLaunchKernelGGL(ns_apply_kernel<true>, dim3(blocks), dim3(ApplyTile::kThreads), ApplyTile::kLdsBytes, stream, a);
        });
    }
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

static int check_steps(const cce_matrix* matrices, int64_t count, const float* coefficients, int32_t steps, float eps,
                       const void* workspace, size_t workspace_bytes) {
    if (!coefficients || steps < 1 || steps > CCE_NS_MAX_STEPS || !(eps >= 0.f)) return CCE_ERR_INVALID;
    if (!workspace || misaligned(workspace, 256) || workspace_bytes < cce_muon_workspace_bytes(matrices, count)) return CCE_ERR_INVALID;
    return check_coefficients(coefficients, steps);
}

}  // namespace cce

using namespace cce;

extern "C" {

size_t cce_muon_workspace_bytes(const cce_matrix* matrices, int64_t count) {
    if (check_sizes(matrices, count) != CCE_OK) return 0;
    int64_t most = 256;
    for (const bool pairs : {false, true})
        for (int64_t i = 0; i < count;) {
            const int64_t bytes = next_group(matrices, count, pairs, i, [](const cce_matrix&, uint64_t) {});
            most = bytes > most ? bytes : most;
        }
    for (int64_t i = 0; i < count;) {
        const int64_t bytes = next_thin_group(matrices, count, i, [](const cce_matrix&, uint64_t) {});
        most = bytes > most ? bytes : most;
    }
    return (size_t)most;
}

int cce_orthogonalize_multi(const cce_matrix* matrices, int64_t count, const float* coefficients, int32_t steps, float eps,
                            void* workspace, size_t workspace_bytes, void* stream_) {
    int rc = check_gradients(matrices, count);
    if (rc == CCE_OK) rc = check_steps(matrices, count, coefficients, steps, eps, workspace, workspace_bytes);
    if (rc != CCE_OK) return rc;
    for (int64_t i = 0; i < count; ++i) {
        const cce_matrix& t = matrices[i];
        if (t.rows != 0 && t.cols != 0 && (!t.out_bf16 || misaligned(t.out_bf16, 2))) return CCE_ERR_INVALID;
    }
    (void)hipGetLastError();
    return run_groups(matrices, count, false, 0.f, 0.f, 0, coefficients, steps, eps, nullptr, workspace, (hipStream_t)stream_);
}

int cce_muon_multi_step(const cce_matrix* matrices, int64_t count, float lr, float mu, int32_t nesterov,
                        const float* coefficients, int32_t steps, float eps, const float* clip_coef,
                        void* workspace, size_t workspace_bytes, void* stream_) {
    int rc = check_gradients(matrices, count);
    if (rc == CCE_OK) rc = check_steps(matrices, count, coefficients, steps, eps, workspace, workspace_bytes);
    if (rc != CCE_OK) return rc;
    if (!(lr >= 0.f && mu >= 0.f && mu < 1.f) || misaligned(clip_coef, 4)) return CCE_ERR_INVALID;
    for (int64_t i = 0; i < count; ++i) {
        const cce_matrix& t = matrices[i];
        if (t.rows == 0 || t.cols == 0) continue;
        if (!t.param || !t.momentum || misaligned(t.param, 4) || misaligned(t.momentum, 4) || misaligned(t.out_bf16, 2)) return CCE_ERR_INVALID;
        if (!(t.lr_scale >= 0.f && t.weight_decay >= 0.f)) return CCE_ERR_INVALID;
    }
    (void)hipGetLastError();
    return run_groups(matrices, count, true, lr, mu, nesterov != 0, coefficients, steps, eps, clip_coef, workspace, (hipStream_t)stream_);
}

}  // extern "C"
