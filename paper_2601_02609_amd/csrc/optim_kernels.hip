// libcce, optimizer kernels over many tensors: gradient norm with its clipping coefficient, AdamW with
// moments in fp32 or in 8 bits.  C ABI declared in include/cce_optim.h.
//
// The tensors of a launch are a table in the kernel's arguments (nothing to copy, nothing to keep): a
// tensor's values are cut into blocks of kStepValues (kNormChunk) and the workgroups are numbered through all of them.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/cce.h"
#include "../../include/cce_optim.h"
#include "host_util.h"
#include "vec_util.h"

namespace cce {

typedef __attribute__((ext_vector_type(2))) unsigned int ou32x2;
typedef __attribute__((ext_vector_type(2))) float of32x2;

constexpr int kStepValues = 1024;                      // values of a workgroup of a step: four a thread
constexpr int kReadValues = 2048;                      // of a workgroup that reads 8-bit moments
constexpr int64_t kMaxTensor = (int64_t)1 << 33;       // values of a tensor
constexpr int64_t kMaxValues = (int64_t)1 << 40;       // of all tensors: 2^28 chunks of the norm and one a tensor, twice that in 32 bits
constexpr int64_t kMaxGrid = (1 << 24) - 1;            // of 256 threads: a launch has fewer than 2^32 threads
constexpr int kStepTensors = 64, kStepTensors8 = 52;   // tensors of a launch: kernel arguments hold 4 KB
constexpr int kNormTensors = 160;
constexpr int kNormBlocks = 2048;                      // workgroups of a launch, each with one partial sum
constexpr int kNormChunk = 4096;                       // values of a workgroup's trip

struct StepTensor {
    float* param;
    uint16_t* param_bf16;
    const void* grad;
    void* m;
    void* v;
    int64_t n;
    float lr, decay;                                   // decay: 1 - lr * weight_decay
};

struct StepTensor8 : StepTensor {
    uint8_t* m_scale;
    uint8_t* v_scale;
};

template <class Tensor, int COUNT>
struct StepArgs {
    static constexpr int kCount = COUNT;
    Tensor t[COUNT];
    uint32_t first[COUNT];                             // twice a tensor's first workgroup, plus 1 if its gradient is bf16
    const float* clip_coef;
    double keep_m, take_m, keep_v, take_v;             // the betas and 1 - beta, exact
    float beta1, beta2, eps, inv_bc1, inv_bc2, root_inv_bc2;
    uint32_t key, count;
};
using StepArgs32 = StepArgs<StepTensor, kStepTensors>;
using StepArgs8 = StepArgs<StepTensor8, kStepTensors8>;
static_assert(sizeof(StepArgs32) <= 4096 && sizeof(StepArgs8) <= 4096, "kernel arguments hold 4 KB");

struct NormTensor {
    const void* grad;
    int64_t n;
};

struct NormArgs {
    NormTensor t[kNormTensors];
    uint32_t first[kNormTensors];                      // a tensor's first chunk; twice that, plus 1 if it is bf16
    double* partials;
    uint32_t count, chunks;
};
static_assert(sizeof(NormArgs) <= 4096, "kernel arguments hold 4 KB");

// Which tensor of the table workgroup (or chunk) w belongs to, b = 2 w + 1: the last one that begins at or before it.  Every
// lane looks at one entry: one load instead of the chain of a binary search.
__device__ __forceinline__ int tensor_of(const uint32_t* first, int count, uint32_t b) {
    int n = 0;
    for (int base = 0; base < count; base += 64) {
        const int i = base + (int)(threadIdx.x & 63);
        n += (int)__popcll(__ballot(i < count && first[i] <= b));
    }
    return __builtin_amdgcn_readfirstlane(n - 1);
}

__device__ __forceinline__ float grad_at(const void* grad, bool bf16, int64_t i) {
    return bf16 ? __uint_as_float((uint32_t)((const uint16_t*)grad)[i] << 16) : ((const float*)grad)[i];
}

// Group q of four gradient values behind `base`.
__device__ __forceinline__ af32x4 load_grad4(const void* grad, bool bf16, int64_t base, int q) {
    if (!bf16) return __builtin_nontemporal_load((const af32x4*)((const float*)grad + base) + q);
    const ou32x2 h = __builtin_nontemporal_load((const ou32x2*)((const uint16_t*)grad + base) + q);
    return af32x4{__uint_as_float(h[0] << 16), __uint_as_float(h[0] & 0xffff0000u),
                  __uint_as_float(h[1] << 16), __uint_as_float(h[1] & 0xffff0000u)};
}

__device__ __forceinline__ ou32x2 pack4(const af32x4& x) {
    union { __bf16 h[4]; ou32x2 u; } cv;
#pragma unroll
    for (int e = 0; e < 4; ++e) cv.h[e] = (__bf16)x[e];
    return cv.u;
}

// Copies that the last-level cache cannot keep for the forward pass are written past it: AdamW of 416 M values 2188 -> 2083 us.
constexpr int64_t kStreamCopies = (int64_t)192 << 20;
template <bool STREAM>
__device__ __forceinline__ void store_copy(uint16_t* to, int q, const ou32x2& copy) {
    if (STREAM) __builtin_nontemporal_store(copy, (ou32x2*)to + q); else ((ou32x2*)to)[q] = copy;
}

// ------------------------------------------------------------------------------------------
// Sum of squares of all gradients.  Squares of fp32 values are exact in fp64, whose sums leave nothing
// to argue about.  Workgroups walk the chunks of all tensors with a grid stride, a chunk's loads in flight
// together.  Bound by HBM reads: 416 M values, a third of them bf16, in 232 us, 5.95 TB/s; chunks of 8192 values
// 282 us, of 2048 287; 1024 workgroups 265.
// ------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void norm_partial_kernel(const NormArgs a) {
    __shared__ double red[4];
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int i = tensor_of(a.first, (int)a.count, 2 * c + 1);
        const int64_t at = (int64_t)(c - (a.first[i] >> 1)) * kNormChunk, left = a.t[i].n - at;
        if (a.first[i] & 1u) {
            const uint16_t* g = (const uint16_t*)a.t[i].grad + at;
            if (left >= kNormChunk) {
                au32x4 v[kNormChunk / 2048];
#pragma unroll
                for (int u = 0; u < kNormChunk / 2048; ++u) v[u] = ((const au32x4*)g)[u * 256 + threadIdx.x];
#pragma unroll
                for (int u = 0; u < kNormChunk / 2048; ++u) {
                    float f[8];
                    unpack8(v[u], f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum = fma((double)f[e], (double)f[e], sum);
                }
            } else {
                for (int64_t j = threadIdx.x; j < left; j += 256) {
                    const double x = (double)__uint_as_float((uint32_t)g[j] << 16);
                    sum = fma(x, x, sum);
                }
            }
        } else {
            const float* g = (const float*)a.t[i].grad + at;
            if (left >= kNormChunk) {
                af32x4 v[kNormChunk / 1024];
#pragma unroll
                for (int u = 0; u < kNormChunk / 1024; ++u) v[u] = ((const af32x4*)g)[u * 256 + threadIdx.x];
#pragma unroll
                for (int u = 0; u < kNormChunk / 1024; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum = fma((double)v[u][e], (double)v[u][e], sum);
            } else {
                for (int64_t j = threadIdx.x; j < left; j += 256) sum = fma((double)g[j], (double)g[j], sum);
            }
        }
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) a.partials[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(1024) void norm_final_kernel(const double* __restrict__ partials, int64_t count, double* __restrict__ sumsq,
                                                          int accumulate, float max_norm, float eps_norm, float* __restrict__ clip_coef) {
    __shared__ double red[16];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < count; i += 8192) {      // eight loads of a thread in flight
        double x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = i + 1024 * u < count ? partials[i + 1024 * u] : 0.0;
#pragma unroll
        for (int u = 0; u < 8; ++u) sum += x[u];
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x != 0) return;
    double total = accumulate ? sumsq[0] : 0.0;
#pragma unroll
    for (int w = 0; w < 16; ++w) total += red[w];
    sumsq[0] = total;
    if (clip_coef) {
        const double c = (double)max_norm / (sqrt(total) + (double)eps_norm);
        clip_coef[0] = c < 1.0 ? (float)c : 1.0f;
    }
}

// ------------------------------------------------------------------------------------------
// AdamW: clip, moments, bias corrections, decoupled decay and update.
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ void adamw_one(float& p, float g, float& m, float& v, float lr, float decay, const StepArgs32& a) {
    m = a.beta1 * m + (1.f - a.beta1) * g;
    v = a.beta2 * v + (1.f - a.beta2) * g * g;
    p = p * decay - lr * ((m * a.inv_bc1) / (sqrtf(v * a.inv_bc2) + a.eps));
}

// Every value is touched once: streaming accesses of 16 bytes, one group of a tensor a thread.  Bound by HBM: 416 M values
// (12.2 GB) in 2071 us, 5.88 TB/s where a copy of 1 GiB reaches 5.15.  Two groups a thread took 2.6 % longer, four 1.3 %; 32 bytes of a thread in a row 3.5 %.
template <bool STREAM>
__global__ __launch_bounds__(256) void adamw_multi_kernel(const StepArgs32 a) {
    const int i = tensor_of(a.first, (int)a.count, 2 * blockIdx.x + 1);
    const StepTensor& t = a.t[i];
    const int64_t base = (int64_t)(blockIdx.x - (a.first[i] >> 1)) * kStepValues, left = t.n - base;
    const float clip = a.clip_coef ? a.clip_coef[0] : 1.f;
    float* p = t.param + base;
    float* m = (float*)t.m + base;
    float* v = (float*)t.v + base;
    const bool bf16 = (a.first[i] & 1u) != 0u;
    const int q = threadIdx.x;
    if (left >= kStepValues) {
        af32x4 pv = __builtin_nontemporal_load((const af32x4*)p + q), mv = __builtin_nontemporal_load((const af32x4*)m + q),
               vv = __builtin_nontemporal_load((const af32x4*)v + q);
        const af32x4 gv = load_grad4(t.grad, bf16, base, q);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float pe = pv[e], me = mv[e], ve = vv[e];
            adamw_one(pe, gv[e] * clip, me, ve, t.lr, t.decay, a);
            pv[e] = pe; mv[e] = me; vv[e] = ve;
        }
        __builtin_nontemporal_store(pv, (af32x4*)p + q);
        __builtin_nontemporal_store(mv, (af32x4*)m + q);
        __builtin_nontemporal_store(vv, (af32x4*)v + q);
        if (t.param_bf16) store_copy<STREAM>(t.param_bf16 + base, q, pack4(pv));
        return;
    }
    for (int j = q; j < left; j += 256) {
        float pe = p[j], me = m[j], ve = v[j];
        adamw_one(pe, grad_at(t.grad, bf16, base + j) * clip, me, ve, t.lr, t.decay, a);
        p[j] = pe; m[j] = me; v[j] = ve;
        if (t.param_bf16) t.param_bf16[base + j] = (uint16_t)pack4(af32x4{pe, 0.f, 0.f, 0.f})[0];
    }
}

// Moments in 8 bits.  BITS mantissa bits: 3 for m (E4M3, signed), 4 for sqrt(v) (unsigned), bias 7 in both.
__device__ __forceinline__ uint32_t mix32(uint32_t h) {
    // two multiplications by LCG multipliers of L'Ecuyer's 1999 tables for modulus 2^32, shifts between
    h ^= h >> 16;
    h *= 2891336453u;
    h ^= h >> 15;
    h *= 29943829u;
    return h ^ (h >> 16);
}

// What a code stands for, without its scale.  Its fields are moved into fp32's, whose bias is 120 larger:
// subnormal codes become subnormal values.
template <int BITS>
__device__ __forceinline__ float decode8(uint32_t code) {
    const uint32_t mag = BITS == 3 ? code & 0x7fu : code;
    float x = __uint_as_float(mag << (23 - BITS)) * 0x1p120f;
    if (mag == (BITS == 3 ? 0x7fu : 0xffu)) x = __uint_as_float(0x7fc00000u);
    return BITS == 3 && code > 0x7fu ? -x : x;
}

__device__ __forceinline__ double power_of_two(int e) { return __longlong_as_double((long long)(1023 + e) << 52); }

__device__ __forceinline__ uint32_t high_word(double x) { return (uint32_t)((uint64_t)__double_as_longlong(x) >> 32); }

// sqrt of x >= 0 from the hardware's reciprocal root and one correction of it: a reciprocal root off by d leaves 1.5 d^2, always
// downward; 2^-47.7 at worst over 65 M values (d some 2^-24).  Infinite x gives NaN, as its code is.
__device__ __forceinline__ double root(double x) {
    const double y = __builtin_amdgcn_rsq(fmax(x, 1e-290)), s = x * y;
    return fma(0.5 * s, fma(-s, y, 1.0), s);
}

// The largest of 32 lanes.
__device__ __forceinline__ uint32_t half_max(uint32_t x) {
    auto step = [&](int other) { x = (uint32_t)other > x ? (uint32_t)other : x; };
    step(__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));                 // row_ror:8, 4, 2, 1
    step(__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, false));
    step(__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, false));
    step(__builtin_amdgcn_ds_swizzle((int)x, 0x401f));                                    // lane ^ 16
    return x;
}

// What four values of a block need to become codes: the high words of their magnitudes, and the block's exponent
// e = ceil(log2(amax / top)), top = 1.75 * 2^8 or 1.875 * 2^8, of the largest finite magnitude.  High words decide it, but
// where the largest one is top's own: then whether a low word is not 0.  fits: no value is NaN, infinite or beyond the largest
// scale.
constexpr uint32_t kNotFinite = 0x7ff00000u;
template <int BITS>
__device__ __forceinline__ int scale_exponent(const double (&x)[4], uint32_t (&word)[4], bool& fits) {
    constexpr uint32_t border = BITS == 3 ? 0xc0000u : 0xe0000u;
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        word[i] = BITS == 3 ? high_word(x[i]) & 0x7fffffffu : high_word(x[i]);
        top = word[i] > top ? word[i] : top;
    }
    fits = top < kNotFinite;
    if (!fits) {
        top = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = word[i] < kNotFinite && word[i] > top ? word[i] : top;
    }
    if ((top & 0xfffffu) == border) {
        uint32_t low = 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) low |= word[i] == top ? (uint32_t)__double_as_longlong(x[i]) : 0u;
        top += low != 0u ? 1u : 0u;
    }
    top = half_max(top);
    if (top == 0u) return 0;
    const int e = (int)(top >> 20) - 1023 - 8 + ((top & 0xfffffu) > border ? 1 : 0);
    fits = fits && e <= 120;
    return e < -100 ? -100 : (e > 120 ? 120 : e);
}

// The code of x 2^-e, rounded down after `dither` steps of 2^-(20 - BITS) of a code's step.  Scaled by 2^-1016 more, what the
// formats' bias of 7 has as exponent field is fp64's own: its high word has the code's bits in front of those that the
// dither meets, and subnormal codes are subnormal numbers.  `word`: of |x|; nothing is said of an x that no scale fits.
template <int BITS>
__device__ __forceinline__ uint32_t encode8(double x, uint32_t word, int e, uint32_t dither) {
    const uint32_t y = high_word(ldexp(x, -1016 - e)) + dither;
    if (BITS == 3) return (y >> 17 & 0x7fu) | (y >> 24 & 0x80u);
    const uint32_t code = y >> 16, least = word < 1u ? word : 1u;                        // a root above 0 does not become 0
    return code < least ? least : code;
}

// 32 lanes share a block of 128 values, four each.  The moments are formed in fp64, so that which way a value next to a
// border goes does not depend on the order or the fusing of the operations.  The update takes sqrt(v / bc2) from the root
// that is stored, and reciprocals to one unit in the last place.  Bound by HBM and by its arithmetic nearly as much: 416 M
// values (6.7 GB) in 1130 us, 5.9 TB/s.
template <bool STREAM>
__global__ __launch_bounds__(256) void adamw_multi8_kernel(const StepArgs8 a) {
    const int i = tensor_of(a.first, (int)a.count, 2 * blockIdx.x + 1);
    const StepTensor8& t = a.t[i];
    const int64_t base = (int64_t)(blockIdx.x - (a.first[i] >> 1)) * kStepValues;
    const int q = threadIdx.x;
    const int64_t at = base + 4 * q, left = t.n - at;
    const bool whole = left >= 4, bf16 = (a.first[i] & 1u) != 0u;
    uint8_t* ms = t.m_scale + at / CCE_STATE8_BLOCK;
    uint8_t* vs = t.v_scale + at / CCE_STATE8_BLOCK;
    uint8_t* mcode = (uint8_t*)t.m + at;
    uint8_t* vcode = (uint8_t*)t.v + at;
    af32x4 p = {0.f, 0.f, 0.f, 0.f}, g = p;                   // zeros behind the end: they take part in the block's largest
    uint32_t mc = 0u, vc = 0u;
    int sm = 127, sv = 127;
    if (whole) {
        p = __builtin_nontemporal_load((const af32x4*)(t.param + base) + q);
        g = load_grad4(t.grad, bf16, base, q);
        mc = *(const uint32_t*)mcode;
        vc = *(const uint32_t*)vcode;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e) {
            if (e >= left) continue;
            p[e] = t.param[at + e];
            g[e] = grad_at(t.grad, bf16, at + e);
            mc |= (uint32_t)mcode[e] << (8 * e);
            vc |= (uint32_t)vcode[e] << (8 * e);
        }
    }
    if (left > 0) { sm = ms[0]; sv = vs[0]; }
    const double clip = a.clip_coef ? (double)a.clip_coef[0] : 1.0;
    const double take_m = a.take_m * clip, take_v = a.take_v * clip * clip;
    const double keep_m = ldexp(a.keep_m, sm - 127), keep_v = ldexp(a.keep_v, 2 * (sv - 127));
    const float rate = t.lr * a.inv_bc1;
    const of32x2 m0[2] = {__builtin_amdgcn_cvt_pk_f32_fp8((int)mc, false), __builtin_amdgcn_cvt_pk_f32_fp8((int)mc, true)};
    double m[4], r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const double ge = (double)g[e];
        const float r0 = decode8<4>(vc >> (8 * e) & 0xffu);                              // whose square has ten bits
        m[e] = fma((double)m0[e >> 1][e & 1], keep_m, ge * take_m);
        r[e] = root(fma((double)(r0 * r0), keep_v, ge * ge * take_v));
        float under = fmaf((float)r[e], a.root_inv_bc2, a.eps);
        under = under < 0x1p-126f ? 0x1p-126f : under;                                   // a NaN stays one
        p[e] = fmaf(-rate * (float)m[e], __builtin_amdgcn_rcpf(under), p[e] * t.decay);
    }
    uint32_t mw[4], rw[4], cm[4], cr[4];
    bool m_fits, r_fits;
    const int em = scale_exponent<3>(m, mw, m_fits), er = scale_exponent<4>(r, rw, r_fits);
    const uint32_t key = (uint32_t)at + (uint32_t)((uint64_t)at >> 32) * 32310901u + a.key;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t h = mix32(key + (uint32_t)e);
        cm[e] = encode8<3>(m[e], mw[e], em, h >> 15);
        cr[e] = encode8<4>(r[e], rw[e], er, h & 0xffffu);
    }
    if (!m_fits || !r_fits) {                                                            // fp32 has no value beyond 2^128 either
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            cm[e] = fabs(m[e]) <= 0x1.cp128 ? cm[e] : 0x7fu;
            cr[e] = r[e] <= 0x1.ep128 ? cr[e] : 0xffu;
        }
    }
    if (left <= 0) return;
    const uint32_t mo = cm[0] | cm[1] << 8 | cm[2] << 16 | cm[3] << 24, vo = cr[0] | cr[1] << 8 | cr[2] << 16 | cr[3] << 24;
    const ou32x2 copy = pack4(p);
    if (whole) {
        __builtin_nontemporal_store(p, (af32x4*)(t.param + base) + q);
        if (t.param_bf16) store_copy<STREAM>(t.param_bf16 + base, q, copy);
        *(uint32_t*)mcode = mo;
        *(uint32_t*)vcode = vo;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e) {
            if (e >= left) continue;
            t.param[at + e] = p[e];
            if (t.param_bf16) t.param_bf16[at + e] = (uint16_t)(copy[e >> 1] >> (16 * (e & 1)));
            mcode[e] = (uint8_t)(mo >> (8 * e));
            vcode[e] = (uint8_t)(vo >> (8 * e));
        }
    }
    if ((q & 31) == 0) {
        ms[0] = (uint8_t)(em + 127);
        vs[0] = (uint8_t)(er + 127);
    }
}

// Four values a thread, two groups of them 1024 values apart.  Bound by HBM, mostly writes: 416 M values (2.1 GB) in 330 us.
template <int BITS>
__global__ __launch_bounds__(256) void state8_read_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                          int64_t n, float* __restrict__ out) {
    auto value = [&](uint32_t code, double power) {
        const float d = decode8<BITS>(code);
        return (float)((double)(BITS == 4 ? d * d : d) * power);
    };
    for (int64_t base = (int64_t)blockIdx.x * kReadValues; base < n; base += (int64_t)gridDim.x * kReadValues) {
        uint32_t c[2];
        int scale[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t at = base + 1024 * u + 4 * (int)threadIdx.x;
            if (at + 4 <= n) c[u] = __builtin_nontemporal_load((const uint32_t*)(codes + at));
            if (at < n) scale[u] = scales[at / CCE_STATE8_BLOCK];
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t at = base + 1024 * u + 4 * (int)threadIdx.x;
            if (at >= n) continue;
            const double power = power_of_two((BITS == 4 ? 2 : 1) * (scale[u] - 127));
            if (at + 4 <= n) {
                af32x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = value(c[u] >> (8 * e) & 0xffu, power);
                __builtin_nontemporal_store(x, (af32x4*)(out + at));
            } else {
                for (int64_t j = at; j < n; ++j) out[j] = value(codes[j], power);
            }
        }
    }
}

static uint32_t mix32_host(uint32_t h) {
    h ^= h >> 16;
    h *= 2891336453u;
    h ^= h >> 15;
    h *= 29943829u;
    return h ^ (h >> 16);
}

static void fill_tensor(StepTensor& to, const cce_optim_tensor& t, float rate) {
    to.param = t.param; to.param_bf16 = (uint16_t*)t.param_bf16; to.grad = t.grad; to.m = t.m; to.v = t.v; to.n = t.n;
    to.lr = rate;
    to.decay = 1.f - rate * t.weight_decay;
}

static void fill_tensor(StepTensor8& to, const cce_optim_tensor& t, float rate) {
    fill_tensor(static_cast<StepTensor&>(to), t, rate);
    to.m_scale = t.m_scale;
    to.v_scale = t.v_scale;
}

static bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

static int check_gradients(const cce_optim_tensor* tensors, int64_t count) {
    if (!tensors || count <= 0) return CCE_ERR_INVALID;
    int64_t values = 0;
    for (int64_t i = 0; i < count; ++i) {
        const cce_optim_tensor& t = tensors[i];
        if (t.n < 0) return CCE_ERR_INVALID;
        if (t.n == 0) continue;
        if (t.n > kMaxTensor || (values += t.n) > kMaxValues) return CCE_ERR_UNSUPPORTED;
        if (!t.grad || misaligned(t.grad, 16) || (t.grad_bf16 != 0 && t.grad_bf16 != 1)) return CCE_ERR_INVALID;
    }
    return CCE_OK;
}

}  // namespace cce

using namespace cce;

extern "C" {

size_t cce_sumsq_multi_workspace_bytes(int64_t count) {
    if (count <= 0) return 0;
    return (size_t)((count + kNormTensors - 1) / kNormTensors) * kNormBlocks * sizeof(double);
}

int cce_grad_sumsq_multi(const cce_optim_tensor* tensors, int64_t count, double* sumsq, int accumulate,
                         float max_norm, float eps_norm, float* clip_coef,
                         void* workspace, size_t workspace_bytes, void* stream_) {
    const int rc = check_gradients(tensors, count);
    if (rc != CCE_OK) return rc;
    if (!sumsq || misaligned(sumsq, 8) || !workspace || misaligned(workspace, 256) || misaligned(clip_coef, 4)) return CCE_ERR_INVALID;
    if (clip_coef && !(max_norm > 0.f && eps_norm >= 0.f)) return CCE_ERR_INVALID;
    if (workspace_bytes < cce_sumsq_multi_workspace_bytes(count)) return CCE_ERR_INVALID;
    hipStream_t stream = (hipStream_t)stream_;
    (void)hipGetLastError();
    NormArgs a;
    int64_t partials = 0;
    for (int64_t i = 0; i < count;) {
        a.count = 0;
        int64_t chunks = 0;
        for (; i < count && a.count < (uint32_t)kNormTensors; ++i) {
            const cce_optim_tensor& t = tensors[i];
            if (t.n == 0) continue;
            a.first[a.count] = 2 * (uint32_t)chunks + (uint32_t)t.grad_bf16;
            a.t[a.count++] = NormTensor{t.grad, t.n};
            chunks += (t.n + kNormChunk - 1) / kNormChunk;
        }
        if (a.count == 0) continue;
        const int blocks = (int)(chunks < kNormBlocks ? chunks : kNormBlocks);
        a.partials = (double*)workspace + partials;
        a.chunks = (uint32_t)chunks;
        hipLaunchKernelGGL(norm_partial_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, a);
        partials += blocks;
    }
    hipLaunchKernelGGL(norm_final_kernel, dim3(1), dim3(1024), 0, stream, (const double*)workspace, partials, sumsq,
                       accumulate ? 1 : 0, max_norm, eps_norm, clip_coef);
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

int cce_adamw_multi_step(const cce_optim_tensor* tensors, int64_t count, float lr, float beta1, float beta2,
                         float eps, int64_t step, const float* clip_coef, uint32_t seed, void* stream_) {
    int rc = check_gradients(tensors, count);
    if (rc != CCE_OK) return rc;
    if (step < 1 || misaligned(clip_coef, 4)) return CCE_ERR_INVALID;
    if (!(beta1 >= 0.f && beta1 < 1.f && beta2 >= 0.f && beta2 < 1.f && eps >= 0.f && lr >= 0.f)) return CCE_ERR_INVALID;
    for (int64_t i = 0; i < count; ++i) {
        const cce_optim_tensor& t = tensors[i];
        if (t.n == 0) continue;
        if (!t.param || !t.m || !t.v) return CCE_ERR_INVALID;
        if (misaligned(t.param, 16) || misaligned(t.param_bf16, 16) || misaligned(t.m, 16) || misaligned(t.v, 16)) return CCE_ERR_INVALID;
        if ((t.state8 != 0 && t.state8 != 1) || (t.state8 && (!t.m_scale || !t.v_scale))) return CCE_ERR_INVALID;
        if (!(t.lr_scale >= 0.f && t.weight_decay >= 0.f)) return CCE_ERR_INVALID;
    }
    hipStream_t stream = (hipStream_t)stream_;
    (void)hipGetLastError();
    bool any32 = false, any8 = false;
    int64_t copies = 0;
    for (int64_t i = 0; i < count; ++i) {
        (tensors[i].state8 ? any8 : any32) = true;
        if (tensors[i].n != 0 && tensors[i].param_bf16) copies += tensors[i].n * 2;
    }
    const bool past_caches = copies >= kStreamCopies;
    // the tensors with moments of one kind, as many a launch as its table and a grid hold
    auto run = [&](auto& a, int state8, auto launch) {
        a.clip_coef = clip_coef;
        a.beta1 = beta1; a.beta2 = beta2; a.eps = eps;
        a.keep_m = (double)beta1; a.take_m = 1.0 - a.keep_m;
        a.keep_v = (double)beta2; a.take_v = 1.0 - a.keep_v;
        a.inv_bc1 = (float)(1.0 / (1.0 - pow((double)beta1, (double)step)));
        a.inv_bc2 = (float)(1.0 / (1.0 - pow((double)beta2, (double)step)));
        a.root_inv_bc2 = (float)sqrt(1.0 / (1.0 - pow((double)beta2, (double)step)));
        a.key = mix32_host(seed + mix32_host((uint32_t)step));
        for (int64_t i = 0; i < count;) {
            a.count = 0;
            int64_t blocks = 0;
            for (; i < count && a.count < (uint32_t)a.kCount; ++i) {
                const cce_optim_tensor& t = tensors[i];
                if (t.n == 0 || t.state8 != state8) continue;
                const int64_t own = (t.n + kStepValues - 1) / kStepValues;
                if (blocks + own > kMaxGrid) break;
                const float rate = lr * t.lr_scale;
                a.first[a.count] = 2 * (uint32_t)blocks + (uint32_t)t.grad_bf16;
                fill_tensor(a.t[a.count++], t, rate);
                blocks += own;
            }
            if (a.count != 0) launch(a, (unsigned)blocks);
        }
    };
    if (any32) {
        StepArgs32 a;
        run(a, 0, [&](const StepArgs32& x, unsigned blocks) {
            if (past_caches) hipLaunchKernelGGL(adamw_multi_kernel<true>, dim3(blocks), dim3(256), 0, stream, x);
            else hipLaunchKernelGGL(adamw_multi_kernel<false>, dim3(blocks), dim3(256), 0, stream, x);
        });
    }
    if (any8) {
        StepArgs8 a;
        run(a, 1, [&](const StepArgs8& x, unsigned blocks) {
            if (past_caches) hipLaunchKernelGGL(adamw_multi8_kernel<true>, dim3(blocks), dim3(256), 0, stream, x);
            else hipLaunchKernelGGL(adamw_multi8_kernel<false>, dim3(blocks), dim3(256), 0, stream, x);
        });
    }
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

int cce_adamw_state8_read(const void* codes, const uint8_t* scales, int64_t n, int second, float* out, void* stream_) {
    if (!codes || !scales || !out || n <= 0 || (second != 0 && second != 1)) return CCE_ERR_INVALID;
    if (misaligned(codes, 8) || misaligned(out, 16)) return CCE_ERR_INVALID;
    const int64_t want = (n + kReadValues - 1) / kReadValues;
    const dim3 grid((unsigned)(want < kMaxGrid ? want : kMaxGrid));
    hipStream_t stream = (hipStream_t)stream_;
    (void)hipGetLastError();
    if (second) hipLaunchKernelGGL(state8_read_kernel<4>, grid, dim3(256), 0, stream, (const uint8_t*)codes, scales, n, out);
    else hipLaunchKernelGGL(state8_read_kernel<3>, grid, dim3(256), 0, stream, (const uint8_t*)codes, scales, n, out);
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

}  // extern "C"
