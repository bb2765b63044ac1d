// libcce, optimizer kernels over many tensors: gradient norm with its clipping coefficient, AdamW with
// moments in fp32 or in 8 bits.  C ABI declared in include/cce_optim.h.
//
// The tensors of a launch are a table in the kernel's arguments (nothing to copy, nothing to keep): a
// tensor's values are cut into blocks of kBlockValues and the workgroups are numbered through all of them.
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

constexpr int kBlockValues = 2048;                     // values of a workgroup: eight a thread
constexpr int64_t kMaxTensor = (int64_t)1 << 34;       // values of a tensor
constexpr int64_t kMaxGrid = (1 << 24) - 1;            // of 256 threads: a launch has fewer than 2^32 threads
constexpr int kStepTensors = 44;                       // tensors of a launch: kernel arguments hold 4 KB
constexpr int kNormTensors = 160;
constexpr int kNormBlocks = 1024;                      // workgroups of a launch, each with one partial sum

struct StepTensor {
    float* param;
    uint16_t* param_bf16;
    const void* grad;
    void* m;
    void* v;
    uint8_t* m_scale;
    uint8_t* v_scale;
    int64_t n;
    float lr, decay;                                   // decay: 1 - lr * weight_decay
    uint32_t first;                                    // its first workgroup
    uint32_t grad_bf16;
};

struct StepArgs {
    StepTensor t[kStepTensors];
    const float* clip_coef;
    float beta1, beta2, eps, inv_bc1, inv_bc2;
    uint32_t key, count;
};
static_assert(sizeof(StepArgs) <= 4096, "kernel arguments hold 4 KB");

struct NormTensor {
    const void* grad;
    int64_t n;
    uint32_t first;                                    // its first chunk
    uint32_t grad_bf16;
};

struct NormArgs {
    NormTensor t[kNormTensors];
    double* partials;
    uint32_t count, chunks;
};
static_assert(sizeof(NormArgs) <= 4096, "kernel arguments hold 4 KB");

// Which tensor of the table workgroup (or chunk) `b` belongs to: the last one that begins at or before it.
template <class Tensor>
__device__ __forceinline__ int tensor_of(const Tensor* t, int count, uint32_t b) {
    int low = 0, high = count - 1;
    while (low < high) {
        const int mid = (low + high + 1) >> 1;
        if (t[mid].first <= b) low = mid; else high = mid - 1;
    }
    return low;
}

// Eight gradient values from `at` on, of which `live` exist; zeros behind them.
__device__ __forceinline__ void load_grad(const void* grad, bool bf16, int64_t at, int live, float (&g)[8]) {
    if (live >= 8) {
        if (bf16) {
            unpack8(*(const au32x4*)((const uint16_t*)grad + at), g);
        } else {
            const af32x4 a = *(const af32x4*)((const float*)grad + at), b = *(const af32x4*)((const float*)grad + at + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { g[e] = a[e]; g[4 + e] = b[e]; }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        g[e] = 0.f;
        if (e < live) g[e] = bf16 ? __uint_as_float((uint32_t)((const uint16_t*)grad)[at + e] << 16) : ((const float*)grad)[at + e];
    }
}

__device__ __forceinline__ void load_f32(const float* p, int64_t at, int live, float (&x)[8]) { load_grad(p, false, at, live, x); }

__device__ __forceinline__ void store_f32(float* p, int64_t at, int live, const float (&x)[8]) {
    if (live >= 8) {
        *(af32x4*)(p + at) = af32x4{x[0], x[1], x[2], x[3]};
        *(af32x4*)(p + at + 4) = af32x4{x[4], x[5], x[6], x[7]};
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < live) p[at + e] = x[e];
}

__device__ __forceinline__ void store_bf16(uint16_t* p, int64_t at, int live, const float (&x)[8]) {
    const au32x4 packed = pack8(x);
    if (live >= 8) { *(au32x4*)(p + at) = packed; return; }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < live) p[at + e] = (uint16_t)(packed[e >> 1] >> (16 * (e & 1)));
}

// ------------------------------------------------------------------------------------------
// Sum of squares of all gradients.  Squares of fp32 values are exact in fp64, whose sums leave nothing
// to argue about.  Workgroups walk the chunks of all tensors with a grid stride.
// ------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void norm_partial_kernel(const NormArgs a) {
    __shared__ double red[4];
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int i = tensor_of(a.t, (int)a.count, c);
        const int64_t at = (int64_t)(c - a.t[i].first) * kBlockValues + threadIdx.x * 8, left = a.t[i].n - at;
        if (left <= 0) continue;
        float g[8];
        load_grad(a.t[i].grad, a.t[i].grad_bf16 != 0, at, left < 8 ? (int)left : 8, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum = fma((double)g[e], (double)g[e], sum);
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
    for (int64_t i = threadIdx.x; i < count; i += 1024) sum += partials[i];
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
// AdamW.  The parameter's part of a step, from its new moments: decoupled decay, bias corrections, update.
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ float adamw_param(float p, float m, float v, float lr, float decay, const StepArgs& a) {
    return p * decay - lr * ((m * a.inv_bc1) / (sqrtf(v * a.inv_bc2) + a.eps));
}

__global__ __launch_bounds__(256) void adamw_multi_kernel(const StepArgs a) {
    const StepTensor& t = a.t[tensor_of(a.t, (int)a.count, blockIdx.x)];
    const int64_t at = (int64_t)(blockIdx.x - t.first) * kBlockValues + threadIdx.x * 8, left = t.n - at;
    if (left <= 0) return;
    const int live = left < 8 ? (int)left : 8;
    const float clip = a.clip_coef ? a.clip_coef[0] : 1.f;
    float p[8], g[8], m[8], v[8];
    load_f32(t.param, at, live, p);
    load_grad(t.grad, t.grad_bf16 != 0, at, live, g);
    load_f32((const float*)t.m, at, live, m);
    load_f32((const float*)t.v, at, live, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float ge = g[e] * clip;
        m[e] = a.beta1 * m[e] + (1.f - a.beta1) * ge;
        v[e] = a.beta2 * v[e] + (1.f - a.beta2) * ge * ge;
        p[e] = adamw_param(p[e], m[e], v[e], t.lr, t.decay, a);
    }
    store_f32(t.param, at, live, p);
    store_f32((float*)t.m, at, live, m);
    store_f32((float*)t.v, at, live, v);
    if (t.param_bf16) store_bf16(t.param_bf16, at, live, p);
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

template <int BITS>
__device__ __forceinline__ double decode8(uint32_t code, int scale) {
    const uint32_t mag = BITS == 3 ? code & 0x7fu : code;
    // the code's fields moved into fp32's, whose bias is 120 larger: subnormal codes become subnormal values
    float x = __uint_as_float(mag << (23 - BITS)) * 0x1p120f;
    if (mag == (BITS == 3 ? 0x7fu : 0xffu)) x = __uint_as_float(0x7fc00000u);
    if (BITS == 3 && code > 0x7fu) x = -x;
    return ldexp((double)x, scale - 127);
}

// The high word of |x|, one more if its low word is not 0, for the block's largest; 0 if x is not finite.
__device__ __forceinline__ uint32_t high_word_up(double x) {
    const uint64_t w = (uint64_t)__double_as_longlong(x) & 0x7fffffffffffffffull;
    const uint32_t high = (uint32_t)(w >> 32);
    return high >= 0x7ff00000u ? 0u : high + ((uint32_t)w != 0u ? 1u : 0u);
}

// e = ceil(log2(amax / top)), top = 1.75 * 2^8 or 1.875 * 2^8, of the largest high_word_up: rounding the
// words up keeps which side of a border (a value with a low word of 0) they are on.
template <int BITS>
__device__ __forceinline__ int scale_exponent(uint32_t amax) {
    if (amax == 0u) return 0;
    const int e = (int)(amax >> 20) - 1023 - 8 + ((amax & 0xfffffu) > (BITS == 3 ? 0xc0000u : 0xe0000u) ? 1 : 0);
    return e < -100 ? -100 : (e > 120 ? 120 : e);
}

// y = |x| 2^-e rounded down after `dither` steps of 2^-(20 - BITS) of a code's step: the high word of a
// normal y has the code's bits in front of those that the dither meets; below 2^-6, y + 2^-6 has the
// subnormal codes' step.
template <int BITS>
__device__ __forceinline__ uint32_t encode8(double x, int e, uint32_t dither) {
    const double a = fabs(x);
    if (!(a < INFINITY)) return BITS == 3 ? 0x7fu : 0xffu;
    const double y = ldexp(a, -e);
    const bool low = y < 0x1p-6;
    const uint32_t high = (uint32_t)((uint64_t)__double_as_longlong(low ? y + 0x1p-6 : y) >> 32);
    uint32_t code = ((high + dither) >> (20 - BITS)) - ((low ? 1017u : 1016u) << BITS);
    if (BITS == 3) { if (x < 0.0) code |= 0x80u; }
    else if (x > 0.0 && code == 0u) code = 1u;
    return code;
}

__device__ __forceinline__ ou32x2 load_codes(const void* codes, int64_t at, int live) {
    const uint8_t* c = (const uint8_t*)codes + at;
    if (live >= 8) return *(const ou32x2*)c;
    ou32x2 r = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < live) r[e >> 2] |= (uint32_t)c[e] << (8 * (e & 3));
    return r;
}

__device__ __forceinline__ void store_codes(void* codes, int64_t at, int live, const ou32x2& r) {
    uint8_t* c = (uint8_t*)codes + at;
    if (live >= 8) { *(ou32x2*)c = r; return; }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < live) c[e] = (uint8_t)(r[e >> 2] >> (8 * (e & 3)));
}

// 16 lanes share a block of 128 values, eight each.  The moments are formed in fp64, so that which way a
// value next to a border goes does not depend on the order or the fusing of the operations.
__global__ __launch_bounds__(256) void adamw_multi8_kernel(const StepArgs a) {
    const StepTensor& t = a.t[tensor_of(a.t, (int)a.count, blockIdx.x)];
    const int64_t at = (int64_t)(blockIdx.x - t.first) * kBlockValues + threadIdx.x * 8, left = t.n - at;
    const int live = left < 8 ? (left > 0 ? (int)left : 0) : 8;         // lanes without a value take part in the block's largest
    const int64_t block = at / CCE_STATE8_BLOCK;
    const double clip = a.clip_coef ? (double)a.clip_coef[0] : 1.0;
    const double b1 = (double)a.beta1, b2 = (double)a.beta2;
    float p[8], g[8];
    load_f32(t.param, at, live, p);
    load_grad(t.grad, t.grad_bf16 != 0, at, live, g);
    const ou32x2 mc = load_codes(t.m, at, live), vc = load_codes(t.v, at, live);
    const int ms = live > 0 ? t.m_scale[block] : 127, vs = live > 0 ? t.v_scale[block] : 127;
    double m[8], r[8];
    uint32_t mtop = 0u, rtop = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double ge = (double)g[e] * clip;
        const double r0 = decode8<4>((vc[e >> 2] >> (8 * (e & 3))) & 0xffu, vs);
        m[e] = b1 * decode8<3>((mc[e >> 2] >> (8 * (e & 3))) & 0xffu, ms) + (1.0 - b1) * ge;
        const double v = b2 * (r0 * r0) + ((1.0 - b2) * ge) * ge;
        r[e] = sqrt(v);
        p[e] = adamw_param(p[e], (float)m[e], (float)v, t.lr, t.decay, a);
        const uint32_t mw = high_word_up(m[e]), rw = high_word_up(r[e]);
        mtop = mw > mtop ? mw : mtop;
        rtop = rw > rtop ? rw : rtop;
    }
#pragma unroll
    for (int o = 1; o <= 8; o <<= 1) {
        const uint32_t mo = (uint32_t)__shfl_xor((int)mtop, o), ro = (uint32_t)__shfl_xor((int)rtop, o);
        mtop = mo > mtop ? mo : mtop;
        rtop = ro > rtop ? ro : rtop;
    }
    if (live == 0) return;
    const int em = scale_exponent<3>(mtop), er = scale_exponent<4>(rtop);
    ou32x2 mo = {0u, 0u}, vo = {0u, 0u};
    const uint32_t base = (uint32_t)at + (uint32_t)((uint64_t)at >> 32) * 32310901u + a.key;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t h = mix32(base + e);
        mo[e >> 2] |= encode8<3>(m[e], em, h >> 15) << (8 * (e & 3));
        vo[e >> 2] |= encode8<4>(r[e], er, h & 0xffffu) << (8 * (e & 3));
    }
    store_f32(t.param, at, live, p);
    if (t.param_bf16) store_bf16(t.param_bf16, at, live, p);
    store_codes(t.m, at, live, mo);
    store_codes(t.v, at, live, vo);
    if ((threadIdx.x & 15) == 0) {
        t.m_scale[block] = (uint8_t)(em + 127);
        t.v_scale[block] = (uint8_t)(er + 127);
    }
}

template <int BITS>
__global__ __launch_bounds__(256) void state8_read_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                          int64_t n, float* __restrict__ out) {
    for (int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; at < n; at += (int64_t)gridDim.x * kBlockValues) {
        const int live = n - at < 8 ? (int)(n - at) : 8;
        const ou32x2 c = load_codes(codes, at, live);
        const int scale = scales[at / CCE_STATE8_BLOCK];
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double d = decode8<BITS>((c[e >> 2] >> (8 * (e & 3))) & 0xffu, scale);
            x[e] = (float)(BITS == 4 ? d * d : d);
        }
        store_f32(out, at, live, x);
    }
}

static uint32_t mix32_host(uint32_t h) {
    h ^= h >> 16;
    h *= 2891336453u;
    h ^= h >> 15;
    h *= 29943829u;
    return h ^ (h >> 16);
}

static bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

static int check_gradients(const cce_optim_tensor* tensors, int64_t count) {
    if (!tensors || count <= 0) return CCE_ERR_INVALID;
    int64_t blocks = 0;
    for (int64_t i = 0; i < count; ++i) {
        const cce_optim_tensor& t = tensors[i];
        if (t.n < 0) return CCE_ERR_INVALID;
        if (t.n == 0) continue;
        blocks += t.n / kBlockValues + 1;
        if (t.n > kMaxTensor || blocks > 0x7fffffff) return CCE_ERR_UNSUPPORTED;
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
            a.t[a.count++] = NormTensor{t.grad, t.n, (uint32_t)chunks, (uint32_t)t.grad_bf16};
            chunks += (t.n + kBlockValues - 1) / kBlockValues;
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
    StepArgs a;
    a.clip_coef = clip_coef;
    a.beta1 = beta1; a.beta2 = beta2; a.eps = eps;
    a.inv_bc1 = (float)(1.0 / (1.0 - pow((double)beta1, (double)step)));
    a.inv_bc2 = (float)(1.0 / (1.0 - pow((double)beta2, (double)step)));
    a.key = mix32_host(seed + mix32_host((uint32_t)step));
    for (int state8 = 0; state8 < 2; ++state8) {
        for (int64_t i = 0; i < count;) {
            a.count = 0;
            int64_t blocks = 0;
            for (; i < count && a.count < (uint32_t)kStepTensors; ++i) {
                const cce_optim_tensor& t = tensors[i];
                if (t.n == 0 || t.state8 != state8) continue;
                const int64_t own = (t.n + kBlockValues - 1) / kBlockValues;
                if (blocks + own > kMaxGrid) break;
                const float rate = lr * t.lr_scale;
                a.t[a.count++] = StepTensor{t.param, (uint16_t*)t.param_bf16, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.n,
                                            rate, 1.f - rate * t.weight_decay, (uint32_t)blocks, (uint32_t)t.grad_bf16};
                blocks += own;
            }
            if (a.count == 0) continue;
            if (state8) hipLaunchKernelGGL(adamw_multi8_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, a);
            else hipLaunchKernelGGL(adamw_multi_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, a);
        }
    }
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

int cce_adamw_state8_read(const void* codes, const uint8_t* scales, int64_t n, int second, float* out, void* stream_) {
    if (!codes || !scales || !out || n <= 0 || (second != 0 && second != 1)) return CCE_ERR_INVALID;
    if (misaligned(codes, 8) || misaligned(out, 16)) return CCE_ERR_INVALID;
    const int64_t want = (n + kBlockValues - 1) / kBlockValues;
    const dim3 grid((unsigned)(want < kMaxGrid ? want : kMaxGrid));
    hipStream_t stream = (hipStream_t)stream_;
    (void)hipGetLastError();
    if (second) hipLaunchKernelGGL(state8_read_kernel<4>, grid, dim3(256), 0, stream, (const uint8_t*)codes, scales, n, out);
    else hipLaunchKernelGGL(state8_read_kernel<3>, grid, dim3(256), 0, stream, (const uint8_t*)codes, scales, n, out);
    return hip_ok(hipGetLastError()) ? CCE_OK : CCE_ERR_HIP;
}

}  // extern "C"
