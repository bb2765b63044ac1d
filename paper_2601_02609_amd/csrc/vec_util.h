// Device helpers of the kernels that stream their tensors: 16-byte vectors, eight bf16 values to and from
// fp32, sums over a wavefront; order of a wavefront's LDS accesses.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cce {

typedef __attribute__((ext_vector_type(4))) unsigned int au32x4;
typedef __attribute__((ext_vector_type(4))) float af32x4;

__device__ __forceinline__ void unpack8(const au32x4& p, float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(p[i] << 16);
        f[2 * i + 1] = __uint_as_float(p[i] & 0xffff0000u);
    }
}

__device__ __forceinline__ au32x4 pack8(const float (&f)[8]) {
    au32x4 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        union { __bf16 h[2]; unsigned int u; } cv;
        cv.h[0] = (__bf16)f[2 * i];
        cv.h[1] = (__bf16)f[2 * i + 1];
        p[i] = cv.u;
    }
    return p;
}

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x += __shfl_xor(x, o);
    return x;
}

// Between LDS accesses of a wavefront's lanes to each other's places: the LDS keeps their order, and the compiler has to.
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

}  // namespace cce
