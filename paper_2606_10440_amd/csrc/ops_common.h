// Shared pieces of the operator kernels (ops_*.hip): element types, 4-bit
// packing, and the launchers that ops_api.cpp calls after its checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "../../include/simgpu_ops.h"
#include "ops_forms.h"

namespace simops {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---- element types: the value of one element, and one value rounded to the type
template <int T> struct Elem;
template <> struct Elem<SIM_TYPE_F32> {
    typedef float type;
    static __device__ float get(float v) { return v; }
    static __device__ float put(float v) { return v; }
};
template <> struct Elem<SIM_TYPE_F16> {
    typedef _Float16 type;
    static __device__ float get(_Float16 v) { return (float)v; }
    static __device__ _Float16 put(float v) { return (_Float16)v; }
};
template <> struct Elem<SIM_TYPE_BF16> {
    typedef __bf16 type;
    static __device__ float get(__bf16 v) { return (float)v; }
    static __device__ __bf16 put(float v) { return (__bf16)v; }
};

// ---- 4-bit blocks

// Scale byte of a block from its largest magnitude (finite: exponent - 2,
// at least 2^-127; NaN and infinity, whose exponent field is 255: byte 255).
__device__ inline uint32_t scale_byte(uint32_t amax_bits) {
    uint32_t field = amax_bits >> 23;
    return field == 255 ? 255u : field < 2 ? 0u : field - 2;
}

// 2^(byte - 127) in 32 bits; byte 0 is the subnormal 2^-127.  255 is NaN.
__device__ inline float scale_value(uint32_t byte) {
    return __uint_as_float(byte == 255 ? 0x7fc00000u : byte ? byte << 23 : 0x00400000u);
}

// Eight values to eight codes (element 0 in the lowest four bits).  The
// conversion divides by the scale, rounds to nearest even and saturates.
__device__ inline uint32_t pack8(const float v[8], float scale) {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
    return r;
}

// ---- lanes

// value of the lane that DPP control word CTRL names, within rows of 16 lanes
template <int CTRL> __device__ inline uint32_t dpp_u32(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
template <int CTRL> __device__ inline float dpp_f32(float v) { return __uint_as_float(dpp_u32<CTRL>(__float_as_uint(v))); }
constexpr int kDppXor1 = 0xB1;    // quad_perm 1,0,3,2
constexpr int kDppXor2 = 0x4E;    // quad_perm 2,3,0,1
constexpr int kDppHalfMirror = 0x141;  // lane i of 8 <-> 7 - i
constexpr int kDppMirror = 0x140;      // lane i of 16 <-> 15 - i

// Between the writes and the reads of LDS through which the lanes of a wave
// exchange values: the wave's accesses are in order, and the compiler has to
// keep them so.  It costs no instruction.
__device__ inline void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Magnitude bits of 32-bit values order as whole numbers, NaN above infinity,
// so a block's largest magnitude is a whole-number maximum.
__device__ inline uint32_t mag(float v) { return __float_as_uint(v) & 0x7fffffffu; }

#define SIM_OPS_LAUNCH_OK() (hipGetLastError() == hipSuccess ? SIM_OK : SIM_ERR_DEVICE)

// ---- launchers (arguments already checked)
sim_status launch_quantize(hipStream_t st, const void *x, int type, int64_t rows, int64_t cols, int64_t stride,
                           bool transpose, uint8_t *codes, uint8_t *scales);
struct QuantizeJob {
    const void *x;
    int64_t rows, cols, stride;  // of x
    bool transpose;
    uint8_t *codes, *scales;
};
constexpr int kMaxJobs = 4;
sim_status launch_quantize_jobs(hipStream_t st, int type, const QuantizeJob *job, int n);
sim_status launch_dequantize(hipStream_t st, const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols,
                             void *out, int type, int64_t stride);
sim_status launch_matmul(hipStream_t st, const uint8_t *ac, const uint8_t *as, const uint8_t *bc, const uint8_t *bs,
                         int64_t M, int64_t N, int64_t K, void *out, int type, int64_t stride);
// for sizes that linear_in_one takes
sim_status launch_linear(hipStream_t st, const void *x, int x_type, int64_t x_stride, const uint8_t *wc, const uint8_t *ws,
                         int64_t M, int64_t N, int64_t K, void *out, int type, int64_t stride);
struct RouteArgs {
    const void *logits;
    int type;
    int64_t T;
    int E;
    int64_t stride;
    const uint8_t *mask;
    int64_t mask_stride;
    int k;
    bool renorm;
};
sim_status launch_route(hipStream_t st, const RouteArgs &a, int32_t *experts, float *weights, int32_t *offsets,
                        int32_t *order, void *ws);
size_t route_workspace(int64_t T, int E, int k);
sim_status launch_route_grad(hipStream_t st, const RouteArgs &a, const int32_t *experts, const float *dw, void *dz);
struct LayerArgs {
    RouteArgs route;
    const void *x;
    int type;
    int64_t D, x_stride;
    const void *w13, *w2;
    const uint8_t *s13, *s2;
    bool mx4;
    int64_t F;
    void *y;
    int64_t y_stride;
};
sim_status launch_layer(hipStream_t st, const LayerArgs &a, void *ws);
size_t layer_workspace(int64_t T, int64_t D, int E, int k, int64_t F);

}  // namespace simops
