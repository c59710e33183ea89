// Pieces of the router that the experts' layer uses too: logits as whole
// numbers that order as the values do, and exchanges among 16 lanes.
#pragma once

#include "ops_common.h"

namespace simops {

// NaN above everything, -infinity 0: never chosen.
__device__ inline uint32_t order_key(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);  // -0 to 0: they tie
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    if (b == 0xff800000u) return 0;
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ inline float key_value(uint32_t k) {
    return __uint_as_float(k == 0xffffffffu ? 0x7fc00000u : k & 0x80000000u ? k & 0x7fffffffu : ~k);
}

// e^x for x <= 0: 2^(x log2 e), whose argument's rounding is the error
__device__ inline float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504f); }

// (key, index) of the higher key, the lower index where they tie
__device__ inline void keep_better(uint32_t &k, uint32_t &i, uint32_t k2, uint32_t i2) {
    const bool take = k2 > k || (k2 == k && i2 < i);
    k = take ? k2 : k;
    i = take ? i2 : i;
}
template <int CTRL> __device__ inline void best_step(uint32_t &k, uint32_t &i) {
    keep_better(k, i, dpp_u32<CTRL>(k), dpp_u32<CTRL>(i));
}
// the same result in all 16 lanes
__device__ inline void best16(uint32_t &k, uint32_t &i) {
    best_step<kDppXor1>(k, i);
    best_step<kDppXor2>(k, i);
    best_step<kDppHalfMirror>(k, i);
    best_step<kDppMirror>(k, i);
}
__device__ inline float sum16(float v) {
    v += dpp_f32<kDppXor1>(v);
    v += dpp_f32<kDppXor2>(v);
    v += dpp_f32<kDppHalfMirror>(v);
    v += dpp_f32<kDppMirror>(v);
    return v;
}
__device__ inline uint32_t max16(uint32_t v) {
    v = max(v, dpp_u32<kDppXor1>(v));
    v = max(v, dpp_u32<kDppXor2>(v));
    v = max(v, dpp_u32<kDppHalfMirror>(v));
    v = max(v, dpp_u32<kDppMirror>(v));
    return v;
}

}  // namespace simops
