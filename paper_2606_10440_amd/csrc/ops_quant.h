// Eight elements at a time into 4 bits; four neighbouring lanes share a block.
#pragma once

#include "ops_common.h"

namespace simops {

typedef u32x4 __attribute__((aligned(2))) u32x4_any;

// Eight consecutive elements of a row, zeros past the end of the row.
// WIDE: the row is a whole number of eights.
template <int T, bool WIDE = false>
__device__ inline void load8(const typename Elem<T>::type *p, int64_t left, float v[8]) {
    typedef typename Elem<T>::type E;
    if (WIDE || left >= 8) {
        if (left > 0) {
            E e[8];
            ((u32x4 *)e)[0] = __builtin_nontemporal_load((const u32x4_any *)p);
            if (sizeof(E) == 4) ((u32x4 *)e)[1] = __builtin_nontemporal_load((const u32x4_any *)p + 1);
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = Elem<T>::get(e[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = 0.f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < left ? Elem<T>::get(p[i]) : 0.f;
    }
}

// The codes of a lane's eight elements and the scale byte of its block, which
// is held by four neighbouring lanes.
__device__ inline uint32_t quantize8(const float v[8], uint32_t &sb) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, mag(v[i]));
    m = max(m, dpp_u32<kDppXor1>(m));
    m = max(m, dpp_u32<kDppXor2>(m));
    sb = scale_byte(m);
    return sb == 255 ? 0u : pack8(v, scale_value(sb));
}

}  // namespace simops
