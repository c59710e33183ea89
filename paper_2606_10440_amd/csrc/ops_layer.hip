// The experts' layer for few tokens: two products per expert over the tokens
// that chose it.  With few tokens the time is that of reading the chosen
// experts' weights once; everything else is kept out of the way of that
// stream.
//
// Both products run on 16x16x32 matrix instructions with sixteen weight rows
// as the first operand and sixteen of the expert's tokens as the second, the
// waves of a workgroup each taking a part of the contraction.  Activations
// and 4-bit weights enter as bf16; values of more than 8 significant bits
// (fp16 inputs, the hidden values between the products) enter as the sum of
// two bf16 parts, which is free where the weights' bytes bound the time.
#include "ops_common.h"

namespace simops {
namespace {

constexpr int kWaves = 4;
constexpr int kStep = 128;  // columns of one step of a wave

typedef u32x4 __attribute__((aligned(2))) u32x4_a2;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// Which expert the a-th non-empty list belongs to; -1 past the last.
__device__ inline int nth_expert(const int32_t *__restrict__ offsets, int E, int a, int *shared) {
    const int lane = threadIdx.x & 63;
    if (threadIdx.x < 64) {
        int seen = 0, found = -1;
        for (int e0 = 0; e0 < E && found < 0; e0 += 64) {
            const int e = e0 + lane;
            const bool some = e < E && offsets[e + 1] > offsets[e];
            const uint64_t all = __ballot(some);
            const bool hit = some && seen + __popcll(all & ((1ull << lane) - 1)) == a;
            const uint64_t at = __ballot(hit);
            if (at) found = e0 + __ffsll((unsigned long long)at) - 1;
            seen += __popcll(all);
        }
        if (lane == 0) *shared = found;
    }
    __syncthreads();
    return *shared;
}

// 16-bit elements k .. k + 7 of a row of K, zeros past its end, as raw bits.
__device__ inline u32x4 load_row8(const uint16_t *__restrict__ row, int64_t k, int64_t K) {
    if (k + 8 <= K) return *(const u32x4_a2 *)(row + k);
    uint16_t v[8];
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = k + i < K ? row[k + i] : 0;
    return *(u32x4 *)v;
}

// fp16 to the two bf16 values that add up to it
__device__ inline void split_f16(u32x4 raw, bf16x8 &hi, bf16x8 &lo) {
    const f16x8 v = __builtin_bit_cast(f16x8, raw);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        hi[i] = (__bf16)(float)v[i];
        lo[i] = (__bf16)((float)v[i] - (float)hi[i]);
    }
}

// eight 4-bit weights to bf16 (exact)
__device__ inline bf16x8 widen8(uint32_t codes, float scale) {
    bf16x8 r;
    bf16x2 *p = (bf16x2 *)&r;
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return r;
}

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// A wave's step of one 16-row weight tile: lane l holds row l % 16 and, of
// 128 columns, elements 32 (l / 16) + 8 s .. + 7 in instruction s.
template <int WT> struct Weights;  // the four instructions' operands
template <> struct Weights<SIM_TYPE_BF16> {
    u32x4 raw[4];
    __device__ void load(const void *base, const uint8_t *, int64_t row, int64_t K, int64_t k) {
        const uint16_t *p = (const uint16_t *)base + row * K;
#pragma unroll
        for (int s = 0; s < 4; s++) raw[s] = load_row8(p, k + 8 * s, K);
    }
    __device__ f32x4 mul(int s, bf16x8 x, f32x4 c) const { return mfma(__builtin_bit_cast(bf16x8, raw[s]), x, c); }
};
template <> struct Weights<SIM_TYPE_F16> {
    u32x4 raw[4];
    __device__ void load(const void *base, const uint8_t *, int64_t row, int64_t K, int64_t k) {
        const uint16_t *p = (const uint16_t *)base + row * K;
#pragma unroll
        for (int s = 0; s < 4; s++) raw[s] = load_row8(p, k + 8 * s, K);
    }
    __device__ f32x4 mul(int s, bf16x8 x, f32x4 c) const {
        bf16x8 hi, lo;
        split_f16(raw[s], hi, lo);
        return mfma(lo, x, mfma(hi, x, c));
    }
};
template <> struct Weights<SIM_TYPE_MX4> {
    u32x4 raw;
    uint32_t sb;
    __device__ void load(const void *base, const uint8_t *scales, int64_t row, int64_t K, int64_t k) {
        const int64_t g = groups_of(K);
        raw = u32x4{0, 0, 0, 0};
        sb = 0;
        if (k < K) {  // the row's last group may end in the middle of a step
            raw = *(const u32x4 *)((const uint8_t *)base + row * g * kGroupCodes + k / 2);
            sb = scales[row * g * kGroupScales + k / 32];
        }
    }
    __device__ f32x4 mul(int s, bf16x8 x, f32x4 c) const { return mfma(widen8(raw[s], scale_value(sb)), x, c); }
};

// Gate and up products of sixteen hidden units of one expert.
template <int T, int WT>
__global__ __launch_bounds__(64 * kWaves) void layer_up(const uint16_t *__restrict__ x, int64_t x_stride, int64_t D,
                                                        const void *__restrict__ w13, const uint8_t *__restrict__ s13,
                                                        int64_t F, int E, int k, const int32_t *__restrict__ offsets,
                                                        const int32_t *__restrict__ order,
                                                        const float *__restrict__ weights, uint32_t tiles,
                                                        __bf16 *__restrict__ h_hi, __bf16 *__restrict__ h_lo,
                                                        int64_t h_pitch) {
    __shared__ int s_expert;
    __shared__ f32x4 part[kWaves][2][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int e = nth_expert(offsets, E, blockIdx.x / tiles, &s_expert);
    if (e < 0) return;
    const int64_t f0 = (int64_t)(blockIdx.x % tiles) * 16;
    const int first = offsets[e], n = offsets[e + 1] - first;
    const int64_t row = (int64_t)e * 2 * F + min(f0 + r, F - 1);
    for (int c0 = 0; c0 < n; c0 += 16) {
        const int slot = order[first + min(c0 + r, n - 1)];
        const uint16_t *xr = x + (int64_t)(slot / k) * x_stride;
        f32x4 g = {0}, u = {0};
        for (int64_t d = wave * kStep; d < D; d += kWaves * kStep) {
            const int64_t kk = d + q * 32;
            Weights<WT> wg, wu;
            wg.load(w13, s13, row, D, kk);
            wu.load(w13, s13, row + F, D, kk);
#pragma unroll
            for (int s = 0; s < 4; s++) {
                const u32x4 raw = load_row8(xr, kk + 8 * s, D);
                if (T == SIM_TYPE_BF16) {
                    const bf16x8 v = __builtin_bit_cast(bf16x8, raw);
                    g = wg.mul(s, v, g);
                    u = wu.mul(s, v, u);
                } else {
                    bf16x8 hi, lo;
                    split_f16(raw, hi, lo);
                    g = wg.mul(s, lo, wg.mul(s, hi, g));
                    u = wu.mul(s, lo, wu.mul(s, hi, u));
                }
            }
        }
        part[wave][0][lane] = g;
        part[wave][1][lane] = u;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 1; w < kWaves; w++) {
                g += part[w][0][lane];
                u += part[w][1][lane];
            }
            if (c0 + r < n) {
                const float w = weights[slot];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int64_t f = f0 + 4 * q + i;
                    const float v = f < F ? g[i] / (1.f + expf(-g[i])) * u[i] * w : 0.f;
                    const __bf16 hi = (__bf16)v;
                    h_hi[slot * h_pitch + f] = hi;
                    h_lo[slot * h_pitch + f] = (__bf16)(v - (float)hi);
                }
            }
        }
        __syncthreads();
    }
}

// Sixteen output columns of one expert, for each of its slots.
template <int WT>
__global__ __launch_bounds__(64 * kWaves) void layer_down(const __bf16 *__restrict__ h_hi, const __bf16 *__restrict__ h_lo,
                                                          int64_t h_pitch, int64_t F, const void *__restrict__ w2,
                                                          const uint8_t *__restrict__ s2, int64_t D, int E,
                                                          const int32_t *__restrict__ offsets,
                                                          const int32_t *__restrict__ order, uint32_t tiles,
                                                          float *__restrict__ out) {
    __shared__ int s_expert;
    __shared__ f32x4 part[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
    const int e = nth_expert(offsets, E, blockIdx.x / tiles, &s_expert);
    if (e < 0) return;
    const int64_t d0 = (int64_t)(blockIdx.x % tiles) * 16;
    const int first = offsets[e], n = offsets[e + 1] - first;
    const int64_t row = (int64_t)e * D + min(d0 + r, D - 1);
    for (int c0 = 0; c0 < n; c0 += 16) {
        const int slot = order[first + min(c0 + r, n - 1)];
        const uint16_t *hr = (const uint16_t *)h_hi + slot * h_pitch, *lr = (const uint16_t *)h_lo + slot * h_pitch;
        f32x4 y = {0};
        for (int64_t f = wave * kStep; f < F; f += kWaves * kStep) {
            const int64_t kk = f + q * 32;
            Weights<WT> w;
            w.load(w2, s2, row, F, kk);
#pragma unroll
            for (int s = 0; s < 4; s++) {
                y = w.mul(s, __builtin_bit_cast(bf16x8, load_row8(hr, kk + 8 * s, F)), y);
                y = w.mul(s, __builtin_bit_cast(bf16x8, load_row8(lr, kk + 8 * s, F)), y);
            }
        }
        part[wave][lane] = y;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int w = 1; w < kWaves; w++) y += part[w][lane];
            if (c0 + r < n)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int64_t d = d0 + 4 * q + i;
                    if (d < D) out[(int64_t)slot * D + d] = y[i];
                }
        }
        __syncthreads();
    }
}

// A token's result: its choices in order.
template <int T>
__global__ __launch_bounds__(256) void layer_join(const float *__restrict__ part, const int32_t *__restrict__ experts, int k,
                                                  int64_t D, typename Elem<T>::type *__restrict__ y, int64_t y_stride,
                                                  uint32_t tiles) {
    const int64_t t = blockIdx.x / tiles, d = (int64_t)(blockIdx.x % tiles) * 256 + threadIdx.x;
    if (d >= D) return;
    float s = 0.f;
    for (int j = 0; j < k; j++)
        if (experts[t * k + j] >= 0) s += part[(t * k + j) * D + d];
    y[t * y_stride + d] = Elem<T>::put(s);
}

inline int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }
inline size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

// The workspace in the order in which it is handed out.
struct Layout {
    size_t experts, weights, offsets, order, route, hi, lo, part, end;
    int64_t pitch;
    Layout(int64_t T, int64_t D, int E, int k, int64_t F) {
        const size_t n = (size_t)T * k;
        pitch = up16(F);
        size_t at = 0;
        const auto take = [&](size_t bytes) { const size_t p = at; at += aligned(bytes); return p; };
        experts = take(n * 4);
        weights = take(n * 4);
        offsets = take((size_t)(E + 1) * 4);
        order = take(n * 4);
        route = take(route_workspace(T, E, k));
        hi = take(n * pitch * 2);
        lo = take(n * pitch * 2);
        part = take(n * D * 4);
        end = at;
    }
};

template <int T, int WT> sim_status layer_t(hipStream_t st, const LayerArgs &a, uint8_t *ws) {
    const RouteArgs &r = a.route;
    const Layout at(r.T, a.D, r.E, r.k, a.F);
    int32_t *experts = (int32_t *)(ws + at.experts), *offsets = (int32_t *)(ws + at.offsets), *order = (int32_t *)(ws + at.order);
    float *weights = (float *)(ws + at.weights), *part = (float *)(ws + at.part);
    __bf16 *hi = (__bf16 *)(ws + at.hi), *lo = (__bf16 *)(ws + at.lo);
    const sim_status s = launch_route(st, r, experts, weights, offsets, order, ws + at.route);
    if (s != SIM_OK) return s;
    const uint32_t lists = (uint32_t)std::min<int64_t>(r.E, r.T * r.k);
    if (a.F > 0) {
        const uint32_t tf = (uint32_t)((a.F + 15) / 16);
        layer_up<T, WT><<<lists * tf, 64 * kWaves, 0, st>>>((const uint16_t *)a.x, a.x_stride, a.D, a.w13, a.s13, a.F, r.E,
                                                           r.k, offsets, order, weights, tf, hi, lo, at.pitch);
    }
    const uint32_t td = (uint32_t)((a.D + 15) / 16), tj = (uint32_t)((a.D + 255) / 256);
    layer_down<WT><<<lists * td, 64 * kWaves, 0, st>>>(hi, lo, at.pitch, a.F, a.w2, a.s2, a.D, r.E, offsets, order, td, part);
    layer_join<T><<<(uint32_t)(r.T * tj), 256, 0, st>>>(part, experts, r.k, a.D, (typename Elem<T>::type *)a.y, a.y_stride, tj);
    return SIM_OPS_LAUNCH_OK();
}

}  // namespace

size_t layer_workspace(int64_t T, int64_t D, int E, int k, int64_t F) { return Layout(T, D, E, k, F).end; }

sim_status launch_layer(hipStream_t st, const LayerArgs &a, void *ws) {
    uint8_t *w = (uint8_t *)ws;
    if (a.type == SIM_TYPE_BF16)
        return a.mx4 ? layer_t<SIM_TYPE_BF16, SIM_TYPE_MX4>(st, a, w) : layer_t<SIM_TYPE_BF16, SIM_TYPE_BF16>(st, a, w);
    return a.mx4 ? layer_t<SIM_TYPE_F16, SIM_TYPE_MX4>(st, a, w) : layer_t<SIM_TYPE_F16, SIM_TYPE_F16>(st, a, w);
}

}  // namespace simops
