// Quantisation to 4 bits with a shared power-of-two scale for 32 elements,
// and back.  Both only move bytes: one pass over the input, wide loads, the
// conversions are single instructions.
#include "ops_quant.h"

namespace simops {
namespace {

// Blocks along the columns.  A lane holds 8 elements, four lanes a block, 32
// lanes a group of 256 columns; a half wave takes U groups at a time, so that
// U loads are under way before the first is used.
template <int T, bool WIDE, int U>
__global__ __launch_bounds__(256) void quantize_rows(const typename Elem<T>::type *__restrict__ x, int64_t cols,
                                                     int64_t stride, int64_t n_groups, uint32_t per_row,
                                                     uint8_t *__restrict__ codes, uint8_t *__restrict__ scales) {
    const int lane = threadIdx.x & 31;
    const int64_t g0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * U;
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t g = g0 + u;
        const int64_t row = (n_groups >> 32) ? g / per_row : (uint32_t)g / per_row;
        const int64_t col = (g - row * per_row) * kGroup + lane * 8;
        load8<T, WIDE>(x + row * stride + col, g < n_groups ? cols - col : 0, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t g = g0 + u;
        uint32_t sb;
        const uint32_t c = quantize8(v[u], sb);
        if (g < n_groups) {
            *(uint32_t *)(codes + g * kGroupCodes + lane * 4) = c;
            if ((lane & 3) == 0) scales[g * kGroupScales + (lane >> 2)] = (uint8_t)sb;
        }
    }
}

// Blocks along the rows of x: the result's row c is column c of x.  A
// workgroup takes 256 rows and, of each, 256 bytes; a lane holds 32 rows (one
// block) of eight bytes, all of them loaded before the first is used, and
// the codes go through LDS so that a result row is written 128 bytes at a
// time.
template <int T>
__global__ __launch_bounds__(256) void quantize_cols(const typename Elem<T>::type *__restrict__ x, int64_t rows,
                                                     int64_t cols, int64_t stride, int64_t row_groups,
                                                     uint32_t col_tiles, uint8_t *__restrict__ codes,
                                                     uint8_t *__restrict__ scales) {
    typedef typename Elem<T>::type E;
    typedef u32x2 __attribute__((aligned(2))) u32x2_any;
    constexpr int VC = 8 / sizeof(E), COLS = 32 * VC, PITCH = kGroupCodes + 16;
    __shared__ __align__(16) uint8_t tile[COLS * PITCH];
    __shared__ __align__(8) uint8_t stile[COLS * kGroupScales];
    const int part = threadIdx.x & 31, blk = threadIdx.x >> 5;  // columns part VC .., rows blk 32 ..
    const int64_t g = blockIdx.x / col_tiles;                   // group of 256 rows
    const int64_t c0 = (int64_t)(blockIdx.x % col_tiles) * COLS, c = c0 + part * VC;
    const int64_t r0 = g * 256 + blk * 32;
    E v[32][VC];
    const E *p = x + r0 * stride + c;
    if (r0 + 32 <= rows && c + VC <= cols) {
#pragma unroll
        for (int i = 0; i < 32; i++) *(u32x2 *)v[i] = *(const u32x2_any *)(p + i * stride);
    } else {
#pragma unroll
        for (int i = 0; i < 32; i++)
#pragma unroll
            for (int j = 0; j < VC; j++) v[i][j] = r0 + i < rows && c + j < cols ? p[i * stride + j] : Elem<T>::put(0.f);
    }
#pragma unroll
    for (int j = 0; j < VC; j++) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 32; i++) m = max(m, mag(Elem<T>::get(v[i][j])));
        const uint32_t sb = scale_byte(m);
        const float s = scale_value(sb);
        u32x4 out;
#pragma unroll
        for (int q = 0; q < 4; q++) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; i++) f[i] = Elem<T>::get(v[q * 8 + i][j]);
            out[q] = sb == 255 ? 0u : pack8(f, s);
        }
        const int col = part * VC + j;
        *(u32x4 *)(tile + col * PITCH + blk * 16) = out;
        stile[col * kGroupScales + blk] = (uint8_t)sb;
    }
    __syncthreads();
#pragma unroll
    for (int n = threadIdx.x; n < COLS * 8; n += 256) {  // 16 bytes each
        const int col = n >> 3, piece = n & 7;
        if (c0 + col < cols)
            *(u32x4 *)(codes + ((c0 + col) * row_groups + g) * kGroupCodes + piece * 16) =
                *(const u32x4 *)(tile + col * PITCH + piece * 16);
    }
    if (threadIdx.x < COLS && c0 + threadIdx.x < cols)
        *(u32x2 *)(scales + ((c0 + threadIdx.x) * row_groups + g) * kGroupScales) =
            *(const u32x2 *)(stile + threadIdx.x * kGroupScales);
}

// Back: a lane takes eight codes.  Their products with the scale are exact in
// 32 bits, so the one rounding is that to the type.
template <int T, bool WIDE, int U>
__global__ __launch_bounds__(256) void dequantize(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                  int64_t n_groups, uint32_t per_row, int64_t cols,
                                                  typename Elem<T>::type *__restrict__ out, int64_t stride) {
    typedef typename Elem<T>::type E;
    const int lane = threadIdx.x & 31;
    const int64_t g0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * U;
    uint32_t c[U], sb[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t g = min(g0 + u, n_groups - 1);
        c[u] = *(const uint32_t *)(codes + g * kGroupCodes + lane * 4);
        sb[u] = scales[g * kGroupScales + (lane >> 2)];
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int64_t g = g0 + u;
        if (g >= n_groups) return;
        const int64_t row = (n_groups >> 32) ? g / per_row : (uint32_t)g / per_row;
        const int64_t col = (g - row * per_row) * kGroup + lane * 8;
        const float s = scale_value(sb[u]);
        E e[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t n = (c[u] >> (4 * i)) & 15, k = n & 7;
            // 0 .5 1 1.5 2 3 4 6 in steps of a half
            const uint32_t halves = (0xC8643210u >> (4 * k)) & 15;
            const float v = (float)halves * 0.5f * s;
            e[i] = Elem<T>::put(n & 8 ? -v : v);
        }
        E *p = out + row * stride + col;
        if (WIDE || col + 8 <= cols) {
            if (col < cols) {
                ((u32x4_any *)p)[0] = ((u32x4 *)e)[0];
                if (sizeof(E) == 4) ((u32x4_any *)p)[1] = ((u32x4 *)e)[1];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (col + i < cols) p[i] = e[i];
        }
    }
}

template <int T>
sim_status quantize_t(hipStream_t st, const void *xv, int64_t rows, int64_t cols, int64_t stride, bool transpose,
                      uint8_t *codes, uint8_t *scales) {
    typedef typename Elem<T>::type E;
    const E *x = (const E *)xv;
    if (transpose) {
        const int64_t rg = groups_of(rows);
        constexpr int COLS = 256 / sizeof(E);
        const uint32_t ct = (uint32_t)((cols + COLS - 1) / COLS);
        quantize_cols<T><<<(uint32_t)(ct * rg), 256, 0, st>>>(x, rows, cols, stride, rg, ct, codes, scales);
        return SIM_OPS_LAUNCH_OK();
    }
    const int64_t per = groups_of(cols), n = rows * per;
    const bool wide = cols % 8 == 0;
    constexpr int U = 4;
    const bool many = n >= 8 * U * 1024;
    const int64_t blocks = many ? (n + 8 * U - 1) / (8 * U) : (n + 7) / 8;
    if (many) {
        if (wide) quantize_rows<T, true, U><<<(uint32_t)blocks, 256, 0, st>>>(x, cols, stride, n, per, codes, scales);
        else quantize_rows<T, false, U><<<(uint32_t)blocks, 256, 0, st>>>(x, cols, stride, n, per, codes, scales);
    } else {
        if (wide) quantize_rows<T, true, 1><<<(uint32_t)blocks, 256, 0, st>>>(x, cols, stride, n, per, codes, scales);
        else quantize_rows<T, false, 1><<<(uint32_t)blocks, 256, 0, st>>>(x, cols, stride, n, per, codes, scales);
    }
    return SIM_OPS_LAUNCH_OK();
}

template <int T>
sim_status dequantize_t(hipStream_t st, const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols,
                        void *out, int64_t stride) {
    typedef typename Elem<T>::type E;
    const int64_t per = groups_of(cols), n = rows * per;
    const bool wide = cols % 8 == 0;
    constexpr int U = 4;
    const bool many = n >= 8 * U * 1024;
    const uint32_t blocks = (uint32_t)(many ? (n + 8 * U - 1) / (8 * U) : (n + 7) / 8);
    if (many) {
        if (wide) dequantize<T, true, U><<<blocks, 256, 0, st>>>(codes, scales, n, per, cols, (E *)out, stride);
        else dequantize<T, false, U><<<blocks, 256, 0, st>>>(codes, scales, n, per, cols, (E *)out, stride);
    } else {
        if (wide) dequantize<T, true, 1><<<blocks, 256, 0, st>>>(codes, scales, n, per, cols, (E *)out, stride);
        else dequantize<T, false, 1><<<blocks, 256, 0, st>>>(codes, scales, n, per, cols, (E *)out, stride);
    }
    return SIM_OPS_LAUNCH_OK();
}

}  // namespace

sim_status launch_quantize(hipStream_t st, const void *x, int type, int64_t rows, int64_t cols, int64_t stride,
                           bool transpose, uint8_t *codes, uint8_t *scales) {
    if (type == SIM_TYPE_F32) return quantize_t<SIM_TYPE_F32>(st, x, rows, cols, stride, transpose, codes, scales);
    if (type == SIM_TYPE_F16) return quantize_t<SIM_TYPE_F16>(st, x, rows, cols, stride, transpose, codes, scales);
    return quantize_t<SIM_TYPE_BF16>(st, x, rows, cols, stride, transpose, codes, scales);
}

sim_status launch_dequantize(hipStream_t st, const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols,
                             void *out, int type, int64_t stride) {
    if (type == SIM_TYPE_F32) return dequantize_t<SIM_TYPE_F32>(st, codes, scales, rows, cols, out, stride);
    if (type == SIM_TYPE_F16) return dequantize_t<SIM_TYPE_F16>(st, codes, scales, rows, cols, out, stride);
    return dequantize_t<SIM_TYPE_BF16>(st, codes, scales, rows, cols, out, stride);
}

}  // namespace simops
