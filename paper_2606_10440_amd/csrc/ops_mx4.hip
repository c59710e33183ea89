// Quantisation to 4 bits with a shared power-of-two scale for 32 elements,
// and back.  Both only move bytes: one pass over the input, wide loads, the
// conversions are single instructions.  Accesses are sixteen bytes at any
// alignment of the type; only the last few elements of a row go one by one.
#include "ops_quant.h"

namespace simops {
namespace {

// Blocks along the columns.  A lane holds 8 elements, four lanes a block, 32
// lanes a group of 256 columns; a half wave takes U groups at a time, so that
// U loads are under way before the first is used.  They go past the caches:
// 16384 x 8192 bf16 57 us, 5.9 TB/s in and out (71 us through them).
template <int T, bool WIDE, int U>
__device__ inline void rows_block(uint32_t block, const typename Elem<T>::type *__restrict__ x, int64_t cols, int64_t stride,
                                  int64_t n_groups, uint32_t per_row, uint8_t *__restrict__ codes,
                                  uint8_t *__restrict__ scales) {
    const int lane = threadIdx.x & 31;
    const int64_t g0 = ((int64_t)block * 8 + (threadIdx.x >> 5)) * U;
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

template <int T, bool WIDE, int U>
__global__ __launch_bounds__(256) void quantize_rows(const typename Elem<T>::type *__restrict__ x, int64_t cols,
                                                     int64_t stride, int64_t n_groups, uint32_t per_row,
                                                     uint8_t *__restrict__ codes, uint8_t *__restrict__ scales) {
    rows_block<T, WIDE, U>(blockIdx.x, x, cols, stride, n_groups, per_row, codes, scales);
}

// A type of two bytes for every T, so that code for those that have them compiles.
template <int T> using E16 = std::conditional_t<T == SIM_TYPE_F32, _Float16, typename Elem<T>::type>;
template <int T> constexpr int kTileCols = 256 / sizeof(typename Elem<T>::type);

// Blocks along the rows of x: the result's row c is column c of x.  A
// workgroup takes 256 rows and, of each, 256 bytes; a lane holds 32 rows (one
// block) of eight bytes, all of them loaded before the first is used, and
// the codes go through LDS so that a result row is written 128 bytes at a
// time.  4096 x 4096 bf16 9.6 us, 4.4 TB/s (15.6 us with 128 bytes of each
// row); 4099 x 5003 fp32 20 us, 4.7 TB/s.
template <int T>
__device__ inline void cols_block(uint32_t block, const typename Elem<T>::type *__restrict__ x, int64_t rows, int64_t cols,
                                  int64_t stride, int64_t row_groups, uint32_t col_tiles, uint8_t *__restrict__ codes,
                                  uint8_t *__restrict__ scales) {
    typedef typename Elem<T>::type E;
    typedef u32x2 __attribute__((aligned(2))) u32x2_any;
    constexpr int VC = 8 / sizeof(E), COLS = kTileCols<T>, PITCH = kGroupCodes + 16;
    __shared__ __align__(16) uint8_t tile[COLS * PITCH];
    __shared__ __align__(8) uint8_t stile[COLS * kGroupScales];
    const int part = threadIdx.x & 31, blk = threadIdx.x >> 5;  // columns part VC .., rows blk 32 ..
    const int64_t g = block / col_tiles;                       // group of 256 rows
    const int64_t c0 = (int64_t)(block % col_tiles) * COLS, c = c0 + part * VC;
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
    // magnitudes of 16-bit values order as whole numbers too: two columns at once
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    typedef uint32_t u32_two __attribute__((may_alias));
    uint32_t top[VC];
    if (sizeof(E) == 2) {
        u16x2 m[VC / 2];
#pragma unroll
        for (int j = 0; j < VC / 2; j++) {
            m[j] = u16x2{0, 0};
#pragma unroll
            for (int i = 0; i < 32; i++)
                m[j] = __builtin_elementwise_max(m[j], __builtin_bit_cast(u16x2, ((const u32_two *)v[i])[j] & 0x7fff7fffu));
            top[2 * j] = mag((float)__builtin_bit_cast(E16<T>, (uint16_t)m[j][0]));
            top[2 * j + 1] = mag((float)__builtin_bit_cast(E16<T>, (uint16_t)m[j][1]));
        }
    } else {
#pragma unroll
        for (int j = 0; j < VC; j++) {
            top[j] = 0;
#pragma unroll
            for (int i = 0; i < 32; i++) top[j] = max(top[j], mag(Elem<T>::get(v[i][j])));
        }
    }
#pragma unroll
    for (int j = 0; j < VC; j++) {
        const uint32_t m = top[j];
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

template <int T>
__global__ __launch_bounds__(256) void quantize_cols(const typename Elem<T>::type *__restrict__ x, int64_t rows, int64_t cols,
                                                     int64_t stride, int64_t row_groups, uint32_t col_tiles,
                                                     uint8_t *__restrict__ codes, uint8_t *__restrict__ scales) {
    cols_block<T>(blockIdx.x, x, rows, cols, stride, row_groups, col_tiles, codes, scales);
}

// Several matrices of one type in one launch, each along its rows or its
// columns: one that is wanted both ways comes from the caches the second
// time.  Four operands of 4096 x 4096 bf16: 36 us (38 one by one, and three
// launches more).
struct Jobs {
    QuantizeJob job[kMaxJobs];
    uint32_t end[kMaxJobs];  // blocks of the jobs up to this one
};
constexpr int kJobUnroll = 4;

template <int T> __global__ __launch_bounds__(256) void quantize_jobs(Jobs jobs) {
    int i = 0;
    while (blockIdx.x >= jobs.end[i]) i++;
    const QuantizeJob &j = jobs.job[i];
    const uint32_t block = blockIdx.x - (i ? jobs.end[i - 1] : 0);
    const typename Elem<T>::type *x = (const typename Elem<T>::type *)j.x;
    if (j.transpose) {
        cols_block<T>(block, x, j.rows, j.cols, j.stride, groups_of(j.rows), (uint32_t)((j.cols + kTileCols<T> - 1) / kTileCols<T>),
                      j.codes, j.scales);
    } else {
        const int64_t per = groups_of(j.cols);
        rows_block<T, false, kJobUnroll>(block, x, j.cols, j.stride, j.rows * per, (uint32_t)per, j.codes, j.scales);
    }
}

template <int T> sim_status jobs_t(hipStream_t st, const QuantizeJob *job, int n) {
    Jobs jobs = {};
    uint32_t blocks = 0;
    for (int i = 0; i < kMaxJobs; i++) {
        if (i < n) {
            const QuantizeJob &j = job[i];
            jobs.job[i] = j;
            blocks += j.transpose ? (uint32_t)(groups_of(j.rows) * ((j.cols + kTileCols<T> - 1) / kTileCols<T>))
                                  : (uint32_t)((j.rows * groups_of(j.cols) + 8 * kJobUnroll - 1) / (8 * kJobUnroll));
        }
        jobs.end[i] = blocks;
    }
    quantize_jobs<T><<<blocks, 256, 0, st>>>(jobs);
    return SIM_OPS_LAUNCH_OK();
}

// Back: a lane takes eight codes.  Their products with the scale are exact in
// 32 bits, so the one rounding is that to the type.  16384 x 8192 to bf16: 58
// us, 5.8 TB/s; 5003 x 4099: 13.5 us (33 with element stores for the odd row
// length).
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
        constexpr int COLS = kTileCols<T>;
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

sim_status launch_quantize_jobs(hipStream_t st, int type, const QuantizeJob *job, int n) {
    if (type == SIM_TYPE_F32) return jobs_t<SIM_TYPE_F32>(st, job, n);
    if (type == SIM_TYPE_F16) return jobs_t<SIM_TYPE_F16>(st, job, n);
    return jobs_t<SIM_TYPE_BF16>(st, job, n);
}

sim_status launch_dequantize(hipStream_t st, const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols,
                             void *out, int type, int64_t stride) {
    if (type == SIM_TYPE_F32) return dequantize_t<SIM_TYPE_F32>(st, codes, scales, rows, cols, out, stride);
    if (type == SIM_TYPE_F16) return dequantize_t<SIM_TYPE_F16>(st, codes, scales, rows, cols, out, stride);
    return dequantize_t<SIM_TYPE_BF16>(st, codes, scales, rows, cols, out, stride);
}

}  // namespace simops
