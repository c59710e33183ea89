// Products of two 4-bit matrices: C[m, n] = sum_k A[m, k] B[n, k], with the
// scaled matrix instructions, which take the codes and the block scales as
// they are stored.
//
// 32x32x64: lane l holds row l % 32 of its operand and one block of 32
// columns, half l / 32 of the 64; its scale is one byte of a register, chosen
// by the instruction.  Which columns meet in one instruction does not matter
// to the sum, so of a group of 256 columns half h takes blocks 4 h .. 4 h + 3
// in four instructions: 64 contiguous bytes of codes and one word of scales
// per lane and group.
#include "ops_common.h"

namespace simops {
namespace {

template <int T>
__global__ __launch_bounds__(256) void matmul_simple(const uint8_t *__restrict__ ac, const uint8_t *__restrict__ as,
                                                     const uint8_t *__restrict__ bc, const uint8_t *__restrict__ bs,
                                                     int64_t M, int64_t N, int groups,
                                                     typename Elem<T>::type *__restrict__ out, int64_t stride) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, h = lane >> 5;
    const int64_t tiles_n = (N + 63) / 64;
    const int64_t m0 = blockIdx.x / tiles_n * 64 + (wave >> 1) * 32, n0 = blockIdx.x % tiles_n * 64 + (wave & 1) * 32;
    const int64_t am = min(m0 + r, M - 1), bn = min(n0 + r, N - 1);  // rows past the end repeat the last one
    const uint8_t *ap = ac + am * groups * kGroupCodes + h * 64, *bp = bc + bn * groups * kGroupCodes + h * 64;
    const uint8_t *asp = as + am * groups * kGroupScales + h * 4, *bsp = bs + bn * groups * kGroupScales + h * 4;
    f32x16 acc = {0};
    for (int g = 0; g < groups; g++) {
        const int sa = *(const int *)(asp + (int64_t)g * kGroupScales), sb = *(const int *)(bsp + (int64_t)g * kGroupScales);
        i32x8 a[4], b[4];
#pragma unroll
        for (int s = 0; s < 4; s++) {
            a[s] = b[s] = i32x8{0};
            *(u32x4 *)&a[s] = *(const u32x4 *)(ap + (int64_t)g * kGroupCodes + s * 16);
            *(u32x4 *)&b[s] = *(const u32x4 *)(bp + (int64_t)g * kGroupCodes + s * 16);
        }
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[0], b[0], acc, 4, 4, 0, sa, 0, sb);
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[1], b[1], acc, 4, 4, 1, sa, 1, sb);
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[2], b[2], acc, 4, 4, 2, sa, 2, sb);
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a[3], b[3], acc, 4, 4, 3, sa, 3, sb);
    }
    if (n0 + r < N) {
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const int64_t m = m0 + 8 * (i >> 2) + 4 * h + (i & 3);
            if (m < M) out[m * stride + n0 + r] = Elem<T>::put(acc[i]);
        }
    }
}

template <int T>
sim_status matmul_t(hipStream_t st, const uint8_t *ac, const uint8_t *as, const uint8_t *bc, const uint8_t *bs, int64_t M,
                    int64_t N, int64_t K, void *out, int64_t stride) {
    const uint32_t grid = (uint32_t)(((M + 63) / 64) * ((N + 63) / 64));
    matmul_simple<T><<<grid, 256, 0, st>>>(ac, as, bc, bs, M, N, (int)groups_of(K), (typename Elem<T>::type *)out, stride);
    return SIM_OPS_LAUNCH_OK();
}

}  // namespace

sim_status launch_matmul(hipStream_t st, const uint8_t *ac, const uint8_t *as, const uint8_t *bc, const uint8_t *bs,
                         int64_t M, int64_t N, int64_t K, void *out, int type, int64_t stride) {
    if (type == SIM_TYPE_F32) return matmul_t<SIM_TYPE_F32>(st, ac, as, bc, bs, M, N, K, out, stride);
    if (type == SIM_TYPE_F16) return matmul_t<SIM_TYPE_F16>(st, ac, as, bc, bs, M, N, K, out, stride);
    return matmul_t<SIM_TYPE_BF16>(st, ac, as, bc, bs, M, N, K, out, stride);
}

}  // namespace simops
