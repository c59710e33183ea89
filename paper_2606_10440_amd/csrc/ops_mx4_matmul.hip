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
#include "ops_quant.h"
#include "ops_stream.h"

namespace simops {
namespace {

// This kernel takes what the others do not: an empty sum, and rows so long
// that offsets within a tile pass 32 bits.
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


// ---- tiles through LDS
//
// A workgroup of WM x WN waves computes a BM x BN tile, each wave TM x TN
// blocks of 32 x 32.  The contraction goes in stages of 128 columns (64 bytes
// of codes a row).  Codes are copied from memory straight into LDS, sixteen
// bytes a lane, three stages ahead of the products through four buffers;
// scales likewise, for two groups of 256 columns at a time (16 bytes a row),
// two such pairs ahead.  Past the end the copies repeat the last stage, so
// that the loop has no branches: it is one run of matrix instructions with
// everything else dealt out between them.  A stage is two rounds of matrix
// instructions, and the operands of each round are read from LDS during the
// round before, the first ones of a stage before its own barrier: that barrier says that the NEXT stage's codes are there.
//
// Of a stage's four blocks half h of the lanes takes blocks 2 h and 2 h + 1.
// In LDS a row's four 16-byte pieces are permuted by bits 2 and 3 of the row
// number, so that the sixteen rows that are read together fill all banks
// once; the copy writes LDS in lane order, so the permutation is applied to
// the addresses that it reads.
//
// The operands change places in the instruction (B first), so that a lane
// ends up with one row of the result and four columns in sequence; the
// results of 32 rows go through LDS once more to be stored sixteen bytes a
// lane.
//
// 8192 x 8192 x 8192 to bf16: 272 to 303 us, 3.6 to 4.0 PFLOP/s; 4096 x 4096 x
// 4096: 44 to 46 us, 3.0 to 3.1 PFLOP/s.  The matrix units are busy 53 % of the cycles, at
// a clock that their load has brought down to 1.77 GHz; the same loop without
// its copies takes 215 us, without its operand reads 251.
constexpr int kStageCodes = 64;  // bytes of a row
constexpr int kBuffers = 4;
constexpr int kScaleGroups = 2;   // groups whose scales are copied together
constexpr int kScaleBuffers = 4;

typedef __attribute__((address_space(3))) uint8_t lds_byte;
typedef u32x4 __attribute__((aligned(2))) u32x4_any;

// Sixteen bytes per lane from base + offset to LDS at dst + 16 lane.  The
// compiler does not count these copies: whoever reads dst waits for them.
// They leave another value in m0, which it has to know for uses of its own
// (it warns of m0 since it would not keep a value there for us: none is).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void copy_to_lds(uint32_t dst, const uint8_t *base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(offset), "s"(base) : "m0");
}
__device__ inline void copy4_to_lds(uint32_t dst, const uint8_t *base, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(dst), "v"(offset), "s"(base) : "m0");
}
#pragma clang diagnostic pop
// All but the newest N copies (or loads) of this wave have arrived, its LDS
// accesses are done, and so it is for the other waves.
template <int N> __device__ inline void wait_and_meet() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Workgroups go round the eight dies in turn, each with an L2 of its own.  A
// die gets a run of neighbouring tiles, eight rows high, so that the tiles
// that it has at one time share as much of A and B as they can (8192 x 7936 x
// 8192: 330 us, 358 in row order; the same at 8192 x 8192, where row order
// happens to do it too).
__device__ inline void tile_of(uint32_t block, uint32_t tiles_m, uint32_t tiles_n, uint32_t &tm, uint32_t &tn) {
    constexpr uint32_t DIES = 8, HIGH = 8;
    const uint32_t total = tiles_m * tiles_n, die = block % DIES, each = total / DIES, more = total % DIES;
    const uint32_t id = die * each + min(die, more) + block / DIES;
    const uint32_t band = id / (HIGH * tiles_n), in = id - band * HIGH * tiles_n, high = min(HIGH, tiles_m - band * HIGH);
    tn = in / high;
    tm = band * HIGH + in - tn * high;
}

template <int T, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(64 * WM * WN, 1) void matmul_tile(const uint8_t *__restrict__ ac, const uint8_t *__restrict__ as,
                                                            const uint8_t *__restrict__ bc, const uint8_t *__restrict__ bs,
                                                            int64_t M, int64_t N, int groups, uint32_t tiles_m,
                                                            uint32_t tiles_n, typename Elem<T>::type *__restrict__ out,
                                                            int64_t stride) {
    constexpr int W = WM * WN, BM = WM * TM * 32, BN = WN * TN * 32, ROWS = BM + BN;
    constexpr int COPIES = ROWS / 16 / W;  // per wave and stage: sixteen rows each
    constexpr int A_COPIES = BM / 16 / W;  // of which rows of A
    constexpr int SCALE_COPIES = ROWS / 16 / W;  // per wave and two groups: sixteen rows each
    constexpr int OPS = TM + TN, PRODUCTS = TM * TN;  // of a round
    static_assert(BM % (16 * W) == 0 && BN % (16 * W) == 0, "rows are dealt evenly");
    constexpr int STAGE_SCALES = (SCALE_COPIES + 3) / 4, STAGE_COPIES = COPIES + STAGE_SCALES;
    // the slot beside a round's products from which the copies start
    constexpr int COPY_SLOT = COPIES < PRODUCTS ? PRODUCTS - COPIES : 0;
    constexpr int SCALE_ROW = kScaleGroups * kGroupScales;
    __shared__ __align__(16) uint8_t codes[kBuffers][ROWS * kStageCodes];
    __shared__ __align__(16) uint8_t scales[kScaleBuffers][ROWS * SCALE_ROW];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 31, h = lane >> 5;
    uint32_t tm, tn;
    tile_of(blockIdx.x, tiles_m, tiles_n, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    const int stages = groups * 2;

    // rows past the end repeat the last one: their products are not stored
    const int64_t code_pitch = (int64_t)groups * kGroupCodes, scale_pitch = (int64_t)groups * kGroupScales;
    const uint8_t *a_base = ac + m0 * code_pitch, *b_base = bc + n0 * code_pitch;
    const int a_last = (int)min((int64_t)BM, M - m0) - 1, b_last = (int)min((int64_t)BN, N - n0) - 1;
    uint32_t src[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; i++) {
        const bool in_a = i < A_COPIES;
        const int row = (in_a ? wave * A_COPIES + i : wave * (COPIES - A_COPIES) + i - A_COPIES) * 16 + (lane >> 2);
        src[i] = (uint32_t)(min(row, in_a ? a_last : b_last) * (uint32_t)code_pitch) + ((lane & 3) ^ ((lane >> 4) & 3)) * 16;
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte *)&codes[0][0];
    const uint32_t dst_a = lds0 + wave * A_COPIES * 1024, dst_b = lds0 + BM * kStageCodes + wave * (COPIES - A_COPIES) * 1024;
    const auto copy = [&](int i, int stage, int at) {
        const uint32_t buffer = (uint32_t)at % kBuffers * (ROWS * kStageCodes);
        if (i < A_COPIES) copy_to_lds(dst_a + buffer + i * 1024, a_base + (int64_t)stage * kStageCodes, src[i]);
        else copy_to_lds(dst_b + buffer + (i - A_COPIES) * 1024, b_base + (int64_t)stage * kStageCodes, src[i]);
    };

    const uint8_t *as_base = as + m0 * scale_pitch, *bs_base = bs + n0 * scale_pitch;
    const uint32_t sdst = (uint32_t)(uintptr_t)(lds_byte *)&scales[0][0] + wave * SCALE_COPIES * 256;
    const auto copy_scale = [&](int i, int g) {  // of the two groups from g on, four lanes a row
        const int first = (wave * SCALE_COPIES + i) * 16, row = first + (lane >> 2);
        const bool in_a = first < BM;
        const int at = in_a ? min(row, a_last) : min(row - BM, b_last);
        // a row's four words are permuted by bits 3 and 4 of its number, against bank conflicts
        const int word = (lane & 3) ^ (((first >> 3) & 2) | (lane >> 5));
        const uint32_t offset = (uint32_t)at * (uint32_t)scale_pitch + min(g + (word >> 1), groups - 1) * kGroupScales + (word & 1) * 4;
        copy4_to_lds(sdst + (uint32_t)(g / kScaleGroups) % kScaleBuffers * (ROWS * SCALE_ROW) + i * 256, in_a ? as_base : bs_base, offset);
    };

    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = f32x16{0};
    const int row_a = wave / WN * TM * 32 + r, row_b = BM + wave % WN * TN * 32 + r;

    // operands of the round in hand and of the next; sixteen bits of scales (a byte for each round) a stage
    u32x4 op[2][OPS];
    int sc[2][OPS];
    const auto row_of = [&](int i) { return i < TM ? row_a + i * 32 : row_b + (i - TM) * 32; };
    // in the order of first use: a row block, the column blocks, the other row blocks
    const auto nth_op = [&](int n) { return n == 0 ? 0 : n <= TN ? TM + n - 1 : n - TN; };
    const auto read_op = [&](int i, int stage, int s) {
        const int piece = (h * 2 + s) ^ ((lane >> 2) & 3);
        op[s][i] = *(const u32x4 *)(codes[(uint32_t)stage % kBuffers] + row_of(i) * kStageCodes + piece * 16);
    };
    const auto read_scale = [&](int i, int stage, int q) {
        const uint8_t *p = scales[(uint32_t)stage / (2 * kScaleGroups) % kScaleBuffers] + ((stage % (2 * kScaleGroups)) ^ ((lane >> 3) & 3)) * 4 + h * 2;
        sc[q][i] = *(const uint16_t *)(p + row_of(i) * SCALE_ROW);
    };
    const auto product = [&](auto sel, auto parity, int n) {
        constexpr int s = decltype(sel)::value, q = decltype(parity)::value;
        const int i = n / TN, j = n % TN;
        i32x8 a = {0}, b = {0};
        *(u32x4 *)&a = op[s][i];
        *(u32x4 *)&b = op[s][TM + j];
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b, a, acc[i][j], 4, 4, s, sc[q][TM + j], s, sc[q][i]);
    };
    typedef std::integral_constant<int, 0> C0;
    typedef std::integral_constant<int, 1> C1;

#pragma unroll
    for (int i = 0; i < SCALE_COPIES; i++) copy_scale(i, 0), copy_scale(i, kScaleGroups);
#pragma unroll
    for (int k = 0; k < 3; k++)
#pragma unroll
        for (int i = 0; i < COPIES; i++) copy(i, min(k, stages - 1), k);
    wait_and_meet<0>();
#pragma unroll
    for (int n = 0; n < OPS; n++) read_op(nth_op(n), 0, 0), read_scale(nth_op(n), 0, 0);

    const auto run_stage = [&](int g, auto half) {
        constexpr int q = decltype(half)::value;
        const int t = 2 * g + q;
        wait_and_meet<STAGE_COPIES>();  // the codes of stage t + 1 are there, and the buffer of stage t - 1 is free
#pragma unroll
        for (int n = 0; n < PRODUCTS; n++) {
#pragma unroll
            for (int o = n; o < OPS; o += PRODUCTS) read_op(nth_op(o), t, 1);
#pragma unroll
            for (int o = n; o < STAGE_SCALES; o += PRODUCTS)
                copy_scale(min(((g & 1) * 2 + q) * STAGE_SCALES + o, SCALE_COPIES - 1), (g & ~1) + 2 * kScaleGroups);
#pragma unroll
            for (int o = n - COPY_SLOT; o < COPIES; o += PRODUCTS)
                if (o >= 0) copy(o, min(t + 3, stages - 1), t + 3);
            product(C0(), half, n);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int n = 0; n < PRODUCTS; n++) {
#pragma unroll
            for (int o = n; o < OPS; o += PRODUCTS) read_op(nth_op(o), t + 1, 0), read_scale(nth_op(o), t + 1, 1 - q);
            product(C1(), half, n);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    for (int g = 0; g < groups; g++) {
        run_stage(g, C0());
        run_stage(g, C1());
    }
    wait_and_meet<0>();

    typedef typename Elem<T>::type E;
    constexpr int COLS = TN * 32, PITCH = COLS + 16 / sizeof(E), PER = 16 / sizeof(E), LANES = COLS / PER;
    static_assert(W * 32 * PITCH * sizeof(E) <= sizeof(codes), "the results of 32 rows of every wave fit");
    E *mine = (E *)&codes[0][0] + wave * 32 * PITCH;
    const int64_t n_wave = n0 + wave % WN * COLS;
#pragma unroll
    for (int i = 0; i < TM; i++) {
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int v = 0; v < 16; v += 4) {
                E e[4];
#pragma unroll
                for (int c = 0; c < 4; c++) e[c] = Elem<T>::put(acc[i][j][v + c]);
                E *p = mine + r * PITCH + j * 32 + 2 * v + 4 * h;
                if (sizeof(E) == 2) *(u32x2 *)p = *(u32x2 *)e;
                else *(u32x4 *)p = *(u32x4 *)e;
            }
        wave_fence();
        const int64_t m_first = m0 + wave / WN * TM * 32 + i * 32, n = n_wave + lane % LANES * PER;
#pragma unroll
        for (int k = 0; k < 32; k += 64 / LANES) {
            const int row = k + lane / LANES;
            const u32x4 v = *(const u32x4 *)(mine + row * PITCH + lane % LANES * PER);
            if (m_first + row < M) {
                E *o = out + (m_first + row) * stride + n;
                if (n + PER <= N) *(u32x4_any *)o = v;
                else
#pragma unroll
                    for (int c = 0; c < PER; c++)
                        if (n + c < N) o[c] = ((const E *)&v)[c];
            }
        }
        wave_fence();
    }
}

template <int T, int WM, int WN, int TM, int TN>
void launch_tile(hipStream_t st, const uint8_t *ac, const uint8_t *as, const uint8_t *bc, const uint8_t *bs, int64_t M,
                 int64_t N, int64_t K, void *out, int64_t stride) {
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32;
    const uint32_t tm = (uint32_t)((M + BM - 1) / BM), tn = (uint32_t)((N + BN - 1) / BN);
    matmul_tile<T, WM, WN, TM, TN><<<tm * tn, 64 * WM * WN, 0, st>>>(ac, as, bc, bs, M, N, (int)groups_of(K), tm, tn,
                                                                   (typename Elem<T>::type *)out, stride);
}

// ---- few rows of A
//
// At most 32 rows: the time is that of reading B once.  A workgroup takes 16 R
// rows of B, its waves each a part of the contraction, with 16x16x128
// instructions, B's rows as the first operand: lane l holds row l % 16 and
// block l / 16 of 128 columns.  The rows of A lie in LDS, where they are put
// into 4 bits first if they are not (XT): a launch less, worth it for a few
// (4 x 8192 x 4096: 8.2 us either way; 8 rows: 11.1 us against 8.5).
// 1 x 8192 x 4096: 5.7 us where the caches hold B (3.1 TB/s), 7.4 us from
// memory, of which some 2.5 us are the launch.
constexpr int kSkinnyWaves = 8;

template <int T, int XT, int R, int MT, int LDS>
__global__ __launch_bounds__(64 * kSkinnyWaves) void matmul_skinny(const void *__restrict__ x, const uint8_t *__restrict__ xs,
                                                                   int64_t x_stride, const uint8_t *__restrict__ bc,
                                                                   const uint8_t *__restrict__ bs, int M, int64_t N, int K,
                                                                   typename Elem<T>::type *__restrict__ out, int64_t stride) {
    constexpr int U = 4, W = kSkinnyWaves;
    __shared__ __align__(16) uint8_t lds[LDS];
    static_assert(W * R * MT * 1024 <= LDS, "the parts of the sum fit");
    const int groups = (int)groups_of(K), pitch = groups * kGroupCodes + 16, scale_pitch = groups * kGroupScales;
    uint8_t *codes = lds, *scales = lds + M * pitch;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 16 * R;
    int64_t row[R];
#pragma unroll
    for (int j = 0; j < R; j++) row[j] = min(n0 + j * 16 + r, N - 1);  // rows past the end repeat the last one
    const int64_t scale_row = min(n0 + Scales<SIM_TYPE_MX4, R, U>::tile() * 16 + r, N - 1);
    u32x4 w[U][R];
    Scales<SIM_TYPE_MX4, R, U> sc[2];
    f32x4 acc[R][MT];
#pragma unroll
    for (int j = 0; j < R; j++)
#pragma unroll
        for (int m = 0; m < MT; m++) acc[j][m] = f32x4{0};
    const int steps = groups * 2;
    bool ready = false;
    const auto prepare = [&] {  // A to LDS, while the first rows of B are on their way
        constexpr int AHEAD = XT == SIM_TYPE_MX4 ? 4 : 2;  // loads under way
        if (XT == SIM_TYPE_MX4) {
            const int pieces = M * groups * 8;  // of sixteen bytes of codes, and as many bytes of scales
            for (int i0 = threadIdx.x; i0 < pieces; i0 += AHEAD * 64 * W) {
                u32x4 c[AHEAD];
                uint8_t sb[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; u++) {
                    const int i = min(i0 + u * 64 * W, pieces - 1);
                    c[u] = ((const u32x4 *)x)[i];
                    sb[u] = xs[i];
                }
#pragma unroll
                for (int u = 0; u < AHEAD; u++) {
                    const int i = i0 + u * 64 * W, m = i / (groups * 8);
                    if (i < pieces) {
                        *(u32x4 *)(codes + m * pitch + (i - m * groups * 8) * 16) = c[u];
                        scales[i] = sb[u];
                    }
                }
            }
        } else {
            constexpr int FT = XT == SIM_TYPE_MX4 ? SIM_TYPE_F32 : XT;
            const int pieces = M * groups * 32;  // of eight columns; whole waves take part to the end
            for (int i0 = threadIdx.x; i0 < pieces; i0 += AHEAD * 64 * W) {
                float v[AHEAD][8];
#pragma unroll
                for (int u = 0; u < AHEAD; u++) {
                    const int i = i0 + u * 64 * W, m = i / (groups * 32), at = i - m * groups * 32;
                    load8<FT>((const typename Elem<FT>::type *)x + (i < pieces ? m : 0) * x_stride + at * 8, i < pieces ? K - at * 8 : 0, v[u]);
                }
#pragma unroll
                for (int u = 0; u < AHEAD; u++) {
                    const int i = i0 + u * 64 * W, m = i / (groups * 32), at = i - m * groups * 32;
                    uint32_t sb;
                    const uint32_t c = quantize8(v[u], sb);
                    if (i < pieces) {
                        *(uint32_t *)(codes + m * pitch + at * 4) = c;
                        if ((at & 3) == 0) scales[m * scale_pitch + at / 4] = (uint8_t)sb;
                    }
                }
            }
        }
        __syncthreads();
    };
    // every wave prepares: a wave without a run would otherwise miss the barrier
    const int runs = (steps + U - 1) / U;
    if (wave >= runs) prepare();
    ring<U, W>(
        runs, wave, [&](int p, int run) { sc[p].load(bs, scale_row, K, run); },
        [&](int i, int run) {
            const int step = min(run * U + i, steps - 1);
#pragma unroll
            for (int j = 0; j < R; j++)
                w[i][j] = *(const u32x4 *)(bc + row[j] * groups * kGroupCodes + step * (kStep / 2) + q * 16);
        },
        [&](int i, int p, int run) {
            if (!ready) {
                ready = true;
                prepare();
            }
            const int step = run * U + i;
            if (step < steps) {
                i32x8 a[MT];
                int sa[MT];
#pragma unroll
                for (int m = 0; m < MT; m++) {
                    const int at = m * 16 + r < M ? m * 16 + r : 0;
                    a[m] = i32x8{0};
                    *(u32x4 *)&a[m] = *(const u32x4 *)(codes + at * pitch + step * (kStep / 2) + q * 16);
                    sa[m] = scales[at * scale_pitch + step * 4 + q];
                }
#pragma unroll
                for (int j = 0; j < R; j++) {
                    i32x8 b = {0};
                    *(u32x4 *)&b = w[i][j];
                    const int sb = sc[p].get_byte(i, j, r, q);
#pragma unroll
                    for (int m = 0; m < MT; m++)
                        acc[j][m] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a[m], acc[j][m], 4, 4, 0, sb, 0, sa[m]);
                }
            }
        });
    __syncthreads();  // A is no longer needed: the parts of the sum take its place
    f32x4 *part = (f32x4 *)lds;
#pragma unroll
    for (int j = 0; j < R; j++)
#pragma unroll
        for (int m = 0; m < MT; m++) part[((wave * R + j) * MT + m) * 64 + lane] = acc[j][m];
    __syncthreads();
    if (wave < R * MT) {
        const int j = wave / MT, m = wave % MT;
        f32x4 v = {0};
#pragma unroll
        for (int p = 0; p < W; p++) v += part[((p * R + j) * MT + m) * 64 + lane];
        const int64_t n = n0 + j * 16 + 4 * q;
        if (m * 16 + r < M)
#pragma unroll
            for (int i = 0; i < 4; i++)
                if (n + i < N) out[(int64_t)(m * 16 + r) * stride + n + i] = Elem<T>::put(v[i]);
    }
}

template <int T, int XT>
void skinny_t(hipStream_t st, const void *x, const uint8_t *xs, int64_t x_stride, const uint8_t *bc, const uint8_t *bs,
              int64_t M, int64_t N, int64_t K, void *out, int64_t stride) {
    typedef typename Elem<T>::type E;
    constexpr int R = 2;
    const uint32_t grid = (uint32_t)((N + 16 * R - 1) / (16 * R));
    const auto launch = [&](auto mt, auto lds) {
        matmul_skinny<T, XT, R, decltype(mt)::value, decltype(lds)::value><<<grid, 64 * kSkinnyWaves, 0, st>>>(
            x, xs, x_stride, bc, bs, (int)M, N, (int)K, (E *)out, stride);
    };
    typedef std::integral_constant<int, kSkinnyLds[0]> Small;
    typedef std::integral_constant<int, kSkinnyLds[1]> Large;
    const bool small = skinny_lds(M, K) <= (size_t)kSkinnyLds[0];
    if constexpr (XT == SIM_TYPE_MX4) {
        if (M <= 16) small ? launch(std::integral_constant<int, 1>(), Small()) : launch(std::integral_constant<int, 1>(), Large());
        else small ? launch(std::integral_constant<int, 2>(), Small()) : launch(std::integral_constant<int, 2>(), Large());
    } else {  // at most kOwnQuantize elements, which always fit
        static_assert(kOwnQuantize * 34 / 64 + kSkinnyRows * (kGroupCodes + kGroupScales + 16) <= kSkinnyLds[0], "they fit");
        if (M <= 16) launch(std::integral_constant<int, 1>(), Small());
        else launch(std::integral_constant<int, 2>(), Small());
    }
}

template <int T>
sim_status matmul_t(hipStream_t st, const uint8_t *ac, const uint8_t *as, const uint8_t *bc, const uint8_t *bs, int64_t M,
                    int64_t N, int64_t K, void *out, int64_t stride) {
    switch (product_form(M, N, K)) {
        case kSkinnySmall:
        case kSkinnyLarge: skinny_t<T, SIM_TYPE_MX4>(st, ac, as, 0, bc, bs, M, N, K, out, stride); break;
        case kTile256x256: launch_tile<T, 2, 2, 4, 4>(st, ac, as, bc, bs, M, N, K, out, stride); break;
        case kTile128x128: launch_tile<T, 2, 2, 2, 2>(st, ac, as, bc, bs, M, N, K, out, stride); break;
        case kTile64x128: launch_tile<T, 2, 2, 1, 2>(st, ac, as, bc, bs, M, N, K, out, stride); break;
        case kTile64x64: launch_tile<T, 2, 2, 1, 1>(st, ac, as, bc, bs, M, N, K, out, stride); break;
        case kSimple:
            matmul_simple<T><<<(uint32_t)(((M + 63) / 64) * ((N + 63) / 64)), 256, 0, st>>>(
                ac, as, bc, bs, M, N, (int)groups_of(K), (typename Elem<T>::type *)out, stride);
    }
    return SIM_OPS_LAUNCH_OK();
}

template <int T>
sim_status linear_t(hipStream_t st, const void *x, int x_type, int64_t x_stride, const uint8_t *wc, const uint8_t *ws,
                    int64_t M, int64_t N, int64_t K, void *out, int64_t stride) {
    if (x_type == SIM_TYPE_F32) skinny_t<T, SIM_TYPE_F32>(st, x, nullptr, x_stride, wc, ws, M, N, K, out, stride);
    else if (x_type == SIM_TYPE_F16) skinny_t<T, SIM_TYPE_F16>(st, x, nullptr, x_stride, wc, ws, M, N, K, out, stride);
    else skinny_t<T, SIM_TYPE_BF16>(st, x, nullptr, x_stride, wc, ws, M, N, K, out, stride);
    return SIM_OPS_LAUNCH_OK();
}

}  // namespace

sim_status launch_linear(hipStream_t st, const void *x, int x_type, int64_t x_stride, const uint8_t *wc, const uint8_t *ws,
                         int64_t M, int64_t N, int64_t K, void *out, int type, int64_t stride) {
    if (type == SIM_TYPE_F32) return linear_t<SIM_TYPE_F32>(st, x, x_type, x_stride, wc, ws, M, N, K, out, stride);
    if (type == SIM_TYPE_F16) return linear_t<SIM_TYPE_F16>(st, x, x_type, x_stride, wc, ws, M, N, K, out, stride);
    return linear_t<SIM_TYPE_BF16>(st, x, x_type, x_stride, wc, ws, M, N, K, out, stride);
}

sim_status launch_matmul(hipStream_t st, const uint8_t *ac, const uint8_t *as, const uint8_t *bc, const uint8_t *bs,
                         int64_t M, int64_t N, int64_t K, void *out, int type, int64_t stride) {
    if (type == SIM_TYPE_F32) return matmul_t<SIM_TYPE_F32>(st, ac, as, bc, bs, M, N, K, out, stride);
    if (type == SIM_TYPE_F16) return matmul_t<SIM_TYPE_F16>(st, ac, as, bc, bs, M, N, K, out, stride);
    return matmul_t<SIM_TYPE_BF16>(st, ac, as, bc, bs, M, N, K, out, stride);
}

}  // namespace simops
