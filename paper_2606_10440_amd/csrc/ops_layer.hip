// The experts' layer for few tokens: two products per expert over the tokens
// that chose it.  With few tokens the time is that of reading the chosen
// experts' weights once; everything else is kept out of the way of that
// stream.
//
// Both products run on 16x16x32 matrix instructions with sixteen weight rows
// as the first operand and sixteen tokens as the second, the waves of a
// workgroup each taking a part of the contraction in steps of 128 columns.
// A wave keeps a ring of U steps' operands in registers and refills a place
// as soon as it has been multiplied, weights and activations alike, since
// loads return in the order in which they were issued.  Activations and 4-bit
// weights enter as bf16; the hidden values between the products, and fp16
// where the other operand is bf16, enter as the sum of two bf16 parts: the
// range of the hidden values needs that of bf16, and the second instruction
// is free where the weights' bytes bound the time.
#include "ops_route_keys.h"
#include "ops_stream.h"

namespace simops {
namespace {

typedef u32x4 __attribute__((aligned(2))) u32x4_a2;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// A row of K 16-bit elements: a whole number of steps, at least one load
// long, or shorter than that.
enum Edge { kWhole, kTail, kTiny };

// Elements k .. k + 7 of a row as raw bits.  Past the end of a kTail row the
// row's last eight are loaded instead, and tail8 puts them in their place: no
// branch stands around the load, so that loads under way are still counted
// (100 tokens, k = 2 of 16 bf16 experts of 2080 x 2080: 127 us, 187 with branches).
template <int EDGE> __device__ inline u32x4 load8(const uint16_t *__restrict__ row, int k, int K) {
    if (EDGE == kTiny) {
        uint16_t v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = k + i < K ? row[k + i] : 0;
        return *(u32x4 *)v;
    }
    return *(const u32x4_a2 *)(row + (EDGE == kTail ? min(k, K - 8) : k));
}
// What load8 gave, with zeros past the end of a kTail row.
template <int EDGE> __device__ inline u32x4 tail8(u32x4 v, int k, int K) {
    if (EDGE != kTail) return v;
    const int n = min(k + 8 - K, 8);  // elements past the end
    if (n <= 0) return v;
    if (n & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
    if (n & 2) v = u32x4{v[1], v[2], v[3], 0};
    if (n & 4) v = u32x4{v[2], v[3], 0, 0};
    return n & 8 ? u32x4{0, 0, 0, 0} : v;
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

// A step is 64 columns of 16-bit weights (two loads, whole cache lines, for
// two instructions) or 128 of 4-bit ones (one load for four).  Elements of
// lane l (q = l / 16) in instruction s: 32 s + 8 q .. + 7, or 32 q + 8 s .. + 7.
template <int WT> constexpr int kCols = WT == SIM_TYPE_MX4 ? 128 : 64;
template <int WT> constexpr int kIns = WT == SIM_TYPE_MX4 ? 4 : 2;
template <int WT> __device__ inline int step_at(int q, int s) { return WT == SIM_TYPE_MX4 ? 32 * q + 8 * s : 32 * s + 8 * q; }

// A step of one tile of sixteen weight rows; lane l holds row l % 16.
template <int WT, int EDGE> struct Weights {
    u32x4 raw[2];
    // base: the weights; row: this lane's; k0: the step's first column
    __device__ void load(const void *base, int64_t row, int K, int k0, int q) {
#pragma unroll
        for (int s = 0; s < 2; s++) raw[s] = load8<EDGE>((const uint16_t *)base + row * K, k0 + step_at<WT>(q, s), K);
    }
    __device__ void tail(int K, int k0, int q) {
#pragma unroll
        for (int s = 0; s < 2; s++) raw[s] = tail8<EDGE>(raw[s], k0 + step_at<WT>(q, s), K);
    }
    struct Operand {
        u32x4 raw;
        bf16x8 hi, lo;
    };
    __device__ Operand operand(int s, float) const {
        Operand o;
        o.raw = raw[s];
        if (WT == SIM_TYPE_F16) split_f16(raw[s], o.hi, o.lo);
        else o.hi = __builtin_bit_cast(bf16x8, raw[s]);
        return o;
    }
    static __device__ f32x4 mul(const Operand &w, bf16x8 x, f32x4 c) {
        c = mfma(w.hi, x, c);
        return WT == SIM_TYPE_F16 ? mfma(w.lo, x, c) : c;
    }
};
template <int EDGE> struct Weights<SIM_TYPE_MX4, EDGE> {
    u32x4 raw;
    __device__ void load(const void *base, int64_t row, int K, int k0, int q) {
        raw = *(const u32x4 *)((const uint8_t *)base + row * groups_of(K) * kGroupCodes + k0 / 2 + q * 16);
    }
    __device__ void tail(int, int, int) {}  // rows are padded
    struct Operand {
        bf16x8 hi;
    };
    __device__ Operand operand(int s, float scale) const { return {widen8(raw[s], scale)}; }
    static __device__ f32x4 mul(const Operand &w, bf16x8 x, f32x4 c) { return mfma(w.hi, x, c); }
};

// A step of sixteen inputs; lane l holds token l % 16.
template <int T, int WT, int EDGE> struct Inputs {
    u32x4 raw[kIns<WT>];
    __device__ void load(const uint16_t *row, int K, int k0, int q) {
#pragma unroll
        for (int s = 0; s < kIns<WT>; s++) raw[s] = load8<EDGE>(row, k0 + step_at<WT>(q, s), K);
    }
    __device__ void tail(int K, int k0, int q) {
#pragma unroll
        for (int s = 0; s < kIns<WT>; s++) raw[s] = tail8<EDGE>(raw[s], k0 + step_at<WT>(q, s), K);
    }
    template <typename W> static __device__ f32x4 mul(u32x4 v, const typename W::Operand &w, f32x4 c) {
        if constexpr (T == SIM_TYPE_F16 && WT == SIM_TYPE_F16)  // as they are
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w.raw), __builtin_bit_cast(f16x8, v), c, 0, 0, 0);
        if (T == SIM_TYPE_BF16) return W::mul(w, __builtin_bit_cast(bf16x8, v), c);
        bf16x8 hi, lo;
        split_f16(v, hi, lo);
        return W::mul(w, lo, W::mul(w, hi, c));
    }
};

// A step of sixteen rows of hidden values in their two parts (rows of a whole
// number of steps), zeros where the lane has none.
template <int WT> struct Hidden {
    u32x4 hi[kIns<WT>], lo[kIns<WT>];
    __device__ void load(const __bf16 *h_hi, const __bf16 *h_lo, int64_t at, bool some, int k0, int q) {
#pragma unroll
        for (int s = 0; s < kIns<WT>; s++) {
            hi[s] = lo[s] = u32x4{0, 0, 0, 0};
            if (some) {
                hi[s] = *(const u32x4 *)(h_hi + at + k0 + step_at<WT>(q, s));
                lo[s] = *(const u32x4 *)(h_lo + at + k0 + step_at<WT>(q, s));
            }
        }
    }
    template <typename W> __device__ f32x4 mul(int s, const typename W::Operand &w, f32x4 c) const {
        return W::mul(w, __builtin_bit_cast(bf16x8, lo[s]), W::mul(w, __builtin_bit_cast(bf16x8, hi[s]), c));
    }
};

// A step of CT tiles of sixteen rows of activations.  Sixteen bytes of an
// operand lie a row apart from lane to lane, and a load of that shape costs a
// cache access for each lane.  STAGED: rows are loaded as they lie, kCols / 8
// lanes to a row, and read from LDS in the operand's order; a wave stages its
// own steps, so nothing waits for others (63 tokens, k = 5 of 9 experts of 3687
// x 1024: bf16 165 -> 135 us, 4-bit 101 -> 78 us; with one tile it costs as
// much as it saves).
template <int WT> constexpr int kStagePitch = kCols<WT> * 2 + 16;  // bytes: sixteen rows start in different banks
template <int WT, int CT, bool STAGED> struct Acts {
    static constexpr int kBytes = STAGED ? CT * 16 * kStagePitch<WT> : 0;  // of LDS for a wave
    static constexpr int kRowLanes = kCols<WT> / 8, kRows = STAGED ? kIns<WT> : 1;
    u32x4 raw[CT][kIns<WT>];
    // the row of a tile and the column of a step of this lane's load s
    static __device__ int row(int s) {
        const int lane = threadIdx.x & 63;
        return STAGED ? s * (64 / kRowLanes) + lane / kRowLanes : lane & 15;
    }
    static __device__ int col(int s) {
        const int lane = threadIdx.x & 63;
        return STAGED ? lane % kRowLanes * 8 : step_at<WT>(lane >> 4, s);
    }
    // between a step's reads and the next one's writes, and between its
    // writes and reads
    static __device__ void fence() {
        if (STAGED) wave_fence();
    }
    __device__ void put(uint8_t *lds) const {
        if (!STAGED) return;
#pragma unroll
        for (int c = 0; c < CT; c++)
#pragma unroll
            for (int s = 0; s < kIns<WT>; s++) *(u32x4 *)(lds + (c * 16 + row(s)) * kStagePitch<WT> + col(s) * 2) = raw[c][s];
    }
    // the operand of instruction s
    __device__ u32x4 get(const uint8_t *lds, int c, int s) const {
        if (!STAGED) return raw[c][s];
        const int lane = threadIdx.x & 63;
        return *(const u32x4 *)(lds + (c * 16 + (lane & 15)) * kStagePitch<WT> + step_at<WT>(lane >> 4, s) * 2);
    }
};

__device__ inline float gated(float g, float u, float w) { return g / (1.f + expf(-g)) * u * w; }

__device__ inline void store_hidden(__bf16 *h_hi, __bf16 *h_lo, int64_t at, const float v[4]) {
    __bf16 hi[4], lo[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        hi[i] = (__bf16)v[i];
        lo[i] = (__bf16)(fabsf((float)hi[i]) < INFINITY ? v[i] - (float)hi[i] : 0.f);  // inf - inf is no part of inf
    }
    *(u32x2 *)(h_hi + at) = *(u32x2 *)hi;
    *(u32x2 *)(h_lo + at) = *(u32x2 *)lo;
}

// ------------------------------------------------------- at most 16 tokens
//
// Two kernels, of as many workgroups as the GPU holds at once.  The tokens
// themselves are the sixteen columns of every product.  The first kernel
// routes, every workgroup for itself, which costs less than a launch, and
// then takes tiles of sixteen hidden units of the used experts in turn.  In
// the second, a step's sums are added to the columns of the tokens that chose
// its expert, so all experts share one accumulator and nothing has to be
// joined but the parts of the split contraction.
//
// 16 tokens, k = 8 of 128 4-bit experts of 4096 x 1280: 102 to 112 us for 459
// MB of gates and ups (4.1 to 4.5 TB/s), 68 to 76 us for 230 MB of downs (3.0
// to 3.4 TB/s, 57 us without the hidden values' loads); one token, k = 6 of 64
// bf16 experts of 2048 x 1408: 22 us for 69 MB that the caches still hold, 25
// from memory, some 7 of which are the launch, the routing and the epilogue,
// and 12 to 13 us for 35 MB.  The kernels for more tokens took 206, 39
// and (both small) 20 us where these took 177, 35 and 14.

constexpr int kFewWaves = 4;
constexpr int kFewGroups = 768;  // workgroups: three on each of 256 compute units
constexpr int kMaxSplits = 16;
constexpr int kJoin = 16;     // parts of a split sum that are loaded together

// What the first kernel leaves for the second.
struct FewPlan {
    int32_t *n_used;    // experts with tokens
    int16_t *expert;    // [n_used]
    int16_t *slot;      // [n_used][16]: token's slot, -1
    uint32_t *arrived;  // [tiles of the second kernel]
};

struct FewRoute {
    uint8_t inputs[kFewInputs];
    float weight[kFewTokens * SIM_MOE_MAX_TOPK];
    uint8_t pos[kFewTokens][kFewExperts];  // which choice of the token the expert is
    uint32_t tokens[kFewExperts];          // bit t: token t chose the expert
    int16_t list[kFewExperts];             // the used experts
    int count[kFewWaves];
};

// A token's choices; lane l of its sixteen holds experts l, l + 16, ... in NV
// registers (16 tokens, k = 8 of 128 bf16 experts of 2048 x 256: the kernel
// takes 36 us, 40.4 with the keys in LDS).
template <int NV> __device__ inline void few_choose(const RouteArgs &a, FewRoute &s, int t, int l) {
    float v[NV];
    const auto load = [&](const auto *z) {
#pragma unroll
        for (int i = 0; i < NV; i++) v[i] = (float)z[t * a.stride + min(l + 16 * i, a.E - 1)];
    };
    if (a.type == SIM_TYPE_F32) load((const float *)a.logits);
    else if (a.type == SIM_TYPE_F16) load((const _Float16 *)a.logits);
    else load((const __bf16 *)a.logits);
    uint32_t ok = ~0u;
    if (a.mask) {
        uint8_t m[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) m[i] = a.mask[t * a.mask_stride + min(l + 16 * i, a.E - 1)];
        ok = 0;
#pragma unroll
        for (int i = 0; i < NV; i++) ok |= (uint32_t)(m[i] != 0) << i;
    }
    uint32_t key[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) key[i] = l + 16 * i < a.E && (ok >> i) & 1 ? order_key(v[i]) : 0;

    float top = 0.f, z = 0.f, w[2];
    uint32_t mine[2] = {0, 0}, mine_e[2] = {0, 0};
    for (int j = 0; j < a.k; j++) {
        uint32_t bk = 0, bi = 0xffffu;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const bool take = key[i] > bk;
            bk = take ? key[i] : bk;
            bi = take ? (uint32_t)(l + 16 * i) : bi;
        }
        best16(bk, bi);
        if (j == 0) {
            top = key_value(bk);
            if (!a.renorm) {
#pragma unroll
                for (int i = 0; i < NV; i++) z += key[i] ? expf(key_value(key[i]) - top) : 0.f;
                z = sum16(z);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; i++) key[i] = (uint32_t)(l + 16 * i) == bi ? 0 : key[i];
        if (l == (j & 15)) {
            if (j < 16) mine[0] = bk, mine_e[0] = bi;
            else mine[1] = bk, mine_e[1] = bi;
        }
    }
#pragma unroll
    for (int q = 0; q < 2; q++) w[q] = mine[q] ? expf(key_value(mine[q]) - top) : 0.f;
    if (a.renorm) z = sum16(w[0] + w[1]);
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const int j = q * 16 + l;
        if (j < a.k && mine[q]) {
            s.weight[t * a.k + j] = w[q] / z;
            s.pos[t][mine_e[q]] = (uint8_t)j;
            atomicOr(&s.tokens[mine_e[q]], 1u << t);
        }
    }
}

// All tokens' choices, sixteen threads a token; returns the number of used
// experts.
__device__ inline int few_route(const RouteArgs &a, FewRoute &s) {
    const int l = threadIdx.x & 15, t = threadIdx.x >> 4, n_tok = (int)a.T, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    static_assert(64 * kFewWaves == kFewExperts && 4 * kFewWaves == kFewTokens, "a thread for each expert, sixteen for each token");
    s.tokens[threadIdx.x] = 0;
    __syncthreads();
    if (t < n_tok) {
        if (a.E <= 64) few_choose<4>(a, s, t, l);
        else if (a.E <= 128) few_choose<8>(a, s, t, l);
        else few_choose<kFewExperts / 16>(a, s, t, l);
    }
    __syncthreads();
    const uint64_t all = __ballot(s.tokens[threadIdx.x] != 0);
    if (lane == 0) s.count[wave] = __popcll(all);
    __syncthreads();
    int at = __popcll(all & ((1ull << lane) - 1)), used = 0;
    for (int w = 0; w < kFewWaves; w++) {
        if (w < wave) at += s.count[w];
        used += s.count[w];
    }
    if (s.tokens[threadIdx.x]) s.list[at] = (int16_t)threadIdx.x;
    __syncthreads();
    return used;
}

// Gate and up products, sixteen hidden units of one expert after another.
template <int T, int WT, int U, int EDGE>
__global__ __launch_bounds__(64 * kFewWaves, 3) void few_up(RouteArgs route, const uint16_t *__restrict__ x, int64_t x_stride,
                                                            int D, const void *__restrict__ w13,
                                                            const uint8_t *__restrict__ s13, int F, int tiles,
                                                            __bf16 *__restrict__ h_hi, __bf16 *__restrict__ h_lo, int h_pitch,
                                                            FewPlan plan, int down_tiles) {
    __shared__ __align__(16) FewRoute rt;
    __shared__ f32x4 part[2][kFewWaves][2][64];
    __shared__ int s_token[16];  // of the inputs in LDS
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int used = few_route(route, rt);
    if (blockIdx.x == 0) {
        if (threadIdx.x == 0) *plan.n_used = used;
        for (int i = threadIdx.x; i < down_tiles; i += blockDim.x) plan.arrived[i] = 0;
        for (int i = threadIdx.x; i < used * 16; i += blockDim.x) {
            const int e = rt.list[i >> 4], t = i & 15;
            plan.slot[i] = (rt.tokens[e] >> t) & 1 ? (int16_t)(t * route.k + rt.pos[t][e]) : (int16_t)-1;
            if (t == 0) plan.expert[i >> 4] = (int16_t)e;
        }
    }
    const int steps = (D + kCols<WT> - 1) / kCols<WT>, items = used * tiles;
    int turn = 0, held = -1;
    bool in_lds = false;
    // neighbours take neighbouring rows at the same time (measured: 109 us;
    // 126 us with a range of items for each workgroup)
    for (int item = blockIdx.x; item < items; item += gridDim.x, turn ^= 1) {
        const int e = __builtin_amdgcn_readfirstlane(rt.list[item / tiles]), f0 = item % tiles * 16;
        const uint32_t tokens = rt.tokens[e];
        const bool has = (tokens >> r) & 1;
        const int pitch = few_input_pitch(D, kCols<WT>);
        if (e != held) {  // the expert's inputs to LDS, where they fit
            held = e;
            in_lds = __popc(tokens) * pitch <= kFewInputs;
            if (in_lds) {
                if (wave == 0 && has && q == 0) s_token[__popc(tokens & ((1u << r) - 1))] = r;
                __syncthreads();
                const int pieces = steps * kCols<WT> / 8, all = __popc(tokens) * pieces;
                for (int c0 = threadIdx.x; c0 < all; c0 += 4 * 64 * kFewWaves) {  // four loads under way
                    u32x4 v[4];
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int c = min(c0 + i * 64 * kFewWaves, all - 1), n = c / pieces;
                        v[i] = load8<EDGE>(x + (int64_t)s_token[n] * x_stride, (c - n * pieces) * 8, D);
                    }
#pragma unroll
                    for (int i = 0; i < 4; i++) {
                        const int c = c0 + i * 64 * kFewWaves, n = c / pieces;
                        if (c < all)
                            *(u32x4 *)(rt.inputs + n * pitch + (c - n * pieces) * 16) = tail8<EDGE>(v[i], (c - n * pieces) * 8, D);
                    }
                }
                __syncthreads();
            }
        }
        const int64_t row = (int64_t)e * 2 * F + min(f0 + r, F - 1), scale_row = row + (int64_t)Scales<WT, 2, 2>::tile() * F;
        typedef Inputs<T, WT, EDGE> In;
        f32x4 g = {0}, u = {0};
        if (in_lds) {
            typedef Weights<WT, EDGE> Wt;
            Wt wg[U], wu[U];
            Scales<WT, 2, U> sc[2];
            // columns without a token repeat the first
            const uint8_t *xr = rt.inputs + (has ? __popc(tokens & ((1u << r) - 1)) : 0) * pitch;
            ring<U, kFewWaves>(
                (steps + U - 1) / U, wave,
                [&](int p, int run) { sc[p].load(s13, scale_row, D, run); },
                [&](int i, int run) {  // a step past the last loads that again and is not used
                    const int k0 = min(run * U + i, steps - 1) * kCols<WT>;
                    wg[i].load(w13, row, D, k0, q);
                    wu[i].load(w13, row + F, D, k0, q);
                },
                [&](int i, int p, int run) {
                    if (run * U + i < steps) {
                        if (EDGE && run * U + i == steps - 1) {
                            wg[i].tail(D, (steps - 1) * kCols<WT>, q);
                            wu[i].tail(D, (steps - 1) * kCols<WT>, q);
                        }
                        const float cg = sc[p].get(i, 0, r, q), cu = sc[p].get(i, 1, r, q);
#pragma unroll
                        for (int s = 0; s < kIns<WT>; s++) {
                            const u32x4 v = *(const u32x4 *)(xr + ((run * U + i) * kCols<WT> + step_at<WT>(q, s)) * 2);
                            g = In::template mul<Wt>(v, wg[i].operand(s, cg), g);
                            u = In::template mul<Wt>(v, wu[i].operand(s, cu), u);
                        }
                    }
                });
        } else {
            constexpr int V = WT == SIM_TYPE_MX4 ? 2 : U;  // (registers)
            typedef Weights<WT, EDGE> Wt;
            Wt wg[V], wu[V];
            Scales<WT, 2, V> sc[2];
            const uint16_t *xr = x + (int64_t)(has ? r : __ffs(tokens) - 1) * x_stride;
            In xi[V];
            ring<V, kFewWaves>(
                (steps + V - 1) / V, wave,
                [&](int p, int run) { sc[p].load(s13, scale_row, D, run); },
                [&](int i, int run) {
                    const int k0 = min(run * V + i, steps - 1) * kCols<WT>;
                    wg[i].load(w13, row, D, k0, q);
                    wu[i].load(w13, row + F, D, k0, q);
                    xi[i].load(xr, D, k0, q);
                },
                [&](int i, int p, int run) {
                    if (run * V + i < steps) {
                        if (EDGE && run * V + i == steps - 1) {
                            wg[i].tail(D, (steps - 1) * kCols<WT>, q);
                            wu[i].tail(D, (steps - 1) * kCols<WT>, q);
                            xi[i].tail(D, (steps - 1) * kCols<WT>, q);
                        }
                        const float cg = sc[p].get(i, 0, r, q), cu = sc[p].get(i, 1, r, q);
#pragma unroll
                        for (int s = 0; s < kIns<WT>; s++) {
                            g = In::template mul<Wt>(xi[i].raw[s], wg[i].operand(s, cg), g);
                            u = In::template mul<Wt>(xi[i].raw[s], wu[i].operand(s, cu), u);
                        }
                    }
                });
        }
        part[turn][wave][0][lane] = g;
        part[turn][wave][1][lane] = u;
        __syncthreads();
        if (wave == 0) {  // the others go on: their next parts go to the other place
#pragma unroll
            for (int w = 1; w < kFewWaves; w++) {
                g += part[turn][w][0][lane];
                u += part[turn][w][1][lane];
            }
            if (has) {
                const int slot = r * route.k + rt.pos[r][e];
                const float weight = rt.weight[slot];
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; i++) v[i] = f0 + 4 * q + i < F ? gated(g[i], u[i], weight) : 0.f;
                const int64_t at = (int64_t)slot * h_pitch + f0 + 4 * q;
                store_hidden(h_hi, h_lo, at, v);
                if (f0 + 16 >= F)  // the rest of the last step
                    for (int f = 16; f0 + f < h_pitch; f += 16) {
                        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
                        store_hidden(h_hi, h_lo, at + f, zero);
                    }
            }
        }
    }
}

template <int WT> constexpr int few_down_run = WT == SIM_TYPE_MX4 ? 2 : 4;  // steps

// 16 R output columns of all tokens; the steps of all used experts are one
// list, dealt to the splits and their waves.
template <int T, int WT, int R, int EDGE>
__global__ __launch_bounds__(64 * kFewWaves, 3) void few_down(const __bf16 *__restrict__ h_hi, const __bf16 *__restrict__ h_lo,
                                                              int h_pitch, int F, const void *__restrict__ w2,
                                                              const uint8_t *__restrict__ s2, int D, int n_tok, FewPlan plan,
                                                              int max_lists, int splits, float *__restrict__ parts,
                                                              typename Elem<T>::type *__restrict__ y, int64_t y_stride) {
    static_assert(R <= kFewWaves, "a wave for each row tile");
    constexpr int U = few_down_run<WT>;
    __shared__ f32x4 part[kFewWaves][R][64];
    __shared__ int16_t s_slot[kFewExperts * 16], s_expert[kFewExperts];
    __shared__ int last;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int tiles = gridDim.x / splits, tile = blockIdx.x % tiles, split = blockIdx.x / tiles, d0 = tile * 16 * R;
    for (int i = threadIdx.x; i < max_lists * 16; i += blockDim.x) {  // the whole plan: not one load after another
        s_slot[i] = plan.slot[i];
        if (i < max_lists) s_expert[i] = plan.expert[i];
    }
    const int steps = (F + kCols<WT> - 1) / kCols<WT>, per = (steps + U - 1) / U, total = *plan.n_used * per;  // runs
    const int begin = (int)((int64_t)total * split / splits), end = (int)((int64_t)total * (split + 1) / splits);
    typedef Weights<WT, EDGE> Wt;
    Wt w[U][R];
    Hidden<WT> h[U];
    f32x4 acc[R];
#pragma unroll
    for (int i = 0; i < R; i++) acc[i] = f32x4{0};
    __syncthreads();
    Scales<WT, R, U> sc[2];
    bool some[2] = {false, false};
    int64_t row[R], hidden = 0;  // of the run that is being loaded
    int k0 = 0, loading = 0;
    ring<U, kFewWaves>(
        end - begin, wave,
        [&](int p, int run) {
            const int a = (begin + run) / per;
            const int64_t first = (int64_t)__builtin_amdgcn_readfirstlane(s_expert[a]) * D;
            const int slot = s_slot[a * 16 + r];
            k0 = begin + run - a * per;
            some[loading = p] = slot >= 0;
            hidden = (int64_t)slot * h_pitch;
#pragma unroll
            for (int j = 0; j < R; j++) row[j] = first + min(d0 + j * 16 + r, D - 1);
            sc[p].load(s2, first + min(d0 + sc[p].tile() * 16 + r, D - 1), F, k0);
        },
        [&](int i, int) {
            const int at = min(k0 * U + i, steps - 1) * kCols<WT>;
            h[i].load(h_hi, h_lo, hidden, some[loading], at, q);
#pragma unroll
            for (int j = 0; j < R; j++) w[i][j].load(w2, row[j], F, at, q);
        },
        [&](int i, int p, int run) {
            const int step = (begin + run) % per * U + i;
            if (step < steps)
#pragma unroll
                for (int j = 0; j < R; j++) {
                    if (EDGE && step == steps - 1) w[i][j].tail(F, step * kCols<WT>, q);
                    const float c = sc[p].get(i, j, r, q);
                    f32x4 sum = {0};
#pragma unroll
                    for (int s = 0; s < kIns<WT>; s++) sum = h[i].template mul<Wt>(s, w[i][j].operand(s, c), sum);
                    acc[j] += some[p] ? sum : f32x4{0};  // zeros times an infinite weight are no zeros
                }
        });
#pragma unroll
    for (int j = 0; j < R; j++) part[wave][j][lane] = acc[j];
    __syncthreads();
    f32x4 v = {0};
    const int j = wave;  // wave j sums and stores row tile j
    const bool mine = j < R && r < n_tok;
    if (mine)
#pragma unroll
        for (int i = 0; i < kFewWaves; i++) v += part[i][j][lane];
    if (splits > 1) {
        // Every split leaves its part; the one that comes last adds them up
        // in their order, so that the result does not depend on which it is.
        // The parts are written and read at device scope, past the caches
        // that are not shared, so that only their order has to be kept: they
        // have left before the count goes up, and are read after it.
        const auto at = [&](int p, int i) { return parts + (((int64_t)tile * splits + p) * R + j) * 256 + (r * 4 + i) * 4 + q; };
        if (mine)
#pragma unroll
            for (int i = 0; i < 4; i++) __hip_atomic_store(at(split, i), v[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0)
            last = __hip_atomic_fetch_add(&plan.arrived[tile], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)splits - 1;
        __syncthreads();
        if (!last) return;
        v = f32x4{0};
        if (mine)
            for (int p0 = 0; p0 < splits; p0 += kJoin) {  // so many under way at once
                float part[kJoin][4];
#pragma unroll
                for (int p = 0; p < kJoin; p++)
#pragma unroll
                    for (int i = 0; i < 4; i++)
                        part[p][i] = __hip_atomic_load(at(min(p0 + p, splits - 1), i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                for (int p = 0; p < kJoin; p++)
#pragma unroll
                    for (int i = 0; i < 4; i++) v[i] += p0 + p < splits ? part[p][i] : 0.f;
            }
    }
    if (mine)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int d = d0 + j * 16 + 4 * q + i;
            if (d < D) y[r * y_stride + d] = Elem<T>::put(v[i]);
        }
}

// ------------------------------------------------------- more tokens
//
// The router's lists give each expert its tokens, CT tiles of sixteen at a
// time as columns.  The second product leaves one row per slot, and a last
// kernel adds a token's rows up.
//
// 150 tokens, k = 2 of 16 bf16 experts of 4096 x 4096, three of them masked: 179
// us for 872 MB of gates and ups, 109 us for 436 MB of downs (4.9 and 4.0
// TB/s; a last round of workgroups that is half full); 64 tokens, k = 4 of 32
// of 4096 x 2048: 298 us in all, 5.4 TB/s.  A list that is longer than the
// others runs on while these are done: all tokens' first choice one expert,
// 426 us in place of 380 (150 tokens, no mask).  What bounds them beside memory are cache accesses, one
// for every lane's sixteen bytes: so several rows of weights share a load of
// activations, and a step is whole cache lines.

constexpr int kWaves = 4;

// Which expert the a-th non-empty list belongs to; -1 past the last.  The
// same in every wave.
__device__ inline int nth_expert(const int32_t *__restrict__ offsets, int E, int a) {
    const int lane = threadIdx.x & 63;
    int seen = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        const int e = e0 + lane;
        const bool some = e < E && offsets[e + 1] > offsets[e];
        const uint64_t all = __ballot(some);
        const uint64_t at = __ballot(some && seen + __popcll(all & ((1ull << lane) - 1)) == a);
        if (at) return e0 + __ffsll((unsigned long long)at) - 1;
        seen += __popcll(all);
    }
    return -1;
}

// 16 RP hidden units of one expert.
template <int T, int WT, int RP, int CT, int U, int EDGE>
__global__ __launch_bounds__(64 * kWaves, 2) void group_up(const uint16_t *__restrict__ x, int64_t x_stride, int D,
                                                           const void *__restrict__ w13, const uint8_t *__restrict__ s13, int F,
                                                           int E, int k, const int32_t *__restrict__ offsets,
                                                           const int32_t *__restrict__ order,
                                                           const float *__restrict__ weights, uint32_t tiles,
                                                           __bf16 *__restrict__ h_hi, __bf16 *__restrict__ h_lo, int h_pitch) {
    constexpr int kPart = 2 * RP * CT * 64;  // sums of a wave
    typedef Acts<WT, CT, (CT > 1)> Ac;
    __shared__ __align__(16) uint8_t lds[kWaves * std::max<int>(Ac::kBytes, kPart * sizeof(f32x4))];
    f32x4 *const part = (f32x4 *)lds;  // once all waves have read what they staged
    typedef Weights<WT, EDGE> Wt;
    typedef Inputs<T, WT, EDGE> In;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    uint8_t *const mine = lds + wave * Ac::kBytes;
    const int e = nth_expert(offsets, E, blockIdx.x / tiles);
    if (e < 0) return;
    const int f0 = (int)(blockIdx.x % tiles) * 16 * RP;
    const int first = offsets[e], n = offsets[e + 1] - first;
    // tiles 2 j are gates, 2 j + 1 ups
    const auto row_of = [&](int j) { return (int64_t)e * 2 * F + min(f0 + (j >> 1) * 16 + r, F - 1) + (int64_t)(j & 1) * F; };
    int64_t row[2 * RP];
#pragma unroll
    for (int j = 0; j < 2 * RP; j++) row[j] = row_of(j);
    const int steps = (D + kCols<WT> - 1) / kCols<WT>;
    for (int c0 = blockIdx.y * 16 * CT; c0 < n; c0 += gridDim.y * 16 * CT) {
        // of token r, needed at the end; on their way before where registers
        // suffice (130 tokens, k = 4 of 64 bf16 experts of 2048 x 1408: 240 ->
        // 230 us; with two tiles some 5 % more time)
        int slot0 = 0;
        float weight0 = 0.f;
        if (CT == 1) {
            slot0 = order[first + min(c0 + r, n - 1)];
            weight0 = weights[slot0];
        }
        const uint16_t *xr[CT][Ac::kRows];
#pragma unroll
        for (int c = 0; c < CT; c++)
#pragma unroll
            for (int s = 0; s < Ac::kRows; s++)
                xr[c][s] = x + (int64_t)(order[first + min(c0 + c * 16 + Ac::row(s), n - 1)] / k) * x_stride;
        Wt w[U][2 * RP];
        Scales<WT, 2 * RP, U> sc[2];
        const int64_t scale_row = row_of(sc[0].tile());
        Ac xi[U];
        f32x4 acc[2 * RP][CT];
#pragma unroll
        for (int j = 0; j < 2 * RP; j++)
#pragma unroll
            for (int c = 0; c < CT; c++) acc[j][c] = f32x4{0};
        ring<U, kWaves>(
            (steps + U - 1) / U, wave, [&](int p, int run) { sc[p].load(s13, scale_row, D, run); },
            [&](int i, int run) {
                const int k0 = min(run * U + i, steps - 1) * kCols<WT>;
#pragma unroll
                for (int j = 0; j < 2 * RP; j++) w[i][j].load(w13, row[j], D, k0, q);
#pragma unroll
                for (int c = 0; c < CT; c++)
#pragma unroll
                    for (int s = 0; s < kIns<WT>; s++) xi[i].raw[c][s] = load8<EDGE>(xr[c][s % Ac::kRows], k0 + Ac::col(s), D);
            },
            [&](int i, int p, int run) {
                if (EDGE && run * U + i == steps - 1) {
#pragma unroll
                    for (int j = 0; j < 2 * RP; j++) w[i][j].tail(D, (steps - 1) * kCols<WT>, q);
#pragma unroll
                    for (int c = 0; c < CT; c++)
#pragma unroll
                        for (int s = 0; s < kIns<WT>; s++)
                            xi[i].raw[c][s] = tail8<EDGE>(xi[i].raw[c][s], (steps - 1) * kCols<WT> + Ac::col(s), D);
                }
                if (run * U + i < steps) {
                    Ac::fence();
                    xi[i].put(mine);
                    Ac::fence();
                    float scale[2 * RP];
#pragma unroll
                    for (int j = 0; j < 2 * RP; j++) scale[j] = sc[p].get(i, j, r, q);
#pragma unroll
                    for (int s = 0; s < kIns<WT>; s++) {
                        u32x4 v[CT];
#pragma unroll
                        for (int c = 0; c < CT; c++) v[c] = xi[i].get(mine, c, s);
#pragma unroll
                        for (int j = 0; j < 2 * RP; j++) {
                            const typename Wt::Operand o = w[i][j].operand(s, scale[j]);
#pragma unroll
                            for (int c = 0; c < CT; c++) acc[j][c] = In::template mul<Wt>(v[c], o, acc[j][c]);
                        }
                    }
                }
            });
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 2 * RP; j++)
#pragma unroll
            for (int c = 0; c < CT; c++) part[wave * kPart + (j * CT + c) * 64 + lane] = acc[j][c];
        __syncthreads();
        for (int p = wave; p < RP * CT; p += kWaves) {
            const int j = p / CT, c = p % CT, f = f0 + j * 16;
            if (c0 + c * 16 + r < n && f < F) {
                f32x4 sg = {0}, su = {0};
#pragma unroll
                for (int w = 0; w < kWaves; w++) {
                    sg += part[w * kPart + (2 * j * CT + c) * 64 + lane];
                    su += part[w * kPart + ((2 * j + 1) * CT + c) * 64 + lane];
                }
                const int slot = CT == 1 ? slot0 : order[first + c0 + c * 16 + r];
                const float weight = CT == 1 ? weight0 : weights[slot];
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; i++) v[i] = f + 4 * q + i < F ? gated(sg[i], su[i], weight) : 0.f;
                const int64_t at = (int64_t)slot * h_pitch + f + 4 * q;
                store_hidden(h_hi, h_lo, at, v);
                if (f + 16 >= F)  // the rest of the last step
                    for (int o = 16; f + o < h_pitch; o += 16) {
                        const float zero[4] = {0.f, 0.f, 0.f, 0.f};
                        store_hidden(h_hi, h_lo, at + o, zero);
                    }
            }
        }
        __syncthreads();
    }
}

template <int WT, int R, int CT, int U, int EDGE>
__global__ __launch_bounds__(64 * kWaves, 2) void group_down(const __bf16 *__restrict__ h_hi, const __bf16 *__restrict__ h_lo,
                                                          int h_pitch, int F, const void *__restrict__ w2,
                                                          const uint8_t *__restrict__ s2, int D, int E,
                                                          const int32_t *__restrict__ offsets,
                                                          const int32_t *__restrict__ order, uint32_t tiles,
                                                          float *__restrict__ out) {
    constexpr int kPart = R * CT * 64;  // sums of a wave
    // (4-bit weights: the registers do not suffice)
    typedef Acts<WT, CT, (CT > 1 && WT != SIM_TYPE_MX4)> Ac;
    __shared__ __align__(16) uint8_t lds[kWaves * std::max<int>(2 * Ac::kBytes, kPart * sizeof(f32x4))];
    f32x4 *const part = (f32x4 *)lds;  // once all waves have read what they staged
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    uint8_t *const mine = lds + wave * 2 * Ac::kBytes, *const mine_lo = mine + Ac::kBytes;
    const int e = nth_expert(offsets, E, blockIdx.x / tiles);
    if (e < 0) return;
    const int d0 = (int)(blockIdx.x % tiles) * 16 * R;
    const int first = offsets[e], n = offsets[e + 1] - first;
    const int steps = (F + kCols<WT> - 1) / kCols<WT>;
    for (int c0 = blockIdx.y * 16 * CT; c0 < n; c0 += gridDim.y * 16 * CT) {
        const int slot0 = CT == 1 ? order[first + min(c0 + r, n - 1)] : 0;
        int64_t at[CT][Ac::kRows];
#pragma unroll
        for (int c = 0; c < CT; c++)
#pragma unroll
            for (int s = 0; s < Ac::kRows; s++)
                at[c][s] = (int64_t)order[first + min(c0 + c * 16 + Ac::row(s), n - 1)] * h_pitch + Ac::col(0);
        typedef Weights<WT, EDGE> Wt;
        Wt w[U][R];
        Scales<WT, R, U> sc[2];
        Ac hi[U], lo[U];
        f32x4 acc[R][CT];
        int64_t row[R];
#pragma unroll
        for (int j = 0; j < R; j++) {
            row[j] = (int64_t)e * D + min(d0 + j * 16 + r, D - 1);
#pragma unroll
            for (int c = 0; c < CT; c++) acc[j][c] = f32x4{0};
        }
        ring<U, kWaves>(
            (steps + U - 1) / U, wave,
            [&](int p, int run) {
                sc[p].load(s2, (int64_t)e * D + min(d0 + sc[p].tile() * 16 + r, D - 1), F, run);
            },
            [&](int i, int run) {
                const int k0 = min(run * U + i, steps - 1) * kCols<WT>;
#pragma unroll
                for (int j = 0; j < R; j++) w[i][j].load(w2, row[j], F, k0, q);
#pragma unroll
                for (int c = 0; c < CT; c++)
#pragma unroll
                    for (int s = 0; s < kIns<WT>; s++) {
                        const int64_t from = at[c][s % Ac::kRows] + k0 + (Ac::col(s) - Ac::col(0));
                        hi[i].raw[c][s] = *(const u32x4 *)(h_hi + from);
                        lo[i].raw[c][s] = *(const u32x4 *)(h_lo + from);
                    }
            },
            [&](int i, int p, int run) {
                if (run * U + i < steps) {
                    Ac::fence();
                    hi[i].put(mine);
                    lo[i].put(mine_lo);
                    Ac::fence();
                    float scale[R];
#pragma unroll
                    for (int j = 0; j < R; j++) {
                        if (EDGE && run * U + i == steps - 1) w[i][j].tail(F, (steps - 1) * kCols<WT>, q);
                        scale[j] = sc[p].get(i, j, r, q);
                    }
#pragma unroll
                    for (int s = 0; s < kIns<WT>; s++) {
                        bf16x8 v[CT], l[CT];
#pragma unroll
                        for (int c = 0; c < CT; c++) {
                            v[c] = __builtin_bit_cast(bf16x8, hi[i].get(mine, c, s));
                            l[c] = __builtin_bit_cast(bf16x8, lo[i].get(mine_lo, c, s));
                        }
#pragma unroll
                        for (int j = 0; j < R; j++) {
                            const typename Wt::Operand o = w[i][j].operand(s, scale[j]);
#pragma unroll
                            for (int c = 0; c < CT; c++) acc[j][c] = Wt::mul(o, l[c], Wt::mul(o, v[c], acc[j][c]));
                        }
                    }
                }
            });
        __syncthreads();
#pragma unroll
        for (int j = 0; j < R; j++)
#pragma unroll
            for (int c = 0; c < CT; c++) part[wave * kPart + (j * CT + c) * 64 + lane] = acc[j][c];
        __syncthreads();
        for (int p = wave; p < R * CT; p += kWaves) {
            const int j = p / CT, c = p % CT;
            if (c0 + c * 16 + r < n) {
                f32x4 v = {0};
#pragma unroll
                for (int w = 0; w < kWaves; w++) v += part[w * kPart + (j * CT + c) * 64 + lane];
                float *o = out + (int64_t)(CT == 1 ? slot0 : order[first + c0 + c * 16 + r]) * D;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int d = d0 + j * 16 + 4 * q + i;
                    if (d < D) o[d] = v[i];
                }
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

inline size_t aligned(size_t n) { return (n + 255) / 256 * 256; }

// Calls f with the kind of rows of K elements as a constant.  Rows of less
// than eight are left to the form of one column tile for more tokens.
template <int WT, int CT, typename Fn> inline void by_edge(int64_t K, Fn &&f) {
    if (K % kCols<WT> == 0) f(std::integral_constant<int, kWhole>());
    else if (K >= 8) f(std::integral_constant<int, kTail>());
    else if constexpr (CT == 1) f(std::integral_constant<int, kTiny>());
}

// The workspace in the order in which it is handed out.
struct Layout {
    size_t experts, weights, offsets, order, route, hi, lo, part, end;
    size_t n_used, expert, slot, arrived;
    int pitch;
    Layout(int64_t T, int64_t D, int E, int k, int64_t F) {
        const size_t n = (size_t)T * k, lists = std::min<size_t>(E, n);
        pitch = (int)((F + kStep - 1) / kStep * kStep);
        size_t at = 0;
        const auto take = [&](size_t bytes) { const size_t p = at; at += aligned(bytes); return p; };
        hi = take(n * pitch * 2);
        lo = take(n * pitch * 2);
        if (few(T, E, D, F)) {
            n_used = take(4);
            expert = take(lists * 2);
            slot = take(lists * 16 * 2);
            arrived = take((size_t)(D + 15) / 16 * 4);
            part = take((size_t)kMaxSplits * ((D + 63) / 64 * 64) * 16 * 4);
        } else {
            experts = take(n * 4);
            weights = take(n * 4);
            offsets = take((size_t)(E + 1) * 4);
            order = take(n * 4);
            route = take(route_workspace(T, E, k));
            part = take(n * D * 4);
        }
        end = at;
    }
};

template <int T, int WT> sim_status few_t(hipStream_t st, const LayerArgs &a, uint8_t *ws) {
    const RouteArgs &r = a.route;
    const Layout at(r.T, a.D, r.E, r.k, a.F);
    __bf16 *hi = (__bf16 *)(ws + at.hi), *lo = (__bf16 *)(ws + at.lo);
    const FewPlan plan = {(int32_t *)(ws + at.n_used), (int16_t *)(ws + at.expert), (int16_t *)(ws + at.slot),
                          (uint32_t *)(ws + at.arrived)};
    constexpr int R = WT == SIM_TYPE_MX4 ? 4 : 2;  // row tiles that share the hidden values
    const int64_t lists = std::min<int64_t>(r.E, r.T * r.k);
    const int tf = (int)((a.F + 15) / 16), td = (int)((a.D + 16 * R - 1) / (16 * R));
    // runs of four steps where there is one for each wave, else of two (8
    // tokens, k = 4 of 64 bf16 experts of 896 x 2048: 60 us, 74 with runs of four)
    const auto up = [&](auto u, auto edge) {
        few_up<T, WT, decltype(u)::value, decltype(edge)::value><<<(uint32_t)std::min<int64_t>(kFewGroups, lists * tf), 64 * kFewWaves, 0, st>>>(
            r, (const uint16_t *)a.x, a.x_stride, (int)a.D, a.w13, a.s13, (int)a.F, tf, hi, lo, at.pitch, plan, td);
    };
    by_edge<WT, 0>(a.D, [&](auto edge) {
        if (a.D >= 4 * kFewWaves * kCols<WT>) up(std::integral_constant<int, 4>(), edge);
        else up(std::integral_constant<int, 2>(), edge);
    });
    // as many parts as workgroups fit, but a run for every wave: joining costs
    // a part about half a microsecond (one token, 11 experts of 1024 x 2869:
    // 25 us in 24 parts, 20 us in 15)
    const int64_t runs = lists * ((a.F + kCols<WT> * few_down_run<WT> - 1) / (kCols<WT> * few_down_run<WT>));
    const int splits = (int)std::max<int64_t>(1, std::min<int64_t>(std::min(kMaxSplits, kFewGroups / td), runs / kFewWaves));
    const auto down = [&](auto edge) {
        few_down<T, WT, R, decltype(edge)::value><<<td * splits, 64 * kFewWaves, 0, st>>>(
            hi, lo, at.pitch, (int)a.F, a.w2, a.s2, (int)a.D, (int)r.T, plan, (int)lists, splits, (float *)(ws + at.part),
            (typename Elem<T>::type *)a.y, a.y_stride);
    };
    if constexpr (WT == SIM_TYPE_MX4) down(std::integral_constant<int, kWhole>());  // rows and hidden values are padded
    else by_edge<WT, 0>(a.F, down);
    return SIM_OPS_LAUNCH_OK();
}

template <int T, int WT, int CT> sim_status group_t(hipStream_t st, const LayerArgs &a, uint8_t *ws) {
    const RouteArgs &r = a.route;
    const Layout at(r.T, a.D, r.E, r.k, a.F);
    int32_t *experts = (int32_t *)(ws + at.experts), *offsets = (int32_t *)(ws + at.offsets), *order = (int32_t *)(ws + at.order);
    float *weights = (float *)(ws + at.weights), *part = (float *)(ws + at.part);
    __bf16 *hi = (__bf16 *)(ws + at.hi), *lo = (__bf16 *)(ws + at.lo);
    const sim_status s = launch_route(st, r, experts, weights, offsets, order, ws + at.route);
    if (s != SIM_OK) return s;
    constexpr bool M = WT == SIM_TYPE_MX4;
    // rows that share the activations' loads, and how far ahead all are loaded
    constexpr int RP = CT == 1 && !M ? 1 : 2, UU = M ? 2 : 4 / CT, R = 4, UD = CT == 4 ? 1 : 2;
    const uint32_t lists = (uint32_t)std::min<int64_t>(r.E, r.T * r.k);
    const uint32_t tf = (uint32_t)((a.F + 16 * RP - 1) / (16 * RP)), td = (uint32_t)((a.D + 16 * R - 1) / (16 * R)), tj = (uint32_t)((a.D + 255) / 256);
    // lists are shared among workgroups where these would leave compute units
    // idle, which costs another read of the weights from the caches (120
    // tokens, k = 4 of 4 4-bit experts of 2048 x 768: 68 -> 41 us; 1000, k = 2
    // of 8 bf16 ones of 1024 x 512: 96 -> 59 us)
    const auto grid = [&](uint32_t tiles) {
        const uint32_t all = (uint32_t)((r.T + 16 * CT - 1) / (16 * CT));
        return dim3(lists * tiles, std::max(1u, std::min(all, kSlots / (lists * tiles))));
    };
    by_edge<WT, CT>(a.D, [&](auto edge) {
        group_up<T, WT, RP, CT, UU, decltype(edge)::value><<<grid(tf), 64 * kWaves, 0, st>>>(
            (const uint16_t *)a.x, a.x_stride, (int)a.D, a.w13, a.s13, (int)a.F, r.E, r.k, offsets, order, weights, tf, hi, lo,
            at.pitch);
    });
    const auto down = [&](auto edge) {
        group_down<WT, R, CT, UD, decltype(edge)::value><<<grid(td), 64 * kWaves, 0, st>>>(
            hi, lo, at.pitch, (int)a.F, a.w2, a.s2, (int)a.D, r.E, offsets, order, td, part);
    };
    if constexpr (M) down(std::integral_constant<int, kWhole>());  // rows and hidden values are padded
    else by_edge<WT, CT>(a.F, down);
    layer_join<T><<<(uint32_t)(r.T * tj), 256, 0, st>>>(part, experts, r.k, a.D, (typename Elem<T>::type *)a.y, a.y_stride, tj);
    return SIM_OPS_LAUNCH_OK();
}

template <int T>
__global__ __launch_bounds__(256) void layer_zero(typename Elem<T>::type *y, int64_t stride, int64_t D) {
    for (int64_t d = threadIdx.x; d < D; d += 256) y[blockIdx.x * stride + d] = Elem<T>::put(0.f);
}

template <int T, int WT> sim_status layer_t(hipStream_t st, const LayerArgs &a, uint8_t *ws) {
    const RouteArgs &r = a.route;
    if (a.F == 0) {
        layer_zero<T><<<(uint32_t)r.T, 256, 0, st>>>((typename Elem<T>::type *)a.y, a.y_stride, a.D);
        return SIM_OPS_LAUNCH_OK();
    }
    switch (layer_form(r.T, r.E, r.k, a.D, a.F, a.mx4)) {
        case kFew: return few_t<T, WT>(st, a, ws);
        case kGroup1: return group_t<T, WT, 1>(st, a, ws);
        case kGroup4:
            if constexpr (WT != SIM_TYPE_MX4) return group_t<T, WT, 4>(st, a, ws);  // (4-bit weights never take it)
        case kGroup2: break;
    }
    return group_t<T, WT, 2>(st, a, ws);
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
