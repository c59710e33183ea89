// Router: the k highest of each token's logits, their softmax weights, the
// tokens' lists by expert, and the gradient.
//
// Sixteen lanes hold a token's logits in registers (NV each), so that a wave
// runs four tokens at once and every exchange stays within a row of 16 lanes.
// A logit is compared as a whole number that orders as the value does, NaN
// highest, 0 for what cannot be chosen (masked, -infinity, past E).
//
// 16385 tokens, 256 bf16 experts, a mask of its own for each token, k = 8:
// choice 11 us (k searches of 16 registers a lane, 1.1 TB/s), lists 8.7 us (a
// workgroup reads the 66 KB of all chunks' counts), gradient 8 us; 8 tokens,
// 64 experts: 4.5 us in one launch.
#include "ops_exp64.h"
#include "ops_route_keys.h"

namespace simops {
namespace {

constexpr int kChunk = 64;           // tokens of one workgroup
constexpr int kThreads = 16 * kChunk;
constexpr int kPart = 16;            // tokens of one where there are few

typedef uint32_t u32_any __attribute__((aligned(1), may_alias));  // words of elements of any type

// N consecutive elements, at any alignment that their type has.
template <int N, typename E> __device__ inline void load_some(const E *p, E v[N]) {
    if (sizeof(E) * N >= 4) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(E) * N / 4); i++) ((u32_any *)v)[i] = ((const u32_any *)p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = p[i];
    }
}
template <int N, typename E> __device__ inline void store_some(E *p, const E v[N]) {
    if (sizeof(E) * N >= 4) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(E) * N / 4); i++) ((u32_any *)p)[i] = ((const u32_any *)v)[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) p[i] = v[i];
    }
}

// A token's logits: lane l of 16 holds experts NV l .. NV l + NV - 1, and ok
// has a bit for each that may be used.
template <int T, int NV>
__device__ inline uint64_t load_logits(const typename Elem<T>::type *__restrict__ z, const uint8_t *__restrict__ mask, int E,
                                       bool live, typename Elem<T>::type v[NV]) {
    const int e0 = (threadIdx.x & 15) * NV;
    uint64_t ok = 0;
    if (live && e0 + NV <= E) {
        uint8_t m[NV];
        load_some<NV>(z + e0, v);
        if (mask) {
            load_some<NV>(mask + e0, m);
#pragma unroll
            for (int i = 0; i < NV; i++) ok |= (uint64_t)(m[i] != 0) << i;
        } else {
            ok = ~0ull;
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const bool in = live && e0 + i < E;
            v[i] = in ? z[e0 + i] : Elem<T>::put(0.f);
            ok |= (uint64_t)(in && (!mask || mask[e0 + i])) << i;
        }
    }
    return ok;
}

// The keys of a lane's experts and the search for the best of all.  16-bit
// logits fit with their index in one word, the lower index higher: a search
// is maxima and nothing else.  32-bit ones are searched as pairs.
template <int T, int NV> struct Keys {
    uint32_t k[NV];
    static __device__ uint32_t of(typename Elem<T>::type v, uint32_t e) {
        const uint16_t b = __builtin_bit_cast(uint16_t, v);
        const uint16_t inf = T == SIM_TYPE_BF16 ? 0x7f80 : 0x7c00;
        const uint16_t key = (b & 0x7fff) > inf ? 0xffff : (b & 0x7fff) == 0 ? 0x8000 : b == (inf | 0x8000) ? 0 : b & 0x8000 ? ~b : b | 0x8000;
        return key ? (uint32_t)key << 16 | (0xffff - e) : 0;
    }
    static __device__ float value(uint32_t k) {
        const uint16_t key = k >> 16;
        return Elem<T>::get(__builtin_bit_cast(typename Elem<T>::type,
                                               (uint16_t)(key == 0xffff ? 0x7fff : key & 0x8000 ? key & 0x7fff : ~key)));
    }
    // the best of 16 lanes and its expert; 0 where nothing is left.  It is
    // taken out.
    __device__ uint32_t take(uint32_t &e) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < NV; i++) m = max(m, k[i]);
        m = max16(m);
#pragma unroll
        for (int i = 0; i < NV; i++) k[i] = k[i] == m ? 0 : k[i];
        e = 0xffff - (m & 0xffff);
        return m;
    }
};
template <int NV> struct Keys<SIM_TYPE_F32, NV> {
    uint32_t k[NV];
    static __device__ uint32_t of(float v, uint32_t) { return order_key(v); }
    static __device__ float value(uint32_t k) { return key_value(k); }
    __device__ uint32_t take(uint32_t &e) {
        const uint32_t e0 = (threadIdx.x & 15) * NV;
        uint32_t m = 0;
        e = 0xffffu;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const bool better = k[i] > m;  // the first of equal ones has the lowest index
            m = better ? k[i] : m;
            e = better ? e0 + i : e;
        }
        best16(m, e);
#pragma unroll
        for (int i = 0; i < NV; i++) k[i] = e0 + i == e ? 0 : k[i];
        return m;
    }
};

// Exclusive prefix sums over kThreads values (one a thread) and their total.
__device__ inline int block_scan(int v, int *wave_sum, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(s, d);
        if (lane >= d) s += o;
    }
    if (lane == 63) wave_sum[wave] = s;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < kThreads / 64; w++) {
        if (w < wave) before += wave_sum[w];
        total += wave_sum[w];
    }
    return before + s - v;
}

__host__ __device__ inline int hist_pitch(int E) { return (E + 3) / 4 * 4; }

// The tokens of a chunk that chose an expert, a bit for each.  A token has an
// expert once at most, so the place of its slot in the expert's list is the
// number of lower bits.
__device__ inline void mark(uint64_t *chose, int e, int tok) { atomicOr((unsigned long long *)&chose[e], 1ull << tok); }
__device__ inline int before_in(uint64_t chose, int tok) { return __popcll(chose & ((1ull << tok) - 1)); }

// The choices of CH tokens, sixteen threads a token with the choices l and l +
// 16 each (had: whether there is one), and what is made of them: their counts,
// or (one chunk only) the lists.
struct Lists {
    uint64_t chose[SIM_MOE_MAX_EXPERTS];  // zeros, before
    int base[SIM_MOE_MAX_EXPERTS];
    int wave_sum[kThreads / 64];
};
template <int CH>
__device__ inline void clear(Lists &s) {
    for (int e = threadIdx.x; e < SIM_MOE_MAX_EXPERTS; e += 16 * CH) s.chose[e] = 0;
}
template <int CH>
__device__ inline void finish(Lists &s, int64_t t, bool live, int k, int E, int n_tok, const uint32_t e[2], const uint32_t had[2],
                              const float w[2], int32_t *__restrict__ experts, float *__restrict__ weights,
                              uint8_t *__restrict__ hist, int32_t *__restrict__ offsets, int32_t *__restrict__ order) {
    const int l = threadIdx.x & 15, tok = threadIdx.x >> 4;
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const int j = q * 16 + l;
        if (live && j < k) {
            experts[t * k + j] = had[q] ? (int)e[q] : -1;
            weights[t * k + j] = had[q] ? w[q] : 0.f;
            if (had[q] && order) mark(s.chose, e[q], tok);
        }
    }
    if (!order) return;
    __syncthreads();
    if (CH < kChunk || gridDim.x > 1) {
        // at most kChunk: a byte
        for (int i = threadIdx.x; i < hist_pitch(E); i += 16 * CH)
            hist[(int64_t)blockIdx.x * hist_pitch(E) + i] = (uint8_t)__popcll(s.chose[i]);
        return;
    }
    int total;
    s.base[threadIdx.x] = block_scan(__popcll(s.chose[threadIdx.x]), s.wave_sum, total);
    if ((int)threadIdx.x < E) offsets[threadIdx.x] = s.base[threadIdx.x];
    if (threadIdx.x == 0) offsets[E] = total;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; q++)
        if (live && had[q]) order[s.base[e[q]] + before_in(s.chose[e[q]], tok)] = tok * k + q * 16 + l;
    for (int i = total + threadIdx.x; i < n_tok * k; i += kThreads) order[i] = -1;
}

// Choice and weights of CH tokens; their counts, or (one chunk only) the lists.
template <int T, int NV, int CH>
__global__ __launch_bounds__(16 * CH) void route_choose(const typename Elem<T>::type *__restrict__ logits, int64_t n_tok,
                                                         int E, int64_t stride, const uint8_t *__restrict__ mask,
                                                         int64_t mask_stride, int k, int renorm,
                                                         int32_t *__restrict__ experts, float *__restrict__ weights,
                                                         uint8_t *__restrict__ hist, int32_t *__restrict__ offsets,
                                                         int32_t *__restrict__ order) {
    __shared__ Lists lists;
    const int l = threadIdx.x & 15, tok = threadIdx.x >> 4;
    const int64_t t = (int64_t)blockIdx.x * CH + tok;
    const bool live = t < n_tok;
    clear<CH>(lists);
    Keys<T, NV> key;
    float z = 0.f, top = 0.f;
    {
        typename Elem<T>::type v[NV];
        const uint64_t ok = load_logits<T, NV>(logits + (live ? t : 0) * stride, mask ? mask + (live ? t : 0) * mask_stride : nullptr, E, live, v);
#pragma unroll
        for (int i = 0; i < NV; i++) key.k[i] = (ok >> i) & 1 ? Keys<T, NV>::of(v[i], l * NV + i) : 0;
    }
    if (!renorm) {  // the sum over all that are allowed
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < NV; i++) m = max(m, key.k[i]);
        top = Keys<T, NV>::value(max16(m));
#pragma unroll
        for (int i = 0; i < NV; i++) z += key.k[i] ? fast_exp(Keys<T, NV>::value(key.k[i]) - top) : 0.f;
        z = sum16(z);
    }
    __syncthreads();

    uint32_t mine[2] = {0, 0}, mine_e[2] = {0, 0};  // the choices l and l + 16
    for (int j = 0; j < k; j++) {
        uint32_t e;
        const uint32_t m = key.take(e);
        if (j == 0) top = Keys<T, NV>::value(m);
        if (l == (j & 15)) {
            mine[j >> 4] = m;
            mine_e[j >> 4] = e;
        }
    }
    float w[2];
#pragma unroll
    for (int q = 0; q < 2; q++) w[q] = mine[q] ? fast_exp(Keys<T, NV>::value(mine[q]) - top) : 0.f;
    if (renorm) z = sum16(w[0] + w[1]);
#pragma unroll
    for (int q = 0; q < 2; q++) w[q] = w[q] / z;
    finish<CH>(lists, t, live, k, E, (int)min(n_tok, (int64_t)CH), mine_e, mine, w, experts, weights, hist, offsets, order);
}

// The sums over the chunks before each; the row past the last gets the totals.
// (Counts are loaded eight at a time: one after another the 512 chunks of 32768
// tokens took 7.1 us, so 4.9.)
__global__ __launch_bounds__(kThreads) void route_scan(const uint8_t *__restrict__ hist, int32_t *__restrict__ sums, int chunks,
                                                       int E) {
    __shared__ int part_sum[64][16];
    const int e = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4, pitch = hist_pitch(E);
    const int per = (chunks + 63) / 64, c0 = part * per, c1 = min(chunks, c0 + per);
    int s = 0;
    const auto load8 = [&](int c, int v[8]) {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = c + i < c1 ? hist[(int64_t)(c + i) * pitch + e] : 0;
    };
    int v[8];
    if (e < E)
        for (int c = c0; c < c1; c += 8) {
            load8(c, v);
#pragma unroll
            for (int i = 0; i < 8; i++) s += v[i];
        }
    part_sum[part][threadIdx.x & 15] = s;
    __syncthreads();
    if (e >= E) return;
    int before = 0, total = 0;
#pragma unroll 16
    for (int p = 0; p < 64; p++) {
        const int n = part_sum[p][threadIdx.x & 15];
        if (p < part) before += n;
        total += n;
    }
    for (int c = c0; c < c1; c += 8) {
        if (per > 8) load8(c, v);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (c + i < c1) sums[(int64_t)(c + i) * E + e] = before;
            before += v[i];
        }
    }
    if (part == 0) sums[(int64_t)chunks * E + e] = total;
}

// Lists of one chunk, from the counts of all (each workgroup adds them up
// itself; of chunks, or of their parts) or from the scanned ones.
__global__ __launch_bounds__(kThreads) void route_place(const int32_t *__restrict__ experts, int64_t n_tok, int E, int k,
                                                        const uint8_t *__restrict__ hist, int parts, int rows,
                                                        const int32_t *__restrict__ sums, int32_t *__restrict__ offsets,
                                                        int32_t *__restrict__ order) {
    __shared__ uint64_t chose[SIM_MOE_MAX_EXPERTS];  // in this chunk
    __shared__ int before[SIM_MOE_MAX_EXPERTS];      // slots of the chunks before
    __shared__ int all[SIM_MOE_MAX_EXPERTS];
    __shared__ int wave_sum[kThreads / 64];
    const int chunk = blockIdx.x, chunks = gridDim.x, t = threadIdx.x;
    const int first = chunk * kChunk * k;
    const int n = (int)min((int64_t)kChunk * k, n_tok * k - first);
    chose[t] = 0;
    before[t] = all[t] = 0;
    int mine[2];  // the experts of this thread's slots
#pragma unroll
    for (int q = 0; q < 2; q++) mine[q] = t + q * kThreads < n ? experts[(int64_t)first + t + q * kThreads] : -1;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; q++)
        if (mine[q] >= 0) mark(chose, mine[q], (t + q * kThreads) / k);
    if (sums) {
        if (t < E) {
            before[t] = sums[(int64_t)chunk * E + t];
            all[t] = sums[(int64_t)chunks * E + t];
        }
    } else {
        // a thread adds up four experts' bytes over every step-th row
        const int pitch = hist_pitch(E);
        int width = 4;
        while (width * 4 < pitch) width <<= 1;
        const int e = (t & (width - 1)) * 4, step = kThreads / width;
        if (e < pitch) {
            int a[4] = {0, 0, 0, 0}, b[4] = {0, 0, 0, 0};
            for (int c = t / width; c < rows; c += 8 * step) {  // eight loads under way
                uint32_t v[8];
#pragma unroll
                for (int i = 0; i < 8; i++)
                    v[i] = c + i * step < rows ? *(const uint32_t *)(hist + (int64_t)(c + i * step) * pitch + e) : 0;
#pragma unroll
                for (int i = 0; i < 8; i++)
#pragma unroll
                    for (int x = 0; x < 4; x++) {
                        const int n = (v[i] >> (8 * x)) & 255;
                        a[x] += n;
                        b[x] += c + i * step < chunk * parts ? n : 0;
                    }
            }
#pragma unroll
            for (int x = 0; x < 4; x++) {
                atomicAdd(&all[e + x], a[x]);
                atomicAdd(&before[e + x], b[x]);
            }
        }
    }
    __syncthreads();
    int total;
    const int base = block_scan(all[t], wave_sum, total);
    before[t] += base;
    if (chunk == 0) {
        if (t < E) offsets[t] = base;
        if (t == 0) offsets[E] = total;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const int s = t + q * kThreads;
        if (mine[q] >= 0) order[before[mine[q]] + before_in(chose[mine[q]], s / k)] = first + s;
    }
    for (int64_t s = max((int64_t)total, (int64_t)first) + t; s < (int64_t)first + n; s += kThreads) order[s] = -1;
}

// Gradient: sixteen lanes a token again.  Lane l has the choices l and l +
// 16; a row in LDS brings their part to the lanes that hold the experts.
template <int T, int NV>
__global__ __launch_bounds__(256) void route_grad(const typename Elem<T>::type *__restrict__ logits, int64_t n_tok, int E,
                                                  int64_t stride, const uint8_t *__restrict__ mask, int64_t mask_stride,
                                                  int k, int renorm, float scale, const int32_t *__restrict__ experts,
                                                  const float *__restrict__ dw, typename Elem<T>::type *__restrict__ dz) {
    typedef typename Elem<T>::type El;
    __shared__ __align__(16) float rows[16][NV * 16];
    const int l = threadIdx.x & 15;
    const int64_t t = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (t >= n_tok) return;  // sixteen lanes at a time: they share no barrier
    float *row = rows[threadIdx.x >> 4];
    const El *zt = logits + t * stride;
    const uint8_t *mt = mask ? mask + t * mask_stride : nullptr;
    int e[2];
    float g[2], v[2];
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const int j = q * 16 + l;
        e[q] = j < k ? experts[t * k + j] : -1;
        if (e[q] < 0 || e[q] >= E || (mt && !mt[e[q]])) e[q] = -1;
        g[q] = e[q] >= 0 ? dw[t * k + j] * scale : 0.f;
        v[q] = e[q] >= 0 ? Elem<T>::get(zt[e[q]]) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < NV; i++) row[i * 16 + l] = 0.f;
    float top, p[NV];
    uint64_t ok = 0;
    if (renorm) {
        uint32_t m = max(order_key(v[0]), order_key(v[1]));
        top = key_value(max16(m));
    } else {
        El all[NV];
        ok = load_logits<T, NV>(zt, mt, E, true, all);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const uint32_t key = (ok >> i) & 1 ? order_key(Elem<T>::get(all[i])) : 0u;
            m = max(m, key);
            if (!key) ok &= ~(1ull << i);  // -infinity takes no part, as in the choice: a row of nothing else has no sum
        }
        top = key_value(max16(m));
#pragma unroll
        for (int i = 0; i < NV; i++) p[i] = (ok >> i) & 1 ? fast_exp(Elem<T>::get(all[i]) - top) : 0.f;
    }
    float w[2], z = 0.f;
#pragma unroll
    for (int q = 0; q < 2; q++) w[q] = e[q] >= 0 ? fast_exp(v[q] - top) : 0.f;
    if (renorm) z = w[0] + w[1];
    else
#pragma unroll
        for (int i = 0; i < NV; i++) z += p[i];
    const float inv = 1.f / sum16(z);
    float dot = 0.f;
#pragma unroll
    for (int q = 0; q < 2; q++) {
        w[q] *= inv;
        dot += e[q] >= 0 ? g[q] * w[q] : 0.f;
    }
    dot = sum16(dot);
    wave_fence();  // the zeros are other lanes' than the values, and both than what is read
#pragma unroll
    for (int q = 0; q < 2; q++)
        if (e[q] >= 0) row[e[q]] = renorm ? w[q] * (g[q] - dot) : g[q];
    wave_fence();
    El out[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const float r = row[l * NV + i];
        out[i] = Elem<T>::put(renorm ? r : (ok >> i) & 1 ? p[i] * inv * (r - dot) : 0.f);
    }
    El *o = dz + t * E + l * NV;
    if (l * NV + NV <= E) store_some<NV>(o, out);
    else
#pragma unroll
        for (int i = 0; i < NV; i++)
            if (l * NV + i < E) o[i] = out[i];
}

// Lists of choices that are given: what route_choose ends with (200 tokens, k =
// 8: 4.9 us).
template <int CH>
__global__ __launch_bounds__(16 * CH) void route_given(RouteArgs a, int32_t *__restrict__ experts, float *__restrict__ weights,
                                                       uint8_t *__restrict__ hist, int32_t *__restrict__ offsets,
                                                       int32_t *__restrict__ order) {
    __shared__ Lists lists;
    const int64_t t = (int64_t)blockIdx.x * CH + (threadIdx.x >> 4);
    const bool live = t < a.T;
    clear<CH>(lists);
    uint32_t e[2], had[2];
    float w[2];
    given_choices(a, live ? t : 0, e, had, w);
    __syncthreads();
    finish<CH>(lists, t, live, a.k, a.E, (int)min(a.T, (int64_t)CH), e, had, w, experts, weights, hist, offsets, order);
}

// ------------------------------------------------------------------ scores, bias, groups

// 1 / x for 1 <= x <= 2^11, to the last place but one
__device__ inline double reciprocal(double x) {
    double y = __builtin_amdgcn_rcp(x);
    y = __builtin_fma(__builtin_fma(-x, y, 1.), y, y);
    return __builtin_fma(__builtin_fma(-x, y, 1.), y, y);
}
__device__ inline double sigmoid64(double z) {
    const double e = exp64(-__builtin_fabs(z));
    return (z < 0. ? e : 1.) * reciprocal(1. + e);
}
template <int CTRL> __device__ inline double dpp_f64(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, dpp_u32<CTRL>((uint32_t)b) | (uint64_t)dpp_u32<CTRL>((uint32_t)(b >> 32)) << 32);
}
__device__ inline double sum16(double v) {
    v += dpp_f64<kDppXor1>(v);
    v += dpp_f64<kDppXor2>(v);
    v += dpp_f64<kDppHalfMirror>(v);
    v += dpp_f64<kDppMirror>(v);
    return v;
}

// The two highest keys of those seen.
struct Two {
    uint32_t a = 0, b = 0;
    __device__ void add(uint32_t k) {
        b = max(b, min(a, k));
        a = max(a, k);
    }
    template <int CTRL> __device__ void merge() {
        const uint32_t a2 = dpp_u32<CTRL>(a), b2 = dpp_u32<CTRL>(b);
        b = max(min(a, a2), max(b, b2));
        a = max(a, a2);
    }
    // of a group, as a key; 0 where nothing of it can be chosen
    __device__ uint32_t value(int best) const { return best == 1 || !b ? a : max(1u, order_key(key_value(a) + key_value(b))); }
};

// Which groups a token keeps, a bit for each, from its experts' keys.  Where a
// group is a whole number of lanes, a power of two, each lane merges with those
// of its own; else the groups are searched one after another.
template <int NV> __device__ inline uint64_t top_groups(const uint32_t key[NV], int E, int groups, int top, int best) {
    const int l = threadIdx.x & 15, size = E / groups, lanes = size / NV;
    uint64_t keep = 0;
    if (lanes * NV == size && (lanes & (lanes - 1)) == 0) {
        Two two;
#pragma unroll
        for (int i = 0; i < NV; i++) two.add(key[i]);
        if (lanes >= 2) two.merge<kDppXor1>();
        if (lanes >= 4) two.merge<kDppXor2>();
        if (lanes >= 8) two.merge<kDppHalfMirror>();
        if (lanes >= 16) two.merge<kDppMirror>();
        const uint32_t mine = l / lanes;
        uint32_t v = two.value(best);
        for (int j = 0; j < top; j++) {
            uint32_t k = v, i = mine;
            best16(k, i);
            if (k) keep |= 1ull << i;
            if (mine == i) v = 0;
        }
        return keep;
    }
    uint32_t v[SIM_MOE_MAX_GROUPS / 16] = {};  // of groups l, l + 16, ...
    for (int g = 0; g < groups; g++) {
        Two two;
#pragma unroll
        for (int i = 0; i < NV; i++) two.add((uint32_t)(l * NV + i - g * size) < (uint32_t)size ? key[i] : 0);
        two.merge<kDppXor1>();
        two.merge<kDppXor2>();
        two.merge<kDppHalfMirror>();
        two.merge<kDppMirror>();
#pragma unroll
        for (int q = 0; q < SIM_MOE_MAX_GROUPS / 16; q++)
            if (g == q * 16 + l) v[q] = two.value(best);
    }
    for (int j = 0; j < top; j++) {
        uint32_t k = 0, i = 0xffffu;
#pragma unroll
        for (int q = 0; q < SIM_MOE_MAX_GROUPS / 16; q++) keep_better(k, i, v[q], q * 16 + l);
        best16(k, i);
        if (k) keep |= 1ull << i;
#pragma unroll
        for (int q = 0; q < SIM_MOE_MAX_GROUPS / 16; q++)
            if ((int)i == q * 16 + l) v[q] = 0;
    }
    return keep;
}

// The choice by scores with a bias, from scores in 32 bits: as whole numbers of
// kBits bits above the experts' complemented indices, so that a search is
// maxima and nothing else.  It is the definition's where no two that it had to
// tell apart, of the groups or of the experts, are nearer to each other than
// their errors; sure says whether that is so.
template <int NV> struct Fast {
    static constexpr int kIndexBits = NV == 1 ? 4 : NV == 2 ? 5 : NV == 4 ? 6 : NV == 8 ? 7 : NV == 16 ? 8 : NV == 32 ? 9 : 10;
    static constexpr int kBits = kIndexBits < 8 ? 24 : 32 - kIndexBits;
    static constexpr uint32_t kIndex = (1u << kIndexBits) - 1;
    // In steps of 2^-24 of the range, how far a value may be from what the
    // definition compares: a sigmoid 4 (its exponent's argument, two results to
    // a unit in the last place, a sum), the definition's own two roundings 2,
    // the bias, the offset and the scale 6, and two whole steps of a conversion
    // beside; a softmax's sum of NV + 4 terms and its division as many more.
    // Two values that are further apart than twice that are in order.
    static constexpr uint32_t near(uint32_t steps) { return 2 * ((steps >> (24 - kBits)) + 3); }
    static constexpr uint32_t kNear = near(12), kNearSum = near(12 + NV + 8);
    uint32_t k[NV];
    uint32_t apart;  // kNear or kNearSum
    bool sure = true;

    __device__ uint32_t take() {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < NV; i++) m = max(m, k[i]);
        m = max16(m);
#pragma unroll
        for (int i = 0; i < NV; i++) k[i] = k[i] == m ? 0 : k[i];
        return m;
    }
    // groups as 64 times their value and, complemented, their index
    __device__ static uint32_t group_key(const Two &two, uint32_t zero, int best, uint32_t g) {
        const uint32_t v = (two.a >> kIndexBits) + (best == 1 ? 0 : two.b ? two.b >> kIndexBits : zero);
        return two.a ? v << 6 | (63 - g) : 0;
    }
    __device__ void keep_groups(int E, int groups, int top, int best, uint32_t zero) {
        const int l = threadIdx.x & 15, size = E / groups, lanes = size / NV;
        uint64_t keep = 0;
        uint32_t last = 0, next = 0;
        if (lanes * NV == size && (lanes & (lanes - 1)) == 0) {
            Two two;
#pragma unroll
            for (int i = 0; i < NV; i++) two.add(k[i]);
            if (lanes >= 2) two.merge<kDppXor1>();
            if (lanes >= 4) two.merge<kDppXor2>();
            if (lanes >= 8) two.merge<kDppHalfMirror>();
            if (lanes >= 16) two.merge<kDppMirror>();
            uint32_t v = group_key(two, zero, best, l / lanes);
            for (int j = 0; j <= top; j++) {
                const uint32_t m = max16(v);
                if (j < top) keep |= m ? 1ull << (63 - (m & 63)) : 0, last = m;
                else next = m;
                v = v == m ? 0 : v;
            }
            const bool kept = (keep >> (l / lanes)) & 1;
#pragma unroll
            for (int i = 0; i < NV; i++) k[i] = kept ? k[i] : 0;
        } else {
            uint32_t v[SIM_MOE_MAX_GROUPS / 16] = {};  // of groups l, l + 16, ...
            for (int g = 0; g < groups; g++) {
                Two two;
#pragma unroll
                for (int i = 0; i < NV; i++) two.add((uint32_t)(l * NV + i - g * size) < (uint32_t)size ? k[i] : 0);
                two.merge<kDppXor1>();
                two.merge<kDppXor2>();
                two.merge<kDppHalfMirror>();
                two.merge<kDppMirror>();
#pragma unroll
                for (int q = 0; q < SIM_MOE_MAX_GROUPS / 16; q++)
                    if (g == q * 16 + l) v[q] = group_key(two, zero, best, g);
            }
            for (int j = 0; j <= top; j++) {
                const uint32_t m = max16(max(max(v[0], v[1]), max(v[2], v[3])));
                if (j < top) keep |= m ? 1ull << (63 - (m & 63)) : 0, last = m;
                else next = m;
#pragma unroll
                for (int q = 0; q < SIM_MOE_MAX_GROUPS / 16; q++) v[q] = v[q] == m ? 0 : v[q];
            }
            int g = l * NV / size, in = l * NV - g * size;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                if (!((keep >> (g & 63)) & 1)) k[i] = 0;
                if (++in == size) in = 0, g++;
            }
        }
        sure = sure && (next == 0 || (last >> 6) - (next >> 6) > best * (apart + 4));  // (the definition's sum is rounded too)
    }
};

// Up to 16 experts, one in each of 16 lanes where had, in the order of their
// sigmoids with the bias, from 64 bits.
__device__ inline uint32_t rank_chosen(bool had, uint32_t e, double z, const float *__restrict__ bias) {
    const uint32_t key = had ? order_key((float)sigmoid64(z) + bias[e]) : 0;
    const int row = threadIdx.x & 48;
    int place = 0;
    for (int j = 0; j < 16; j++) {
        const uint32_t k2 = __shfl(key, row | j), e2 = __shfl(e, row | j);
        place += k2 > key || (k2 == key && (k2 ? e2 < e : j < (int)(threadIdx.x & 15)));
    }
    return (uint32_t)__builtin_amdgcn_ds_permute((row | place) << 2, (int)e);
}

// The choice by scores.  Which of two experts is higher must not depend on how
// a score was computed, so scores are those of 64 bits, rounded to 32, in which
// the bias and the groups' sums are added: what is compared is the definition's
// but where a 64-bit value lies within its own error of the middle between two
// 32-bit ones.  With a bias 32 bits are tried first, which suffice but for one
// token in a thousand (scores of 256 experts, k = 8).
//
// 32768 tokens, 256 bf16 experts in 8 groups, k = 8: 33 us (49 with all scores
// in 64 bits; 39 where a token whose choices are near to each other is done
// anew with these, so that one wave in seventy holds up its workgroup).
template <int T, int NV, int CH>
__global__ __launch_bounds__(16 * CH) void route_scored(RouteArgs a, int32_t *__restrict__ experts, float *__restrict__ weights,
                                                        uint8_t *__restrict__ hist, int32_t *__restrict__ offsets,
                                                        int32_t *__restrict__ order) {
    typedef typename Elem<T>::type El;
    __shared__ Lists lists;
    const int l = threadIdx.x & 15, tok = threadIdx.x >> 4, E = a.E, k = a.k;
    const int64_t t = (int64_t)blockIdx.x * CH + tok;
    const bool live = t < a.T, grouped = a.groups > a.top_groups, sigmoid = a.score == SIM_SCORE_SIGMOID;
    const El *const z = (const El *)a.logits + (live ? t : 0) * a.stride;
    const uint8_t *const mask = a.mask ? a.mask + (live ? t : 0) * a.mask_stride : nullptr;
    clear<CH>(lists);
    float x[NV];  // -infinity where nothing can be chosen
    {
        El v[NV];
        const uint64_t ok = load_logits<T, NV>(z, mask, E, live, v);
#pragma unroll
        for (int i = 0; i < NV; i++) x[i] = (ok >> i) & 1 ? Elem<T>::get(v[i]) : -INFINITY;
    }

    uint32_t mine[2] = {0, 0}, mine_e[2] = {0, 0};  // the choices l and l + 16
    bool sure = false;
    if (a.bias) {
        Fast<NV> fast;
        float b[NV], most = 0.f, all = 0.f, high = 1.f, top = -INFINITY, inv = 1.f;
        if (l * NV + NV <= E) load_some<NV>(a.bias + l * NV, b);
        else
#pragma unroll
            for (int i = 0; i < NV; i++) b[i] = a.bias[min(l * NV + i, E - 1)];
#pragma unroll
        for (int i = 0; i < NV; i++) {
            most = fmaxf(most, fabsf(b[i]));
            top = fmaxf(top, x[i]);
        }
        most = __uint_as_float(max16(__float_as_uint(most)));
        if (!sigmoid) {
            top = fmaxf(top, dpp_f32<kDppXor1>(top));
            top = fmaxf(top, dpp_f32<kDppXor2>(top));
            top = fmaxf(top, dpp_f32<kDppHalfMirror>(top));
            top = fmaxf(top, dpp_f32<kDppMirror>(top));
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < NV; i++) sum += x[i] == -INFINITY ? 0.f : fast_exp(x[i] - top);
            high = inv = 1.f / sum16(sum);
        }
        const float scale = (float)((1 << Fast<NV>::kBits) - 16) / (high + 2.f * most);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const float c = sigmoid ? __builtin_amdgcn_rcpf(1.f + fast_exp(-x[i])) + b[i] : fast_exp(x[i] - top) * inv + b[i];
            const uint32_t key = ((uint32_t)((c + most) * scale) + 1) << Fast<NV>::kIndexBits | (Fast<NV>::kIndex - (l * NV + i));
            all += x[i] == -INFINITY ? 0.f : c;
            fast.k[i] = x[i] == -INFINITY ? 0 : key;
        }
        all = sum16(all);
        fast.apart = sigmoid ? Fast<NV>::kNear : Fast<NV>::kNearSum;
        // nothing is infinite or NaN (most past 2^64 is left to the other way too)
        fast.sure = fabsf(all) < 1.8446744e19f && most < 1.8446744e19f;
        if (grouped) fast.keep_groups(E, a.groups, a.top_groups, a.group_best, (uint32_t)(most * scale) + 1);
        // two more than are wanted: who of those that are near is higher is a
        // question of few then, unless the last is near the last wanted too
        const bool ranked = sigmoid && k <= 14;
        const int n = ranked ? k + 2 : k + 1;
        bool near = false;
        uint32_t before = 0, wanted = 0;
        for (int j = 0; j < n; j++) {
            const uint32_t m = fast.take(), gap = (before >> Fast<NV>::kIndexBits) - (m >> Fast<NV>::kIndexBits);
            near |= j && m && gap <= fast.apart;
            before = m;
            if (j == k - 1) wanted = m;
            if ((j < k || ranked) && l == (j & 15)) {  // (of 32 and one more the last has no place)
                mine[j >> 4] = m;
                mine_e[j >> 4] = Fast<NV>::kIndex - (m & Fast<NV>::kIndex);
            }
        }
        if (!ranked) {
            fast.sure = fast.sure && !near;
        } else {
            if (before && (wanted >> Fast<NV>::kIndexBits) - (before >> Fast<NV>::kIndexBits) <= fast.apart) fast.sure = false;
            if (__ballot(near && live)) mine_e[0] = rank_chosen(mine[0] != 0, mine_e[0], mine[0] ? (double)Elem<T>::get(z[mine_e[0]]) : 0., a.bias);
            if (l >= k) mine[0] = 0;
        }
        sure = fast.sure || !live;
    }
    if (__ballot(!sure)) {
        Keys<SIM_TYPE_F32, NV> key;
        uint32_t top = 0;  // the highest of the allowed logits
#pragma unroll
        for (int i = 0; i < NV; i++) {
            key.k[i] = order_key(x[i]);
            top = max(top, key.k[i]);
        }
        const bool by_score = a.bias || (grouped && a.group_best == 2);
        if (by_score) {
            double high = 0., inv = 0.;
            if (!sigmoid) {
                high = key_value(max16(top));
                double sum = 0.;
#pragma unroll
                for (int i = 0; i < NV; i++) sum += x[i] == -INFINITY ? 0. : exp64(x[i] - high);
                inv = 1. / sum16(sum);
            }
#pragma unroll
            for (int i = 0; i < NV; i++) {
                const float s = (float)(sigmoid ? sigmoid64(x[i]) : exp64(x[i] - high) * inv);
                key.k[i] = x[i] == -INFINITY ? 0 : order_key(a.bias ? s + a.bias[min(l * NV + i, E - 1)] : s);
            }
        }
        if (grouped) {
            const uint64_t keep = top_groups<NV>(key.k, E, a.groups, a.top_groups, a.group_best);
            const int size = E / a.groups;
            int g = l * NV / size, in = l * NV - g * size;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                // without a bias the logits have the scores' order, and a finer one
                if (by_score && !a.bias && key.k[i]) key.k[i] = order_key(x[i]);
                if (!((keep >> (g & 63)) & 1)) key.k[i] = 0;
                if (++in == size) in = 0, g++;
            }
        }
        for (int j = 0; j < k; j++) {
            uint32_t e;
            const uint32_t m = key.take(e);
            if (l == (j & 15)) {
                mine[j >> 4] = m;
                mine_e[j >> 4] = e;
            }
        }
    }
    // the weights from the chosen logits again, relative to the highest chosen
    // one where they are divided by their sum
    const int rows = k > 16 ? 2 : 1;
    double high = 0., inv = 0., chosen[2] = {0., 0.}, w64[2] = {0., 0.};
    uint32_t first = 0;
#pragma unroll
    for (int q = 0; q < 2; q++)
        if (q < rows) {
            chosen[q] = mine[q] ? (double)Elem<T>::get(z[mine_e[q]]) : 0.;
            first = max(first, mine[q] ? order_key((float)chosen[q]) : 0u);
        }
    if (a.renorm) {
        high = key_value(max16(first));
        if (sigmoid && high > 0.) high = 0.;
    } else if (!sigmoid) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < NV; i++) top = max(top, order_key(x[i]));
        high = key_value(max16(top));
        double sum = 0.;
#pragma unroll
        for (int i = 0; i < NV; i++) sum += x[i] == -INFINITY ? 0. : exp64(x[i] - high);
        inv = 1. / sum16(sum);
    }
#pragma unroll
    for (int q = 0; q < 2; q++)
        if (q < rows) {
            if (!sigmoid) w64[q] = exp64(chosen[q] - high);
            else if (a.renorm) w64[q] = exp64((chosen[q] > 0. ? 0. : chosen[q]) - high) * reciprocal(1. + exp64(-__builtin_fabs(chosen[q])));
            else w64[q] = sigmoid64(chosen[q]);
            if (!mine[q]) w64[q] = 0.;
        }
    if (a.renorm) inv = 1. / sum16(w64[0] + w64[1]);
    else if (sigmoid) inv = 1.;
    float w[2];
#pragma unroll
    for (int q = 0; q < 2; q++) w[q] = (float)(w64[q] * inv * a.scale);
    __syncthreads();  // the lists are clear
    finish<CH>(lists, t, live, k, E, (int)min(a.T, (int64_t)CH), mine_e, mine, w, experts, weights, hist, offsets, order);
}

// The same for a decode step's few tokens, where one wave's chain of operations
// is all of the time: a wave for a token, so that a lane has a quarter of the
// experts, and scores in 64 bits at once (256 fp32 experts in 8 groups, k = 8:
// one token 6.8 us, 15.7 by route_scored; 16 tokens 10.3 and 14.8).
constexpr int kRouteFew = 16;

__device__ inline uint32_t max64(uint32_t v) {
    v = max16(v);
    const auto row = [&](int r) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 16 * r); };
    return max(max(row(0), row(1)), max(row(2), row(3)));
}
__device__ inline double sum64(double v) {
    v = sum16(v);
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const auto row = [&](int r) {
        return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)b, 16 * r) |
                                              (uint64_t)__builtin_amdgcn_readlane((int)(b >> 32), 16 * r) << 32);
    };
    return (row(0) + row(1)) + (row(2) + row(3));
}

template <int T, int NV>
__global__ __launch_bounds__(64 * kRouteFew) void route_few(RouteArgs a, int32_t *__restrict__ experts, float *__restrict__ weights,
                                                           int32_t *__restrict__ offsets, int32_t *__restrict__ order) {
    typedef typename Elem<T>::type El;
    static_assert(64 * kRouteFew == kThreads, "a thread for each expert");
    __shared__ Lists lists;
    const int l = threadIdx.x & 63, t = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), E = a.E, k = a.k, e0 = l * NV;
    const bool live = t < a.T, grouped = a.groups > a.top_groups, sigmoid = a.score == SIM_SCORE_SIGMOID;
    clear<kChunk>(lists);
    __syncthreads();
    int mine = -1;
    if (live) {
        const El *const z = (const El *)a.logits + t * a.stride;
        const uint8_t *const mask = a.mask ? a.mask + t * a.mask_stride : nullptr;
        El raw[NV];
        uint8_t m[NV];
        if (e0 + NV <= E) {
            load_some<NV>(z + e0, raw);
            if (mask) load_some<NV>(mask + e0, m);
        } else {
#pragma unroll
            for (int i = 0; i < NV; i++) {
                raw[i] = e0 + i < E ? z[e0 + i] : Elem<T>::put(-INFINITY);
                m[i] = mask && e0 + i < E ? mask[e0 + i] : 0;
            }
        }
        float x[NV];  // -infinity where nothing can be chosen
        uint32_t key[NV], top = 0;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            x[i] = e0 + i < E && (!mask || m[i]) ? Elem<T>::get(raw[i]) : -INFINITY;
            key[i] = order_key(x[i]);
            top = max(top, key[i]);
        }
        const bool by_score = a.bias || (grouped && a.group_best == 2);
        double high = 0., inv = 1.;
        if (!sigmoid && (by_score || !a.renorm)) {
            high = key_value(max64(top));
            double sum = 0.;
#pragma unroll
            for (int i = 0; i < NV; i++) sum += x[i] == -INFINITY ? 0. : exp64(x[i] - high);
            inv = 1. / sum64(sum);
        }
        if (by_score) {
#pragma unroll
            for (int i = 0; i < NV; i++) {
                const float s = (float)(sigmoid ? sigmoid64(x[i]) : exp64(x[i] - high) * inv);
                key[i] = x[i] == -INFINITY ? 0 : order_key(a.bias ? s + a.bias[min(e0 + i, E - 1)] : s);
            }
        }
        if (grouped) {
            // a group's value in one lane each: its first where it is a whole
            // number of lanes, a power of two up to 16, else lane g
            const int size = E / a.groups, lanes = size / NV;
            const bool whole = lanes * NV == size && (lanes & (lanes - 1)) == 0 && lanes <= 16;
            uint32_t v = 0;
            if (whole) {
                Two two;
#pragma unroll
                for (int i = 0; i < NV; i++) two.add(key[i]);
                if (lanes >= 2) two.merge<kDppXor1>();
                if (lanes >= 4) two.merge<kDppXor2>();
                if (lanes >= 8) two.merge<kDppHalfMirror>();
                if (lanes >= 16) two.merge<kDppMirror>();
                v = l % lanes ? 0 : two.value(a.group_best);
            }
            for (int g = whole ? a.groups : 0; g < a.groups; g++) {
                Two two;
#pragma unroll
                for (int i = 0; i < NV; i++) two.add((uint32_t)(e0 + i - g * size) < (uint32_t)size ? key[i] : 0);
                two.merge<kDppXor1>();
                two.merge<kDppXor2>();
                two.merge<kDppHalfMirror>();
                two.merge<kDppMirror>();
                Two all;
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    all.add((uint32_t)__builtin_amdgcn_readlane((int)two.a, 16 * r));
                    all.add((uint32_t)__builtin_amdgcn_readlane((int)two.b, 16 * r));
                }
                if (l == g) v = all.value(a.group_best);
            }
            uint64_t keep = 0;
            for (int j = 0; j < a.top_groups; j++) {
                const uint32_t best = max64(v);
                if (!best) break;
                const int from = __ffsll((unsigned long long)__ballot(v == best)) - 1;
                keep |= 1ull << (whole ? from / lanes : from);
                v = l == from ? 0 : v;
            }
            int g = e0 / size, in = e0 - g * size;
#pragma unroll
            for (int i = 0; i < NV; i++) {
                // without a bias the logits have the scores' order, and a finer one
                if (by_score && !a.bias && key[i]) key[i] = order_key(x[i]);
                if (!((keep >> (g & 63)) & 1)) key[i] = 0;
                if (++in == size) in = 0, g++;
            }
        }
        for (int j = 0; j < k; j++) {
            uint32_t best = 0;
            int at = 0;  // the first of equal ones has the lowest index, in the lane and among the lanes
#pragma unroll
            for (int i = 0; i < NV; i++) {
                at = key[i] > best ? i : at;
                best = max(best, key[i]);
            }
            const uint32_t all = max64(best);
            if (!all) break;
            const int from = __ffsll((unsigned long long)__ballot(best == all)) - 1, e = from * NV + __builtin_amdgcn_readlane(at, from);
            mine = l == j ? e : mine;
#pragma unroll
            for (int i = 0; i < NV; i++) key[i] = e0 + i == e ? 0 : key[i];
        }
        // the weights, as in route_scored
        const double chosen = mine >= 0 ? (double)Elem<T>::get(z[mine]) : 0.;
        if (a.renorm) {
            high = key_value(max64(mine >= 0 ? order_key((float)chosen) : 0u));
            if (sigmoid && high > 0.) high = 0.;
        }
        double w;
        if (!sigmoid) w = exp64(chosen - high);
        else if (a.renorm) w = exp64((chosen > 0. ? 0. : chosen) - high) * reciprocal(1. + exp64(-__builtin_fabs(chosen)));
        else w = sigmoid64(chosen);
        w = mine >= 0 ? w : 0.;
        if (a.renorm) inv = 1. / sum64(w);
        if (l < k) {
            experts[t * k + l] = mine;
            weights[t * k + l] = mine >= 0 ? (float)(w * inv * a.scale) : 0.f;
            if (mine >= 0 && order) mark(lists.chose, mine, t);
        }
    }
    if (!order) return;
    __syncthreads();
    int total;
    lists.base[threadIdx.x] = block_scan(__popcll(lists.chose[threadIdx.x]), lists.wave_sum, total);
    if ((int)threadIdx.x < E) offsets[threadIdx.x] = lists.base[threadIdx.x];
    if (threadIdx.x == 0) offsets[E] = total;
    __syncthreads();
    if (mine >= 0) order[lists.base[mine] + before_in(lists.chose[mine], t)] = t * k + l;
    for (int i = total + threadIdx.x; i < (int)a.T * k; i += kThreads) order[i] = -1;
}

// Gradient of sigmoid weights: at the chosen experts only, so it writes and reads
// few of them.  As in route_grad, lane l has the choices l and l + 16 (32768
// tokens, 256 bf16 experts, k = 8: 8.5 us for 19 MB).
template <int T, int NV>
__global__ __launch_bounds__(256) void route_grad_sigmoid(RouteArgs a, const int32_t *__restrict__ experts,
                                                          const float *__restrict__ dw, typename Elem<T>::type *__restrict__ dz) {
    typedef typename Elem<T>::type El;
    __shared__ __align__(16) float rows[16][NV * 16];
    const int l = threadIdx.x & 15, E = a.E, k = a.k;
    const int64_t t = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (t >= a.T) return;  // sixteen lanes at a time: they share no barrier
    float *row = rows[threadIdx.x >> 4];
    const El *zt = (const El *)a.logits + t * a.stride;
    const uint8_t *mt = a.mask ? a.mask + t * a.mask_stride : nullptr;
    int e[2];
    float g[2], z[2], w[2];
    uint32_t top = 0;
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const int j = q * 16 + l;
        e[q] = j < k ? experts[t * k + j] : -1;
        if (e[q] < 0 || e[q] >= E || (mt && !mt[e[q]])) e[q] = -1;
        z[q] = e[q] >= 0 ? Elem<T>::get(zt[e[q]]) : 0.f;
        if (z[q] == -INFINITY) e[q] = -1;
        g[q] = e[q] >= 0 ? dw[t * k + j] * a.scale : 0.f;
        top = max(top, e[q] >= 0 ? order_key(z[q]) : 0u);
    }
#pragma unroll
    for (int i = 0; i < NV; i++) row[i * 16 + l] = 0.f;
    float high = 0.f, dot = 0.f, inv = 1.f;
    if (a.renorm) {
        high = key_value(max16(top));
        high = high > 0.f ? 0.f : high;
    }
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const float s = fast_exp((z[q] > 0.f ? 0.f : z[q]) - high) / (1.f + fast_exp(-fabsf(z[q])));  // times e^-high
        w[q] = e[q] >= 0 ? s : 0.f;
    }
    if (a.renorm) {
        inv = 1.f / sum16(w[0] + w[1]);
        dot = sum16((e[0] >= 0 ? g[0] * w[0] : 0.f) + (e[1] >= 0 ? g[1] * w[1] : 0.f)) * inv;
    }
    wave_fence();  // the zeros are other lanes' than the values, and both than what is read
#pragma unroll
    for (int q = 0; q < 2; q++)
        if (e[q] >= 0) {
            const float far = fast_exp(-fabsf(z[q])), rest = (z[q] < 0.f ? 1.f : far) / (1.f + far);  // 1 - s
            row[e[q]] = w[q] * inv * (g[q] - dot) * rest;
        }
    wave_fence();
    El out[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) out[i] = Elem<T>::put(row[l * NV + i]);
    El *o = dz + t * E + l * NV;
    if (l * NV + NV <= E) store_some<NV>(o, out);
    else
#pragma unroll
        for (int i = 0; i < NV; i++)
            if (l * NV + i < E) o[i] = out[i];
}

// Calls f with the smallest register count that holds E experts in 16 lanes.
template <typename F> void with_nv(int E, F &&f) {
    if (E <= 16) f(std::integral_constant<int, 1>());
    else if (E <= 32) f(std::integral_constant<int, 2>());
    else if (E <= 64) f(std::integral_constant<int, 4>());
    else if (E <= 128) f(std::integral_constant<int, 8>());
    else if (E <= 256) f(std::integral_constant<int, 16>());
    else if (E <= 512) f(std::integral_constant<int, 32>());
    else f(std::integral_constant<int, 64>());
}

// How many groups of tokens are counted by themselves: those of kPart tokens
// while these do not yet fill the GPU (119 tokens, k = 8 of 457: 16 us, 24 in
// groups of 64; 1000, k = 8 of 256: 10.1 and 12.0), but one of 64 where no
// second launch is needed and the search (registers times k) is not long (64
// tokens of 512 fp32 experts: 19 and 13.7 us with k = 8, 14 and 11 with k = 4;
// bf16: 12.6 and 11.5, 10.2 and 10.3).
inline uint32_t count_rows(int64_t T, int E, int k) {
    const bool parts = T > kPart && T <= kPart * 256 && (T > kChunk || (E > 256 && k > 4));
    const int64_t n = parts ? kPart : kChunk;
    return (uint32_t)((T + n - 1) / n);
}

// Whether the counts are scanned by a kernel of their own: where each workgroup
// that places would read more than 64 KB of them (20000 tokens of 256 experts,
// k = 8: 22.2 us, 23.9 by themselves; 12000: 16.6 and 14.9; of 1000 37 and 40), or
// there are many workgroups to read them.  (Never where parts are counted: at most
// 64 chunks, 64 KB of 1024 experts.)
inline bool scanned(size_t chunks, int E) { return chunks > 384 || chunks * (size_t)hist_pitch(E) > 65536; }

inline size_t hist_bytes(size_t chunks, int E) { return (chunks * hist_pitch(E) + 15) / 16 * 16; }

template <int T>
sim_status route_t(hipStream_t st, const RouteArgs &a, int32_t *experts, float *weights, int32_t *offsets, int32_t *order,
                   void *ws) {
    const uint32_t chunks = (uint32_t)((a.T + kChunk - 1) / kChunk), rows = count_rows(a.T, a.E, a.k);
    uint8_t *hist = (uint8_t *)ws;
    int32_t *sums = scanned(chunks, a.E) ? (int32_t *)(hist + hist_bytes(rows, a.E)) : nullptr;
    const auto choose = [&](auto nv, auto ch) {
        constexpr int CH = decltype(ch)::value;
        if (a.scored) {
            route_scored<T, decltype(nv)::value, CH><<<(uint32_t)((a.T + CH - 1) / CH), 16 * CH, 0, st>>>(a, experts, weights, hist, offsets, order);
            return;
        }
        route_choose<T, decltype(nv)::value, CH><<<(uint32_t)((a.T + CH - 1) / CH), 16 * CH, 0, st>>>(
            (const typename Elem<T>::type *)a.logits, a.T, a.E, a.stride, a.mask, a.mask_stride, a.k, a.renorm, experts,
            weights, hist, offsets, order);
    };
    if (a.scored && a.T <= kRouteFew) {
        const auto few = [&](auto nv) {
            route_few<T, decltype(nv)::value><<<1, 64 * kRouteFew, 0, st>>>(a, experts, weights, offsets, order);
        };
        if (a.E <= 64) few(std::integral_constant<int, 1>());
        else if (a.E <= 128) few(std::integral_constant<int, 2>());
        else if (a.E <= 256) few(std::integral_constant<int, 4>());
        else if (a.E <= 512) few(std::integral_constant<int, 8>());
        else few(std::integral_constant<int, 16>());
        return SIM_OPS_LAUNCH_OK();
    }
    if (a.given) {
        if (rows > chunks) route_given<kPart><<<rows, 16 * kPart, 0, st>>>(a, experts, weights, hist, offsets, order);
        else route_given<kChunk><<<chunks, kThreads, 0, st>>>(a, experts, weights, hist, offsets, order);
    } else {
        with_nv(a.E, [&](auto nv) {
            if (rows > chunks) choose(nv, std::integral_constant<int, kPart>());
            else choose(nv, std::integral_constant<int, kChunk>());
        });
    }
    if (order && rows > 1) {
        if (sums) route_scan<<<(a.E + 15) / 16, kThreads, 0, st>>>(hist, sums, (int)chunks, a.E);
        route_place<<<chunks, kThreads, 0, st>>>(experts, a.T, a.E, a.k, hist, rows > chunks ? kChunk / kPart : 1, (int)rows, sums,
                                                 offsets, order);
    }
    return SIM_OPS_LAUNCH_OK();
}

template <int T>
sim_status route_grad_t(hipStream_t st, const RouteArgs &a, const int32_t *experts, const float *dw, void *dz) {
    with_nv(a.E, [&](auto nv) {
        const uint32_t grid = (uint32_t)((a.T + 15) / 16);
        if (a.score == SIM_SCORE_SIGMOID)
            route_grad_sigmoid<T, decltype(nv)::value><<<grid, 256, 0, st>>>(a, experts, dw, (typename Elem<T>::type *)dz);
        else
            route_grad<T, decltype(nv)::value><<<grid, 256, 0, st>>>(
                (const typename Elem<T>::type *)a.logits, a.T, a.E, a.stride, a.mask, a.mask_stride, a.k, a.renorm, a.scale, experts,
                dw, (typename Elem<T>::type *)dz);
    });
    return SIM_OPS_LAUNCH_OK();
}

__global__ void no_tokens(int32_t *offsets, int E) {
    for (int e = threadIdx.x; e <= E; e += blockDim.x) offsets[e] = 0;
}

}  // namespace

size_t route_workspace(int64_t T, int E, int k) {
    const size_t rows = count_rows(T, E, k), chunks = (size_t)((T + kChunk - 1) / kChunk);
    if (rows <= 1) return 0;
    return hist_bytes(rows, E) + (scanned(chunks, E) ? (chunks + 1) * (size_t)E * sizeof(int32_t) : 0);
}

sim_status launch_route(hipStream_t st, const RouteArgs &a, int32_t *experts, float *weights, int32_t *offsets,
                        int32_t *order, void *ws) {
    if (a.T == 0) {
        if (offsets) no_tokens<<<1, 256, 0, st>>>(offsets, a.E);
        return SIM_OPS_LAUNCH_OK();
    }
    if (a.type == SIM_TYPE_F32) return route_t<SIM_TYPE_F32>(st, a, experts, weights, offsets, order, ws);
    if (a.type == SIM_TYPE_F16) return route_t<SIM_TYPE_F16>(st, a, experts, weights, offsets, order, ws);
    return route_t<SIM_TYPE_BF16>(st, a, experts, weights, offsets, order, ws);
}

sim_status launch_route_grad(hipStream_t st, const RouteArgs &a, const int32_t *experts, const float *dw, void *dz) {
    if (a.T == 0) return SIM_OK;
    if (a.type == SIM_TYPE_F32) return route_grad_t<SIM_TYPE_F32>(st, a, experts, dw, dz);
    if (a.type == SIM_TYPE_F16) return route_grad_t<SIM_TYPE_F16>(st, a, experts, dw, dz);
    return route_grad_t<SIM_TYPE_BF16>(st, a, experts, dw, dz);
}

}  // namespace simops
