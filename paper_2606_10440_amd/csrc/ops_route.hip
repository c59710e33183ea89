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
#include "ops_route_keys.h"

namespace simops {
namespace {

constexpr int kChunk = 64;           // tokens of one workgroup
constexpr int kThreads = 16 * kChunk;
constexpr int kPart = 16;            // tokens of one where there are few
constexpr int kScanChunks = 512;     // above it, counts are scanned by a kernel of their own

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

// Choice and weights of CH tokens; their counts, or (one chunk only) the lists.
template <int T, int NV, int CH>
__global__ __launch_bounds__(16 * CH) void route_choose(const typename Elem<T>::type *__restrict__ logits, int64_t n_tok,
                                                         int E, int64_t stride, const uint8_t *__restrict__ mask,
                                                         int64_t mask_stride, int k, int renorm,
                                                         int32_t *__restrict__ experts, float *__restrict__ weights,
                                                         uint8_t *__restrict__ hist, int32_t *__restrict__ offsets,
                                                         int32_t *__restrict__ order) {
    __shared__ uint64_t chose[SIM_MOE_MAX_EXPERTS];
    __shared__ int base[SIM_MOE_MAX_EXPERTS];
    __shared__ int wave_sum[kThreads / 64];
    const int l = threadIdx.x & 15, tok = threadIdx.x >> 4;
    const int64_t t = (int64_t)blockIdx.x * CH + tok;
    const bool live = t < n_tok;
    for (int e = threadIdx.x; e < SIM_MOE_MAX_EXPERTS; e += 16 * CH) chose[e] = 0;
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
    for (int q = 0; q < 2; q++) {
        const int j = q * 16 + l;
        if (live && j < k) {
            experts[t * k + j] = mine[q] ? (int)mine_e[q] : -1;
            weights[t * k + j] = mine[q] ? w[q] / z : 0.f;
            if (mine[q] && order) mark(chose, mine_e[q], tok);
        }
    }
    if (!order) return;
    __syncthreads();
    if (CH < kChunk || gridDim.x > 1) {
        // at most kChunk: a byte
        for (int e = threadIdx.x; e < hist_pitch(E); e += 16 * CH)
            hist[(int64_t)blockIdx.x * hist_pitch(E) + e] = (uint8_t)__popcll(chose[e]);
        return;
    }
    int total;
    base[threadIdx.x] = block_scan(__popcll(chose[threadIdx.x]), wave_sum, total);
    if ((int)threadIdx.x < E) offsets[threadIdx.x] = base[threadIdx.x];
    if (threadIdx.x == 0) offsets[E] = total;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; q++)
        if (live && mine[q]) order[base[mine_e[q]] + before_in(chose[mine_e[q]], tok)] = tok * k + q * 16 + l;
    for (int s = total + threadIdx.x; s < (int)n_tok * k; s += kThreads) order[s] = -1;
}

// The sums over the chunks before each; the row past the last gets the totals.
__global__ __launch_bounds__(kThreads) void route_scan(const uint8_t *__restrict__ hist, int32_t *__restrict__ sums, int chunks,
                                                       int E) {
    __shared__ int part_sum[64][16];
    const int e = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4, pitch = hist_pitch(E);
    const int per = (chunks + 63) / 64, c0 = part * per, c1 = min(chunks, c0 + per);
    int s = 0;
    if (e < E)
        for (int c = c0; c < c1; c++) s += hist[(int64_t)c * pitch + e];
    part_sum[part][threadIdx.x & 15] = s;
    __syncthreads();
    if (e >= E) return;
    int before = 0, total = 0;
    for (int p = 0; p < 64; p++) {
        const int v = part_sum[p][threadIdx.x & 15];
        if (p < part) before += v;
        total += v;
    }
    for (int c = c0; c < c1; c++) {
        sums[(int64_t)c * E + e] = before;
        before += hist[(int64_t)c * pitch + e];
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
                                                  int k, int renorm, const int32_t *__restrict__ experts,
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
        g[q] = e[q] >= 0 ? dw[t * k + j] : 0.f;
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

inline size_t hist_bytes(size_t chunks, int E) { return (chunks * hist_pitch(E) + 15) / 16 * 16; }

template <int T>
sim_status route_t(hipStream_t st, const RouteArgs &a, int32_t *experts, float *weights, int32_t *offsets, int32_t *order,
                   void *ws) {
    const uint32_t chunks = (uint32_t)((a.T + kChunk - 1) / kChunk), rows = count_rows(a.T, a.E, a.k);
    uint8_t *hist = (uint8_t *)ws;
    int32_t *sums = chunks > kScanChunks ? (int32_t *)(hist + hist_bytes(rows, a.E)) : nullptr;
    const auto choose = [&](auto nv, auto ch) {
        constexpr int CH = decltype(ch)::value;
        route_choose<T, decltype(nv)::value, CH><<<(uint32_t)((a.T + CH - 1) / CH), 16 * CH, 0, st>>>(
            (const typename Elem<T>::type *)a.logits, a.T, a.E, a.stride, a.mask, a.mask_stride, a.k, a.renorm, experts,
            weights, hist, offsets, order);
    };
    with_nv(a.E, [&](auto nv) {
        if (rows > chunks) choose(nv, std::integral_constant<int, kPart>());
        else choose(nv, std::integral_constant<int, kChunk>());
    });
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
        route_grad<T, decltype(nv)::value><<<(uint32_t)((a.T + 15) / 16), 256, 0, st>>>(
            (const typename Elem<T>::type *)a.logits, a.T, a.E, a.stride, a.mask, a.mask_stride, a.k, a.renorm, experts, dw,
            (typename Elem<T>::type *)dz);
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
    return hist_bytes(rows, E) + (chunks > kScanChunks ? (chunks + 1) * (size_t)E * sizeof(int32_t) : 0);
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
