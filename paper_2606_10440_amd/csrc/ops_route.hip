// Router: the k highest of each token's logits, their softmax weights, the
// tokens' lists by expert, and the gradient.
//
// Sixteen lanes hold a token's logits in registers (NV each), so that a wave
// runs four tokens at once and every exchange stays within a row of 16 lanes.
// A logit is compared as a whole number that orders as the value does, NaN
// highest, 0 for what cannot be chosen (masked, -infinity, past E).
#include "ops_route_keys.h"

namespace simops {
namespace {

constexpr int kChunk = 64;           // tokens of one workgroup
constexpr int kThreads = 16 * kChunk;
constexpr int kScanChunks = 512;     // above it, counts are scanned by a kernel of their own

// A token's keys: lane l of 16 holds experts 16 i + l.
template <int T, int NV>
__device__ inline void load_keys(const typename Elem<T>::type *__restrict__ z, const uint8_t *__restrict__ mask, int E,
                                 bool live, uint32_t key[NV]) {
    const int l = threadIdx.x & 15;
    typename Elem<T>::type v[NV];
    uint8_t ok[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int e = i * 16 + l;
        const bool in = live && e < E;
        v[i] = in ? z[e] : Elem<T>::put(0.f);
        ok[i] = in ? (mask ? mask[e] : 1) : 0;
    }
#pragma unroll
    for (int i = 0; i < NV; i++) key[i] = ok[i] ? order_key(Elem<T>::get(v[i])) : 0;
}

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

// Slots of one chunk to their places: base[e] = place of its first slot of
// expert e.  A wave takes one expert after another and looks 64 slots over at
// a time, so that equal experts stay in slot order.
__device__ inline void place_slots(const int16_t *slot_expert, int n, int first_slot, const int *count, const int *base,
                                   int E, int32_t *__restrict__ order) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int e = wave; e < E; e += kThreads / 64) {
        if (!count[e]) continue;
        int at = base[e];
        for (int s = 0; s < n; s += 64) {
            const bool mine = s + lane < n && slot_expert[s + lane] == e;
            const uint64_t all = __ballot(mine);
            if (mine) order[at + __popcll(all & ((1ull << lane) - 1))] = first_slot + s + lane;
            at += __popcll(all);
        }
    }
}

// Choice and weights; counts of the chunk, or (one chunk only) the lists.
template <int T, int NV>
__global__ __launch_bounds__(kThreads) void route_choose(const typename Elem<T>::type *__restrict__ logits, int64_t n_tok,
                                                         int E, int64_t stride, const uint8_t *__restrict__ mask,
                                                         int64_t mask_stride, int k, int renorm,
                                                         int32_t *__restrict__ experts, float *__restrict__ weights,
                                                         int32_t *__restrict__ hist, int32_t *__restrict__ offsets,
                                                         int32_t *__restrict__ order) {
    __shared__ int count[SIM_MOE_MAX_EXPERTS];
    __shared__ int base[SIM_MOE_MAX_EXPERTS];
    __shared__ int wave_sum[kThreads / 64];
    __shared__ int16_t slot_expert[kChunk * SIM_MOE_MAX_TOPK];
    const int l = threadIdx.x & 15, tok = threadIdx.x >> 4;
    const int64_t t0 = (int64_t)blockIdx.x * kChunk, t = t0 + tok;
    const bool live = t < n_tok;
    count[threadIdx.x] = 0;
    uint32_t key[NV];
    load_keys<T, NV>(logits + (live ? t : 0) * stride, mask ? mask + (live ? t : 0) * mask_stride : nullptr, E, live, key);
    __syncthreads();

    uint32_t mine[2] = {0, 0}, mine_e[2] = {0, 0};  // the choices l and l + 16
    float top = 0.f, z = 0.f;
    for (int j = 0; j < k; j++) {
        uint32_t bk = 0, bi = 0xffffu;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const bool take = key[i] > bk;  // the first of equal ones has the lowest index
            bk = take ? key[i] : bk;
            bi = take ? (uint32_t)(i * 16 + l) : bi;
        }
        best16(bk, bi);
        if (j == 0) {
            top = key_value(bk);
#pragma unroll
            for (int i = 0; i < NV; i++) z += key[i] ? expf(key_value(key[i]) - top) : 0.f;
            z = sum16(z);
        }
#pragma unroll
        for (int i = 0; i < NV; i++)
            if ((uint32_t)(i * 16 + l) == bi) key[i] = 0;
        if (l == (j & 15)) {
            mine[j >> 4] = bk;
            mine_e[j >> 4] = bi;
        }
    }
    float w[2];
#pragma unroll
    for (int q = 0; q < 2; q++) w[q] = mine[q] ? expf(key_value(mine[q]) - top) : 0.f;
    const float chosen = sum16(w[0] + w[1]);
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const int j = q * 16 + l;
        if (live && j < k) {
            const int e = mine[q] ? (int)mine_e[q] : -1;
            experts[t * k + j] = e;
            weights[t * k + j] = mine[q] ? w[q] / (renorm ? chosen : z) : 0.f;
            slot_expert[tok * k + j] = (int16_t)e;
            if (e >= 0) atomicAdd(&count[e], 1);
        }
    }
    if (!order) return;
    __syncthreads();
    if (gridDim.x > 1) {
        if ((int)threadIdx.x < E) hist[(int64_t)blockIdx.x * E + threadIdx.x] = count[threadIdx.x];
        return;
    }
    int total;
    const int mine_base = block_scan(count[threadIdx.x], wave_sum, total);
    base[threadIdx.x] = mine_base;
    if ((int)threadIdx.x < E) offsets[threadIdx.x] = mine_base;
    if (threadIdx.x == 0) offsets[E] = total;
    __syncthreads();
    const int n = (int)n_tok * k;
    place_slots(slot_expert, n, 0, count, base, E, order);
    for (int s = total + threadIdx.x; s < n; s += kThreads) order[s] = -1;
}

// Counts of each chunk to the sums over the chunks before it; the row past
// the last gets the totals.
__global__ __launch_bounds__(kThreads) void route_scan(int32_t *__restrict__ hist, int chunks, int E) {
    __shared__ int part_sum[64][16];
    const int e = blockIdx.x * 16 + (threadIdx.x & 15), part = threadIdx.x >> 4;
    const int per = (chunks + 63) / 64, c0 = part * per, c1 = min(chunks, c0 + per);
    int s = 0;
    if (e < E)
        for (int c = c0; c < c1; c++) s += hist[(int64_t)c * E + e];
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
        const int v = hist[(int64_t)c * E + e];
        hist[(int64_t)c * E + e] = before;
        before += v;
    }
    if (part == 0) hist[(int64_t)chunks * E + e] = total;
}

// Lists of one chunk, from the counts of all (each workgroup adds them up
// itself) or from the scanned ones.
__global__ __launch_bounds__(kThreads) void route_place(const int32_t *__restrict__ experts, int64_t n_tok, int E, int k,
                                                        const int32_t *__restrict__ hist, int scanned,
                                                        int32_t *__restrict__ offsets, int32_t *__restrict__ order) {
    __shared__ int count[SIM_MOE_MAX_EXPERTS];   // of this chunk
    __shared__ int before[SIM_MOE_MAX_EXPERTS];  // of the chunks before
    __shared__ int all[SIM_MOE_MAX_EXPERTS];
    __shared__ int wave_sum[kThreads / 64];
    __shared__ int16_t slot_expert[kChunk * SIM_MOE_MAX_TOPK];
    const int chunk = blockIdx.x, chunks = gridDim.x, t = threadIdx.x;
    const int first = chunk * kChunk * k;
    const int n = (int)min((int64_t)kChunk * k, n_tok * k - first);
    count[t] = before[t] = all[t] = 0;
    __syncthreads();
    for (int s = t; s < n; s += kThreads) {
        const int e = experts[(int64_t)first + s];
        slot_expert[s] = (int16_t)e;
        if (e >= 0) atomicAdd(&count[e], 1);
    }
    if (scanned) {
        if (t < E) {
            before[t] = hist[(int64_t)chunk * E + t];
            all[t] = hist[(int64_t)chunks * E + t];
        }
    } else {
        int width = 16;  // lanes over the experts, the rest over the chunks
        while (width < E) width <<= 1;
        const int e = t & (width - 1), step = kThreads / width;
        if (e < E) {
            int b = 0, a = 0;
            for (int c = t / width; c < chunks; c += step) {
                const int v = hist[(int64_t)c * E + e];
                a += v;
                b += c < chunk ? v : 0;
            }
            atomicAdd(&all[e], a);
            atomicAdd(&before[e], b);
        }
    }
    __syncthreads();
    int total;
    const int mine = block_scan(all[t], wave_sum, total);
    before[t] += mine;
    if (chunk == 0) {
        if (t < E) offsets[t] = mine;
        if (t == 0) offsets[E] = total;
    }
    __syncthreads();
    place_slots(slot_expert, n, first, count, before, E, order);
    for (int64_t s = max((int64_t)total, (int64_t)first) + t; s < (int64_t)first + n; s += kThreads) order[s] = -1;
}

// Gradient: sixteen lanes a token again; each chosen expert's w g is taken up
// by the lane that holds that expert.
template <int T, int NV>
__global__ __launch_bounds__(256) void route_grad(const typename Elem<T>::type *__restrict__ logits, int64_t n_tok, int E,
                                                  int64_t stride, const uint8_t *__restrict__ mask, int64_t mask_stride,
                                                  int k, int renorm, const int32_t *__restrict__ experts,
                                                  const float *__restrict__ dw, typename Elem<T>::type *__restrict__ dz) {
    const int l = threadIdx.x & 15;
    const int64_t t = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const bool live = t < n_tok;
    const int64_t tt = live ? t : 0;
    uint32_t key[NV];
    load_keys<T, NV>(logits + tt * stride, mask ? mask + tt * mask_stride : nullptr, E, live, key);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NV; i++) m = max(m, key[i]);
    const float top = key_value(max16(m));
    // g and whether it was chosen, of the experts held here
    float g[NV];
    uint64_t chosen = 0;
#pragma unroll
    for (int i = 0; i < NV; i++) g[i] = 0.f;
    for (int j = 0; j < k; j++) {
        const int e = live ? experts[t * k + j] : -1;
        const float gj = live ? dw[t * k + j] : 0.f;
#pragma unroll
        for (int i = 0; i < NV; i++)
            if (e == i * 16 + l && key[i]) {
                g[i] = gj;
                chosen |= 1ull << i;
            }
    }
    float p[NV], z = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const bool counts = renorm ? (chosen >> i) & 1 : key[i] != 0;
        p[i] = counts ? expf(key_value(key[i]) - top) : 0.f;
        z += p[i];
    }
    const float inv = 1.f / sum16(z);
#pragma unroll
    for (int i = 0; i < NV; i++) {
        p[i] *= inv;
        dot += (chosen >> i) & 1 ? g[i] * p[i] : 0.f;
    }
    dot = sum16(dot);
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int e = i * 16 + l;
        const bool sel = (chosen >> i) & 1;
        const float d = key[i] && (sel || !renorm) ? p[i] * ((sel ? g[i] : 0.f) - dot) : 0.f;
        if (live && e < E) dz[t * E + e] = Elem<T>::put(d);
    }
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

template <int T>
sim_status route_t(hipStream_t st, const RouteArgs &a, int32_t *experts, float *weights, int32_t *offsets, int32_t *order,
                   void *ws) {
    const uint32_t chunks = (uint32_t)((a.T + kChunk - 1) / kChunk);
    int32_t *hist = (int32_t *)ws;
    with_nv(a.E, [&](auto nv) {
        route_choose<T, decltype(nv)::value><<<chunks, kThreads, 0, st>>>(
            (const typename Elem<T>::type *)a.logits, a.T, a.E, a.stride, a.mask, a.mask_stride, a.k, a.renorm, experts,
            weights, hist, offsets, order);
    });
    if (order && chunks > 1) {
        const int scanned = chunks > kScanChunks;
        if (scanned) route_scan<<<(a.E + 15) / 16, kThreads, 0, st>>>(hist, (int)chunks, a.E);
        route_place<<<chunks, kThreads, 0, st>>>(experts, a.T, a.E, a.k, hist, scanned, offsets, order);
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

size_t route_workspace(int64_t T, int E, int) {
    const size_t chunks = (size_t)((T + kChunk - 1) / kChunk);
    return chunks > 1 ? (chunks + 1) * (size_t)E * sizeof(int32_t) : 0;
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
