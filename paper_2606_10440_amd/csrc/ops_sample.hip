// The next token of each row of logits: what temperature, top-k, top-p and
// min-p keep, and of that the one that a given random number points at.
//
// What is kept is a run of the logits' falling order, so it is known by the
// lowest kept logit and how many of the logits that tie with it are kept, in
// the order of their indices.  That logit is searched digit by digit of a key
// that orders as the logits do, by the number of logits to a digit (top-k) or
// by the sum of their weights (top-p).
#include "ops_exp64.h"

namespace simops {
namespace {

constexpr int kThreads = 1024;
constexpr int kWaves = kThreads / 64;
constexpr int kDigit = 11;
constexpr int kBins = 1 << kDigit;
// Weights are at most 1: as whole multiples of 2^-44, of 2^20 of them, their
// sums fit 64 bits, and do not depend on the order in which they are added.
constexpr double kUnit = 17592186044416.;

// Keys that order as logits do: NaN above everything, -infinity 0.
template <int T> __device__ inline uint32_t key_of(typename Elem<T>::type v) {
    if constexpr (T == SIM_TYPE_F32) {
        const uint32_t b = __float_as_uint(v + 0.f);  // -0 to 0: they tie
        return (b & 0x7fffffffu) > 0x7f800000u ? 0xffffffffu : b == 0xff800000u ? 0 : b & 0x80000000u ? ~b : b | 0x80000000u;
    } else {
        constexpr uint32_t inf = T == SIM_TYPE_BF16 ? 0x7f80 : 0x7c00;
        const uint32_t b = __builtin_bit_cast(uint16_t, v), m = b & 0x7fff;
        return m > inf ? 0xffff : m == 0 ? 0x8000 : b == (inf | 0x8000) ? 0 : b & 0x8000 ? ~b & 0xffff : b | 0x8000;
    }
}
template <int T> __device__ inline float value_of(uint32_t key) {
    if constexpr (T == SIM_TYPE_F32) return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
    else return Elem<T>::get(__builtin_bit_cast(typename Elem<T>::type, (uint16_t)(key & 0x8000 ? key & 0x7fff : ~key)));
}
template <int T> constexpr uint32_t kInfinite = T == SIM_TYPE_F32 ? 0xff800000u : T == SIM_TYPE_BF16 ? 0xff80u : 0xfc00u;  // key of +infinity
template <int T> constexpr int kKeyBits = T == SIM_TYPE_F32 ? 32 : 16;

__device__ inline double wave_sum(double v) {
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

struct Shared {
    uint64_t bin[kBins];
    uint64_t wave64[kWaves];
    double wave_d[kWaves];
    uint32_t wave_key[kWaves], wave_at[kWaves];
    uint32_t digit;
    uint64_t above;
    int found;
};

template <int T> struct Row {
    typedef typename Elem<T>::type El;
    const El *z;
    int V;
    double top, per;  // the highest logit; 1 / temperature
    __device__ double weight(uint32_t key) const { return exp64(((double)value_of<T>(key) - top) * per); }
    __device__ uint32_t key(int i) const { return key_of<T>(z[i]); }
};

// Sum over the workgroup, in an order of its own.
__device__ inline double block_sum(double v, Shared &s) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.wave_d[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.;
    for (int w = 0; w < kWaves; w++) sum += s.wave_d[w];
    return sum;
}

// The key at which the sum of add(key) over the keys from the highest down
// reaches target (whole numbers; at least 1), and the sum above it; false where
// all together do not.
template <int T, typename Add>
__device__ inline bool search(const Row<T> &row, Shared &s, uint64_t target, uint32_t extra_key, uint64_t extra, Add &&add, uint32_t &key,
                              uint64_t &above) {
    uint32_t prefix = 0;
    above = 0;
    for (int left = kKeyBits<T>; left > 0;) {
        const int bits = min(left, kDigit), shift = left - bits;
        __syncthreads();
        for (int i = threadIdx.x; i < kBins; i += kThreads) s.bin[i] = 0;
        if (threadIdx.x == 0) s.found = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < row.V; i += kThreads) {
            const uint32_t k = row.key(i);
            if (left < 32 && (k >> left) != prefix) continue;
            const uint64_t n = add(k);
            if (n) atomicAdd((unsigned long long *)&s.bin[(k >> shift) & ((1u << bits) - 1)], (unsigned long long)n);
        }
        if (threadIdx.x == 0 && extra && (left == 32 || (extra_key >> left) == prefix))
            atomicAdd((unsigned long long *)&s.bin[(extra_key >> shift) & ((1u << bits) - 1)], (unsigned long long)extra);
        __syncthreads();
        // two bins a thread, from the highest down
        const int hi = kBins - 1 - 2 * threadIdx.x;
        const uint64_t a = s.bin[hi], b = s.bin[hi - 1];
        uint64_t sum = a + b;
        for (int d = 1; d < 64; d <<= 1) {
            const uint64_t o = __shfl_up((unsigned long long)sum, d);
            if ((int)(threadIdx.x & 63) >= d) sum += o;
        }
        if ((threadIdx.x & 63) == 63) s.wave64[threadIdx.x >> 6] = sum;
        __syncthreads();
        uint64_t before = above + sum - a - b;
        for (int w = 0; w < (int)(threadIdx.x >> 6); w++) before += s.wave64[w];
        if (before < target && before + a >= target) s.digit = hi, s.above = before, s.found = 1;
        else if (before + a < target && before + a + b >= target) s.digit = hi - 1, s.above = before + a, s.found = 1;
        __syncthreads();
        if (!s.found) return false;
        prefix = (left < 32 ? prefix << bits : 0) | s.digit;
        above = s.above;
        left = shift;
    }
    key = prefix;
    return true;
}

// The first index at which the running sum of weight(i) is above target(sum of
// all); of one with a weight above 0, the last such if rounding leaves none.
template <typename Weight, typename Target>
__device__ inline int locate(Shared &s, int V, Weight &&weight, Target &&target_of) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int lo = 0, hi = V;
    double before = 0., target = 0.;
    bool first = true;
    do {
        const int seg = (hi - lo + kWaves - 1) / kWaves, a = min(hi, lo + wave * seg), b = min(hi, a + seg);
        double sum = 0.;
        for (int i = a + lane; i < b; i += 64) sum += weight(i);
        sum = wave_sum(sum);
        __syncthreads();
        if (lane == 0) s.wave_d[wave] = sum;
        __syncthreads();
        if (first) {
            double all = 0.;
            for (int w = 0; w < kWaves; w++) all += s.wave_d[w];
            target = target_of(all);
            first = false;
        }
        int at = 0;
        double run = before, start = before;
        for (int w = 0; w < kWaves; w++) {
            const double v = s.wave_d[w];
            if (v > 0.) at = w, start = run;
            run += v;
            if (v > 0. && run > target) break;
        }
        before = start;
        lo = min(hi, lo + at * seg);
        hi = min(hi, lo + seg);
    } while (hi - lo > 64);
    const double mine = lo + lane < hi ? weight(lo + lane) : 0.;
    double run = mine;
    for (int d = 1; d < 64; d <<= 1) {
        const double o = __shfl_up(run, d);
        if (lane >= d) run += o;
    }
    const uint64_t some = __ballot(mine > 0.), past = __ballot(mine > 0. && before + run > target);
    return lo + (past ? __ffsll((unsigned long long)past) - 1 : some ? 63 - __clzll((long long)some) : 0);
}

template <int T> __global__ __launch_bounds__(kThreads) void sample_rows(SampleArgs a) {
    typedef typename Elem<T>::type El;
    __shared__ Shared s;
    const int64_t b = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Row<T> row;
    row.z = (const El *)a.logits + b * a.stride;
    row.V = a.V;

    // the highest and its first index
    uint32_t best = 0, at = 0;
    for (int i = threadIdx.x; i < a.V; i += kThreads) {
        const uint32_t k = row.key(i);
        if (k > best) best = k, at = i;
    }
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t k = __shfl_xor(best, d), i = __shfl_xor(at, d);
        if (k > best || (k == best && i < at)) best = k, at = i;
    }
    if (lane == 0) s.wave_key[wave] = best, s.wave_at[wave] = at;
    __syncthreads();
    for (int w = 0; w < kWaves; w++)
        if (s.wave_key[w] > best || (s.wave_key[w] == best && s.wave_at[w] < at)) best = s.wave_key[w], at = s.wave_at[w];
    const float temperature = a.temperature ? a.temperature[b] : a.all_temperature, min_p = a.min_p ? a.min_p[b] : a.all_min;
    const float top_p = a.top_p ? a.top_p[b] : a.all_p;
    const int top_k = a.top_k ? a.top_k[b] : a.all_k;
    if (best == 0 || best >= kInfinite<T> || !(temperature > 0.f) || top_k == 1 || top_p <= 0.f || min_p > 1.f) {
        if (threadIdx.x == 0) a.tokens[b] = best == 0 || best >= kInfinite<T> ? -1 : (int)at;
        return;
    }
    row.top = value_of<T>(best);
    row.per = 1. / temperature;

    uint32_t lowest = 0;     // the lowest kept key
    uint64_t ties = ~0ull;   // how many of it are kept
    if (top_k >= 1 && top_k < a.V) {
        uint64_t above;
        if (search(row, s, (uint64_t)top_k, 0, 0, [](uint32_t k) { return (uint64_t)(k != 0); }, lowest, above)) ties = top_k - above;
        else lowest = 0;  // so many are not there
    }
    if (top_p < 1.f) {
        const uint32_t low_k = lowest;
        const double w_k = low_k ? row.weight(low_k) : 0.;
        double sum = 0.;
        for (int i = threadIdx.x; i < a.V; i += kThreads) {
            const uint32_t k = row.key(i);
            if (k > low_k) sum += row.weight(k);
        }
        const double most = (block_sum(sum, s) + (low_k ? (double)ties * w_k : 0.)) * (double)top_p;
        const auto fixed = [](double w) { return (uint64_t)(w * kUnit + .5); };
        uint32_t low_p;
        uint64_t above;
        if (search(row, s, max((uint64_t)1, (uint64_t)__builtin_ceil(most * kUnit)), low_k, low_k ? ties * fixed(w_k) : 0,
                   [&](uint32_t k) { return k > low_k ? fixed(row.weight(k)) : 0; }, low_p, above)) {
            double over = 0., same = 0.;
            for (int i = threadIdx.x; i < a.V; i += kThreads) {
                const uint32_t k = row.key(i);
                if (k > low_p) over += row.weight(k);
                same += k == low_p;
            }
            over = block_sum(over, s);
            same = block_sum(same, s);
            const double w = row.weight(low_p), n = __builtin_ceil((most - over) / w);
            lowest = low_p;
            ties = min(low_p == low_k ? ties : (uint64_t)same, (uint64_t)max(1., min(n, 4294967296.)));
        }
    }
    // the last kept one of those that tie
    int cut = a.V;
    if (lowest && ties < (uint64_t)a.V)
        cut = locate(s, a.V, [&](int i) { return row.key(i) == lowest ? 1. : 0.; }, [&](double all) { return (double)ties < all ? (double)ties - .5 : all; });
    const double u = a.u[b] > 0.f ? (double)min(a.u[b], 1.f - 5.9604644775390625e-8f) : 0.;
    const int token = locate(
        s, a.V,
        [&](int i) {
            const uint32_t k = row.key(i);
            if (k == 0 || k < lowest || (k == lowest && i > cut)) return 0.;
            const double w = row.weight(k);
            return w >= (double)min_p || !(min_p > 0.f) ? w : 0.;
        },
        [&](double all) { return u * all; });
    if (threadIdx.x == 0) a.tokens[b] = token;
}

}  // namespace

size_t sample_workspace(int64_t, int) { return 0; }

sim_status launch_sample(hipStream_t st, const SampleArgs &a, void *) {
    if (a.type == SIM_TYPE_F32) sample_rows<SIM_TYPE_F32><<<(uint32_t)a.B, kThreads, 0, st>>>(a);
    else if (a.type == SIM_TYPE_F16) sample_rows<SIM_TYPE_F16><<<(uint32_t)a.B, kThreads, 0, st>>>(a);
    else sample_rows<SIM_TYPE_BF16><<<(uint32_t)a.B, kThreads, 0, st>>>(a);
    return SIM_OPS_LAUNCH_OK();
}

}  // namespace simops
