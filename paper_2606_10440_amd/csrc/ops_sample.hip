// The next token of each row of logits: what temperature, top-k, top-p and
// min-p keep, and of that the one that a given random number points at.
//
// What is kept is a run of the logits' falling order, so it is known by the
// lowest kept logit and how many of the logits that tie with it are kept, in
// the order of their indices.  A row is read by several workgroups, a slice
// each, in up to five launches:
//   tops    the highest logit of each slice, and of each eight;
//   bins    the sums of the weights, or the numbers of logits, by how far they
//           are below the highest, in steps of 1/128 of that distance;
//   border  the logits of the bin in which the border lies as a list;
//   sorted  one workgroup sorts it.  For a small top-k the list is made here:
//           where k of the eights' highest are above a border, k logits are, so
//           that only the eights whose highest is need be read.  Such a row is
//           done with that;
//   pick    the sums of the kept weights of 512 logits each; the row's last
//           workgroup finds the 512 that the token is in, and the token.
// A row whose border bin holds more than can be sorted (logits that are nearly
// all the same; half a million or more that are normal, of which so many are as
// far from the highest), and one with a top-k above 2048 and a top-p, is searched
// by one workgroup alone, digit by digit of a key that orders as the logits do,
// which takes some 15 to 30 times as long: top-p 0.9 alone, one row of 400000
// normal fp32 80 us, of 524288 1460, of 2^20 2900; top-k 3000 and top-p 0.9, one
// row of 131072 0.4 ms, 64 of 400000 1.6 ms.
//
// One row of 131072 fp32, top-k 50 and top-p 0.95: 18 us (tops 4, sorted 14, which
// is one workgroup's chain of barriers and of 64-bit operations); all of its
// logits kept 15.  192 rows of 100003 bf16, each with settings of its own: 103 us (tops 11,
// bins 22, border 13, sorted 34, pick 25) for 38 MB, 7.4 us of memory: the 64-bit
// weights of the rows without top-k, and the sorted lists, of 700 where top-k is
// 500, take the rest.
#include "ops_exp64.h"

namespace simops {
namespace {

constexpr int kThreads = 256;  // of a workgroup that has a slice
constexpr int kWaves = kThreads / 64;
constexpr int kAll = 1024;     // of one that has what is left of a row, or all of it
constexpr int kAllWaves = kAll / 64;
constexpr int kDigit = 11;
constexpr int kBins = 1 << kDigit;
constexpr double kUnit = kWeightUnit;
static_assert(kUnit * SIM_SAMPLE_MAX_V < 18446744073709551616., "the sum of a row's weights fits 64 bits");

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
template <int T> constexpr uint32_t kLowest = T == SIM_TYPE_F32 ? 0x800000u : T == SIM_TYPE_BF16 ? 0x80u : 0x400u;  // of the lowest finite value
template <int T> constexpr int kKeyBits = T == SIM_TYPE_F32 ? 32 : 16;

// Sums over the lanes up to each, of 64-bit whole numbers or values, by moves
// between registers (an exchange through LDS takes some 100 cycles, and there
// are six, one after another).
template <int CTRL, int ROWS, typename V> __device__ inline V moved(V v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, CTRL, ROWS, 0xf, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), CTRL, ROWS, 0xf, false);
    return __builtin_bit_cast(V, lo | (uint64_t)hi << 32);
}
template <int CTRL, int ROWS, typename V> __device__ inline V add_from(V v) { return v + moved<CTRL, ROWS>(v); }
template <typename V> __device__ inline V row_scan(V v) {  // of 16 lanes
    v = add_from<0x111, 0xf>(v);                           // from the lane before
    v = add_from<0x112, 0xf>(v);                           // two before
    v = add_from<0x114, 0xf>(v);
    return add_from<0x118, 0xf>(v);
}
template <typename V> __device__ inline V wave_scan(V v) {
    v = row_scan(v);
    v = add_from<0x142, 0xa>(v);     // lane 15's and 47's to the rows after
    return add_from<0x143, 0xc>(v);  // lane 31's to the upper half
}
template <typename V> __device__ inline V lane_of(V v, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(V, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)b, lane) |
                                     (uint64_t)__builtin_amdgcn_readlane((int)(b >> 32), lane) << 32);
}
__device__ inline uint64_t wave_max(uint64_t v) {
    v = max(v, moved<0x111, 0xf>(v));
    v = max(v, moved<0x112, 0xf>(v));
    v = max(v, moved<0x114, 0xf>(v));
    v = max(v, moved<0x118, 0xf>(v));
    v = max(v, moved<0x142, 0xa>(v));
    return lane_of(max(v, moved<0x143, 0xc>(v)), 63);
}
// Sums over the workgroup's threads before each, and over all, from own values.
template <int NT, typename V> __device__ inline V block_scan(V own, V *wave_sums, V &all) {
    static_assert(NT / 64 <= 16, "a lane of a row for each wave");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const V sum = wave_scan(own);
    __syncthreads();
    if (lane == 63) wave_sums[wave] = sum;
    __syncthreads();
    const V waves = row_scan((lane & 15) < NT / 64 ? wave_sums[lane & 15] : V(0));
    all = lane_of(waves, 15);
    const V before = __shfl_up(sum, 1);
    return (lane ? before : V(0)) + (wave ? lane_of(waves, wave - 1) : V(0));
}
__device__ inline double wave_sum(double v) { return lane_of(wave_scan(v), 63); }

struct Shared {
    uint64_t bin[kBins];
    uint64_t wave64[kAllWaves];
    double wave_d[kAllWaves];
    uint32_t digit;
    uint64_t above;
};

template <int T> struct Row {
    typedef typename Elem<T>::type El;
    const El *z;
    int V;
    double top, per;  // the highest logit; 1 / temperature
    __device__ double weight(uint32_t key) const { return exp64(((double)value_of<T>(key) - top) * per); }
    __device__ uint32_t key(int i) const { return key_of<T>(z[i]); }
};

// The first of kBins values at which their running sum reaches target, in all
// threads, and the sum before it; -1 where all together do not.  The caller
// keeps to barriers around it.
template <int NT, typename Bin> __device__ inline int crossing(Bin &&bin, uint64_t target, uint64_t *wave_sums, uint64_t &before) {
    constexpr int kEach = kBins / NT;
    __shared__ int s_at;
    __shared__ uint64_t s_before;
    typedef unsigned long long u64;
    uint64_t v[kEach], own = 0;
#pragma unroll
    for (int i = 0; i < kEach; i++) own += v[i] = bin(threadIdx.x * kEach + i);
    if (threadIdx.x == 0) s_at = -1;
    u64 all;
    uint64_t run = block_scan<NT>((u64)own, (u64 *)wave_sums, all);
#pragma unroll
    for (int i = 0; i < kEach; i++) {
        if (run < target && run + v[i] >= target) s_at = threadIdx.x * kEach + i, s_before = run;
        run += v[i];
    }
    __syncthreads();
    before = s_before;
    return s_at;
}

// Sum over the workgroup, in an order of its own.
__device__ inline double block_sum(double v, Shared &s) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.wave_d[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.;
    for (int w = 0; w < kAllWaves; w++) sum += s.wave_d[w];
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
        for (int i = threadIdx.x; i < kBins; i += kAll) s.bin[i] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < row.V; i += kAll) {
            const uint32_t k = row.key(i);
            if (left < 32 && (k >> left) != prefix) continue;
            const uint64_t n = add(k);
            if (n) atomicAdd((unsigned long long *)&s.bin[(k >> shift) & ((1u << bits) - 1)], (unsigned long long)n);
        }
        if (threadIdx.x == 0 && extra && (left == 32 || (extra_key >> left) == prefix))
            atomicAdd((unsigned long long *)&s.bin[(extra_key >> shift) & ((1u << bits) - 1)], (unsigned long long)extra);
        __syncthreads();
        // from the highest bin down
        const auto bin = [&](int i) { return s.bin[kBins - 1 - i]; };
        uint64_t before;
        const int at = crossing<kAll>(bin, target - above, s.wave64, before);
        if (at < 0) return false;
        s.digit = kBins - 1 - at, s.above = above + before;
        __syncthreads();
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
        const int seg = (hi - lo + kAllWaves - 1) / kAllWaves, a = min(hi, lo + wave * seg), b = min(hi, a + seg);
        double sum = 0.;
        for (int i = a + lane; i < b; i += 64) sum += weight(i);
        sum = wave_sum(sum);
        __syncthreads();
        if (lane == 0) s.wave_d[wave] = sum;
        __syncthreads();
        if (first) {
            double all = 0.;
            for (int w = 0; w < kAllWaves; w++) all += s.wave_d[w];
            target = target_of(all);
            first = false;
        }
        int at = 0;
        double run = before, start = before;
        for (int w = 0; w < kAllWaves; w++) {
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

// A row by one workgroup alone.
template <int T>
__device__ inline int search_row(const Row<T> &row, Shared &s, int top_k, float top_p, float min_p, double u) {
    uint32_t lowest = 0;     // the lowest kept key
    uint64_t ties = ~0ull;   // how many of it are kept
    if (top_k >= 1 && top_k < row.V) {
        uint64_t above;
        if (search(row, s, (uint64_t)top_k, 0, 0, [](uint32_t k) { return (uint64_t)(k != 0); }, lowest, above)) ties = top_k - above;
        else lowest = 0;  // so many are not there
    }
    if (top_p < 1.f) {
        const uint32_t low_k = lowest;
        const double w_k = low_k ? row.weight(low_k) : 0.;
        double sum = 0.;
        for (int i = threadIdx.x; i < row.V; i += kAll) {
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
            for (int i = threadIdx.x; i < row.V; i += kAll) {
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
    int cut = row.V;
    if (lowest && ties < (uint64_t)row.V)
        cut = locate(s, row.V, [&](int i) { return row.key(i) == lowest ? 1. : 0.; }, [&](double all) { return (double)ties < all ? (double)ties - .5 : all; });
    return locate(
        s, row.V,
        [&](int i) {
            const uint32_t k = row.key(i);
            if (k == 0 || k < lowest || (k == lowest && i > cut)) return 0.;
            const double w = row.weight(k);
            return w >= (double)min_p || !(min_p > 0.f) ? w : 0.;
        },
        [&](double all) { return u * all; });
}

// ------------------------------------------------------------------ rows in slices

constexpr int kChunk = 512;       // logits of one step of a wave, eight a lane
constexpr int kMaxSlices = 64;    // of a row
constexpr int kMaxChunks = (SIM_SAMPLE_MAX_V + 7 + kChunk - 1) / kChunk;
constexpr int kList = 4096;       // logits that a workgroup sorts
constexpr int kStage = 512;       // logits that a slice's workgroup collects before it adds them to the list
constexpr int kMaxSorted = 2048;  // up to this top-k all that are above the border are sorted too
constexpr int kSliceGroups = 2048;  // workgroups of a launch
constexpr int kRows = 1024;       // of one set of launches, and of the workspace

enum Mode : uint32_t { kOpen, kBordered, kDone };

// What the launches find out about a row.
struct RowState {
    uint32_t binned, listed, picked;  // workgroups that have come, and logits in the list
    int border;                                // the bin of the border; -1: there are fewer logits than top-k
    Mode mode;
    uint32_t lowest, cut;                      // kBordered: the lowest kept key and the last kept index that has it
    uint64_t above, all;                       // the bins' sums above the border, and all of them
};

// Where the rows' parts of the workspace are, and how a row is cut.
struct Plan {
    uint64_t *tops;    // [row][slice]: key and, complemented, index of the highest
    void *eights;      // [row][chunks * kChunk / 8]: the highest of each eight
    uint64_t *bins;    // [row][kBins]
    uint64_t *list;    // [row][kList]
    double *sums;      // [row][chunks]
    RowState *state;
    int64_t row0;
    int chunks, slices, chunks_of_slice;
};

enum Kind {
    kToken,   // the highest, or -1
    kSorted,  // a small top-k: all that is above its border is sorted
    kListed,  // the same, of a row with few eights for it
    kNumber,  // a large top-k
    kWeight,  // top-p
    kEvery,   // every logit, or what min-p leaves
    kAlone,   // a large top-k with top-p: one workgroup searches
};
template <int T> struct Task {
    Row<T> row;
    Kind kind;
    uint32_t best;
    int first;  // index of the highest
    float top, min_p, top_p;
    int top_k;
    __device__ int token() const { return best == 0 || best >= kInfinite<T> ? -1 : first; }
};

// Whether a row has so many eights that the k-th highest of theirs leaves no
// more logits than can be sorted (with twice k eights that is four thirds of
// k), or so few logits that all can.
__host__ __device__ inline bool by_eights(int V, int k) { return V <= kList || V / 16 >= k; }

// What is to be done with a row, from its highest logit's key and, complemented,
// index.
template <int T> __device__ inline Task<T> task_from(const SampleArgs &a, int64_t b, uint64_t top) {
    typedef typename Elem<T>::type El;
    Task<T> t;
    t.row.z = (const El *)a.logits + b * a.stride;
    t.row.V = a.V;
    t.best = __builtin_amdgcn_readfirstlane((uint32_t)(top >> 32));
    t.first = (int)~__builtin_amdgcn_readfirstlane((uint32_t)top);
    t.top = value_of<T>(t.best);
    const float temperature = a.temperature ? a.temperature[b] : a.all_temperature;
    t.min_p = a.min_p ? a.min_p[b] : a.all_min;
    t.top_p = a.top_p ? a.top_p[b] : a.all_p;
    t.top_k = a.top_k ? a.top_k[b] : a.all_k;
    t.row.top = t.top;
    t.row.per = 1. / temperature;
    if (t.best == 0 || t.best >= kInfinite<T> || !(temperature > 0.f) || t.top_k == 1 || t.top_p <= 0.f || t.min_p > 1.f) t.kind = kToken;
    else if (t.top_k < 1 || t.top_k >= a.V) t.kind = t.top_p < 1.f ? kWeight : kEvery;
    else if (t.top_k <= kMaxSorted) t.kind = by_eights(a.V, t.top_k) ? kSorted : kListed;
    else t.kind = t.top_p < 1.f ? kAlone : kNumber;
    return t;
}
// The same from its slices' tops, in every wave.
template <int T> __device__ inline Task<T> task_of(const SampleArgs &a, const Plan &p, int64_t b) {
    const int lane = threadIdx.x & 63;
    return task_from<T>(a, b, wave_max(lane < p.slices ? p.tops[(b - p.row0) * p.slices + lane] : 0));
}
__device__ inline double number_of(const SampleArgs &a, int64_t b) {
    return a.u[b] > 0.f ? (double)min(a.u[b], 1.f - 5.9604644775390625e-8f) : 0.;
}

// Rows are cut where memory is aligned, so that their first logits have
// indices below 0 before them.  The index of a lane's first logit of a chunk:
template <int T> __device__ inline int index_of(const Row<T> &row, int chunk) {
    return chunk * kChunk + (int)(threadIdx.x & 63) * 8 - (int)((uintptr_t)row.z / sizeof(*row.z) % 8);
}
// Eight consecutive logits from i on; -infinity outside the row.
typedef u32x4 u32x4_alias __attribute__((may_alias));
template <int T> __device__ inline void load8(const Row<T> &row, int i, typename Elem<T>::type v[8]) {
    if (i >= 0 && i + 8 <= row.V) {
#pragma unroll
        for (int j = 0; j < (int)sizeof(v[0]) / 2; j++) ((u32x4_alias *)v)[j] = ((const u32x4_alias *)(row.z + i))[j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = i + j >= 0 && i + j < row.V ? row.z[i + j] : Elem<T>::put(-INFINITY);
    }
}
constexpr int kAhead = 4;  // chunks that are loaded together
// Calls f(first chunk, end of the slice, logits) for this wave's part of a
// slice, every NW-th chunk.
template <int T, int NW, typename F> __device__ inline void each_group(const Row<T> &row, const Plan &p, int slice, F &&f) {
    const int end = min(p.chunks, (slice + 1) * p.chunks_of_slice);
    for (int c0 = slice * p.chunks_of_slice + (int)(threadIdx.x >> 6); c0 < end; c0 += kAhead * NW) {
        typename Elem<T>::type v[kAhead][8];
#pragma unroll
        for (int n = 0; n < kAhead; n++) load8(row, index_of(row, min(c0 + n * NW, end - 1)), v[n]);
        f(c0, end, v);
    }
}
// Calls f(index, eight logits, chunk) for each of them.
template <int T, int NW, typename F> __device__ inline void each_chunk(const Row<T> &row, const Plan &p, int slice, F &&f) {
    each_group<T, NW>(row, p, slice, [&](int c0, int end, const typename Elem<T>::type v[kAhead][8]) {
#pragma unroll
        for (int n = 0; n < kAhead; n++)
            if (c0 + n * NW < end) f(index_of(row, c0 + n * NW), v[n], c0 + n * NW);
    });
}

// How far a logit is below the highest, as one of kBins: 128 to each doubling
// of the distance plus 1/32, from 1/32 to 2048.
__device__ inline int bin_of(float top, float z) {
    return min((int)(__float_as_uint(top - z + 0.03125f) >> 16) - 0x3d00, kBins - 1);
}
// Weights of many logits: e^((z - top) / T) = 2^(n / 64) e^r, n the nearest whole
// number, from a table of 2^(j / 64) in LDS and the series of e^r up to r^4 / 24
// (r is at most ln 2 / 128, the next term below 2^-44; the argument's rounding is
// below 2^-42 for the farthest).  A 64-bit fused operation
// takes as long as two others here, and a constant that the compiler knows costs
// it two moves, so constants are kept from it, in scalar registers (192 rows of
// 131072 without top-k 68 us by the series alone, 55 so).
constexpr int kTable = 64;
__device__ inline double scalar(double c) {
    asm("" : "+s"(c));
    return c;
}
__device__ inline void fill(double *table) {
    if (threadIdx.x < kTable) table[threadIdx.x] = 2. * exp64(((int)threadIdx.x - kTable) * (0.69314718055994531 / kTable));
}
template <int T> struct Exp {
    const double *table;
    double top, steps;  // 64 / (T ln 2)
    float high, far;    // beyond this below the highest, weights are below 2^-1022: 0
    __device__ Exp(const Row<T> &row, const double *table_) : table(table_), top(row.top), steps(row.per * (kTable * 1.4426950408889634)) {
        high = (float)top;
        far = (float)min(708. / row.per, 3.4028234e38);
    }
    __device__ bool none(float z) const { return high - z > far; }
    // where not none(z)
    __device__ double operator()(float z) const {
        const double d = (double)z - top, t = __builtin_fma(d, steps, scalar(6755399441055744.)), n = t - scalar(6755399441055744.);
        const double f = __builtin_fma(d, steps, -n);
        const int i = (int)__builtin_bit_cast(uint64_t, t);
        constexpr double c = 0.69314718055994531 / kTable;
        double p = __builtin_fma(f, scalar(c * c * c * c / 24.), scalar(c * c * c / 6.));
        p = __builtin_fma(p, f, scalar(c * c / 2.));
        p = __builtin_fma(p, f, scalar(c));
        const uint64_t b = __builtin_bit_cast(uint64_t, table[i & (kTable - 1)]);
        const double s = __builtin_bit_cast(double, b + ((uint64_t)(uint32_t)((i >> 6) << 20) << 32));
        return __builtin_fma(s * f, p, s);
    }
    // Eight at once, without a branch around each, so that their operations fill
    // each other's waits; 0 where not in.
    __device__ void eight(const float z[8], const bool in[8], double w[8]) const {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; j++) x[j] = in[j] ? z[j] : high;
#pragma unroll
        for (int j = 0; j < 8; j++) w[j] = (*this)(x[j]);
#pragma unroll
        for (int j = 0; j < 8; j++) w[j] = in[j] ? w[j] : 0.;
    }
};

// A weight as a whole multiple of 1 / kUnit: it lands in the low bits of 2^52 + w kUnit
__device__ inline uint64_t fixed(double w) {
    return __builtin_bit_cast(uint64_t, __builtin_fma(w, kUnit, 4503599627370496.)) & 0xfffffffffffffull;
}

// Key and, complemented, index of the highest logit of a wave's part of a slice;
// eight(value, chunk) gets the highest of each eight.
template <int T, int NW, typename F> __device__ inline uint64_t highest(const Row<T> &row, const Plan &p, int slice, F &&eight) {
    typedef typename Elem<T>::type El;
    // the highest of eight at a time; which of them it is, only where they hold
    // a lane's highest
    float best = -INFINITY;
    int at = 0;
    each_chunk<T, NW>(row, p, slice, [&](int i, const El v[8], int c) {
        float m = Elem<T>::get(v[0]);
#pragma unroll
        for (int j = 1; j < 8; j++) m = __builtin_elementwise_maximum(m, Elem<T>::get(v[j]));
        if (!(m <= best) && best == best) at = i, best = __builtin_elementwise_maximum(best, m);
        eight(m, c);
    });
    uint32_t key = 0;
    if (best != -INFINITY) {
        El v[8];
        load8(row, at, v);
        int first = 0;
#pragma unroll
        for (int j = 7; j >= 0; j--) {
            const uint32_t k = key_of<T>(v[j]);
            first = k >= key ? j : first;
            key = max(key, k);
        }
        at += first;
    }
    return wave_max((uint64_t)key << 32 | (uint32_t)~at);
}

template <int T> __global__ __launch_bounds__(kThreads) void sample_tops(SampleArgs a, Plan p, bool with_eights) {
    typedef typename Elem<T>::type El;
    __shared__ uint64_t s_top[kWaves];
    const int64_t r = blockIdx.x / p.slices, b = p.row0 + r;
    const int slice = (int)(blockIdx.x % p.slices);
    Row<T> row;
    row.z = (const El *)a.logits + b * a.stride;
    row.V = a.V;
    uint64_t top = highest<T, kWaves>(row, p, slice, [&](float m, int c) {
        if (with_eights) ((El *)p.eights)[r * p.chunks * (kChunk / 8) + c * (kChunk / 8) + (threadIdx.x & 63)] = Elem<T>::put(m);
    });
    if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
    // what the launches after this one count up from
    for (int i = slice * kThreads + threadIdx.x; i < kBins; i += p.slices * kThreads) p.bins[r * kBins + i] = 0;
    if (slice == 0 && threadIdx.x == 0) p.state[r] = RowState{};
    __syncthreads();
    if (threadIdx.x == 0) p.tops[r * p.slices + slice] = max(max(s_top[0], s_top[1]), max(s_top[2], s_top[3]));
}

template <typename V> __device__ inline V at_device(const V *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// Whether this workgroup is the last of a row's: what the others have written at
// device scope before is there then.
__device__ inline bool last_of(uint32_t *arrived, int of, int *s_last) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) *s_last = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)of - 1;
    __syncthreads();
    return *s_last;
}

template <int T> __global__ __launch_bounds__(kThreads) void sample_bins(SampleArgs a, Plan p) {
    typedef typename Elem<T>::type El;
    __shared__ uint64_t s_bin[kBins], wave64[kWaves];
    __shared__ double s_table[kTable];
    __shared__ int s_last;
    const int64_t r = blockIdx.x / p.slices;
    const int slice = (int)(blockIdx.x % p.slices);
    const Task<T> t = task_of<T>(a, p, p.row0 + r);
    if (t.kind != kListed && t.kind != kNumber && t.kind != kWeight) return;
    for (int i = threadIdx.x; i < kBins; i += kThreads) s_bin[i] = 0;
    fill(s_table);
    const Exp<T> weight(t.row, s_table);
    const bool weights = t.kind == kWeight;
    __syncthreads();
    each_chunk<T, kWaves>(t.row, p, slice, [&](int, const El v[8], int) {
        float z[8];
        bool in[8];
        double w[8];
#pragma unroll
        for (int j = 0; j < 8; j++) z[j] = Elem<T>::get(v[j]), in[j] = !(weights ? weight.none(z[j]) : z[j] == -INFINITY);
        if (weights) weight.eight(z, in, w);
#pragma unroll
        for (int j = 0; j < 8; j++)
            if (in[j]) atomicAdd((unsigned long long *)&s_bin[bin_of(t.top, z[j])], (unsigned long long)(weights ? fixed(w[j]) : 1));
    });
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads)
        if (s_bin[i]) __hip_atomic_fetch_add(&p.bins[r * kBins + i], s_bin[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    RowState &state = p.state[r];
    if (!last_of(&state.binned, p.slices, &s_last)) return;
    for (int i = threadIdx.x; i < kBins; i += kThreads) s_bin[i] = at_device(&p.bins[r * kBins + i]);
    __syncthreads();
    uint64_t target = (uint64_t)t.top_k, above = 0, all = 0;
    if (t.kind == kWeight) {
        for (int i = threadIdx.x; i < kBins; i += kThreads) all += s_bin[i];
        all = lane_of(wave_scan(all), 63);
        if ((threadIdx.x & 63) == 0) wave64[threadIdx.x >> 6] = all;
        __syncthreads();
        all = wave64[0] + wave64[1] + wave64[2] + wave64[3];
        __syncthreads();
        target = max((uint64_t)1, (uint64_t)__builtin_ceil((double)all * (double)t.top_p));
    }
    const int border = crossing<kThreads>([&](int i) { return s_bin[i]; }, target, wave64, above);
    if (threadIdx.x == 0) state.border = border, state.above = above, state.all = all;
}

// Sorts 1024 E values in registers, the highest first, by exchanges between
// values that are further and further apart: value 1024 e + t is thread t's
// e-th, so only those 64 to 512 apart go through LDS.
template <int E> __device__ inline void sort_registers(uint64_t *lds, int n) {
    const int t = threadIdx.x;
    uint64_t v[E];
#pragma unroll
    for (int e = 0; e < E; e++) v[e] = e * kAll + t < n ? lds[e * kAll + t] : 0;
    const auto across = [&](int run, int d) {
        if (d >= 64) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; e++) lds[e * kAll + t] = v[e];
            __syncthreads();
        }
#pragma unroll
        for (int e = 0; e < E; e++) {
            const uint64_t o = d >= 64 ? lds[e * kAll + (t ^ d)] : (uint64_t)__shfl_xor((unsigned long long)v[e], d);
            const bool high = ((t & d) == 0) == (((e * kAll + t) & run) == 0);
            v[e] = high ? max(v[e], o) : min(v[e], o);
        }
    };
    for (int run = 2; run <= kAll; run <<= 1)
        for (int d = run >> 1; d; d >>= 1) across(run, d);
#pragma unroll
    for (int r = 2; r <= E; r *= 2) {
#pragma unroll
        for (int d = r / 2; d; d /= 2)
#pragma unroll
            for (int e = 0; e < E; e++)
                if (!(e & d)) {
                    const uint64_t x = max(v[e], v[e | d]), y = min(v[e], v[e | d]);
                    v[e] = e & r ? y : x, v[e | d] = e & r ? x : y;
                }
        for (int d = kAll / 2; d; d >>= 1) across(r * kAll, d);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; e++) lds[e * kAll + t] = v[e];
    __syncthreads();
}

// Sorts n of kList (4 kAll) different values; what is past them may be overwritten.  Few
// are put where the number of higher ones says.
__device__ inline void sort(uint64_t *v, int n) {
    if (n <= 128) {
        const uint64_t own = (int)threadIdx.x < n ? v[threadIdx.x] : 0;
        int place = 0;
        // (a wave that has none of them would read them all the same)
        for (int i = 0; i < n && (int)(threadIdx.x & ~63) < n; i += 8) {
            uint64_t o[8];
#pragma unroll
            for (int j = 0; j < 8; j++) o[j] = v[min(i + j, n - 1)];
#pragma unroll
            for (int j = 0; j < 8; j++) place += i + j < n && o[j] > own;
        }
        __syncthreads();
        if ((int)threadIdx.x < n) v[place] = own;
        __syncthreads();
    } else if (n <= kAll) {
        sort_registers<1>(v, n);
    } else if (n <= 2 * kAll) {
        sort_registers<2>(v, n);
    } else {
        sort_registers<4>(v, n);
    }
}

// Running sums over n values, a run of them to each thread: before(i) of each is
// passed to f(i, before, value); returns the sum of all.
template <int NT, typename Value, typename F> __device__ inline double scan(int n, double *wave_d, Value &&value, F &&f) {
    const int each = (n + NT - 1) / NT, i0 = threadIdx.x * each, i1 = min(n, i0 + each);
    double own = 0.;
    for (int i = i0; i < i1; i++) own += value(i);
    double all, run = block_scan<NT>(own, wave_d, all);
    for (int i = i0; i < i1; i++) {
        const double v = value(i);
        f(i, run, v);
        run += v;
    }
    return all;
}
__device__ inline int count(int n, int *wave_n) {
    for (int d = 1; d < 64; d <<= 1) n += __shfl_xor(n, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) wave_n[threadIdx.x >> 6] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < kAllWaves; w++) n += wave_n[w];
    return n;
}

// The weights of the highest kMaxSorted, once these are sorted, take the place
// of the rest of the list.
struct Sorting {
    union {
        uint64_t list[kList];
        struct {
            uint64_t highest[kMaxSorted];
            double w[kMaxSorted];
        };
    };
};

// The token of a small top-k, from the n sorted logits down to its border.
template <int T>
__device__ inline int pick_sorted(const Task<T> &t, Sorting &s, int n, double u, double *wave_d, int *wave_n) {
    const int k = min(n, t.top_k);
    for (int i = threadIdx.x; i < k; i += kAll) s.w[i] = t.row.weight((uint32_t)(s.list[i] >> 32));
    __syncthreads();
    const auto w = [&](int i) { return s.w[i]; };
    int kept = 0;
    const double all = scan<kAll>(k, wave_d, w, [](int, double, double) {});
    const double most = all * (double)t.top_p;
    scan<kAll>(k, wave_d, w, [&](int i, double before, double v) {
        kept += i == 0 || ((t.top_p >= 1.f || before < most || t.top_p != t.top_p) && (!(t.min_p > 0.f) || v >= (double)t.min_p));
    });
    kept = count(kept, wave_n);
    // in the order of the indices: their complements, the highest first, with the places of the weights
    for (int i = threadIdx.x; i < kept; i += kAll) s.list[i] = s.list[i] << 32 | (uint32_t)i;
    __syncthreads();
    sort(s.list, kept);
    const auto in_order = [&](int i) { return s.w[(uint32_t)s.list[i]]; };
    const double target = u * scan<kAll>(kept, wave_d, in_order, [](int, double, double) {});
    int first = kept, some = 0;  // the first that is above it; the last that has a weight, and one
    scan<kAll>(kept, wave_d, in_order, [&](int i, double run, double v) {
        if (v > 0.) some = i + 1;
        if (v > 0. && run + v > target) first = min(first, i);
    });
    for (int d = 1; d < 64; d <<= 1) first = min(first, __shfl_xor(first, d)), some = max(some, __shfl_xor(some, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) wave_n[threadIdx.x >> 6] = first, wave_n[kAllWaves + (threadIdx.x >> 6)] = some;
    __syncthreads();
    for (int w = 0; w < kAllWaves; w++) first = min(first, wave_n[w]), some = max(some, wave_n[kAllWaves + w]);
    return (int)~(uint32_t)(s.list[first < kept ? first : some - 1] >> 32);
}

// The same of few, by one wave without barriers: two to a lane, in the order
// of their ranks.
constexpr int kFew = 128;
template <int T> __device__ inline int pick_few(const Task<T> &t, Sorting &s, int n, double u) {
    const int lane = threadIdx.x & 63, k = min(n, t.top_k);
    uint32_t index[2];
    double w[2];
#pragma unroll
    for (int e = 0; e < 2; e++) {
        const int i = e * 64 + lane;
        const uint64_t v = i < k ? s.list[i] : 0;
        index[e] = ~(uint32_t)v;
        w[e] = i < k ? t.row.weight((uint32_t)(v >> 32)) : 0.;
    }
    const double run[2] = {wave_scan(w[0]), wave_scan(w[1])};
    const double half = lane_of(run[0], 63), most = (half + lane_of(run[1], 63)) * (double)t.top_p;
    const double lower[2] = {__shfl_up(run[0], 1), __shfl_up(run[1], 1)};
    int kept = 0;
#pragma unroll
    for (int e = 0; e < 2; e++) {
        const double before = (e ? half : 0.) + (lane ? lower[e] : 0.);
        const bool in = e * 64 + lane < k && (t.top_p >= 1.f || before < most || t.top_p != t.top_p) && (!(t.min_p > 0.f) || w[e] >= (double)t.min_p);
        kept += __popcll(__ballot(in));
    }
    kept = max(kept, 1);
    // the running sums in the order of the indices
    double sum[2] = {0., 0.}, all = 0.;
    for (int i = 0; i < kept; i++) {
        const uint32_t o = __builtin_amdgcn_readlane(i < 64 ? index[0] : index[1], i & 63);
        const uint64_t b = __builtin_bit_cast(uint64_t, i < 64 ? w[0] : w[1]);
        const double v = __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)b, i & 63) |
                                                        (uint64_t)__builtin_amdgcn_readlane((uint32_t)(b >> 32), i & 63) << 32);
        all += v;
#pragma unroll
        for (int e = 0; e < 2; e++) sum[e] += o <= index[e] ? v : 0.;
    }
    uint32_t past = ~0u, some = 0;  // the first index above, the last with a weight, and one
#pragma unroll
    for (int e = 0; e < 2; e++)
        if (e * 64 + lane < kept && w[e] > 0.) {
            some = max(some, index[e] + 1);
            if (sum[e] > u * all) past = min(past, index[e]);
        }
    for (int d = 1; d < 64; d <<= 1) past = min(past, (uint32_t)__shfl_xor((int)past, d)), some = max(some, (uint32_t)__shfl_xor((int)some, d));
    return (int)(past != ~0u ? past : some - 1);
}

template <int T> __global__ __launch_bounds__(kThreads) void sample_border(SampleArgs a, Plan p) {
    typedef typename Elem<T>::type El;
    __shared__ uint64_t s_list[kStage];
    __shared__ int s_n;
    __shared__ uint32_t s_base;
    const int64_t r = blockIdx.x / p.slices;
    const int slice = (int)(blockIdx.x % p.slices);
    const Task<T> t = task_of<T>(a, p, p.row0 + r);
    if (t.kind != kListed && t.kind != kNumber && t.kind != kWeight) return;
    RowState &state = p.state[r];
    const bool whole = t.kind == kListed;
    int border = state.border;
    if (border < 0) {  // all of them
        if (!whole) return;
        border = kBins - 1;
    }
    uint64_t *const list = p.list + r * kList;
    if (threadIdx.x == 0) s_n = 0;
    __syncthreads();
    each_chunk<T, kWaves>(t.row, p, slice, [&](int i, const El v[8], int) {
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const float z = Elem<T>::get(v[j]);
            const int bin = bin_of(t.top, z);
            if (z != -INFINITY && (bin == border || (whole && bin < border))) {
                const int n = atomicAdd(&s_n, 1);
                const uint64_t what = (uint64_t)key_of<T>(v[j]) << 32 | (uint32_t)~(i + j);
                if (n < kStage) {
                    s_list[n] = what;
                } else {
                    const uint32_t at = atomicAdd(&state.listed, 1u);
                    if (at < kList) list[at] = what;
                }
            }
        }
    });
    __syncthreads();
    const int mine = min(s_n, kStage);
    if (mine == 0) return;
    if (threadIdx.x == 0) s_base = atomicAdd(&state.listed, (uint32_t)mine);
    __syncthreads();
    for (int i = threadIdx.x; i < mine; i += kThreads)
        if (s_base + i < kList) list[s_base + i] = s_list[i];
}

// The list of a small top-k, from the highest of each eight; its length.
template <int T> __device__ inline int list_by_eights(const Task<T> &t, const Plan &p, int64_t r, Sorting &s, int *s_n) {
    typedef typename Elem<T>::type El;
    __shared__ union {
        uint32_t bin[kBins];
        int32_t first[kList];  // of the eights that are read
    } e;
    __shared__ uint64_t wave64[kAllWaves];
    __shared__ int s_eights;
    constexpr int kAt = 8;  // loads under way
    const int n = p.chunks * (kChunk / 8), before_row = (int)((uintptr_t)t.row.z / sizeof(El) % 8);
    const El *const eights = (const El *)p.eights + r * n;
    const auto each = [&](auto &&f) {
        for (int g0 = threadIdx.x; g0 < n; g0 += kAt * kAll) {
            float m[kAt];
#pragma unroll
            for (int x = 0; x < kAt; x++) m[x] = Elem<T>::get(eights[min(g0 + x * kAll, n - 1)]);
#pragma unroll
            for (int x = 0; x < kAt; x++)
                if (g0 + x * kAll < n && m[x] != -INFINITY) f(g0 + x * kAll, bin_of(t.top, m[x]));
        }
    };
    for (int i = threadIdx.x; i < kBins; i += kAll) e.bin[i] = 0;
    if (threadIdx.x == 0) *s_n = s_eights = 0;
    __syncthreads();
    each([&](int, int bin) { atomicAdd(&e.bin[bin], 1u); });
    __syncthreads();
    uint64_t above;
    int border = crossing<kAll>([&](int i) { return (uint64_t)e.bin[i]; }, (uint64_t)t.top_k, wave64, above);
    if (border < 0) border = kBins - 1;  // all of them
    __syncthreads();
    each([&](int g, int bin) {
        if (bin > border) return;
        const int at = atomicAdd(&s_eights, 1);
        if (at < kList) e.first[at] = g * 8 - before_row;
    });
    __syncthreads();
    if (s_eights > kList) return kList + 1;  // of which each has one at least
    for (int x0 = threadIdx.x; x0 < s_eights * 8; x0 += kAt * kAll) {
        El v[kAt];
        int at[kAt];
#pragma unroll
        for (int x = 0; x < kAt; x++) {
            const int of = min(x0 + x * kAll, s_eights * 8 - 1);
            at[x] = e.first[of / 8] + of % 8;
            const bool in = x0 + x * kAll < s_eights * 8 && at[x] >= 0 && at[x] < t.row.V;
            v[x] = in ? t.row.z[at[x]] : Elem<T>::put(-INFINITY);
        }
#pragma unroll
        for (int x = 0; x < kAt; x++) {
            const float z = Elem<T>::get(v[x]);
            if (z == -INFINITY || bin_of(t.top, z) > border) continue;
            const int n = atomicAdd(s_n, 1);
            if (n < kList) s.list[n] = (uint64_t)key_of<T>(v[x]) << 32 | (uint32_t)~at[x];
        }
    }
    __syncthreads();
    return min(*s_n, kList + 1);
}

// The token of a row's sorted list; -2 where that has the border alone: then
// lowest and cut are that of thread 0.  above and all: the bins' sums above the
// border and all of them.
template <int T>
__device__ inline int resolve(const Task<T> &t, Sorting &s, int n, double u, uint64_t above, uint64_t all, double *wave_d, int *wave_n,
                              uint32_t &lowest, uint32_t &cut) {
    sort(s.list, n);
    if (t.kind == kSorted || t.kind == kListed) {
        if (n > kFew) return pick_sorted<T>(t, s, n, u, wave_d, wave_n);
        return threadIdx.x < 64 ? pick_few<T>(t, s, n, u) : 0;
    }
    int kept = 0;
    if (t.kind == kNumber) {
        kept = (int)((uint64_t)t.top_k - above);
    } else {
        const double most = (double)all * (double)t.top_p / kUnit, over = (double)above / kUnit;
        scan<kAll>(n, wave_d, [&](int i) { return t.row.weight((uint32_t)(s.list[i] >> 32)); },
                   [&](int, double before, double) { kept += over + before < most; });
        kept = count(kept, wave_n);
    }
    const uint64_t last = s.list[min(max(kept, 1), n) - 1];
    lowest = (uint32_t)(last >> 32);
    cut = ~(uint32_t)last;
    return -2;
}

// What the list says: the border, or the token.
template <int T> __global__ __launch_bounds__(kAll) void sample_sorted(SampleArgs a, Plan p) {
    __shared__ union {
        Sorting sorting;
        Shared alone;
    } s;
    __shared__ double wave_d[kAllWaves];
    __shared__ int wave_n[2 * kAllWaves], s_n;
    const int64_t r = blockIdx.x, b = p.row0 + r;
    const Task<T> t = task_of<T>(a, p, b);
    RowState &state = p.state[r];
    if (t.kind == kEvery) return;
    const double u = number_of(a, b);
    int n = (int)min(state.listed, (uint32_t)kList + 1);
    if (t.kind == kSorted) n = list_by_eights<T>(t, p, r, s.sorting, &s_n);
    int token = -2;
    if (t.kind == kToken) {
        token = t.token();
    } else if (t.kind == kAlone || n > kList) {
        token = search_row<T>(t.row, s.alone, t.top_k, t.top_p, t.min_p, u);
    } else if (t.kind != kListed && state.border < 0) {  // a top-k beyond the logits that there are: all of them
        if (threadIdx.x == 0) state.lowest = kLowest<T>, state.cut = (uint32_t)a.V, state.mode = kBordered;
    } else {
        const uint64_t *const list = p.list + r * kList;
        if (t.kind != kSorted)
            for (int i = threadIdx.x; i < n; i += kAll) s.sorting.list[i] = list[i];
        __syncthreads();
        uint32_t lowest, cut;
        token = resolve<T>(t, s.sorting, n, u, state.above, state.all, wave_d, wave_n, lowest, cut);
        if (token == -2 && threadIdx.x == 0) state.lowest = lowest, state.cut = cut, state.mode = kBordered;
    }
    if (threadIdx.x == 0 && token != -2) a.tokens[b] = token, state.mode = kDone;
}

// The weights of what is kept of a row, 0 for the others.
template <int T> struct Kept {
    Row<T> row;
    Exp<T> exp;
    float top, far, low, min_p;
    int cut;
    __device__ Kept(const Task<T> &t, const double *table, bool all, uint32_t lowest, int cut_)
        : row(t.row), exp(t.row, table), top(t.top), min_p(t.min_p) {
        low = all ? -INFINITY : value_of<T>(lowest);
        cut = all ? INT32_MIN : cut_;
        // further below the highest than this nothing is left by min-p, whatever the rounding (a weight of 1 - 10^-9
        // is below 1, one of 1 - 10^-17 is not: of a min-p of 1 a high temperature may leave all)
        far = min_p > 0.f ? (float)min((1e-9 - log((double)min_p) * 1.0001) / row.per, (double)exp.far) : exp.far;
    }
    __device__ bool in(float z, int i) const { return (z > low || (z == low && i <= cut)) && !(top - z > far); }
    __device__ double weight(typename Elem<T>::type v, int i) const {
        const float z = Elem<T>::get(v);
        if (!in(z, i)) return 0.;
        const double w = exp(z);
        return !(min_p > 0.f) || w >= (double)min_p ? w : 0.;
    }
    // Of a wave's part of a slice: put(chunk, sum of its weights), by one lane.
    template <int NW, typename F> __device__ void sums(const Plan &p, int slice, F &&put) const {
        each_group<T, NW>(row, p, slice, [&](int c0, int end, const typename Elem<T>::type v[kAhead][8]) {
            double sum[kAhead];
#pragma unroll
            for (int n = 0; n < kAhead; n++) {
                sum[n] = 0.;
                if (c0 + n * NW < end) {
                    const int i = index_of(row, c0 + n * NW);
                    float z[8];
                    bool is[8], any = false;
                    double w[8];
#pragma unroll
                    for (int j = 0; j < 8; j++) z[j] = Elem<T>::get(v[n][j]), is[j] = in(z[j], i + j), any |= is[j];
                    if (__ballot(any)) {
                        exp.eight(z, is, w);
#pragma unroll
                        for (int j = 0; j < 8; j++) sum[n] += !(min_p > 0.f) || w[j] >= (double)min_p ? w[j] : 0.;
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < kAhead; n++) sum[n] = wave_sum(sum[n]);
#pragma unroll
            for (int n = 0; n < kAhead; n++)
                if ((int)(threadIdx.x & 63) == n && c0 + n * NW < end) put(c0 + n * NW, sum[n]);
        });
    }
    // The token, from all chunks' sums (in LDS); in all threads.
    template <int NT> __device__ int find(const double *s_sum, int chunks, double u, double *wave_d, int *wave_n) const {
        __shared__ double s_before;
        const int lane = threadIdx.x & 63;
        double target = 0., before = 0.;
        int n = chunks, i0 = 0, at = 0;
#pragma unroll 1
        for (int step = 0; step < 2; step++) {  // the chunk, and the logit in it
            const auto value = [&](int i) {
                if (step == 0) return s_sum[i];
                return i0 + i >= 0 && i0 + i < row.V ? weight(row.z[i0 + i], i0 + i) : 0.;
            };
            int first = n, some = -1;  // the first above the target; the last that has a weight
            double before_first = 0., before_some = 0.;
            for (int pass = step; pass < 2; pass++) {
                const double sum = scan<NT>(n, wave_d, value, [&](int i, double run, double v) {
                    if (pass == 0 || !(v > 0.)) return;
                    some = i, before_some = before + run;
                    if (first == n && before + run + v > target) first = i, before_first = before + run;
                });
                if (pass == 0) target = u * sum;
            }
            int f = first, o = some;
            for (int d = 1; d < 64; d <<= 1) f = min(f, __shfl_xor(f, d)), o = max(o, __shfl_xor(o, d));
            __syncthreads();
            if (lane == 0) wave_n[threadIdx.x >> 6] = f, wave_n[NT / 64 + (threadIdx.x >> 6)] = o;
            if (threadIdx.x == 0) s_before = before;
            __syncthreads();
            for (int w = 0; w < NT / 64; w++) f = min(f, wave_n[w]), o = max(o, wave_n[NT / 64 + w]);
            at = f < n ? f : max(o, 0);
            if (f < n ? first == f : o >= 0 && some == o) s_before = f < n ? before_first : before_some;
            __syncthreads();
            before = s_before;
            if (step == 0) i0 = at * kChunk - (int)((uintptr_t)row.z / sizeof(*row.z) % 8), n = kChunk;
        }
        return i0 + at;
    }
};

template <int T> __global__ __launch_bounds__(kThreads) void sample_pick(SampleArgs a, Plan p) {
    __shared__ double wave_d[kWaves], s_sum[kMaxChunks], s_table[kTable];
    __shared__ int wave_n[2 * kWaves], s_last;
    const int64_t r = blockIdx.x / p.slices, b = p.row0 + r;
    const int slice = (int)(blockIdx.x % p.slices);
    const Task<T> t = task_of<T>(a, p, b);
    RowState &state = p.state[r];
    if (t.kind == kToken) {
        if (slice == 0 && threadIdx.x == 0) a.tokens[b] = t.token();
        return;
    }
    if (t.kind != kEvery && state.mode != kBordered) return;
    fill(s_table);
    __syncthreads();
    const Kept<T> kept(t, s_table, t.kind == kEvery, state.lowest, (int)state.cut);
    double *const sums = p.sums + r * p.chunks;
    kept.template sums<kWaves>(p, slice, [&](int c, double sum) { __hip_atomic_store(&sums[c], sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); });
    if (!last_of(&state.picked, p.slices, &s_last)) return;
    for (int i = threadIdx.x; i < p.chunks; i += kThreads) s_sum[i] = at_device(&sums[i]);
    __syncthreads();
    const int token = kept.template find<kThreads>(s_sum, p.chunks, number_of(a, b), wave_d, wave_n);
    if (threadIdx.x == 0) a.tokens[b] = token;
}

// How rows are cut: into slices that together fill the GPU several times.
Plan plan_of(int64_t rows, int V, uint8_t *ws) {
    Plan p = {};
    p.chunks = (V + 7 + kChunk - 1) / kChunk;  // wherever a row begins
    const int most = (int)std::min<int64_t>({(int64_t)kMaxSlices, std::max<int64_t>(1, kSliceGroups / rows), (int64_t)(p.chunks + kWaves - 1) / kWaves});
    p.chunks_of_slice = (p.chunks + most - 1) / most;
    p.slices = (p.chunks + p.chunks_of_slice - 1) / p.chunks_of_slice;
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t n = at; at += (bytes + 255) / 256 * 256; return ws + n; };
    p.tops = (uint64_t *)take((size_t)rows * p.slices * 8);
    p.eights = take((size_t)rows * p.chunks * (kChunk / 8) * 4);
    p.bins = (uint64_t *)take((size_t)rows * kBins * 8);
    p.list = (uint64_t *)take((size_t)rows * kList * 8);
    p.sums = (double *)take((size_t)rows * p.chunks * 8);
    p.state = (RowState *)take((size_t)rows * sizeof(RowState));
    p.row0 = (int64_t)at;  // the size, for the query
    return p;
}

template <int T> sim_status sample_t(hipStream_t st, const SampleArgs &a, uint8_t *ws) {
    const bool some_k = a.top_k || (a.all_k > 1 && a.all_k < a.V), some_p = a.top_p || a.all_p < 1.f;
    // where one top-k is for all rows, what they need is known; else all of it may be
    const bool small = !a.top_k && some_k && a.all_k <= kMaxSorted, sorted = small && by_eights(a.V, a.all_k);
    for (int64_t row0 = 0; row0 < a.B; row0 += kRows) {
        const int64_t rows = std::min<int64_t>(kRows, a.B - row0);
        Plan p = plan_of(rows, a.V, ws);
        p.row0 = row0;
        const uint32_t grid = (uint32_t)(rows * p.slices);
        sample_tops<T><<<grid, kThreads, 0, st>>>(a, p, some_k);
        if ((some_k || some_p) && !sorted) {
            sample_bins<T><<<grid, kThreads, 0, st>>>(a, p);
            sample_border<T><<<grid, kThreads, 0, st>>>(a, p);
        }
        if (some_k || some_p) sample_sorted<T><<<(uint32_t)rows, kAll, 0, st>>>(a, p);
        if (!small) sample_pick<T><<<grid, kThreads, 0, st>>>(a, p);
    }
    return SIM_OPS_LAUNCH_OK();
}

}  // namespace

size_t sample_workspace(int64_t B, int V) { return (size_t)plan_of(std::min<int64_t>(B, kRows), V, nullptr).row0; }

sim_status launch_sample(hipStream_t st, const SampleArgs &a, void *ws) {
    if (a.type == SIM_TYPE_F32) return sample_t<SIM_TYPE_F32>(st, a, (uint8_t *)ws);
    if (a.type == SIM_TYPE_F16) return sample_t<SIM_TYPE_F16>(st, a, (uint8_t *)ws);
    return sample_t<SIM_TYPE_BF16>(st, a, (uint8_t *)ws);
}

}  // namespace simops
