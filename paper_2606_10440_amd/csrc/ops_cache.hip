// Paged key-value cache: new rows into it, and the attention of one new token
// of each sequence over it.
//
// A cache is pages of [kv heads][page size][D]; a sequence's tokens lie on the
// pages of its row of the page table.
#include "ops_common.h"

namespace simops {
namespace {

typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------------ append

// A thread moves one piece of PIECE elements: sixteen bytes where the rows are
// aligned to that.  It is a copy, bound by memory: 20011 tokens of 8 x 128, 164 MB
// read and written, 27 us (6 TB/s); 64 tokens 3.0 us, launch.
template <int PIECE>
__global__ __launch_bounds__(256) void append_rows(AppendArgs a, int pieces_of_row, int64_t pieces) {
    const bool is_v = blockIdx.y;
    const uint16_t *const from = (const uint16_t *)(is_v ? a.v : a.k);
    uint16_t *const to = (uint16_t *)(is_v ? a.v_cache : a.k_cache);
    const int64_t stride = is_v ? a.v_stride : a.k_stride, head_stride = is_v ? a.v_head_stride : a.k_head_stride;
    const int64_t page_stride = is_v ? a.v_page_stride : a.k_page_stride;
    const int pieces_of_token = pieces_of_row * a.heads;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t t = pieces <= 0x7fffffff ? (uint32_t)i / (uint32_t)pieces_of_token : i / pieces_of_token;
        const int64_t slot = a.slots[t];
        if (slot < 0 || slot >= a.pages * a.page_size) continue;
        const int in_token = (int)(i - t * pieces_of_token), h = in_token / pieces_of_row, d = (in_token - h * pieces_of_row) * PIECE;
        const int64_t page = slot <= 0x7fffffff ? (uint32_t)slot / (uint32_t)a.page_size : slot / a.page_size;
        const int64_t at = slot - page * a.page_size;
        const uint16_t *const p = from + t * stride + h * head_stride + d;
        uint16_t *const o = to + page * page_stride + (h * (int64_t)a.page_size + at) * a.D + d;
        if (PIECE == 8) *(u32x4 *)o = *(const u32x4 *)p;
        else *o = *p;
    }
}

// ------------------------------------------------------------------ attention

constexpr int kWaves = 4;
constexpr int kKeys = kAttendKeys;  // keys of one step of a wave

template <int T> __device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (T == SIM_TYPE_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

template <int T> __device__ inline uint32_t pack(float x, float y) {
    typedef typename Elem<T>::type E;
    const E v[2] = {Elem<T>::put(x), Elem<T>::put(y)};
    return __builtin_bit_cast(uint16_t, v[0]) | (uint32_t)__builtin_bit_cast(uint16_t, v[1]) << 16;
}
template <int T> __device__ inline float half_of(uint32_t w, int i) {
    return Elem<T>::get(__builtin_bit_cast(typename Elem<T>::type, (uint16_t)(i ? w >> 16 : w)));
}

// What the highest weight is.
template <int T> constexpr float kLog2Times = T == SIM_TYPE_F16 ? 15.f : 0.f;
template <int T> constexpr float kTimes = T == SIM_TYPE_F16 ? 32768.f : 1.f;

// Sums over the lanes up to each, by moves between registers: every workgroup
// begins with two of them.
template <int CTRL, int ROWS> __device__ inline uint32_t add_from(uint32_t v) {
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
__device__ inline uint32_t wave_scan(uint32_t v) {
    v = add_from<0x111, 0xf>(v);  // from the lane before, of its row of 16
    v = add_from<0x112, 0xf>(v);
    v = add_from<0x114, 0xf>(v);
    v = add_from<0x118, 0xf>(v);
    v = add_from<0x142, 0xa>(v);     // lane 15's and 47's to the rows after
    return add_from<0x143, 0xc>(v);  // lane 31's to the upper half
}

// Where a sequence's keys lie: steps of kKeys from first_step on.
struct Span {
    int start, end, first_step, steps;
};
__device__ inline Span span_of(const AttendArgs &a, int64_t b) {
    Span s;
    b = min(b, a.B - 1);
    s.end = (int)min((int64_t)max(a.lengths[b], 0), a.capacity);
    s.start = a.window > 0 ? max(0, s.end - a.window) : 0;
    s.first_step = s.start / kKeys;
    s.steps = (s.end + kKeys - 1) / kKeys - s.first_step;
    return s;
}

// How the sequences are cut: into units of so many steps, the same for all,
// so that long sequences among short ones are shared alike; a sequence has one
// unit at least.  Every wave works that out from all lengths by itself; first
// is what lane holds of the first 64, which are not loaded twice.
__device__ inline int steps_of_unit(const AttendArgs &a, const Span &first) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int64_t b0 = 0; b0 < a.B; b0 += 64) {  // (64 times 2^25 fit 32 bits without a sign)
        const int steps = b0 ? span_of(a, b0 + lane).steps : first.steps;
        total += (uint32_t)__builtin_amdgcn_readlane((int)wave_scan(b0 + lane < a.B ? steps : 0), 63);
    }
    return attend_unit(total, a.units);
}
__device__ inline int units_of(int steps, int unit) { return max(1, (steps + unit - 1) / unit); }
// The units up to sequence b0 + lane from b0 on, whose span is s.
__device__ inline int scan_units(const AttendArgs &a, int64_t b0, const Span &s, int unit) {
    return (int)wave_scan(b0 + (int)(threadIdx.x & 63) < a.B ? units_of(s.steps, unit) : 0);
}

// One unit of one sequence and kv head, for up to 16 HT of the heads that
// share it.  Everything is computed transposed, scores as [key][head] and
// results as [d][head], so that a lane's scores are of one head, and are the
// second product's operand where they stand: the products' k axis may take
// the keys in any order, so lane (r, g) of 16 x 4 has keys 4 g + i and 16 + 4 g
// + i of a step in both.  Of the values it loads, for these eight keys, eight
// consecutive d: an 8 x 8 block whose columns, put together in registers, are
// the operands for rows d = 8 r + m.  Nothing goes through LDS but the waves'
// results at the end.
//
// Weights are rounded in two parts, which keep 16 bits (bf16) or 22 (fp16) of
// them: rounded once they would add as much error as rounding the result does.
// fp16 weights are 2^15 times as large as the highest's 1, so that small ones,
// of which a long sequence may have many, are not lost: multiplied by that, since
// a distance of 15 would be rounded with the scores (from 2^24 on to 16, whose 2^16
// fp16 does not hold).
//
// Memory bounds it: 64 sequences of up to 8192 tokens, 8 heads of 128 for 32, 183
// us for 1.1 GB; two of 131072, 64 heads, 175 us (5.9 TB/s), and 7 to 8 us for
// joining the units.  More heads to a kv head than 16 (32 up to D = 128) read the
// keys again from the caches: 64 heads on one of D = 256, 296 us for 0.5 GB.  One
// sequence of 300: 8 us, the chain of lengths, table, keys and values and the
// waves' joint.  Pages of no whole 16 tokens exchange a row's offset for each key,
// which costs 2 to 4 % (64 sequences of up to 8192, fresh ones: 221 us, pages of 24, and 216 of 16).
template <int T, int DP, int HT, bool PAGE16>
__global__ __launch_bounds__(64 * kWaves, attend_resident(DP, 16 * HT)) void attend(AttendArgs a) {
    constexpr int CH = DP / 32;                // 32 d of keys
    constexpr int NV = DP == 64 ? 4 : 8;       // consecutive d of values in a lane
    constexpr int NH = DP / (16 * NV);         // times that
    constexpr int kPitch = DP + 4;
    __shared__ float s_o[kWaves][16][kPitch];
    __shared__ float s_m[kWaves][HT * 16], s_l[kWaves][HT * 16];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    // workgroups that read the same keys for other heads are eight apart: on one XCD
    const int per8 = 8 * a.tiles, tile = (int)(blockIdx.x % per8 / 8), at = (int)(blockIdx.x / per8 * 8 + blockIdx.x % 8);
    const int kvh = at % a.kv_heads, u = at / a.kv_heads;

    // the unit's sequence
    int64_t b = a.splits || u >= a.B ? -1 : u;
    int before = u, n_units = 1, unit = kAttendWhole;
    const Span first = span_of(a, a.splits ? lane : u);
    Span sp = first;
    if (a.splits) unit = __builtin_amdgcn_readfirstlane(steps_of_unit(a, first));
    for (int64_t b0 = 0, base = 0; a.splits && b0 < a.B; b0 += 64) {
        const Span s = b0 ? span_of(a, b0 + lane) : first;
        const int n = scan_units(a, b0, s, unit);
        const uint64_t past = __ballot((int64_t)u < base + n);
        if (past) {
            const int l = __ffsll((unsigned long long)past) - 1;
            b = b0 + l;
            const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
            sp = {of(s.start), of(s.end), of(s.first_step), of(s.steps)};
            before = (int)base + (l ? __builtin_amdgcn_readlane(n, l - 1) : 0);
            n_units = (int)base + of(n) - before;
            break;
        }
        base += __builtin_amdgcn_readlane(n, 63);
    }
    if (b < 0) return;  // the whole workgroup: no such unit
    b = __builtin_amdgcn_readfirstlane((int)b);
    before = __builtin_amdgcn_readfirstlane(before);
    n_units = __builtin_amdgcn_readfirstlane(n_units);
    sp.start = __builtin_amdgcn_readfirstlane(sp.start);
    sp.end = __builtin_amdgcn_readfirstlane(sp.end);
    const int step_end = sp.first_step + min(sp.steps, (u - before + 1) * unit);
    int step = __builtin_amdgcn_readfirstlane(sp.first_step + (u - before) * unit + wave);
    const int last = __builtin_amdgcn_readfirstlane(step_end);

    const int group = a.q_heads / a.kv_heads, h0 = tile * 16 * HT, D = a.D;
    const bool partial = D != DP;
    u32x4 q[HT][CH];
#pragma unroll
    for (int t = 0; t < HT; t++)
#pragma unroll
        for (int c = 0; c < CH; c++) {
            const int h = h0 + t * 16 + r, d = c * 32 + g * 8;
            q[t][c] = u32x4{0};
            if (h < group && d < D) {
                const uint16_t *p = (const uint16_t *)a.q + b * a.q_stride + (int64_t)(kvh * group + h) * a.q_head_stride + d;
                if (a.q_aligned) {
                    q[t][c] = *(const u32x4 *)p;
                } else {
                    u16x8 v;
#pragma unroll
                    for (int i = 0; i < 8; i++) v[i] = p[i];
                    q[t][c] = __builtin_bit_cast(u32x4, v);
                }
            }
        }

    const int32_t *const table = a.table + b * a.table_stride;
    const uint16_t *const kc = (const uint16_t *)a.k_cache + (int64_t)kvh * a.page_size * D;
    const uint16_t *const vc = (const uint16_t *)a.v_cache + (int64_t)kvh * a.page_size * D;

    // lane's key of a step (32 of them, twice) and its page
    const auto page_of = [&](int s) {
        const int key = min(s * kKeys + (lane & (kKeys - 1)), sp.end - 1);
        return s < last ? table[(uint32_t)key / (uint32_t)a.page_size] : -1;
    };
    // which of the step's keys there are
    const auto keys_of = [&](int s, int page) {
        const int key = s * kKeys + (lane & (kKeys - 1));
        return (uint32_t)__ballot(key >= sp.start && key < sp.end && page >= 0 && page < a.pages);
    };
    // offsets of this lane's rows of a step of which there is a key; a key
    // that is not there takes another's row
    struct Rows {
        int64_t base[2];  // PAGE16: of sixteen keys, the same in all lanes
        int64_t mine;     // else: of key lane & 31
    };
    const auto rows_of = [&](int s, int page, uint32_t there, int64_t page_stride) {
        Rows o;
        const int key = s * kKeys;
        if (PAGE16) {
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const int from = (there >> (16 * j)) & 0xffff ? j : 1 - j;
                const int p = __builtin_amdgcn_readlane(page, 16 * from);
                const int in = (int)((uint32_t)(key + 16 * from) % (uint32_t)a.page_size);
                o.base[j] = p * page_stride + (int64_t)in * D;
            }
        } else {
            const int l = lane & (kKeys - 1), from = (there >> l) & 1 ? l : __ffs(there) - 1;
            const int p = __shfl(page, from), in = (int)((uint32_t)(key + from) % (uint32_t)a.page_size);
            o.mine = p * page_stride + (int64_t)in * D;
        }
        return o;
    };
    const auto row_at = [&](const Rows &o, int j, int i) {  // key i of 16 in half j
        if (PAGE16) return o.base[j] + (int64_t)i * D;
        return (int64_t)__shfl((long long)o.mine, j * 16 + i);
    };

    u32x4 k[2][CH];
    const auto load_keys = [&](int s, int page, uint32_t there) {
        const Rows o = rows_of(s, page, there, a.k_page_stride);
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const uint16_t *p = kc + row_at(o, j, r);
#pragma unroll
            for (int c = 0; c < CH; c++) {
                const int d = c * 32 + g * 8;
                k[j][c] = __builtin_nontemporal_load((const u32x4 *)(p + (partial ? min(d, D - 8) : d)));
            }
        }
    };

    f32x4 o[HT][NH * NV];
    float m[HT], l[HT];
#pragma unroll
    for (int t = 0; t < HT; t++) {
        m[t] = -INFINITY;
        l[t] = 0.f;
#pragma unroll
        for (int i = 0; i < NH * NV; i++) o[t][i] = f32x4{0};
    }

    int page = page_of(step), page_next = page_of(step + kWaves);
    uint32_t there = 0;
    if (step < last) {
        there = keys_of(step, page);
        if (there) load_keys(step, page, there);
    }
    for (; step < last; step += kWaves) {
        const int page_after = page_of(step + 2 * kWaves);
        uint32_t w[NH][8][NV / 2];  // values of the lane's eight keys
        f32x4 s[HT][2];
        if (there) {
            const Rows rows = rows_of(step, page, there, a.v_page_stride);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const uint16_t *p = vc + row_at(rows, e >> 2, g * 4 + (e & 3));
#pragma unroll
                for (int h = 0; h < NH; h++) {
                    const int d = h * 128 + r * NV;
                    const uint16_t *at = p + (partial ? min(d, D - NV) : d);
                    if constexpr (NV == 8) {
                        const u32x4 v = __builtin_nontemporal_load((const u32x4 *)at);
#pragma unroll
                        for (int i = 0; i < 4; i++) w[h][e][i] = v[i];
                    } else {
                        const u32x2 v = __builtin_nontemporal_load((const u32x2 *)at);
                        w[h][e][0] = v[0], w[h][e][1] = v[1];
                    }
                }
            }
            if (partial) {
#pragma unroll
                for (int j = 0; j < 2; j++)
#pragma unroll
                    for (int c = 0; c < CH; c++) k[j][c] = c * 32 + g * 8 < D ? k[j][c] : u32x4{0};
            }
#pragma unroll
            for (int t = 0; t < HT; t++)
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    s[t][j] = f32x4{0};
#pragma unroll
                    for (int c = 0; c < CH; c++) s[t][j] = mfma<T>(k[j][c], q[t][c], s[t][j]);
                }
        }
        const uint32_t now = there;
        there = 0;
        if (step + kWaves < last) {
            there = keys_of(step + kWaves, page_next);
            if (there) load_keys(step + kWaves, page_next, there);
        }
        page = page_next;
        page_next = page_after;
        if (!now) continue;

        if (now != 0xffffffffu) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const bool is = (now >> ((e >> 2) * 16 + g * 4 + (e & 3))) & 1;
#pragma unroll
                for (int h = 0; h < NH; h++)
#pragma unroll
                    for (int i = 0; i < NV / 2; i++) w[h][e][i] = is ? w[h][e][i] : 0;  // 0 times what lies there may be NaN
            }
        }
        u32x4 hi[HT], lo[HT];
#pragma unroll
        for (int t = 0; t < HT; t++) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = s[t][e >> 2][e & 3] * a.scale_log2;
            if (now != 0xffffffffu) {
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = (now >> ((e >> 2) * 16 + g * 4 + (e & 3))) & 1 ? v[e] : -INFINITY;
            }
            float top = m[t];
#pragma unroll
            for (int e = 0; e < 8; e++) top = fmaxf(top, v[e]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float off = top == -INFINITY ? 0.f : top;
            if (__ballot(top > m[t])) {
                const float less = __builtin_amdgcn_exp2f(m[t] - off);
                m[t] = top;
                l[t] *= less;
#pragma unroll
                for (int i = 0; i < NH * NV; i++) o[t][i] *= less;
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {
                v[e] = __builtin_amdgcn_exp2f(v[e] - off) * kTimes<T>;
                l[t] += v[e];
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                hi[t][i] = pack<T>(v[2 * i], v[2 * i + 1]);
                lo[t][i] = pack<T>(v[2 * i] - half_of<T>(hi[t][i], 0), v[2 * i + 1] - half_of<T>(hi[t][i], 1));
            }
        }
#pragma unroll
        for (int h = 0; h < NH; h++)
#pragma unroll
            for (int c = 0; c < NV; c++) {
                u32x4 x;
#pragma unroll
                for (int i = 0; i < 4; i++)
                    x[i] = __builtin_amdgcn_perm(w[h][2 * i + 1][c / 2], w[h][2 * i][c / 2], c & 1 ? 0x07060302 : 0x05040100);
#pragma unroll
                for (int t = 0; t < HT; t++) o[t][h * NV + c] = mfma<T>(x, hi[t], mfma<T>(x, lo[t], o[t][h * NV + c]));
            }
    }

    // the waves' results together; lane (r, g): head r, d = 128 h + (4 g + i) NV + c
#pragma unroll
    for (int t = 0; t < HT; t++) {
        l[t] += __shfl_xor(l[t], 16);
        l[t] += __shfl_xor(l[t], 32);
        if (g == 0) s_m[wave][t * 16 + r] = m[t], s_l[wave][t * 16 + r] = l[t];
    }
    __syncthreads();
    float *const part = a.part;  // [unit][q head][D], then [unit][q head] of maximum and sum
    float *const stat = a.part + (int64_t)a.max_units * a.q_heads * D;
#pragma unroll
    for (int t = 0; t < HT; t++) {
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWaves; w++) top = fmaxf(top, s_m[w][t * 16 + r]);
        const float less = m[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[t] - top);
        if (t) __syncthreads();
#pragma unroll
        for (int h = 0; h < NH; h++)
#pragma unroll
            for (int i = 0; i < 4; i++)
#pragma unroll
                for (int c = 0; c < NV; c += 4) {
                    f32x4 v;
#pragma unroll
                    for (int x = 0; x < 4; x++) v[x] = o[t][h * NV + c + x][i] * less;
                    *(f32x4 *)&s_o[wave][r][h * 128 + (g * 4 + i) * NV + c] = v;
                }
        __syncthreads();
        const int pieces = D / 8;
        for (int x = threadIdx.x; x < 16 * pieces; x += 64 * kWaves) {
            const int head = x / pieces, d = (x - head * pieces) * 8, h = h0 + t * 16 + head;
            if (h >= group) break;
            float top = -INFINITY, sum = 0.f, v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < kWaves; w++) top = fmaxf(top, s_m[w][t * 16 + head]);
#pragma unroll
            for (int w = 0; w < kWaves; w++) {
                const float mw = s_m[w][t * 16 + head];
                sum += s_l[w][t * 16 + head] * (mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - top));
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] += s_o[w][head][d + i];
            }
            const int qh = kvh * group + h;
            if (n_units == 1) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                u32x4 out;
#pragma unroll
                for (int i = 0; i < 4; i++) out[i] = pack<T>(v[2 * i] * inv, v[2 * i + 1] * inv);
                uint16_t *p = (uint16_t *)a.out + b * a.out_stride + (int64_t)qh * D + d;
                if (a.out_aligned) {
                    *(u32x4 *)p = out;
                } else {
#pragma unroll
                    for (int i = 0; i < 8; i++) p[i] = (uint16_t)(out[i / 2] >> (16 * (i & 1)));
                }
                if (a.lse && d == 0) a.lse[b * a.q_heads + qh] = sum == 0.f ? -INFINITY : (top + (log2f(sum) - kLog2Times<T>)) * 0.69314718056f;
            } else {
                float *p = part + ((int64_t)u * a.q_heads + qh) * D + d;
                *(f32x4 *)p = f32x4{v[0], v[1], v[2], v[3]};
                *(f32x4 *)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
                if (d == 0) {
                    stat[((int64_t)u * a.q_heads + qh) * 2] = top;
                    stat[((int64_t)u * a.q_heads + qh) * 2 + 1] = sum;
                }
            }
        }
    }
}

// The units of a sequence together: a workgroup for each head; threads in
// groups of D / 4, each with every n-th unit, added up in the groups' order.  A
// launch of its own, since the last workgroup to arrive could not know how many
// there are to wait for without a count that something has cleared before.
template <int T> __global__ __launch_bounds__(256) void attend_join(AttendArgs a) {
    __shared__ f32x4 s_v[256];
    __shared__ float s_top[4];
    const int64_t b = blockIdx.x / a.q_heads;
    const int h = (int)(blockIdx.x % a.q_heads), lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.D;
    const Span first = span_of(a, lane);
    const int unit = steps_of_unit(a, first), n = units_of(span_of(a, b).steps, unit);
    if (n == 1) return;  // it is written
    int u0 = 0;
    for (int64_t b0 = 0; b0 < b; b0 += 64) {
        const int s = scan_units(a, b0, b0 ? span_of(a, b0 + lane) : first, unit);
        u0 += __builtin_amdgcn_readlane(s, (int)min((int64_t)63, b - 1 - b0));
    }
    const float *const part = a.part + ((int64_t)u0 * a.q_heads + h) * D;
    const float *const stat = a.part + (int64_t)a.max_units * a.q_heads * D + ((int64_t)u0 * a.q_heads + h) * 2;
    const int64_t next = (int64_t)a.q_heads;  // from one unit to the next
    float top = -INFINITY;
    for (int i = threadIdx.x; i < n; i += 256) top = fmaxf(top, stat[i * next * 2]);
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    if (lane == 0) s_top[wave] = top;
    __syncthreads();
    top = fmaxf(fmaxf(s_top[0], s_top[1]), fmaxf(s_top[2], s_top[3]));
    const int lanes = D / 4, groups = 256 / lanes, mine = threadIdx.x / lanes, d = (threadIdx.x - mine * lanes) * 4;
    f32x4 v = {0};
    float sum = 0.f;
    if (mine < groups)
        for (int i0 = mine; i0 < n; i0 += 4 * groups) {
            f32x4 x[4];
            float w[4], y[4];
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int c = min(i0 + j * groups, n - 1);
                x[j] = *(const f32x4 *)(part + c * next * D + d);
                w[j] = stat[c * next * 2];
                y[j] = stat[c * next * 2 + 1];
            }
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (i0 + j * groups < n) {
                    const float f = w[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w[j] - top);  // (0 times NaN is kept)
                    v += x[j] * f;
                    sum += y[j] * f;
                }
        }
    s_v[threadIdx.x] = v;
    // the sum over the groups, of any d
    __shared__ float s_part[256];
    s_part[threadIdx.x] = sum;
    __syncthreads();
    if ((int)threadIdx.x >= lanes) return;
    for (int j = 1; j < groups; j++) {
        v += s_v[j * lanes + threadIdx.x];
        sum += s_part[j * lanes + threadIdx.x];
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t *p = (uint16_t *)a.out + b * a.out_stride + (int64_t)h * D + d;
    const u32x2 out = {pack<T>(v[0] * inv, v[1] * inv), pack<T>(v[2] * inv, v[3] * inv)};
    if (a.out_aligned) {
        *(u32x2 *)p = out;
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) p[i] = (uint16_t)(out[i / 2] >> (16 * (i & 1)));
    }
    if (a.lse && threadIdx.x == 0)
        a.lse[b * a.q_heads + h] = sum == 0.f ? -INFINITY : (top + (log2f(sum) - kLog2Times<T>)) * 0.69314718056f;
}

template <int T, int DP, int HT> void attend_t(hipStream_t st, const AttendArgs &a) {
    const uint32_t units = (uint32_t)(a.max_units * a.kv_heads), grid = (units + 7) / 8 * 8 * a.tiles;
    if (a.page_size % 16 == 0) attend<T, DP, HT, true><<<grid, 64 * kWaves, 0, st>>>(a);
    else attend<T, DP, HT, false><<<grid, 64 * kWaves, 0, st>>>(a);
}

template <int T> sim_status attention_t(hipStream_t st, const AttendArgs &a) {
    const int heads = attend_heads(a.q_heads / a.kv_heads, a.D);
    if (a.D <= 64) heads == 16 ? attend_t<T, 64, 1>(st, a) : attend_t<T, 64, 2>(st, a);
    else if (a.D <= 128) heads == 16 ? attend_t<T, 128, 1>(st, a) : attend_t<T, 128, 2>(st, a);
    else attend_t<T, 256, 1>(st, a);
    if (a.splits) attend_join<T><<<(uint32_t)(a.B * a.q_heads), 256, 0, st>>>(a);
    return SIM_OPS_LAUNCH_OK();
}

}  // namespace

sim_status launch_append(hipStream_t st, const AppendArgs &a) {
    const bool wide = ((uintptr_t)a.k | (uintptr_t)a.v | (uint64_t)(a.k_stride | a.v_stride | a.k_head_stride | a.v_head_stride) * 2) % 16 == 0;
    const int of_row = wide ? a.D / 8 : a.D;
    const int64_t pieces = a.T * a.heads * of_row;
    const dim3 grid((uint32_t)std::min<int64_t>((pieces + 255) / 256, 1 << 20), 2);
    if (wide) append_rows<8><<<grid, 256, 0, st>>>(a, of_row, pieces);
    else append_rows<1><<<grid, 256, 0, st>>>(a, of_row, pieces);
    return SIM_OPS_LAUNCH_OK();
}

sim_status launch_attention(hipStream_t st, const AttendArgs &a) {
    return a.type == SIM_TYPE_F16 ? attention_t<SIM_TYPE_F16>(st, a) : attention_t<SIM_TYPE_BF16>(st, a);
}

}  // namespace simops
