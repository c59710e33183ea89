// Which of its kernels' forms an operator takes for given sizes: plain host
// rules, so that tests can ask which form a size runs.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <utility>

namespace simops {

constexpr int kGroup = 256;       // columns to which a 4-bit row is padded
constexpr int kGroupCodes = 128;  // its bytes of codes
constexpr int kGroupScales = 8;   // and of scales

constexpr int64_t groups_of(int64_t K) { return (K + kGroup - 1) / kGroup; }

// ------------------------------------------------------------------ 4-bit products

constexpr int kSkinnyRows = 32;
constexpr int kSkinnyLds[2] = {49152, 147456};  // bytes of A: three workgroups on a compute unit, or one
constexpr int64_t kOwnQuantize = 16384;         // elements of A that every workgroup puts into 4 bits itself

enum ProductForm { kSkinnySmall, kSkinnyLarge, kTile256x256, kTile128x128, kTile64x128, kTile64x64, kSimple };

inline size_t skinny_lds(int64_t M, int64_t K) { return (size_t)(M * (groups_of(K) * (kGroupCodes + kGroupScales) + 16)); }
inline bool skinny(int64_t M, int64_t K) {
    return M <= kSkinnyRows && K > 0 && K < (1 << 20) && skinny_lds(M, K) <= (size_t)kSkinnyLds[1];
}
// A launch less where every workgroup can put the few rows into 4 bits itself.
inline bool linear_in_one(int64_t M, int64_t K) { return skinny(M, K) && M * K <= kOwnQuantize; }

inline ProductForm product_form(int64_t M, int64_t N, int64_t K) {
    if (skinny(M, K)) return skinny_lds(M, K) <= (size_t)kSkinnyLds[0] ? kSkinnySmall : kSkinnyLarge;
    if (K == 0 || K >= (1 << 23)) return kSimple;  // else offsets within a tile fit in 32 bits
    // The tile by what 256 of it at a time cost, in microseconds for 4096
    // columns (measured, beside some 4 for each launch: 64 tiles or 256 of
    // a kind take the same time; 4096 x 4096 in 256 tiles of 256 x 256
    // 43 us, in 1024 of 128 x 128 54; 333 x 5001 x 2056 9.1, 11.1 and 11.3
    // us in tiles of 64 x 128, 64 x 64 and 128 x 128).
    const auto cost = [&](int64_t bm, int64_t bn, double each) {
        return (double)((((M + bm - 1) / bm) * ((N + bn - 1) / bn) + 255) / 256) * each;
    };
    const double c[4] = {cost(256, 256, 38.), cost(128, 128, 12.5), cost(64, 128, 9.2), cost(64, 64, 6.6)};
    return (ProductForm)(kTile256x256 + (std::min_element(c, c + 4) - c));
}

// ------------------------------------------------------------------ experts' layer

constexpr int kFewTokens = 16;
constexpr int kFewExperts = 256;
constexpr int kFewInputs = 24576;  // bytes of inputs that a workgroup of the first kernel keeps in LDS
constexpr uint32_t kSlots = 512;   // workgroups of the forms for more tokens that run at once: two on each of 256 compute units

constexpr int kShortList = 10;     // tokens: up to this average, one column tile

enum LayerForm { kFew, kGroup1, kGroup2, kGroup4 };  // with so many column tiles of sixteen tokens

inline bool few(int64_t T, int E, int64_t D, int64_t F) { return T <= kFewTokens && E <= kFewExperts && D >= 8 && F >= 8; }
// Bytes from one input to the next in LDS, of D columns in steps of cols:
// sixteen rows start in different banks.
constexpr int few_input_pitch(int D, int cols) { return (D + cols - 1) / cols * cols * 2 + 16; }

inline LayerForm layer_form(int64_t T, int E, int k, int64_t D, int64_t F, bool mx4) {
    if (few(T, E, D, F)) return kFew;
    // columns by the tokens of an average expert (lists of 19 of 150 tokens,
    // 4096 x 4096 bf16: 397 us with two column tiles, 482 with one; lists of
    // 98, 2048 x 2710: 137 us with four, 214 with two; 4-bit weights, whose
    // activations take twice the registers, gain nothing from four), but fewer
    // where there are so few workgroups that sharing the lists among more of
    // them gains more than the weights' loads cost: one tile (30 tokens, k = 2
    // of 2 of 4096 x 512 bf16: 27 us, 33 with two; 60, k = 2 of 4 4-bit ones of
    // 2048 x 512: 20.5 and 25), or two (160, k = 1 of 4 of 2048 x 2048 fp16:
    // 50 us, 65 with four; 64, k = 2 of 4 of 1024 x 1024: 23.5 and 30), except
    // for rows of an odd length, whose loads cost twice (120, k = 4 of 4 of
    // 3520 x 545 fp16: 86 us, 62 with four)
    const int64_t mean = T * k / E, tiles = std::min<int64_t>(E, T * k) * ((F + 31) / 32);
    const bool odd = (D | F) & 1;
    if (mean <= kShortList || D < 8 || F < 8 || (tiles * ((mean + 31) / 32) <= kSlots / 8 && !odd)) return kGroup1;
    if (!mx4 && mean > 24 && (tiles > kSlots / 2 || odd)) return kGroup4;
    return kGroup2;
}

// ------------------------------------------------------------------ paged cache

// Whether the pages of two arrays share memory: of so many bytes each, at a, a +
// a_stride, ... and b, b + b_stride, ..., none within its own array.  Arrays of
// one stride may lie between each other; of two that reach into each other with
// different strides none is known to be apart.
inline bool pages_meet(uint64_t a, uint64_t a_stride, uint64_t b, uint64_t b_stride, uint64_t pages, uint64_t page) {
    typedef unsigned __int128 u128;
    if (pages == 0) return false;
    if (b < a) std::swap(a, b), std::swap(a_stride, b_stride);
    if (b - a >= (u128)(pages - 1) * a_stride + page) return false;  // behind it
    if (pages == 1) return true;
    if (a_stride != b_stride) return true;
    // a's last page that begins before b, and the next one
    const uint64_t i = (b - a) / a_stride, before = (b - a) % a_stride;
    return before < page || (i + 1 < pages && a_stride - before < page);
}

// ------------------------------------------------------------------ attention over a paged cache

constexpr int kAttendKeys = 32;       // keys of one step of a wave
constexpr int kAttendMinUnit = 4;     // steps of a unit: one for each wave
constexpr int kAttendWhole = 16;      // sequences of so many are not cut: joining costs more than three steps of a wave
constexpr int kAttendGoodUnit = 16;   // where units fill the GPU more than once they are no shorter
constexpr int kAttendLongUnit = 32;   // up to which they fill it once
constexpr int kAttendRounds = 4;
constexpr int kAttendMostSteps = 1 << 26;  // a sequence has at most 2^30 tokens

// Heads of one workgroup, of those that share a kv head: each sixteen cost D /
// 2 registers for their results.
constexpr int attend_heads(int group, int D) { return group > 16 && D <= 128 ? 32 : 16; }
constexpr int attend_tiles(int group, int D) { return (group + attend_heads(group, D) - 1) / attend_heads(group, D); }

// Workgroups on a compute unit, by the registers of a wave: keys and values of
// a step and the results take 192 at D = 128, more of which in flight gain less
// than values that the registers do not hold cost (64 sequences of up to 8192, D
// = 128: 217 us with two workgroups, 255 with three).
constexpr int attend_resident(int D, int heads) { return D > 128 ? 1 : D <= 64 && heads == 16 ? 3 : 2; }

// Units that fill the GPU once, with so many workgroups to a unit.
constexpr int64_t attend_units(int64_t workgroups, int resident) {
    return workgroups >= 256 * resident ? 1 : 256 * resident / workgroups;
}

// Steps of a unit where all sequences have total: what fills the GPU once, if
// that is little; else small enough that the last ones to run are a small part
// of the whole.  Once up to 32 steps, since somewhat more than once is the worst
// of both (16 sequences of up to 4096, 32 heads on 8, D = 128: 38 us, 46 with the
// limit at 16 steps; 16 of 8192, 128 heads on 4: 64 and 75).  A whole number for
// each wave: the last part of one takes as long (30 sequences, a window of 1000:
// 31.8 us, 34.4 without).
constexpr int attend_unit(int64_t total, int64_t units) {
    const int64_t once = (total + units - 1) / units, part = (total + units * kAttendRounds - 1) / (units * kAttendRounds);
    const int64_t unit = once <= kAttendLongUnit ? (once > kAttendMinUnit ? once : kAttendMinUnit) : part > kAttendGoodUnit ? part : kAttendGoodUnit;
    const int64_t whole = (unit + kAttendMinUnit - 1) / kAttendMinUnit * kAttendMinUnit;
    return whole < kAttendMostSteps ? (int)whole : kAttendMostSteps;  // no sequence has more
}

// Steps that a sequence has at most.
constexpr int64_t attend_steps(int64_t capacity, int32_t window) {
    const int64_t all = (capacity + kAttendKeys - 1) / kAttendKeys, in = (int64_t)window / kAttendKeys + 2;
    return window > 0 && in < all ? in : all;
}
constexpr bool attend_splits(int64_t capacity, int32_t window) { return attend_steps(capacity, window) > kAttendWhole; }
// Units that B sequences have at most: one each and what the cuts add, and as
// many as the smallest units would be.
constexpr int64_t attend_max_units(int64_t B, int64_t units, int64_t capacity, int32_t window) {
    const int64_t each = (attend_steps(capacity, window) + kAttendMinUnit - 1) / kAttendMinUnit, cut = B + units * kAttendRounds;
    return !attend_splits(capacity, window) ? B : each < (cut + B - 1) / B ? B * each : cut;
}

// ------------------------------------------------------------------ sampling

// Weights are at most 1: as whole multiples of 2^-43, their sums over a row of
// 2^20 fit 64 bits, and do not depend on the order in which they are added.
constexpr double kWeightUnit = 8796093022208.;

}  // namespace simops
