// Which of its kernels' forms an operator takes for given sizes: plain host
// rules, so that tests can ask which form a size runs.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <algorithm>

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
    if (mean <= 10 || D < 8 || F < 8 || (tiles * ((mean + 31) / 32) <= kSlots / 8 && !odd)) return kGroup1;
    if (!mx4 && mean > 24 && (tiles > kSlots / 2 || odd)) return kGroup4;
    return kGroup2;
}

}  // namespace simops
