// Streaming weights once through registers: the wave's loop and the scales of
// 4-bit weights.
#pragma once

#include "ops_common.h"

namespace simops {

constexpr int kStep = 128;  // columns of one step of a wave

// The scales of a run of U steps of R tiles of 4-bit weights: sixteen bytes a
// row for four steps, eight for two.  The rows' pieces of eight bytes lie one
// in a lane, piece-major, and each lane asks the one that has its row: loads
// that every lane makes for itself would cost more cache accesses than the
// codes (measured for 459 MB of 4-bit weights: 147 us with a byte load a
// step, 128 us with sixteen bytes a run).
template <int WT, int R, int U> struct Scales {
    __device__ void load(const uint8_t *, int64_t, int, int) {}
    __device__ float get(int, int, int, int) const { return 1.f; }
    static __device__ int tile() { return 0; }
};
template <int R, int U> struct Scales<SIM_TYPE_MX4, R, U> {
    static_assert(R * 16 * (U / 2) <= 64, "a lane for each piece");
    u32x2 v;
    // the tile whose row (lane % 16) this lane loads
    static __device__ int tile() { return (threadIdx.x >> 4 & 3) % R; }
    // row: of that tile; rows are whole groups of 256 columns, two steps: a
    // run of four may have half of it past the end, a step never
    __device__ void load(const uint8_t *scales, int64_t row, int K, int run) {
        const int g = (int)groups_of(K), piece = min((int)(threadIdx.x & 63) / (16 * R), U / 2 - 1);
        v = ((const u32x2 *)scales)[row * g + min(run * (U / 2) + piece, g - 1)];
    }
    // of step i, tile j: row r, quarter q
    __device__ float get(int i, int j, int r, int q) const {
        const uint32_t four = (uint32_t)__builtin_amdgcn_ds_bpermute(((i >> 1) * 16 * R + j * 16 + r) * 4, (int)v[i & 1]);
        return scale_value((four >> (8 * q)) & 255);
    }
    // the same as the scale operand of a matrix instruction: in the lowest byte
    __device__ int get_byte(int i, int j, int r, int q) const {
        return (int)((uint32_t)__builtin_amdgcn_ds_bpermute(((i >> 1) * 16 * R + j * 16 + r) * 4, (int)v[i & 1]) >> (8 * q));
    }
};

// Runs of U steps, this wave's of every W, through a ring of U places:
// head(parity, run) loads what belongs to a whole run, load(place, run), use(
// place, parity, run).  The loop that does the work has no conditions around
// its loads, so the waits in it count them exactly.
template <int U, int W, typename Head, typename Load, typename Use>
__device__ inline void ring(int runs, int wave, Head &&head, Load &&load, Use &&use) {
    if (wave >= runs) return;
    const auto turn = [&](auto parity, int run) {  // uses one run and loads the next of this wave
        constexpr int p = decltype(parity)::value;
        head(1 - p, run + W);
#pragma unroll
        for (int i = 0; i < U; i++) {
            use(i, p, run);
            load(i, run + W);
        }
    };
    const auto end = [&](auto parity, int run) {
        constexpr int p = decltype(parity)::value;
#pragma unroll
        for (int i = 0; i < U; i++) use(i, p, run);
    };
    typedef std::integral_constant<int, 0> P0;
    typedef std::integral_constant<int, 1> P1;
    int run = wave;
    head(0, run);
#pragma unroll
    for (int i = 0; i < U; i++) load(i, run);
    for (; run + 2 * W < runs; run += 2 * W) {
        turn(P0(), run);
        turn(P1(), run + W);
    }
    if (run + W < runs) {
        turn(P0(), run);
        end(P1(), run + W);
    } else {
        end(P0(), run);
    }
}

}  // namespace simops
