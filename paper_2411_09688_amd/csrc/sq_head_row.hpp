// One row (the 128 dimensions of one head of one token) normed and rotated by 16 lanes.
//
// A lane holds 8 of the row's dimensions as two pieces of 4 that lie where the rotation's pairs need them, so that both
// halves of a pair are the lane's own and nothing is exchanged: with pairs (i, i + r/2), lane j < r/8 holds dimensions
// 4j.. and r/2 + 4j.., the remaining lanes 8 consecutive ones behind r; with pairs (2i, 2i + 1) a lane holds 8 consecutive
// ones.  Either way its pairs are 4j .. 4j + 3, 32 bytes of the table.
#pragma once
#include "sq_common.hpp"
#include "sq_e4m3.hpp"

namespace sq {

struct RotaryArgs {
    const float *cos_sin;
    const _Float16 *weight[2];     // queries, keys; null: no norm
    int rot_dim, adjacent, n_positions;
    float eps;
};

struct LanePieces {
    int a, b;                      // first dimensions of the two pieces
    bool turns;                    // they are rotated
};

__device__ __forceinline__ LanePieces lane_pieces(int j, int rot_dim, bool adjacent)
{
    const int n = rot_dim >> 3;
    if (adjacent) return {8 * j, 8 * j + 4, j < n};
    if (j < n) return {4 * j, (rot_dim >> 1) + 4 * j, true};
    return {rot_dim + 8 * (j - n), rot_dim + 8 * (j - n) + 4, false};
}

// The four pairs' cosines and sines of a lane; 1 and 0 where it does not rotate.
__device__ __forceinline__ void load_turn(float (&cs)[8], const RotaryArgs &ra, int position, int j, bool turns)
{
    f4 x = {1.f, 0.f, 1.f, 0.f}, y = x;
    if (turns) {
        const int p = min(max(position, 0), ra.n_positions - 1);
        const float *t = ra.cos_sin + (size_t)p * ra.rot_dim + 8 * j;
        x = *reinterpret_cast<const f4 *>(t);
        y = *reinterpret_cast<const f4 *>(t + 4);
    }
    cs[0] = x[0]; cs[1] = x[1]; cs[2] = x[2]; cs[3] = x[3];
    cs[4] = y[0]; cs[5] = y[1]; cs[6] = y[2]; cs[7] = y[3];
}

template <typename T>
__device__ __forceinline__ T row16_total(T v)
{
    if constexpr (sizeof(T) == 4) {
        return row16_sum(v);
    } else {
#pragma unroll
        for (int k = 8; k > 0; k >>= 1) v += __shfl_xor(v, k, 16);
        return v;
    }
}

// e: the lane's dimensions (pieces a, b); w: the weight's, same places.  T is the type of the arithmetic.
template <typename T>
__device__ __forceinline__ void norm_rotate(T (&e)[8], const T (&w)[8], bool norm, T eps, const float (&cs)[8], bool turns, bool adjacent)
{
    if (norm) {
        T ss = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += e[i] * e[i];
        const T r = (T)1 / sqrt(row16_total(ss) / (T)D + eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = e[i] * r * w[i];
    }
    if (!turns) return;
    if (adjacent) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const T a = e[2 * i], b = e[2 * i + 1], c = cs[2 * i], s = cs[2 * i + 1];
            e[2 * i] = a * c - b * s;
            e[2 * i + 1] = b * c + a * s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const T a = e[i], b = e[i + 4], c = cs[2 * i], s = cs[2 * i + 1];
            e[i] = a * c - b * s;
            e[i + 4] = b * c + a * s;
        }
    }
}

template <typename T>
__device__ __forceinline__ void load_pieces(T (&e)[8], const _Float16 *row, const LanePieces &lp)
{
    const h4 x = *reinterpret_cast<const h4 *>(row + lp.a), y = *reinterpret_cast<const h4 *>(row + lp.b);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        e[i] = (T)(float)x[i];
        e[i + 4] = (T)(float)y[i];
    }
}

// A query or key row to f16, fp32 arithmetic.
__device__ __forceinline__ void store_turned_row(_Float16 *dst, const _Float16 *src, const _Float16 *weight, const RotaryArgs &ra,
                                                 const LanePieces &lp, const float (&cs)[8])
{
    float e[8], w[8] = {};
    load_pieces(e, src, lp);
    if (weight) load_pieces(w, weight, lp);
    norm_rotate<float>(e, w, weight != nullptr, ra.eps, cs, lp.turns, ra.adjacent != 0);
    h4 x, y;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = (_Float16)e[i];
        y[i] = (_Float16)e[i + 4];
    }
    *reinterpret_cast<h4 *>(dst + lp.a) = x;
    *reinterpret_cast<h4 *>(dst + lp.b) = y;
}

}  // namespace sq
