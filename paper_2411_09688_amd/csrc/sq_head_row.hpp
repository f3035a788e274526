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

template <bool ADJACENT, bool PARTIAL>
__device__ __forceinline__ LanePieces lane_pieces(int j, int rot_dim)
{
    const int r = PARTIAL ? rot_dim : D, n = r >> 3;
    if (ADJACENT) return {8 * j, 8 * j + 4, !PARTIAL || j < n};
    if (!PARTIAL || j < n) return {4 * j, (r >> 1) + 4 * j, true};
    return {r + 8 * (j - n), r + 8 * (j - n) + 4, false};
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

// The kernels are compiled for each kind of rotation, which costs a row a third of its instructions as selects otherwise: pairs
// (2i, 2i + 1) or not (ADJACENT), and lanes that do not rotate or none (PARTIAL: rot_dim < 128).
#define SQ_FOR_ROTARY(ra, call)                                                       \
    ((ra).adjacent ? ((ra).rot_dim < D ? call(true, true) : call(true, false))        \
                   : ((ra).rot_dim < D ? call(false, true) : call(false, false)))

// The lane's dimensions x, y (pieces a, b) normed and rotated, fp32 arithmetic; wa, wb: the weight's, same places; turns: this lane
// rotates.
template <bool ADJACENT, bool PARTIAL>
__device__ __forceinline__ void norm_rotate(float (&e)[8], h4 x, h4 y, h4 wa, h4 wb, bool norm, float eps, const float (&cs)[8], bool turns)
{
    if (norm) {
        float ss = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ss = __builtin_fmaf((float)x[i], (float)x[i], ss);
            ss = __builtin_fmaf((float)y[i], (float)y[i], ss);
        }
        const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(row16_sum(ss), 1.0f / D, eps));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[i] = (float)x[i] * ((float)wa[i] * r);
            e[i + 4] = (float)y[i] * ((float)wb[i] * r);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[i] = (float)x[i];
            e[i + 4] = (float)y[i];
        }
    }
    auto turn = [&](int ia, int ib, int i) {
        const float a = e[ia], b = e[ib], c = cs[2 * i], s = cs[2 * i + 1];
        const float u = __builtin_fmaf(a, c, -(b * s)), v = __builtin_fmaf(b, c, a * s);
        e[ia] = PARTIAL && !turns ? a : u;
        e[ib] = PARTIAL && !turns ? b : v;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) ADJACENT ? turn(2 * i, 2 * i + 1, i) : turn(i, i + 4, i);
}

// Up to four heads of one token by 16 lanes, fp32 arithmetic, rounded to f16 once; kind 0: query, 1: key, 2: value (copied).  All of
// the rows are read before the first is turned, and the token's cosines and sines once for all of them.
constexpr int ROWS_AT_ONCE = 4;
struct TurnRows {
    const _Float16 *src[ROWS_AT_ONCE];
    _Float16 *dst[ROWS_AT_ONCE];
    int kind[ROWS_AT_ONCE];
    int n;
};
template <bool ADJACENT, bool PARTIAL, bool STREAM>
__device__ __forceinline__ void turn_rows(const TurnRows &t, const RotaryArgs &ra, int position, int j)
{
    const LanePieces lp = lane_pieces<ADJACENT, PARTIAL>(j, ra.rot_dim);
    h4 x[ROWS_AT_ONCE], y[ROWS_AT_ONCE];
#pragma unroll
    for (int i = 0; i < ROWS_AT_ONCE; ++i) {                // (behind the last the last again, without a branch)
        x[i] = load_once<STREAM>(reinterpret_cast<const h4 *>(t.src[i] + lp.a));
        y[i] = load_once<STREAM>(reinterpret_cast<const h4 *>(t.src[i] + lp.b));
    }
    float cs[8];
    load_turn(cs, ra, position, j, lp.turns && t.kind[0] != 2);   // (values come last)
    h4 wa[2] = {}, wb[2] = {};
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (ra.weight[k]) {
            wa[k] = *reinterpret_cast<const h4 *>(ra.weight[k] + lp.a);
            wb[k] = *reinterpret_cast<const h4 *>(ra.weight[k] + lp.b);
        }
#pragma unroll
    for (int i = 0; i < ROWS_AT_ONCE; ++i)
        if (i < t.n) {
            if (t.kind[i] != 2) {
                const bool key = t.kind[i] == 1;
                float e[8];
                norm_rotate<ADJACENT, PARTIAL>(e, x[i], y[i], key ? wa[1] : wa[0], key ? wb[1] : wb[0], ra.weight[key] != nullptr, ra.eps, cs, lp.turns);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    x[i][c] = (_Float16)e[c];
                    y[i][c] = (_Float16)e[c + 4];
                }
            }
            store_once<STREAM>(reinterpret_cast<h4 *>(t.dst[i] + lp.a), x[i]);
            store_once<STREAM>(reinterpret_cast<h4 *>(t.dst[i] + lp.b), y[i]);
        }
}

}  // namespace sq
