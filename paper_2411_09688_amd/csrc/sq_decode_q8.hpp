// What the decode attention kernels on e4m3 keys and values share: a tile of 32 keys on the matrix cores, and the joining of waves.
//
// A tile, 16 columns = queries:
//   S^T [32 keys x 16] = K [32 x 128] q^T, the codes converted to f16 (exact), fp32 accumulation; the key's scale afterwards
//   O^T [128 x 16]    += V^T [128 x 32] P^T, the codes converted to bf16 (exact); p times the value's scale as the sum of two bf16
//                       (16 significant bits, and fp32's range: a scale may be anything)
// The order of the 32 keys is the same in both products: a lane's scores of S^T are the operand that P^T wants of it.  V is read row
// by row, 8 bytes a lane, and turned in registers (4 x 4 byte transposes).
#pragma once
#include <type_traits>

#include "sq_e4m3.hpp"
#include "sq_internal.hpp"

namespace sq {

typedef int i2v __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));

constexpr int QT = 32;                       // keys per tile
constexpr int O_STRIDE = 132;

// 64 keys of a wave: where they stand (bytes from the first of the fixed context's head, or of the pool's) and their scales.
// Offsets of 32 bits go straight into the loads, beside a scalar base: a pool of more than 4 GB takes those of 64 (WIDE).
template <bool WIDE>
struct KeyList {
    std::conditional_t<WIDE, unsigned long long, uint32_t> at[64];   // (0 for a slot without a key: the first row, which there is where a list is made)
    float ks[64], vs[64];                                            // ks: times the softmax's
};
struct WaveOut {                             // the four waves' results of a row
    float o[4][16][O_STRIDE];
};

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
template <typename T>
using global = const __attribute__((address_space(1))) T *;
template <typename T>
__device__ __forceinline__ global<T> uniform(const T *p)
{
    const unsigned long long v = reinterpret_cast<unsigned long long>(p);
    const uint32_t lo = uniform((int)(uint32_t)v), hi = uniform((int)(uint32_t)(v >> 32));
    return reinterpret_cast<global<T>>((unsigned long long)hi << 32 | lo);
}

// A row by its place in the order in which rows are dealt: head by head, so that the sequences (and query heads) that read the same
// head of the fixed context are on the same XCD at about the same time, where its L2 holds what several of them keep.
struct Row {
    int r, b, h;                             // row, sequence, K/V head
};
__device__ __forceinline__ Row dealt_row(const DecodeQ8Args &a, int i)
{
    if (a.B * a.per == 1) return Row{i, 0, i};
    const int n = a.B * a.per, h = i / n, rest = i - h * n;
    if (a.per == 1) return Row{rest * a.H + h, rest, h};
    const int b = rest / a.per;
    return Row{(b * a.H + h) * a.per + rest - b * a.per, b, h};
}
// Codes (four in a word) of keys 0..3 by rows to the four words of one dimension each.
__device__ __forceinline__ void transpose4(uint32_t &a, uint32_t &b, uint32_t &c, uint32_t &d)
{
    const uint32_t t0 = __builtin_amdgcn_perm(b, a, 0x05010400u), t1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
    const uint32_t u0 = __builtin_amdgcn_perm(d, c, 0x05010400u), u1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
    a = __builtin_amdgcn_perm(u0, t0, 0x05040100u);
    b = __builtin_amdgcn_perm(u0, t0, 0x07060302u);
    c = __builtin_amdgcn_perm(u1, t1, 0x05040100u);
    d = __builtin_amdgcn_perm(u1, t1, 0x07060302u);
}

__device__ __forceinline__ b8 codes_bf16(uint32_t lo, uint32_t hi)
{
    const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
    const b2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
    return b8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Dimension d of a query's result: l is zero where it sees no key, and NaN where it sees one.
__device__ __forceinline__ void store_result(const DecodeQ8Args &a, size_t query, int d, float m, float l, float o)
{
    const bool any = l > 0.0f || l != l;
    a.out[query * D + d] = (_Float16)(any ? o / l : 0.0f);
    if (d == 0 && a.lse) a.lse[query] = any ? (m + log2f(l)) * 0.69314718055994531f : SQ_NEG_INF;
}

// The thread's index as a value that the compiler cannot move: what is computed from it is computed where it stands, and takes no
// registers elsewhere.
__device__ __forceinline__ int thread_here()
{
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// A wave's attention so far: a column per query (lane: column c16), its running maximum (base 2) and sum (of a quarter of the keys in
// each group of 16 lanes), and the output, dimension 32 g4 + 8 i + dt of the column in o[dt][i].
struct Attending {
    h8 q[4];                                 // second operand of S^T: lane = column c16, dimensions 32 g4 + 8 s ..
    float m, l;
    f4 o[8];
};
__device__ __forceinline__ void begin(Attending &st)
{
    st.m = SQ_NEG_INF;
    st.l = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) st.o[i] = f4{0.f, 0.f, 0.f, 0.f};
}

// Slots of the tile without a key (bits i and 16 + i of `mine`: this lane's slots): what stands in their row is not looked at.
__device__ __forceinline__ void hide_empty(float (&s)[8], uint32_t (&w)[2][8], uint32_t mine)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (!(mine >> (i < 4 ? i : 12 + i) & 1u)) {
            s[i] = SQ_NEG_INF;
            w[0][i] = w[1][i] = 0u;
        }
}

// Folds 32 keys: k, v as the lanes read them (keys c16 and 16 + c16, dimensions 32 g4 ..; keys 4 g4 .. and 16 + 4 g4 .., dimensions
// 8 c16 ..), ks, vs the scales of the lane's keys 4 g4 ..  used_k: called when k may be overwritten; hide: sets the scores (and words of
// values) of keys that are not to be seen.
template <class UsedK, class Hide>
__device__ __forceinline__ void fold_tile(Attending &st, const u4v (&k)[2][2], const u2v (&v)[8], const float *ks, const float *vs, UsedK used_k,
                                          Hide hide)
{
    f4 acc[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const u4v x = k[u][s >> 1];
            acc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(s & 1 ? codes_f16(x.z, x.w) : codes_f16(x.x, x.y), st.q[s], acc[u], 0, 0, 0);
        }
    used_k();
    float s[8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const f4 f = *reinterpret_cast<const f4 *>(ks + 16 * u);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[4 * u + i] = acc[u][i] * f[i];
    }
    uint32_t w[2][8];                        // V: words of dimensions 8 c16 .. + 3 and .. + 7
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        w[0][i] = v[i].x;
        w[1][i] = v[i].y;
    }
    hide(s, w);
    const float mx = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    const float mn = fmaxf(st.m, cross16_max(mx));
    const float mu = mn == SQ_NEG_INF ? 0.0f : mn;
    const float alpha = __builtin_amdgcn_exp2f(st.m - mu);
    st.m = mn;
    st.l *= alpha;
    b8 hi8, lo8;
    const f4 v0 = *reinterpret_cast<const f4 *>(vs), v1 = *reinterpret_cast<const f4 *>(vs + 16);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = __builtin_amdgcn_exp2f(s[i] - mu);
        st.l += x;
        const float pv = x * (i < 4 ? v0[i & 3] : v1[i & 3]);
        hi8[i] = (__bf16)pv;
        lo8[i] = (__bf16)(pv - (float)hi8[i]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        transpose4(w[i][0], w[i][1], w[i][2], w[i][3]);
        transpose4(w[i][4], w[i][5], w[i][6], w[i][7]);
    }
    if (__any(alpha != 1.0f)) {              // (the maximum rarely moves behind the first tiles)
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) st.o[dt] *= alpha;
    }
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) {
        const b8 vf = codes_bf16(w[dt >> 2][dt & 3], w[dt >> 2][4 + (dt & 3)]);
        st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, hi8, st.o[dt], 0, 0, 0);
        st.o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, lo8, st.o[dt], 0, 0, 0);
    }
}

// The waves' results of the workgroup's columns to LDS, for join().
__device__ __forceinline__ void hand_over(const Attending &st, int columns, int wave, WaveOut &out, float (&ml)[2][4][16])
{
    const int lane = thread_here() & 63, c16 = lane & 15, g4 = lane >> 4;
    const float l = cross16_sum(st.l);
    if (g4 == 0) {
        ml[0][wave][c16] = st.m;
        ml[1][wave][c16] = l;
    }
    if (c16 < columns) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float *dst = &out.o[wave][c16][32 * g4 + 8 * i];
            *reinterpret_cast<f4 *>(dst) = f4{st.o[0][i], st.o[1][i], st.o[2][i], st.o[3][i]};
            *reinterpret_cast<f4 *>(dst + 4) = f4{st.o[4][i], st.o[5][i], st.o[6][i], st.o[7][i]};
        }
    }
}
struct Joined {
    float m, l, o;
};
__device__ __forceinline__ Joined join(const WaveOut &out, const float (&ml)[2][4][16], int column, int d)
{
    Joined x;
    x.m = fmaxf(fmaxf(ml[0][0][column], ml[0][1][column]), fmaxf(ml[0][2][column], ml[0][3][column]));
    const float mu = x.m == SQ_NEG_INF ? 0.0f : x.m;
    x.l = x.o = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const float f = __builtin_amdgcn_exp2f(ml[0][w][column] - mu);
        x.l += f * ml[1][w][column];
        x.o += f * out.o[w][column][d];
    }
    return x;
}
__device__ __forceinline__ void store_partial(float *p, int d, const Joined &x)
{
    p[4 + d] = x.o;
    if (d == 0) {
        p[0] = x.m;
        p[1] = x.l;
    }
}

}  // namespace sq
