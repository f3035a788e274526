// sq_sparse_attn_decode_q8: decode attention over e4m3 keys and values, kept ranges of the fixed context and the pages of the
// user cache, one softmax over both.
//
// A row is a (sequence, K/V head) with its g query heads (one kept set) or a single query head.  Its keys, laid end to end --
// the kept keys of the fixed context, then the user's -- are cut into tiles of 32; the tiles of all rows, laid end to end, are cut
// into equal shares, one per workgroup, so rows that keep more get more of the chip.  What bounds it is the 256 bytes of a key and
// its value, read once per row.
//
// A tile of a wave on the matrix cores, 16 columns = query heads:
//   S^T [32 keys x 16] = K [32 x 128] q^T, the codes converted to f16 (exact), fp32 accumulation; the key's scale afterwards
//   O^T [128 x 16]    += V^T [128 x 32] P^T, the codes converted to bf16 (exact); p times the value's scale as the sum of two bf16
//                       (16 significant bits, and fp32's range: a scale may be anything)
// The order of the 32 keys is the same in both products: a lane's scores of S^T are the operand that P^T wants of it.  V is read row
// by row, 8 bytes a lane, and turned in registers (4 x 4 byte transposes).
#include "sq_e4m3.hpp"
#include "sq_internal.hpp"

namespace sq {

namespace {

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));

constexpr int QT = 32;                       // keys per tile
constexpr int QCHUNK = 32;                   // tiles whose key rows are listed at a time
constexpr int QLIST = QT * QCHUNK;           // ... 1024 keys
constexpr uint32_t NO_KEY = 0xffffffffu;
constexpr int SENTINEL = INT32_MIN;
constexpr int O_STRIDE = 132;

struct KeyList {                             // the rows (of 128 codes) of a chunk's keys and their scales
    uint32_t row[QLIST];
    float ks[QLIST], vs[QLIST];
};
struct Tile {                                // what a lane reads of 32 keys
    u4v k[2][2];                             // keys c16 and 16 + c16, dimensions 32 g4 ..
    u2v v[8];                                // keys 4 g4 .. and 16 + 4 g4 .., dimensions 8 c16 ..
};
struct WaveOut {                             // the four waves' results of a row
    float o[4][16][O_STRIDE];
};
union SharedMem {
    KeyList list;
    WaveOut out;
};

struct RowTiles {
    int nf, nu, tf, total;                   // fixed and user keys, tiles of fixed keys, all tiles (at least one)
};

__device__ __forceinline__ RowTiles row_tiles(const DecodeQ8Args &a, int r)
{
    RowTiles t;
    t.nf = a.ranges ? min(max(a.n_keys[r], 0), a.L) : 0;
    t.nu = a.seq_len ? min(max(a.seq_len[r / (a.H * a.per)], 0), a.max_pages * a.P) : 0;
    t.tf = (t.nf + QT - 1) / QT;
    t.total = max(1, t.tf + (t.nu + QT - 1) / QT);
    return t;
}

__device__ __forceinline__ int block_exclusive(int v, int tid, int *s_w /*[4]*/, int &total)
{
    const int inc = wave_inclusive_scan(v, tid & 63);
    __syncthreads();
    if ((tid & 63) == 63) s_w[tid >> 6] = inc;
    __syncthreads();
    int ex = inc - v;
    for (int w = 0; w < (tid >> 6); ++w) ex += s_w[w];
    total = s_w[0] + s_w[1] + s_w[2] + s_w[3];
    return ex;
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

__device__ __forceinline__ h8 codes_f16(uint32_t lo, uint32_t hi)
{
    const h2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    const h2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
    return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
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

}  // namespace

// Rows in the order in which they are dealt: head by head, so that the sequences (and query heads) that read the same head of the
// fixed context are on the same XCD at about the same time, where its L2 holds what several of them keep.
__device__ __forceinline__ int dealt_row(const DecodeQ8Args &a, int i)
{
    const int n = a.B * a.per, h = i / n, rest = i - h * n, b = rest / a.per;
    return (b * a.H + h) * a.per + rest - b * a.per;
}

__global__ __launch_bounds__(256, 2) void decode_q8_kernel(DecodeQ8Args a)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c16 = lane & 15, g4 = lane >> 4;
    __shared__ __align__(16) SharedMem sm;
    __shared__ int s_delta[QLIST];
    __shared__ unsigned long long s_bal[QLIST / 64];
    __shared__ int s_w[4], s_found[2];
    __shared__ float s_ml[2][4][16];

    // This workgroup's share of the tiles.  Workgroups go round the 8 XCDs: each XCD takes consecutive shares.
    const int R = a.B * a.H * a.per;
    const int each = (R + 255) / 256, i_lo = min(R, tid * each), i_hi = min(R, i_lo + each);
    int mine = 0, all;
    for (int i = i_lo; i < i_hi; ++i) mine += row_tiles(a, dealt_row(a, i)).total;
    int before = block_exclusive(mine, tid, s_w, all);
    const int shares = min((int)gridDim.x, (all + 3) / 4);
    const int per = (all + shares - 1) / shares, per_xcd = (shares + 7) / 8;
    const int share = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per_xcd || (long long)share * per >= all) return;
    const int t0 = share * per, t1 = min(all, t0 + per);
    if (before <= t0 && t0 < before + mine) {
        int i = i_lo;
        for (;; ++i) {
            const int n = row_tiles(a, dealt_row(a, i)).total;
            if (t0 < before + n) break;
            before += n;
        }
        s_found[0] = i;
        s_found[1] = before;
    }
    __syncthreads();
    int ri = s_found[0], row_start = s_found[1];

    for (; row_start < t1; ++ri) {
        const int r = dealt_row(a, ri);
        const RowTiles rt = row_tiles(a, r);
        const int bh = r / a.per, h = bh % a.H, b = bh / a.H;
        const int lo = max(t0 - row_start, 0), hi = min(t1 - row_start, rt.total);
        // q^T as the second operand of S^T: lane = query column c16, dimensions 32 g4 + 8 s ..
        h8 qf[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const h8 zero = {};
            qf[s] = c16 < a.g ? *reinterpret_cast<const h8 *>(a.q + ((size_t)r * a.g + c16) * D + 32 * g4 + 8 * s) : zero;
        }
        float m = SQ_NEG_INF, l = 0.0f;
        f4 o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = f4{0.f, 0.f, 0.f, 0.f};

        int range0 = 0, range_before = 0;                   // first range of the batch that holds the next position; keys before it
        for (int c0 = lo; c0 < hi; c0 += QCHUNK) {
            const int c1 = min(hi, c0 + QCHUNK), n = (c1 - c0) * QT;
            // fixed keys: positions [p0, p1) of the row's list
            const int p0 = min(c0 * QT, rt.nf), p1 = min(c1 * QT, rt.nf);
            const int nfix = p1 - p0;
            int listed = 0;                                 // of them, those that the ranges really have
            __syncthreads();
            if (nfix > 0) {
                for (int i = tid; i < QLIST; i += 256) s_delta[i] = SENTINEL;
                const int nr = min(max(a.n_ranges[r], 0), a.C);
                const int2 *rg = reinterpret_cast<const int2 *>(a.ranges) + (size_t)r * a.C;
                int total = 0;
                for (; range0 < nr; range0 += 1024) {
                    int2 e[4];
                    int sum = 0;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int i = range0 + tid * 4 + k;
                        e[k] = i < nr ? rg[i] : int2{0, 0};
                        e[k].x = min(max(e[k].x, -MAX_L), MAX_L);
                        e[k].y = min(max(e[k].y, 0), a.L);
                        sum += e[k].y;
                    }
                    // (counts that sum to more than a row can have are cut, far from overflow)
                    int at = block_exclusive(min(sum, MAX_L), tid, s_w, total) + range_before;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int from = max(at, p0), to = min(at + e[k].y, p1);
                        if (from < to) s_delta[from - p0] = e[k].x - at;
                        at += e[k].y;
                    }
                    if (range_before + total >= p1) break;
                    range_before = min(range_before + total, MAX_L);
                }
                listed = range0 < nr ? nfix : max(0, min(p1, range_before) - p0);
                __syncthreads();
            }
            unsigned long long bal[QLIST / 256] = {};
            if (nfix > 0) {
#pragma unroll
                for (int i = 0; i < QLIST / 256; ++i) {
                    bal[i] = __ballot(s_delta[(i * 4 + wave) * 64 + lane] != SENTINEL);
                    if (lane == 0) s_bal[i * 4 + wave] = bal[i];
                }
                __syncthreads();
            }
            // Each thread lists up to four keys.  Their scales are read while the first tile is: they are stored behind its loads.
            const int ntf = max(0, min(c1, rt.tf) - c0) * QT;   // slots of tiles with fixed keys; the user's are behind them
            const int u0 = (max(c0, rt.tf) - rt.tf) * QT;        // first user key of the chunk
            float ks[QLIST / 256], vs[QLIST / 256];
#pragma unroll
            for (int i = 0; i < QLIST / 256; ++i) {
                const int grp = i * 4 + wave, pos = grp * 64 + lane;
                ks[i] = vs[i] = 0.0f;
                if (pos >= n) continue;
                uint32_t row = NO_KEY;
                if (pos < nfix) {
                    unsigned long long w = bal[i] & (~0ull >> (63 - lane));
                    int from = grp;
                    while (w == 0ull && from > 0) w = s_bal[--from];
                    if (w != 0ull && pos < listed) {
                        const int d = s_delta[from * 64 + 63 - __clzll((long long)w)];
                        const int key = min(max(p0 + pos + d, 0), a.L - 1);
                        row = (uint32_t)(h * a.L + key);
                        const int sb = h * a.sblocks + (key >> 6);
                        ks[i] = a.ks[sb];
                        vs[i] = a.vs[sb];
                    }
                } else if (pos >= ntf && u0 + pos - ntf < rt.nu) {
                    const int t = u0 + pos - ntf;
                    const int page = a.page_table[(size_t)b * a.max_pages + t / a.P];
                    if (page >= 0 && page < a.n_pages) {
                        const int ph = page * a.H + h;
                        row = (uint32_t)(ph * a.P + t % a.P);
                        ks[i] = a.cks[ph];
                        vs[i] = a.cvs[ph];
                    }
                }
                sm.list.row[pos] = row;
            }
            __syncthreads();

            const int tiles = c1 - c0;
            auto load = [&](Tile &x, int t) {
                const bool fixed = c0 + t < rt.tf;
                const uint8_t *Kb = (fixed ? a.K8 : a.cK) + 32 * g4, *Vb = (fixed ? a.V8 : a.cV) + 8 * c16;
                const uint32_t *rows = sm.list.row + t * QT;
                // (a slot without a key reads row 0, which there is)
                auto at = [](uint32_t row) { return (size_t)(row == NO_KEY ? 0u : row) * D; };
                const size_t k0 = at(rows[c16]), k1 = at(rows[16 + c16]);
                const u4v v0 = *reinterpret_cast<const u4v *>(rows + 4 * g4), v1 = *reinterpret_cast<const u4v *>(rows + 16 + 4 * g4);
                x.k[0][0] = *reinterpret_cast<const u4v *>(Kb + k0);
                x.k[0][1] = *reinterpret_cast<const u4v *>(Kb + k0 + 16);
                x.k[1][0] = *reinterpret_cast<const u4v *>(Kb + k1);
                x.k[1][1] = *reinterpret_cast<const u4v *>(Kb + k1 + 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x.v[i] = *reinterpret_cast<const u2v *>(Vb + at(v0[i]));
                    x.v[4 + i] = *reinterpret_cast<const u2v *>(Vb + at(v1[i]));
                }
            };
            auto fold = [&](Tile &x, int t) {
                const uint32_t *rows = sm.list.row + t * QT;
                float s[8], mx = SQ_NEG_INF;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    f4 acc = {0.f, 0.f, 0.f, 0.f};
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(x.k[u][0].x, x.k[u][0].y), qf[0], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(x.k[u][0].z, x.k[u][0].w), qf[1], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(x.k[u][1].x, x.k[u][1].y), qf[2], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_f16(x.k[u][1].z, x.k[u][1].w), qf[3], acc, 0, 0, 0);
                    const f4 f = *reinterpret_cast<const f4 *>(sm.list.ks + t * QT + 16 * u + 4 * g4);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[4 * u + i] = acc[i] * (f[i] * a.scale);
                }
                uint32_t w[2][8];                            // V: words of dimensions 8 c16 .. + 3 and .. + 7
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[0][i] = x.v[i].x;
                    w[1][i] = x.v[i].y;
                }
                if (__any(rows[lane & 31] == NO_KEY)) {      // what stands in such a slot's row is not looked at
                    const u4v v0 = *reinterpret_cast<const u4v *>(rows + 4 * g4), v1 = *reinterpret_cast<const u4v *>(rows + 16 + 4 * g4);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if ((i < 4 ? v0[i & 3] : v1[i & 3]) == NO_KEY) {
                            s[i] = SQ_NEG_INF;
                            w[0][i] = w[1][i] = 0u;
                        }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) mx = fmaxf(mx, s[i]);
                const float mn = fmaxf(m, cross16_max(mx));
                const float mu = mn == SQ_NEG_INF ? 0.0f : mn;
                const float alpha = __builtin_amdgcn_exp2f(m - mu);
                m = mn;
                l *= alpha;
                b8 hi8, lo8;
                const f4 f0 = *reinterpret_cast<const f4 *>(sm.list.vs + t * QT + 4 * g4);
                const f4 f1 = *reinterpret_cast<const f4 *>(sm.list.vs + t * QT + 16 + 4 * g4);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p = __builtin_amdgcn_exp2f(s[i] - mu);
                    l += p;
                    const float pv = p * (i < 4 ? f0[i & 3] : f1[i & 3]);
                    hi8[i] = (__bf16)pv;
                    lo8[i] = (__bf16)(pv - (float)hi8[i]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    transpose4(w[i][0], w[i][1], w[i][2], w[i][3]);
                    transpose4(w[i][4], w[i][5], w[i][6], w[i][7]);
                }
                if (__any(alpha != 1.0f)) {                  // (the maximum rarely moves behind the first tiles)
#pragma unroll
                    for (int dt = 0; dt < 8; ++dt) o[dt] *= alpha;
                }
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    const b8 vf = codes_bf16(w[dt >> 2][dt & 3], w[dt >> 2][4 + (dt & 3)]);
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, hi8, o[dt], 0, 0, 0);
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, lo8, o[dt], 0, 0, 0);
                }
            };
            // A wave's tiles, the next one on its way while one is folded.
            Tile x, y;
            if (wave < tiles) load(x, wave);
#pragma unroll
            for (int i = 0; i < QLIST / 256; ++i) {
                const int pos = (i * 4 + wave) * 64 + lane;
                if (pos < n) {
                    sm.list.ks[pos] = ks[i];
                    sm.list.vs[pos] = vs[i];
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
            for (int t = wave; t < tiles; t += 8) {
                if (t + 4 < tiles) load(y, t + 4);
                fold(x, t);
                if (t + 8 < tiles) load(x, t + 8);
                if (t + 4 < tiles) fold(y, t + 4);
            }
        }
        // The four waves' results of the row.
        l = cross16_sum(l);
        __syncthreads();                                    // (the list has been read)
        if (g4 == 0) {
            s_ml[0][wave][c16] = m;
            s_ml[1][wave][c16] = l;
        }
        if (c16 < a.g) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float *dst = &sm.out.o[wave][c16][32 * g4 + 8 * i];
                *reinterpret_cast<f4 *>(dst) = f4{o[0][i], o[1][i], o[2][i], o[3][i]};
                *reinterpret_cast<f4 *>(dst + 4) = f4{o[4][i], o[5][i], o[6][i], o[7][i]};
            }
        }
        __syncthreads();
        const bool whole = lo == 0 && hi == rt.total;
        const int slot = share + ri;
        for (int i = tid; i < a.g * D; i += 256) {
            const int qi = i >> 7, d = i & 127;
            float M = fmaxf(fmaxf(s_ml[0][0][qi], s_ml[0][1][qi]), fmaxf(s_ml[0][2][qi], s_ml[0][3][qi]));
            const float mu = M == SQ_NEG_INF ? 0.0f : M;
            float ls = 0.0f, os = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = exp2f(s_ml[0][w][qi] - mu);
                ls += f * s_ml[1][w][qi];
                os += f * sm.out.o[w][qi][d];
            }
            if (whole) {
                store_result(a, (size_t)r * a.g + qi, d, M, ls, os);
            } else {
                float *p = a.part + ((size_t)slot * a.g + qi) * PART_STRIDE;
                p[4 + d] = os;
                if (d == 0) {
                    p[0] = M;
                    p[1] = ls;
                }
            }
        }
        if (tid == 0 && lo == 0) {
            const int last = (row_start + rt.total - 1) / per;
            a.info[r] = int2{slot, whole ? 0 : last - share + 1};
        }
        __syncthreads();
        row_start += rt.total;
    }
}

// Rows that several workgroups took: one workgroup per row and query.  Eight groups of 32 lanes fold every eighth partial result,
// a lane four dimensions, and are folded in LDS.
__global__ __launch_bounds__(256) void decode_q8_merge_kernel(DecodeQ8Args a)
{
    const int r = blockIdx.x / a.g, qi = blockIdx.x - r * a.g, tid = threadIdx.x, grp = tid >> 5, quad = tid & 31;
    __shared__ float s_m[8], s_l[8];
    __shared__ __align__(16) float s_o[8][D];
    const int2 info = a.info[r];
    if (info.y == 0) return;
    float M = SQ_NEG_INF, ls = 0.0f;
    f4 os = {0.f, 0.f, 0.f, 0.f};
    auto part = [&](int i) { return a.part + ((size_t)(info.x + i) * a.g + qi) * PART_STRIDE; };
    auto fold = [&](float pm, float pl, f4 po) {
        const float mn = fmaxf(M, pm), mu = mn == SQ_NEG_INF ? 0.0f : mn;
        const float fa = exp2f(M - mu), fb = exp2f(pm - mu);
        ls = ls * fa + pl * fb;
        os = os * fa + po * fb;
        M = mn;
    };
    int i = grp;
    for (; i + 8 < info.y; i += 16) {
        const float *p = part(i), *n = part(i + 8);
        const float2 a0 = *reinterpret_cast<const float2 *>(p), a1 = *reinterpret_cast<const float2 *>(n);
        const f4 o0 = *reinterpret_cast<const f4 *>(p + 4 + 4 * quad), o1 = *reinterpret_cast<const f4 *>(n + 4 + 4 * quad);
        fold(a0.x, a0.y, o0);
        fold(a1.x, a1.y, o1);
    }
    if (i < info.y) {
        const float *p = part(i);
        fold(p[0], p[1], *reinterpret_cast<const f4 *>(p + 4 + 4 * quad));
    }
    *reinterpret_cast<f4 *>(&s_o[grp][4 * quad]) = os;
    if (quad == 0) {
        s_m[grp] = M;
        s_l[grp] = ls;
    }
    __syncthreads();
    if (tid >= D) return;
    float MM = s_m[0];
#pragma unroll
    for (int g = 1; g < 8; ++g) MM = fmaxf(MM, s_m[g]);
    const float mu = MM == SQ_NEG_INF ? 0.0f : MM;
    float lt = 0.0f, ot = 0.0f;
#pragma unroll
    for (int g = 0; g < 8; ++g) {
        const float f = exp2f(s_m[g] - mu);
        lt += f * s_l[g];
        ot += f * s_o[g][tid];
    }
    store_result(a, (size_t)r * a.g + qi, tid, MM, lt, ot);
}

hipError_t launch_decode_q8(const DecodeQ8Args &a, hipStream_t s)
{
    hipEvent_t ev0, ev1;
    if (profile_pair(&ev0, &ev1))
        hipExtLaunchKernelGGL(decode_q8_kernel, dim3(Q8_GRID), dim3(256), 0, s, ev0, ev1, 0, a);
    else
        hipLaunchKernelGGL(decode_q8_kernel, dim3(Q8_GRID), dim3(256), 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(decode_q8_merge_kernel, dim3((unsigned)(a.B * a.H * a.per * a.g)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace sq
