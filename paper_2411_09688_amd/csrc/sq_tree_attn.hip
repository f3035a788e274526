// sq_tree_attn_q8: attention of many query tokens of a sequence (a tree or a chain of drafts) over e4m3 keys and values -- kept ranges of
// the fixed context and the pages of the user cache -- and over the drafts' own f16 rows behind a mask, one softmax over all of them.
//
// The G * T query rows of a (sequence, K/V head) read the same keys.  They are cut into blocks, row t * G + g the g-th head of draft
// t, so that a block of a chain sees a prefix of the drafts.  A wave has 16, 32 or 64 rows of a block (TILES of 16 columns of the matrix
// products); the four waves of a workgroup have the same rows and a quarter of the keys each, or rows of their own (row_waves) and
// the same keys.  Keys, laid end to end -- kept ones, the user's, drafts -- are cut into tiles of 32 and the tiles of all blocks into
// equal shares, one per workgroup; a second launch merges the blocks that several workgroups took.
//
//   S^T [32 keys x 16 TILES] = K q^T    codes to f16 (exact), once for all columns
//   t = S * (key's scale * sm_scale * log2 e) + log2(value's scale),   M = running maximum of t,   p = 2^(t - M + 14)
//   O^T [128 x 16 TILES]    += V^T P^T  codes to f16 (exact), P rounded to f16
//   l                       += p / value's scale                       (the unrounded p)
// With the value's scale in the exponent P needs no factor, whatever the scales are: it lies in (0, 2^14], and has its 11 bits down to 2^-28
// of the largest.  out = O / l, log-sum-exp = (M - 14 + log2 l) ln 2.
#include "sq_decode_q8.hpp"

namespace sq {

namespace {

constexpr int SENTINEL = INT32_MIN;
constexpr int GROUP = 64;                    // ranges that a wave holds at a time
constexpr int MAX_GROUPS = SELECT_MAX_C / GROUP;
constexpr float LIFT = 14.0f;                // p is at most 2^14

// 64 keys of a wave: where they stand (as in KeyList), and what their scales make of a score and of a probability.
template <bool WIDE>
struct TreeList {
    std::conditional_t<WIDE, unsigned long long, uint32_t> at[64];
    float mul[64], add[64], inv[64];
};

struct Unit {
    int b, h, block;
    int n;                                   // drafts of the sequence
    int nf, nu, tf, tu, td, total;           // keys and tiles: fixed, user's, drafts'
};

__device__ __forceinline__ int unit_rows(const TreeAttnArgs &a, int tiles) { return 16 * tiles * a.row_waves; }

// Unit i: the blocks of rows of a head follow one another, head by head, as rows of sq_decode_q8.
__device__ __forceinline__ Unit unit_of(const TreeAttnArgs &a, int i, int tiles)
{
    Unit u;
    u.block = i % a.blocks;
    const int hb = i / a.blocks;
    u.b = hb % a.B;
    u.h = hb / a.B;
    // (read side by side without a branch: of what is not there, some number that is not used)
    const int32_t *some = a.ranges ? a.n_keys : a.seq_len ? a.seq_len : a.n_drafts;
    const int32_t *pf = a.ranges ? a.n_keys + u.b * a.H + u.h : some, *pu = a.seq_len ? a.seq_len + u.b : some, *pn = a.n_drafts ? a.n_drafts + u.b : some;
    const int nf = pf ? *pf : 0, nu = pu ? *pu : 0, n = pn ? *pn : 0;
    u.n = a.n_drafts ? min(max(n, 0), a.T) : a.T;
    u.nf = a.ranges ? min(max(nf, 0), a.L) : 0;
    u.nu = a.seq_len ? min(max(nu, 0), a.max_pages << a.p_log) : 0;
    u.tf = (u.nf + QT - 1) / QT;
    u.tu = (u.nu + QT - 1) / QT;
    const int row0 = u.block * unit_rows(a, tiles), rows = min(u.n * a.G, row0 + unit_rows(a, tiles));
    const int seen = !a.Kd ? 0 : a.mask ? u.n : (rows - 1) / a.G + 1;       // (a chain's last row sees the drafts up to its own)
    u.td = (seen + QT - 1) / QT;
    u.total = rows > row0 ? max(1, u.tf + u.tu + u.td) : 0;                 // (a unit without rows has no tiles, one without keys one)
    return u;
}

__device__ __forceinline__ int block_exclusive(int v, int tid, int *s_w /*[4]*/, int &total)
{
    const int inc = wave_inclusive_scan(v, tid & 63);
    __syncthreads();
    if ((tid & 63) == 63) s_w[tid >> 6] = inc;
    __syncthreads();
    int ex = inc - v;
    for (int w = 0; w < (tid >> 6); ++w) ex += s_w[w];
    total = uniform(s_w[0] + s_w[1] + s_w[2] + s_w[3]);
    return ex;
}

__device__ __forceinline__ void store_row(const TreeAttnArgs &a, const Unit &u, int row, int d, float m, float l, float o)
{
    const int t = row / a.G, g = row - t * a.G;
    const size_t at = (((size_t)u.b * a.H + u.h) * a.G + g) * a.T + t;
    const bool any = l > 0.0f || l != l;
    a.out[at * D + d] = (_Float16)(any ? o / l : 0.0f);
    if (d == 0 && a.lse) a.lse[at] = any ? (m - LIFT + log2f(l)) * 0.69314718055994531f : SQ_NEG_INF;
}

// A wave's attention so far, as in Attending, for TILES times 16 columns.
template <int TILES>
struct Columns {
    float m[TILES], l[TILES];
    f4 o[TILES][8];
};

// Folds a tile's scores t (key 16 u + 4 g4 + i of column c16 in t[n][4 u + i]) into maximum and sum; p in f16 for the second product.
template <int TILES>
__device__ __forceinline__ void fold_scores(Columns<TILES> &st, const float (&t)[TILES][8], const float (&inv)[8], h8 (&p)[TILES])
{
#pragma unroll
    for (int n = 0; n < TILES; ++n) {
        const float mx = fmaxf(fmaxf(fmaxf(t[n][0], t[n][1]), fmaxf(t[n][2], t[n][3])), fmaxf(fmaxf(t[n][4], t[n][5]), fmaxf(t[n][6], t[n][7])));
        if (__any(mx > st.m[n])) {                          // (rare behind the first tiles)
            const float mn = fmaxf(st.m[n], cross16_max(mx));
            const float alpha = mn == SQ_NEG_INF ? 1.0f : __builtin_amdgcn_exp2f(st.m[n] - mn);
            st.m[n] = mn;
            st.l[n] *= alpha;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) st.o[n][dt] *= alpha;
        }
        const float base = st.m[n] == SQ_NEG_INF ? 0.0f : st.m[n] - LIFT;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = __builtin_amdgcn_exp2f(t[n][i] - base);
            st.l[n] += x * inv[i];
            p[n][i] = (_Float16)x;
        }
    }
}

}  // namespace

template <int TILES, bool WIDE>
__global__ __launch_bounds__(256, 2) void tree_attn_kernel(TreeAttnArgs a, int units, int grid)
{
    typedef std::conditional_t<WIDE, unsigned long long, uint32_t> offset_t;
    constexpr bool Q_IN_LDS = TILES == 4;
    constexpr int Q_BYTES = Q_IN_LDS ? 4 * 64 * D * 2 : 0;
    // The queries (64 rows of 256 bytes for each wave that has its own, 16 bytes at place p of row r standing at p ^ (r & 15)) and, behind the
    // keys, the waves' results of 16 rows.
    __shared__ __align__(16) char s_mem[Q_BYTES > (int)sizeof(WaveOut) ? Q_BYTES : (int)sizeof(WaveOut)];
    __shared__ __align__(16) TreeList<WIDE> s_list[4][2];
    __shared__ __align__(16) offset_t s_none[QT];           // where a wave reads ahead behind its last tile: the first row
    __shared__ int s_delta[4][64];
    __shared__ int s_group[MAX_GROUPS];
    __shared__ int s_w[4], s_found[2];
    __shared__ float s_ml[2][4][16];

    const int wave = uniform(threadIdx.x >> 6), tid = threadIdx.x;
    const int row_wave = wave % a.row_waves, key_wave = wave / a.row_waves, key_waves = 4 / a.row_waves;
    if (tid < QT) s_none[tid] = 0;
    __syncthreads();
    // This workgroup's share: tiles [t0, t1), counted from unit ui's first less unit_start.
    int share, per, t0, t1, ui, unit_start;
    Unit u;
    if (grid == 0) {
        ui = (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);       // (each XCD takes consecutive units)
        if (ui >= units) return;
        u = unit_of(a, ui, TILES);
        if (u.total == 0) return;
        share = ui;
        per = t1 = u.total;
        t0 = unit_start = 0;
    } else {
        const int each = (units + 255) / 256, i_lo = min(units, tid * each), i_hi = min(units, i_lo + each);
        int mine = 0, all;
        for (int i = i_lo; i < i_hi; ++i) mine += unit_of(a, i, TILES).total;
        int before = block_exclusive(mine, tid, s_w, all);
        const int shares = min(grid, (all + key_waves - 1) / key_waves), per_xcd = (shares + 7) / 8;      // (at least a tile for each wave)
        if (all == 0) return;
        per = (all + shares - 1) / shares;
        share = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
        if ((int)(blockIdx.x >> 3) >= per_xcd || (long long)share * per >= all) return;
        t0 = share * per;
        t1 = min(all, t0 + per);
        if (before <= t0 && t0 < before + mine) {
            int i = i_lo;
            for (;; ++i) {
                const int n = unit_of(a, i, TILES).total;
                if (t0 < before + n) break;
                before += n;
            }
            s_found[0] = i;
            s_found[1] = before;
        }
        __syncthreads();
        ui = uniform(s_found[0]);
        unit_start = uniform(s_found[1]);
        u = unit_of(a, ui, TILES);
    }

    for (;;) {
        const int lane = thread_here() & 63, c16 = lane & 15, g4 = lane >> 4;
        const int b = uniform(u.b), h = uniform(u.h), n_drafts = uniform(u.n), tf = uniform(u.tf), tu = uniform(u.tu);
        const int nf = uniform(u.nf), nu = uniform(u.nu), total = uniform(u.total);
        const size_t bh = (size_t)b * a.H + h;
        const int lo = max(t0 - unit_start, 0), hi = min(t1 - unit_start, total);
        const int row0 = u.block * unit_rows(a, TILES), end_row = n_drafts * a.G;      // rows from end_row on are nobody's
        // The queries.
        auto query = [&](int row) -> const h8 * {
            const int t = row / a.G, g = row - t * a.G;
            return reinterpret_cast<const h8 *>(a.q + ((bh * a.G + g) * a.T + t) * D);
        };
        h8 q[Q_IN_LDS ? 1 : TILES][4];
        h8 *const sq_ = reinterpret_cast<h8 *>(s_mem);
        if constexpr (Q_IN_LDS) {
            for (int i = tid; i < 64 * a.row_waves * 16; i += 256) {
                const int r = i >> 4, p = i & 15;
                h8 v = {};
                if (row0 + r < end_row) v = query(row0 + r)[p];
                sq_[r * 16 + (p ^ (r & 15))] = v;
            }
            __syncthreads();
        } else {
#pragma unroll
            for (int n = 0; n < TILES; ++n) {
                const int row = row0 + (row_wave * TILES + n) * 16 + c16;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const h8 zero = {};
                    q[n][s] = row < end_row ? query(row)[4 * g4 + s] : zero;
                }
            }
        }
        auto q_of = [&](int n, int s) {
            if constexpr (Q_IN_LDS) return sq_[((row_wave * 4 + n) * 16 + c16) * 16 + ((4 * g4 + s) ^ c16)];
            else return q[n][s];
        };
        Columns<TILES> st;
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            st.m[n] = SQ_NEG_INF;
            st.l[n] = 0.0f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) st.o[n][dt] = f4{0.f, 0.f, 0.f, 0.f};
        }

        // The head's ranges in groups of 64: how many keys lie before each group, for a wave to find its first.
        const global<i2v> rg = uniform(reinterpret_cast<const i2v *>(a.ranges) + bh * a.C);
        auto range_of = [&](int gi) { return rg[min(gi * GROUP + lane, a.C - 1)]; };   // as it stands in memory: see in_bounds
        const bool has_fixed = lo < tf;
        const int nr = uniform(has_fixed ? min(max(a.n_ranges[bh], 0), a.C) : 0), groups = (nr + GROUP - 1) / GROUP;
        auto in_bounds = [&](i2v e, int gi) {               // a lane's range of a group; (0, 0) behind the last
            const bool ok = gi * GROUP + lane < nr;
            return i2v{min(max(e.x, -MAX_L), MAX_L), ok ? min(max(e.y, 0), a.L) : 0};
        };
        if (has_fixed) {
            for (int gi = wave; gi < groups; gi += 4) {
                // (counts that sum to more than a head can have are cut, far from overflow)
                const int n = min(wave_sum_i(in_bounds(range_of(gi), gi).y), MAX_L);
                if (lane == 0) s_group[gi] = n;
            }
            __syncthreads();
        }

        // This wave's part of the tiles.
        const int w0 = lo + (int)((long long)(hi - lo) * key_wave / key_waves), w1 = lo + (int)((long long)(hi - lo) * (key_wave + 1) / key_waves);
        int phase = 0;
#pragma clang loop unroll(disable)
        for (; phase < 2; ++phase) {
            asm volatile("" : "+s"(phase));                 // (one copy of the loop below for both)
            const bool fixed = phase == 0;
            const int f0 = fixed ? w0 : max(w0 - tf, 0);    // first tile of the phase, and how many
            const int tiles = (fixed ? min(w1, tf) : min(w1 - tf, tu)) - f0;
            if (tiles <= 0) continue;
            const size_t head = fixed ? (size_t)h * a.L * D : 0;
            const global<uint8_t> Kb = uniform((fixed ? a.K8 : a.cK) + head), Vb = uniform((fixed ? a.V8 : a.cV) + head);
            const global<float> kscale = uniform(fixed ? a.ks : a.cks), vscale = uniform(fixed ? a.vs : a.cvs);
            const global<int32_t> pages = uniform(a.page_table + (size_t)b * a.max_pages);
            int p = f0 * QT;                                // the next position to list
            int end;                                        // where the keys end
            // ranges in hand: group gi, its lanes' first positions, where it ends; the group behind it is on its way
            int gi = 0, first = 0, ends = 0;
            i2v e = {0, 0}, e_next = {0, 0};                 // user: e.x is the page of position p + lane, read ahead
            if (fixed) {
                int sum[MAX_GROUPS / 64], at = 0, start = 0;
#pragma unroll
                for (int i = 0; i < MAX_GROUPS / 64; ++i) {
                    sum[i] = 4 * lane + i < groups ? s_group[4 * lane + i] : 0;
                    at += sum[i];
                }
                const int inc = wave_inclusive_scan(at, lane), listed = __builtin_amdgcn_readlane(inc, 63);
                at = inc - at;
                int here = 0;                               // groups that end at or before p
#pragma unroll
                for (int i = 0; i < MAX_GROUPS / 64; ++i) {
                    const bool passed = 4 * lane + i < groups && at + sum[i] <= p;
                    here += __popcll(__ballot(passed));
                    start += passed ? sum[i] : 0;
                    at += sum[i];
                }
                gi = uniform(max(min(here, groups - 1), 0));
                start = uniform(wave_sum_i(start));
                e = in_bounds(range_of(gi), gi);
                end = min(nf, listed);
                e_next = range_of(gi + 1);
                const int c = wave_inclusive_scan(e.y, lane);
                first = start + c - e.y;
                ends = uniform(start + __builtin_amdgcn_readlane(c, 63));
            } else {
                end = nu;
                e.x = pages[min(p + lane, end - 1) >> a.p_log];
            }

            float ks = 0.0f, vs = 1.0f;
            unsigned long long seen = 0ull, seen_next = 0ull;   // slots with a key, of the list in use and the next
            // Lists positions p .. p + 63 and starts to read their scales.
            auto list = [&](int buf) {
                bool ok = p + lane < end;
                offset_t at = 0;
                int sc = 0;
                if (fixed) {
                    s_delta[wave][lane] = SENTINEL;
                    wave_lds_sync();
                    for (;;) {
                        const int from = max(first, p), to = min(first + e.y, p + 64);
                        if (from < to) s_delta[wave][from - p] = e.x - first;
                        if (ends >= p + 64 || gi + 1 >= groups) break;
                        gi = uniform(gi + 1);
                        e = in_bounds(e_next, gi);
                        e_next = range_of(gi + 1);
                        const int c = wave_inclusive_scan(e.y, lane);
                        first = ends + c - e.y;
                        ends = uniform(min(ends + __builtin_amdgcn_readlane(c, 63), MAX_L + MAX_L));
                    }
                    wave_lds_sync();
                    const unsigned long long marks = __ballot(s_delta[wave][lane] != SENTINEL) & (~0ull >> (63 - lane));
                    ok = ok && marks != 0ull;
                    if (ok) {
                        const int d = s_delta[wave][63 - __clzll((long long)marks)];
                        const int key = min(max(p + lane + d, 0), a.L - 1);
                        at = (offset_t)key * D;
                        sc = h * a.sblocks + (key >> 6);
                    }
                } else {
                    const int t = p + lane;
                    ok = ok && e.x >= 0 && e.x < a.n_pages;
                    if (ok) {
                        sc = e.x * a.H + h;
                        at = (((offset_t)sc << a.p_log) + (t & ((1 << a.p_log) - 1))) * D;
                    }
                    e.x = pages[min(t + 64, end - 1) >> a.p_log];
                }
                ks = 0.0f;
                vs = 1.0f;
                if (ok) {
                    ks = kscale[sc];
                    vs = vscale[sc];
                }
                s_list[wave][buf].at[lane] = at;
                seen_next = __ballot(ok);
                p += 64;
                wave_lds_sync();
            };
            auto list_scales = [&](int buf) {
                s_list[wave][buf].mul[lane] = ks * a.scale;
                s_list[wave][buf].add[lane] = log2f(vs);
                s_list[wave][buf].inv[lane] = 1.0f / vs;
                wave_lds_sync();
            };
            u4v k[2][2];                                    // keys c16 and 16 + c16, dimensions 32 g4 ..
            u2v v[8];                                       // keys 4 g4 .. and 16 + 4 g4 .., dimensions 8 c16 ..
            auto load_k = [&](int t) {
                const auto *at = t < tiles ? s_list[wave][(t >> 1) & 1].at + (t & 1) * QT : s_none;
                const offset_t k0 = at[c16] + 32 * g4, k1 = at[16 + c16] + 32 * g4;
                k[0][0] = *reinterpret_cast<global<u4v>>(Kb + k0);
                k[0][1] = *reinterpret_cast<global<u4v>>(Kb + k0 + 16);
                k[1][0] = *reinterpret_cast<global<u4v>>(Kb + k1);
                k[1][1] = *reinterpret_cast<global<u4v>>(Kb + k1 + 16);
            };
            auto load_v = [&](int t) {
                const auto *at = (t < tiles ? s_list[wave][(t >> 1) & 1].at + (t & 1) * QT : s_none) + 4 * g4;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = *reinterpret_cast<global<u2v>>(Vb + (offset_t)(at[(i < 4 ? 0 : 12) + i] + 8 * c16));
            };

            list(0);
            load_k(0);
            load_v(0);
            list_scales(0);
            for (int t = 0; t < tiles; ++t) {
                const int buf = (t >> 1) & 1, slot = (t & 1) * QT;
                const bool even = !(t & 1);
                if (even) {
                    seen = seen_next;
                    if (t + 2 < tiles) list(buf ^ 1);
                }
                f4 acc[TILES][2];
#pragma unroll
                for (int n = 0; n < TILES; ++n) acc[n][0] = acc[n][1] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const u4v x0 = k[0][s >> 1], x1 = k[1][s >> 1];
                    const h8 k0 = s & 1 ? codes_f16(x0.z, x0.w) : codes_f16(x0.x, x0.y), k1 = s & 1 ? codes_f16(x1.z, x1.w) : codes_f16(x1.x, x1.y);
#pragma unroll
                    for (int n = 0; n < TILES; ++n) {
                        const h8 qv = q_of(n, s);
                        acc[n][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qv, acc[n][0], 0, 0, 0);
                        acc[n][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qv, acc[n][1], 0, 0, 0);
                    }
                }
                load_k(t + 1);                              // (as soon as the scores have used this tile's)
                float x[TILES][8], inv[8];
                {
                    const TreeList<WIDE> &ls = s_list[wave][buf];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int at = slot + 16 * j + 4 * g4;
                        const f4 mul = *reinterpret_cast<const f4 *>(ls.mul + at), add = *reinterpret_cast<const f4 *>(ls.add + at),
                                 iv = *reinterpret_cast<const f4 *>(ls.inv + at);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            inv[4 * j + i] = iv[i];
#pragma unroll
                            for (int n = 0; n < TILES; ++n) x[n][4 * j + i] = fmaf(acc[n][j][i], mul[i], add[i]);
                        }
                    }
                }
                uint32_t w[2][8];                           // V: words of dimensions 8 c16 .. + 3 and .. + 7
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    w[0][i] = v[i].x;
                    w[1][i] = v[i].y;
                }
                const uint32_t keys = (uint32_t)(seen >> slot);
                if (keys != 0xffffffffu) {                  // slots without a key: what stands in their row is not looked at
                    const uint32_t mine = keys >> (4 * g4);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (!(mine >> (i < 4 ? i : 12 + i) & 1u)) {
#pragma unroll
                            for (int n = 0; n < TILES; ++n) x[n][i] = SQ_NEG_INF;
                            w[0][i] = w[1][i] = 0u;
                        }
                }
                h8 pr[TILES];
                fold_scores(st, x, inv, pr);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    transpose4(w[i][0], w[i][1], w[i][2], w[i][3]);
                    transpose4(w[i][4], w[i][5], w[i][6], w[i][7]);
                }
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    const h8 vf = codes_f16(w[dt >> 2][dt & 3], w[dt >> 2][4 + (dt & 3)]);
#pragma unroll
                    for (int n = 0; n < TILES; ++n) st.o[n][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pr[n], st.o[n][dt], 0, 0, 0);
                }
                load_v(t + 1);
                if (even && t + 2 < tiles) list_scales(buf ^ 1);
            }
        }

        // The drafts: f16 rows, read as they are needed.
        if (w1 > tf + tu && a.Kd) {
            const _Float16 *Kd = a.Kd + bh * a.T * D, *Vd = a.Vd + bh * a.T * D;
            const int words = (a.T + 31) / 32;
            int draft[TILES];                               // of the lane's columns
#pragma unroll
            for (int n = 0; n < TILES; ++n) draft[n] = min(row0 + (row_wave * TILES + n) * 16 + c16, end_row - 1) / a.G;
            for (int t = max(w0 - tf - tu, 0); t < w1 - tf - tu; ++t) {
                const int key0 = t * QT;
                auto row_at = [&](int key) { return (size_t)min(key0 + key, n_drafts - 1) * D; };
                f4 acc[TILES][2];
#pragma unroll
                for (int n = 0; n < TILES; ++n) acc[n][0] = acc[n][1] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    const h8 k0 = *reinterpret_cast<const h8 *>(Kd + row_at(c16) + 32 * g4 + 8 * s);
                    const h8 k1 = *reinterpret_cast<const h8 *>(Kd + row_at(16 + c16) + 32 * g4 + 8 * s);
#pragma unroll
                    for (int n = 0; n < TILES; ++n) {
                        const h8 qv = q_of(n, s);
                        acc[n][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k0, qv, acc[n][0], 0, 0, 0);
                        acc[n][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k1, qv, acc[n][1], 0, 0, 0);
                    }
                }
                h8 v[8];
                uint32_t odd = 0;                           // bit 15 or 31: an infinity or NaN among the lane's values
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[i] = *reinterpret_cast<const h8 *>(Vd + row_at(4 * g4 + (i < 4 ? i : 12 + i)) + 8 * c16);
                    const u4v bits = __builtin_bit_cast(u4v, v[i]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) odd |= (bits[c] & 0x7fff7fffu) + 0x04000400u;
                }
                const bool strange = __any((odd & 0x80008000u) != 0u);
                float x[TILES][8], inv[8];
                uint32_t sees[TILES];
                const uint32_t there = n_drafts - key0 >= 32 ? ~0u : (1u << (n_drafts - key0)) - 1u;
#pragma unroll
                for (int n = 0; n < TILES; ++n) {
                    const int own = draft[n] - key0;        // a chain: keys up to the draft itself
                    sees[n] = a.mask ? a.mask[((size_t)b * a.T + draft[n]) * words + t] : own >= 31 ? ~0u : own < 0 ? 0u : (2u << own) - 1u;
                    sees[n] &= there;
                    const uint32_t mine = sees[n] >> (4 * g4);
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[n][i] = mine >> (i < 4 ? i : 12 + i) & 1u ? acc[n][i >> 2][i & 3] * a.scale : SQ_NEG_INF;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) inv[i] = 1.0f;
                h8 pr[TILES];
                fold_scores(st, x, inv, pr);
                if (__builtin_expect(strange, 0)) {
                    // Infinities and NaN among the values reach the columns that see their draft, and no others: they are taken out of the
                    // product and added one by one.
                    for (int key = 0; key < 32; ++key) {
                        const int from = (key & 15) >> 2, i = (key & 3) + (key >> 4) * 4;
#pragma unroll
                        for (int n = 0; n < TILES; ++n) {
                            float mine = 0.0f;
#pragma unroll
                            for (int c = 0; c < 8; ++c) mine = c == i ? (float)pr[n][c] : mine;
                            const float pv = __shfl(mine, from * 16 + c16);
                            if (sees[n] >> key & 1u) {
#pragma unroll
                                for (int c = 0; c < 4; ++c) {
                                    const h8 z = *reinterpret_cast<const h8 *>(Vd + row_at(key) + 32 * g4 + 8 * c);
#pragma unroll
                                    for (int dt = 0; dt < 8; ++dt)
                                        if (!((float)z[dt] - (float)z[dt] == 0.0f)) st.o[n][dt][c] += pv * (float)z[dt];
                                }
                            }
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            if (!((float)v[i][c] - (float)v[i][c] == 0.0f)) v[i][c] = (_Float16)0.0f;
                }
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    const h8 vf = h8{v[0][dt], v[1][dt], v[2][dt], v[3][dt], v[4][dt], v[5][dt], v[6][dt], v[7][dt]};
#pragma unroll
                    for (int n = 0; n < TILES; ++n) st.o[n][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pr[n], st.o[n][dt], 0, 0, 0);
                }
            }
        }

        // The waves' results, 16 rows of each at a time; those of the same rows are joined.
        __syncthreads();                                    // (the queries have been read)
        WaveOut &out = *reinterpret_cast<WaveOut *>(s_mem);
        const bool whole = lo == 0 && hi == total;
        const int slot = share + ui;
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            const float l = cross16_sum(st.l[n]);
            if (g4 == 0) {
                s_ml[0][wave][c16] = st.m[n];
                s_ml[1][wave][c16] = l;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float *dst = &out.o[wave][c16][32 * g4 + 8 * i];
                *reinterpret_cast<f4 *>(dst) = f4{st.o[n][0][i], st.o[n][1][i], st.o[n][2][i], st.o[n][3][i]};
                *reinterpret_cast<f4 *>(dst + 4) = f4{st.o[n][4][i], st.o[n][5][i], st.o[n][6][i], st.o[n][7][i]};
            }
            __syncthreads();
            const int here = thread_here();
            for (int i = here; i < a.row_waves * 16 * D; i += 256) {
                const int d = i & 127, c = i >> 7 & 15, rw = i >> 11;
                const int in_block = (rw * TILES + n) * 16 + c;
                if (row0 + in_block >= end_row) continue;
                float m = SQ_NEG_INF, ls = 0.0f, o = 0.0f;
                for (int kw = 0; kw < key_waves; ++kw) m = fmaxf(m, s_ml[0][kw * a.row_waves + rw][c]);
                const float mu = m == SQ_NEG_INF ? 0.0f : m;
                for (int kw = 0; kw < key_waves; ++kw) {
                    const int w = kw * a.row_waves + rw;
                    const float f = __builtin_amdgcn_exp2f(s_ml[0][w][c] - mu);
                    ls += f * s_ml[1][w][c];
                    o += f * out.o[w][c][d];
                }
                if (whole) store_row(a, u, row0 + in_block, d, m, ls, o);
                else store_partial(a.part + ((size_t)slot * unit_rows(a, TILES) + in_block) * PART_STRIDE, d, Joined{m, ls, o});
            }
            __syncthreads();
        }
        if (grid == 0) return;
        if (tid == 0 && lo == 0) {
            const int last = (unit_start + total - 1) / per;
            a.info[ui] = int2{slot, whole ? 0 : last - share + 1};
        }
        unit_start += total;
        if (unit_start >= t1) break;
        do u = unit_of(a, ++ui, TILES);
        while (u.total == 0);
    }
}

// Rows of blocks that several workgroups took, a wave each: two halves fold every other partial result, a lane four dimensions.
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeAttnArgs a, int tiles)
{
    const int rows = unit_rows(a, tiles), at = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, quad = lane & 31;
    const int ui = at / rows, in_block = at - ui * rows;
    if (ui >= a.B * a.H * a.blocks) return;
    const Unit u = unit_of(a, ui, tiles);
    const int row = u.block * rows + in_block;
    if (row >= u.n * a.G) return;
    const int2 info = a.info[ui];
    if (info.y == 0) return;
    float M = SQ_NEG_INF, ls = 0.0f;
    f4 os = {0.f, 0.f, 0.f, 0.f};
    auto fold = [&](float pm, float pl, f4 po) {
        const float mn = fmaxf(M, pm), mu = mn == SQ_NEG_INF ? 0.0f : mn;
        const float fa = exp2f(M - mu), fb = exp2f(pm - mu);
        ls = ls * fa + pl * fb;
        os = os * fa + po * fb;
        M = mn;
    };
    auto part = [&](int i) { return a.part + ((size_t)(info.x + i) * rows + in_block) * PART_STRIDE; };
    int i = half;
    for (; i + 2 < info.y; i += 4) {
        const float *p = part(i), *q = part(i + 2);
        const float2 a0 = *reinterpret_cast<const float2 *>(p), a1 = *reinterpret_cast<const float2 *>(q);
        const f4 o0 = *reinterpret_cast<const f4 *>(p + 4 + 4 * quad), o1 = *reinterpret_cast<const f4 *>(q + 4 + 4 * quad);
        fold(a0.x, a0.y, o0);
        fold(a1.x, a1.y, o1);
    }
    if (i < info.y) {
        const float *p = part(i);
        fold(p[0], p[1], *reinterpret_cast<const f4 *>(p + 4 + 4 * quad));
    }
    const float m2 = __shfl_xor(M, 32), l2 = __shfl_xor(ls, 32);
    f4 o2;
#pragma unroll
    for (int c = 0; c < 4; ++c) o2[c] = __shfl_xor(os[c], 32);
    if (half) return;
    fold(m2, l2, o2);
#pragma unroll
    for (int c = 0; c < 4; ++c) store_row(a, u, row, 4 * quad + c, M, ls, os[c]);
}

TreePlan tree_plan(int B, int H, int rows)
{
    TreePlan p{};
    p.tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    p.row_waves = rows <= 64 ? 1 : rows <= 128 ? 2 : 4;
    const int block = 16 * p.tiles * p.row_waves;
    p.blocks = (rows + block - 1) / block;
    p.units = (long long)B * H * p.blocks;
    p.grid = p.units < TREE_GRID ? TREE_GRID : 0;
    p.parts = p.grid ? (size_t)(TREE_GRID + p.units) * block : 0;
    return p;
}

hipError_t launch_tree_attn(TreeAttnArgs a, hipStream_t s)
{
    const TreePlan p = tree_plan(a.B, a.H, a.G * a.T);
    const bool wide = ((size_t)a.n_pages * a.H << a.p_log) * D > (1ull << 32);
    a.row_waves = p.row_waves;
    a.blocks = p.blocks;
    const int units = (int)p.units, grid = p.grid ? p.grid : (units + 7) / 8 * 8;
    auto *kernel = p.tiles == 1 ? (wide ? tree_attn_kernel<1, true> : tree_attn_kernel<1, false>)
                   : p.tiles == 2 ? (wide ? tree_attn_kernel<2, true> : tree_attn_kernel<2, false>)
                                  : (wide ? tree_attn_kernel<4, true> : tree_attn_kernel<4, false>);
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, s, a, units, p.grid);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.grid) return e;
    const long long rows = p.units * 16 * p.tiles * p.row_waves;
    hipLaunchKernelGGL(tree_merge_kernel, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a, p.tiles);
    return hipGetLastError();
}

}  // namespace sq
