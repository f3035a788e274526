// sq_tree_attn_q8: attention of many query tokens of a sequence (a tree or a chain of drafts) over e4m3 keys and values -- kept ranges of
// the fixed context and the pages of the user cache -- and over the drafts' own f16 rows behind a mask, one softmax over all of them.
//
// The G * T query rows of a (sequence, K/V head) read the same keys.  They are cut into blocks of 16, 32, 48 or 64 (TILES times the 16 columns
// of a matrix product; see tree_plan), row t * G + g the g-th head of draft t, so that a block of a chain sees a prefix of the drafts.  The four
// waves of a workgroup have the same rows and a quarter of the keys each.  Keys, laid end to end -- kept ones, the user's, drafts -- are cut into
// tiles of 32 and the tiles of all blocks into equal shares, one per workgroup; a second launch merges the blocks that several workgroups took.
//
//   S^T [32 keys x 16 TILES] = K q^T    codes to f16 (exact), once for all columns
//   t = S * (key's scale * sm_scale * log2 e) + log2(value's scale),   M: a reference near the maximum of t,   p = 2^(t - M + 8)
//   O^T [128 x 16 TILES]    += V^T P^T  codes to f16 (exact), P rounded to f16
//   l                       += p / value's scale                       (the unrounded p)
// With the value's scale in the exponent P needs no factor: it is at most 2^15, and has its 11 bits down to 2^-22 of the largest.
// (Rounded to f16 as in the prefill steps: as two bf16 numbers, as in decode, the second product would be made twice, where the units are the
// bound.  Against 64 bits the results are off by 2.8e-4 of their size, 2.1e-4 of it the f16 output's own rounding.)
// out = O / l, log-sum-exp = (M - 8 + log2 l) ln 2.
// The sum takes p / scale from p, so that scales must not lie too far apart: those below 2^-40 count as 2^-40 (LEAST_SCALE; a value is then off by
// less than 448 * 2^-40 < 2^-31, where f16 has steps of 2^-24), and above 2^40 is outside the contract.  Within 2^80 of one another a key drops
// out of the sum (its p, or the factor by which a reference moves, below fp32's 2^-126) only where its weight is under 2^-46 of the largest: 2^23
// such keys are one part in 2^23.  And no term overflows: 2^15 * 2^40 a key.
//
// What bounds it, and what a call takes, both launches, one call after the other (us; 8 K/V heads of 4 query heads):
//   4 heads of 8 drafts, 4K + 128 keys, 1/4 kept     11.5   the launches, and a search, a prologue and a tile whose reads come from HBM
//   1 sequence of 64 drafts, 32K + 512 keys, 1/8 kept     27.5   the same, and 2 to 3 tiles a wave: floor 4.2
//   16 sequences of 13 drafts, 128K keys, 1/16 kept, 4K user's     98 to 102 by card   the reads: 370 MB, at 5 TB/s while the loops run (72 us), the
//     rest beginning and ending blocks.  (Sequences are not joined: the keys that any of them keeps are 280 MB.)
//   a chain of 2048, 32K + 1K keys, 1/8 kept     297   the vector units (conversion, softmax) and the matrix units, which at two waves
//     a SIMD hardly overlap: 205 GFLOP at 690 TFLOP/s in all, 850 to 890 in the loop over codes, half as much in the loop over drafts
//   the cache alone, 32K tokens of 64 drafts     68   34 GFLOP and 68 MB, the same units; 16 sequences of up to 4K of 13 drafts     44   106 MB
// The merge is 4 to 7 of it, of the chain 10.
// Tried there: three workgroups a CU at 32 rows 31.5 -> 37 us, one wave a SIMD 1.55 times the time, 48 / 32 rows of a long chain 303 -> 333 / 372,
// raised or lowered wave priority 5 to 10 % slower either way.
#include <algorithm>

#include "sq_decode_q8.hpp"

namespace sq {

namespace {

constexpr int GROUP = 64;                    // ranges that a wave holds at a time
constexpr int MAX_GROUPS = SELECT_MAX_C / GROUP;
// The reference M of a column follows its largest t once that is more than 2^SLACK times it: of 64 columns one finds a new maximum in most
// tiles, and moving a reference costs as much as half a tile.
constexpr float LIFT = 8.0f, SLACK = 7.0f;   // p is at most 2^15
constexpr float LEAST_SCALE = 0x1p-40f;      // of values

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
struct Counts {
    int nf, nu, n;                           // as they stand in memory
};

// Unit i: the blocks of rows of a head follow one another, head by head, as rows of sq_decode_q8.
__device__ __forceinline__ Unit place_of(const TreeAttnArgs &a, int i)
{
    Unit u;
    const int hb = i / a.blocks;
    u.block = i - hb * a.blocks;
    u.h = hb / a.B;
    u.b = hb - u.h * a.B;
    return u;
}
// A unit's numbers, read side by side without a branch (of what is not there, some number that is not used).
__device__ __forceinline__ Counts counts_of(const TreeAttnArgs &a, const Unit &u)
{
    const int32_t *any = a.ranges ? a.n_keys : a.seq_len ? a.seq_len : a.n_drafts ? a.n_drafts : reinterpret_cast<const int32_t *>(a.q);
    const int32_t *nf = a.ranges ? a.n_keys + u.b * a.H + u.h : any, *nu = a.seq_len ? a.seq_len + u.b : any, *n = a.n_drafts ? a.n_drafts + u.b : any;
    return Counts{*nf, *nu, *n};
}
__device__ __forceinline__ void count(const TreeAttnArgs &a, const Counts &c, int tiles, Unit &u)
{
    u.n = a.n_drafts ? min(max(c.n, 0), a.T) : a.T;
    u.nf = a.ranges ? min(max(c.nf, 0), a.L) : 0;
    u.nu = a.seq_len ? min(max(c.nu, 0), a.max_pages << a.p_log) : 0;
    u.tf = (u.nf + QT - 1) / QT;
    u.tu = (u.nu + QT - 1) / QT;
    const int row0 = u.block * 16 * tiles, rows = min(u.n * a.G, row0 + 16 * tiles);
    const int seen = !a.Kd ? 0 : a.mask ? u.n : (rows - 1) / a.G + 1;       // (a chain's last row sees the drafts up to its own)
    u.td = (seen + QT - 1) / QT;
    u.total = rows > row0 ? max(1, u.tf + u.tu + u.td) : 0;                 // (a unit without rows has no tiles, one without keys one)
}
__device__ __forceinline__ Unit unit_of(const TreeAttnArgs &a, int i, int tiles)
{
    Unit u = place_of(a, i);
    count(a, counts_of(a, u), tiles, u);
    return u;
}

// The kernel's arguments, read again from where they stand: what is read from the one reference is not kept for the other, some 60 scalar
// registers that the loops need.
__device__ __forceinline__ const TreeAttnArgs &arguments()
{
    auto p = (const __attribute__((address_space(4))) TreeAttnArgs *)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const TreeAttnArgs *)p;
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

// Dimensions d .. d + 7 of a row's result: l is zero where it sees no key, and NaN where it sees one.
__device__ __forceinline__ void store_dims(const TreeAttnArgs &a, const Unit &u, int row, int d, float m, float l, f4 x, f4 y)
{
    const int t = row / a.G, g = row - t * a.G;
    const size_t at = (((size_t)u.b * a.H + u.h) * a.G + g) * a.T + t;
    const bool any = l > 0.0f || l != l;
    h8 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = (_Float16)(any ? x[i] / l : 0.0f);
        v[4 + i] = (_Float16)(any ? y[i] / l : 0.0f);
    }
    *reinterpret_cast<h8 *>(a.out + at * D + d) = v;
    if (d == 0 && a.lse) a.lse[at] = any ? (m - LIFT + log2f(l)) * 0.69314718055994531f : SQ_NEG_INF;
}

// A wave's attention so far, as in Attending, for TILES times 16 columns.
template <int TILES>
struct Columns {
    float m[TILES], l[TILES];
    f4 o[TILES][8];
};

// The lane's number, computed where it stands, so that nothing is held for it (or kept in memory, and waited for behind the keys).
__device__ __forceinline__ int lane_here()
{
    int l;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
    return l;
}

// The largest of eight numbers in four instructions (fmaxf takes as many again to quiet its operands, which here are results).
__device__ __forceinline__ float largest8(const float (&x)[8])
{
    float a, b;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(a) : "v"(x[0]), "v"(x[1]), "v"(x[2]));
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(b) : "v"(x[3]), "v"(x[4]), "v"(x[5]));
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(a) : "v"(x[6]), "v"(x[7]), "v"(a));
    asm("v_max_f32 %0, %1, %2" : "=v"(a) : "v"(a), "v"(b));
    return a;
}

// Folds a tile's scores x (key 16 u + 4 g4 + i of column c16 in x[n][4 u + i]) into the maxima and sums of N tiles of columns; p in f16 for
// the second product.
template <int N>
__device__ __forceinline__ void fold_scores(float *m, float *l, f4 (*o)[8], const float (&x)[N][8], const float (&inv)[8], h8 *p)
{
    float mx[N];
    bool more = false;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        mx[n] = largest8(x[n]);
        more = more || mx[n] > m[n] + SLACK;
    }
    if (__any(more)) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const float mn = fmaxf(m[n], cross16_max(mx[n]));
            const float alpha = mn == SQ_NEG_INF ? 1.0f : __builtin_amdgcn_exp2f(m[n] - mn);
            m[n] = mn;
            l[n] *= alpha;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) o[n][dt] *= alpha;
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const float base = m[n] == SQ_NEG_INF ? 0.0f : m[n] - LIFT;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = __builtin_amdgcn_exp2f(x[n][i] - base);
            l[n] += e * inv[i];
            p[n][i] = (_Float16)e;
        }
    }
}

}  // namespace

template <int TILES, bool WIDE>
__global__ __launch_bounds__(256, 2) void tree_attn_kernel(TreeAttnArgs /* see arguments() */, TreePlan plan)
{
    typedef std::conditional_t<WIDE, unsigned long long, uint32_t> offset_t;
    constexpr bool Q_IN_LDS = TILES >= 2;
    // The queries (rows of 256 bytes, 16 bytes at place p of row r standing at p ^ (r & 15)), behind them a tile of the drafts' values for each
    // wave; when all keys are done, in their place two sums of results (of 512 bytes a row, likewise).
    constexpr int V_AT = Q_IN_LDS ? 16 * TILES * D * 2 : 0, V_TILE = QT * D * 2, RESULTS = 2 * 16 * TILES * D * sizeof(float);
    __shared__ __align__(16) char s_mem[RESULTS > V_AT + 4 * V_TILE ? RESULTS : V_AT + 4 * V_TILE];
    __shared__ __align__(16) TreeList<WIDE> s_list[4][2];
    __shared__ __align__(16) offset_t s_none[QT];           // where a wave reads ahead behind its last tile: the first row
    __shared__ int s_group[MAX_GROUPS];
    __shared__ int s_w[4], s_found[5];
    __shared__ float s_ml[2][4][16 * TILES];

    const int wave = uniform(threadIdx.x >> 6), tid = threadIdx.x;
    if (tid < QT) s_none[tid] = 0;
    __syncthreads();
    // This workgroup's share: [t0, t1) of the units' tiles, laid end to end with `ahead` more in front of each unit's for what it costs to
    // begin one (a share that begins inside a unit pays as much); unit ui begins at unit_start.
    int share, share0, per, t0, t1, ui, unit_start, ahead;   // share0 + t / per is who has tile t
    Unit u;
    if (plan.splits > 0) {
        // A workgroup per unit and part of it, without a look at the other units.
        const TreeAttnArgs &a = arguments();
        // (the last units first: of a chain those with the most drafts to see)
        share = gridDim.x - 1 - blockIdx.x;
        ui = share / plan.splits;
        u = unit_of(a, ui, TILES);
        per = max(4, (u.total + plan.splits - 1) / plan.splits);
        share0 = ui * plan.splits;
        t0 = (share - share0) * per;
        t1 = min(u.total, t0 + per);
        if (t0 >= t1) return;
        unit_start = ahead = 0;
    } else {
        const TreeAttnArgs &a = arguments();
        // Every thread counts up to four consecutive units, read side by side.
        const int units = plan.units, each = (units + 255) / 256, i_lo = tid * each;
        ahead = TREE_AHEAD;
        int totals[TREE_SHARED_UNITS / 256], mine = 0, all;
        Counts c[TREE_SHARED_UNITS / 256];
        {
            Unit v[TREE_SHARED_UNITS / 256];
            v[0] = place_of(a, min(i_lo, units - 1));
#pragma unroll
            for (int k = 0; k < TREE_SHARED_UNITS / 256; ++k) {
                if (k > 0) {                                // the unit behind it (the last one again where it ends)
                    v[k] = v[k - 1];
                    if (i_lo + k < units && ++v[k].block == a.blocks) {
                        v[k].block = 0;
                        if (++v[k].b == a.B) {
                            v[k].b = 0;
                            ++v[k].h;
                        }
                    }
                }
                c[k] = counts_of(a, v[k]);
            }
#pragma unroll
            for (int k = 0; k < TREE_SHARED_UNITS / 256; ++k) {
                count(a, c[k], TILES, v[k]);
                totals[k] = k < each && i_lo + k < units && v[k].total > 0 ? v[k].total + ahead : 0;
                mine += totals[k];
            }
        }
        int before = block_exclusive(mine, tid, s_w, all);
        const int shares = min(TREE_SHARES, (all + 3) / 4), per_xcd = (shares + 7) / 8;      // (at least a tile for each wave)
        if (all == 0) return;
        per = (all + shares - 1) / shares;
        share = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);             // (each XCD takes consecutive shares)
        if ((int)(blockIdx.x >> 3) >= per_xcd || (long long)share * per >= all) return;
        share0 = 0;
        t0 = share * per;
        t1 = min(all, t0 + per);
        if (before <= t0 && t0 < before + mine) {
            int i = i_lo;
            Counts found = c[0];
#pragma unroll
            for (int k = 0; k + 1 < TREE_SHARED_UNITS / 256; ++k)
                if (i == i_lo + k && t0 >= before + totals[k]) {
                    before += totals[k];
                    found = c[k + 1];
                    ++i;
                }
            s_found[0] = i;
            s_found[1] = before;
            s_found[2] = found.nf;
            s_found[3] = found.nu;
            s_found[4] = found.n;
        }
        __syncthreads();
        ui = uniform(s_found[0]);
        unit_start = uniform(s_found[1]);
        u = place_of(a, ui);
        count(a, Counts{s_found[2], s_found[3], s_found[4]}, TILES, u);
    }
    // (a share may end, or begin, in what stands in front of a unit's tiles)
    int slot = 2 * share;                                   // of its first unit's partial result; one of a later unit comes behind it
    for (;;) {
        const int lane = thread_here() & 63, c16 = lane & 15, g4 = lane >> 4;
        const int b = uniform(u.b), h = uniform(u.h), n_drafts = uniform(u.n), tf = uniform(u.tf), tu = uniform(u.tu);
        const int nf = uniform(u.nf), nu = uniform(u.nu), total = uniform(u.total);
        const size_t bh = (size_t)b * arguments().H + h;
        const int lo = max(t0 - unit_start - ahead, 0), hi = min(t1 - unit_start - ahead, total);
        if (lo >= hi) break;                                // (only of a last unit)
        const int row0 = u.block * 16 * TILES, end_row = n_drafts * arguments().G;      // rows from end_row on are nobody's
        const TreeAttnArgs &a = arguments();
        // The queries, and what says which keys: read side by side.
        auto query = [&](int row) {                         // of a row behind the last, the last row's
            const int r = min(row, end_row - 1), t = r / a.G, g = r - t * a.G;
            return reinterpret_cast<const h8 *>(a.q + ((bh * a.G + g) * a.T + t) * D);
        };
        const global<i2v> rg = uniform(reinterpret_cast<const i2v *>(a.ranges) + bh * a.C);
        auto range_of = [&](int gi) { return rg[min(gi * GROUP + lane, a.C - 1)]; };   // as it stands in memory: see in_bounds
        const bool has_fixed = lo < tf;
        i2v near[4] = {};                                   // up to four groups of 64 ranges every wave has in registers
        int nr = 0;
        if (has_fixed) {
#pragma unroll
            for (int k = 0; k < 4; ++k) near[k] = range_of(k);
            nr = a.n_ranges[bh];
        }
        h8 q[Q_IN_LDS ? 1 : TILES][4];
        h8 *const sq_ = reinterpret_cast<h8 *>(s_mem);
        if constexpr (Q_IN_LDS) {
            h8 v[TILES];
#pragma unroll
            for (int k = 0; k < TILES; ++k) v[k] = query(row0 + k * 16 + (tid >> 4))[tid & 15];
#pragma unroll
            for (int k = 0; k < TILES; ++k) sq_[(k * 16 + (tid >> 4)) * 16 + ((tid & 15) ^ (tid >> 4))] = v[k];
            __syncthreads();
        } else {
#pragma unroll
            for (int n = 0; n < TILES; ++n)
#pragma unroll
                for (int s = 0; s < 4; ++s) q[n][s] = query(row0 + n * 16 + c16)[4 * g4 + s];
        }
        auto q_of = [&](int n, int s) {
            if constexpr (Q_IN_LDS) return sq_[(n * 16 + c16) * 16 + ((4 * g4 + s) ^ c16)];
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

        // How many keys lie before each group of ranges, for a wave to find its first.
        nr = uniform(min(max(nr, 0), a.C));
        const int groups = (nr + GROUP - 1) / GROUP;
        auto in_bounds = [&](i2v e, int gi) {               // a lane's range of a group; (0, 0) behind the last
            const bool ok = gi * GROUP + lane < nr;
            return i2v{min(max(e.x, -MAX_L), MAX_L), ok ? min(max(e.y, 0), a.L) : 0};
        };
        if (groups > 4) {
            for (int g0 = wave; g0 < groups; g0 += 16) {    // (four groups read side by side: 77 groups 49.9 -> 47.2 us)
                i2v some[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) some[k] = range_of(g0 + 4 * k);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    // (counts that sum to more than a head can have are cut, far from overflow)
                    const int n = min(wave_sum_i(in_bounds(some[k], g0 + 4 * k).y), MAX_L);
                    if (lane == 0 && g0 + 4 * k < groups) s_group[g0 + 4 * k] = n;
                }
            }
            __syncthreads();
        }

        // This wave's part of the tiles: a quarter of the keys in 8 bits, and of the drafts, from the other end, so that what is left over of
        // the one goes to other waves than of the other.
        const int in8 = tf + tu, lo8 = min(lo, in8), n8 = min(hi, in8) - lo8, lod = max(lo - in8, 0), nd = max(hi - in8, 0) - lod;
        auto quarter = [](int n, int i) { return (int)((long long)n * i / 4); };
        const int w0 = lo8 + quarter(n8, wave), w1 = lo8 + quarter(n8, wave + 1);
        const int d0 = lod + quarter(nd, 3 - wave), d1 = lod + quarter(nd, 4 - wave);
        int phase = 0;
#pragma clang loop unroll(disable)
        for (; phase < 2; ++phase) {
            asm volatile("" : "+s"(phase));                 // (one copy of the loop below for both)
            const bool fixed = phase == 0;
            const TreeAttnArgs &a = arguments();
            const int f0 = fixed ? w0 : max(w0 - tf, 0);    // first tile of the phase, and how many
            const int tiles = (fixed ? min(w1, tf) : w1 - tf) - f0;
            if (tiles <= 0) continue;
            const size_t head = fixed ? (size_t)h * a.L * D : 0;
            const global<uint8_t> Kb = uniform((fixed ? a.K8 : a.cK) + head), Vb = uniform((fixed ? a.V8 : a.cV) + head);
            const global<float> kscale = uniform(fixed ? a.ks : a.cks), vscale = uniform(fixed ? a.vs : a.cvs);
            int p = f0 * QT;                                // the next position to list
            int end;                                        // where the keys end
            // ranges in hand: group gi, its lanes' first positions, where it ends
            int gi = 0, first = 0, ends = 0;
            i2v e = {0, 0};
            // the user's pages: that of position p + lane, read ahead (of kept keys some number that is not used)
            const global<int32_t> ids = fixed ? (global<int32_t>)rg : uniform(a.page_table + (size_t)b * a.max_pages);
            int id = 0;
            if (fixed) {
                int start = 0, listed = 0;                  // keys before group gi, keys of all groups
                if (groups <= 4) {
                    e = in_bounds(near[0], 0);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        listed += wave_sum_i(in_bounds(near[k], k).y);
                        if (k + 1 < groups && listed <= p) {
                            gi = k + 1;
                            start = listed;
                            e = in_bounds(near[k < 3 ? k + 1 : 3], k + 1);
                        }
                    }
                    listed = uniform(listed);
                } else {
                    int sum[MAX_GROUPS / 64], at = 0;
#pragma unroll
                    for (int i = 0; i < MAX_GROUPS / 64; ++i) {
                        sum[i] = 4 * lane + i < groups ? s_group[4 * lane + i] : 0;
                        at += sum[i];
                    }
                    const int inc = wave_inclusive_scan(at, lane);
                    listed = __builtin_amdgcn_readlane(inc, 63);
                    at = inc - at;
                    int here = 0;                           // groups that end at or before p
#pragma unroll
                    for (int i = 0; i < MAX_GROUPS / 64; ++i) {
                        const bool passed = 4 * lane + i < groups && at + sum[i] <= p;
                        here += __popcll(__ballot(passed));
                        start += passed ? sum[i] : 0;
                        at += sum[i];
                    }
                    gi = min(here, groups - 1);
                    start = wave_sum_i(start);
                    e = in_bounds(range_of(uniform(gi)), gi);
                }
                gi = uniform(gi);
                start = uniform(start);
                end = min(nf, listed);
                const int c = wave_inclusive_scan(e.y, lane);
                first = start + c - e.y;
                ends = uniform(start + __builtin_amdgcn_readlane(c, 63));
            } else {
                end = nu;
                id = ids[min(p + lane, end - 1) >> a.p_log];
            }

            // (The loop below reads memory in the same order in every round, without a branch around it: what is waited for is then counted
            // exactly, and the tile ahead stays on its way.  With reads under conditions the compiler drained them all, twice a tile.)
            float ks, vs;
            unsigned long long seen, seen_next;             // slots with a key, of the list in use and the next
            // Lists positions p .. p + 63 and starts to read their scales.
            auto list = [&](int buf) {
                const int lane = lane_here();
                bool ok = p + lane < end;
                int key = 0, sc = 0;
                offset_t at = 0;
                if (fixed) {
                    // The ranges that reach into these positions, one after the other.
                    bool found = false;
                    for (;;) {
                        unsigned long long here = __ballot(first < p + 64 && first + e.y > p && e.y > 0);
                        while (here != 0ull) {
                            const int r = __ffsll((long long)here) - 1;
                            here &= here - 1;
                            const int i = p + lane - __builtin_amdgcn_readlane(first, r);
                            const bool in = i >= 0 && i < __builtin_amdgcn_readlane(e.y, r);
                            key = in ? __builtin_amdgcn_readlane(e.x, r) + i : key;
                            found = found || in;
                        }
                        if (ends >= p + 64 || gi + 1 >= groups) break;
                        gi = uniform(gi + 1);
                        e = in_bounds(range_of(gi), gi);
                        const int c = wave_inclusive_scan(e.y, lane);
                        first = ends + c - e.y;
                        ends = uniform(min(ends + __builtin_amdgcn_readlane(c, 63), MAX_L + MAX_L));
                    }
                    ok = ok && found;
                    key = min(max(key, 0), a.L - 1);
                    at = (offset_t)key * D;
                    sc = h * a.sblocks + (key >> 6);
                } else {
                    const int t = p + lane;
                    ok = ok && id >= 0 && id < a.n_pages;
                    sc = id * a.H + h;
                    at = (((offset_t)sc << a.p_log) + (t & ((1 << a.p_log) - 1))) * D;
                }
                at = ok ? at : 0;
                sc = ok ? sc : 0;
                ks = kscale[sc];
                vs = vscale[sc];
                id = ids[fixed ? 0 : max(min(p + 64 + lane, end - 1), 0) >> a.p_log];
                s_list[wave][buf].at[lane] = at;
                seen_next = __ballot(ok);
                p += 64;
                wave_lds_sync();
            };
            auto list_scales = [&](int buf) {
                const int lane = lane_here();
                // (a slot without a key: not looked at, but for this.  A comparison in fmaxf's place keeps 50 more registers in memory at 64 rows:
                // chain 302 -> 337 us)
                const float v = seen_next >> lane & 1u ? fmaxf(vs, LEAST_SCALE) : 1.0f;
                s_list[wave][buf].mul[lane] = ks * a.scale;
                s_list[wave][buf].add[lane] = __builtin_amdgcn_logf(v);
                s_list[wave][buf].inv[lane] = __builtin_amdgcn_rcpf(v);
                wave_lds_sync();
            };
            u4v k[2][2];                                    // keys c16 and 16 + c16, dimensions 32 g4 ..
            u2v v[8];                                       // keys 4 g4 .. and 16 + 4 g4 .., dimensions 8 c16 ..
            auto load_k = [&](const offset_t *at) {
                const int l = lane_here(), c16 = l & 15, g4 = l >> 4;
                const offset_t k0 = at[c16] + 32 * g4, k1 = at[16 + c16] + 32 * g4;
                k[0][0] = *reinterpret_cast<global<u4v>>(Kb + k0);
                k[0][1] = *reinterpret_cast<global<u4v>>(Kb + k0 + 16);
                k[1][0] = *reinterpret_cast<global<u4v>>(Kb + k1);
                k[1][1] = *reinterpret_cast<global<u4v>>(Kb + k1 + 16);
            };
            auto load_v = [&](const offset_t *at) {
                const int l = lane_here(), c16 = l & 15, g4 = l >> 4;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = *reinterpret_cast<global<u2v>>(Vb + (offset_t)(at[4 * g4 + (i < 4 ? 0 : 12) + i] + 8 * c16));
            };
            // Folds slots slot .. + 31 of list buf and reads the tile at `next` in their place.
            auto tile = [&](int buf, int slot, const offset_t *next) {
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
                    if (Q_IN_LDS) __builtin_amdgcn_sched_barrier(0);      // (the queries of one step in registers at a time)
                }
                load_k(next);                               // (as soon as the scores have used this tile's)
                float x[TILES][8], inv[8];
                const TreeList<WIDE> &ls = s_list[wave][buf];
                const int g4 = lane_here() >> 4;
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
                    for (int i = 0; i < 8; ++i) {
                        const bool there = mine >> (i < 4 ? i : 12 + i) & 1u;
#pragma unroll
                        for (int n = 0; n < TILES; ++n) x[n][i] = there ? x[n][i] : SQ_NEG_INF;
                        w[0][i] = there ? w[0][i] : 0u;
                        w[1][i] = there ? w[1][i] : 0u;
                    }
                }
                h8 pr[TILES];
                fold_scores<TILES>(st.m, st.l, st.o, x, inv, pr);
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
                load_v(next);
            };

            list(0);
            load_k(s_list[wave][0].at);
            load_v(s_list[wave][0].at);
            list_scales(0);
#pragma clang loop unroll(disable)
            for (int t = 0, buf = 0; t < tiles; t += 2, buf ^= 1) {
                const offset_t *here = s_list[wave][buf].at, *next = t + 2 < tiles ? s_list[wave][buf ^ 1].at : s_none;
                seen = seen_next;
                list(buf ^ 1);
                tile(buf, 0, t + 1 < tiles ? here + QT : s_none);
                list_scales(buf ^ 1);
                if (t + 1 >= tiles) break;
                tile(buf, QT, next);
            }
        }

        // The drafts: f16 rows.
        if (d0 < d1 && arguments().Kd) {
            const TreeAttnArgs &a = arguments();
            typedef global<char> bytes;
            const bytes Kd = (bytes)uniform(a.Kd + bh * a.T * D), Vd = (bytes)uniform(a.Vd + bh * a.T * D);
            const int words = (a.T + 31) / 32;
            const global<uint32_t> mask = uniform(a.mask + (size_t)b * a.T * words);
            // (in LDS, where the results' maxima stand later: registers are short here)
            float *const s_draft = s_ml[0][wave];           // drafts of the columns, as a float's bits
#pragma unroll
            for (int n = 0; n < TILES; ++n) s_draft[n * 16 + c16] = __builtin_bit_cast(float, min(row0 + n * 16 + c16, end_row - 1) / a.G);
            wave_lds_sync();
            auto draft_of = [&](int n) { return __builtin_bit_cast(int, s_draft[n * 16 + c16]); };
            auto row_at = [&](int key) { return (uint32_t)min(key, n_drafts - 1) * (uint32_t)(D * sizeof(_Float16)); };
            // Values go to LDS past the registers: with them on their way in registers, 128 of which hold the output, some were kept in memory.
            char *const s_v = s_mem + V_AT + wave * V_TILE;
            const uint32_t lds_v = uniform((int)(uint32_t)(size_t)(__attribute__((address_space(3))) void *)s_v);
            auto load_v = [&](int t) {                      // rows 4 i + g4, 16 bytes a lane, one after the other
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // (the values in their place have been read)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds_v + (uint32_t)(i * 1024)),
                                 "v"(row_at(t * QT + 4 * i + g4) + 16 * c16), "s"(Vd) : "m0", "memory");
            };
            h8 k[2][4];
            auto load_k = [&](int t) {                      // (behind the last tile the last draft, again and again)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t at = row_at(t * QT + 16 * j + c16) + 64 * g4;
#pragma unroll
                    for (int s = 0; s < 4; ++s) k[j][s] = *reinterpret_cast<global<h8>>(Kd + at + 16 * s);
                }
            };
            bool strange = false;
            load_k(d0);
#pragma clang loop unroll(disable)
            for (int t = d0; t < d1; ++t) {
                const int key0 = t * QT;
                const uint32_t there = n_drafts - key0 >= 32 ? ~0u : (1u << (n_drafts - key0)) - 1u;
                float one[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) one[i] = 1.0f;
                h8 pr[TILES];
                // (two columns at a time, which leaves registers for the tile of values that is on its way)
                constexpr int PAIR = TILES == 4 ? 2 : TILES;
#pragma unroll
                for (int n0 = 0; n0 < TILES; n0 += PAIR) {
                    f4 acc[PAIR][2];
#pragma unroll
                    for (int n = 0; n < PAIR; ++n) acc[n][0] = acc[n][1] = f4{0.f, 0.f, 0.f, 0.f};
                    h8 qs[PAIR];
#pragma unroll
                    for (int n = 0; n < PAIR; ++n) qs[n] = q_of(n0 + n, 0);
#pragma unroll
                    for (int s = 0; s < 4; ++s) {
                        h8 next[PAIR];                      // (a step ahead: else the products wait for LDS four times)
#pragma unroll
                        for (int n = 0; n < PAIR; ++n) next[n] = s < 3 ? q_of(n0 + n, s + 1) : qs[n];
#pragma unroll
                        for (int n = 0; n < PAIR; ++n) {
                            acc[n][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[0][s], qs[n], acc[n][0], 0, 0, 0);
                            acc[n][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[1][s], qs[n], acc[n][1], 0, 0, 0);
                        }
                        if (Q_IN_LDS) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int n = 0; n < PAIR; ++n) qs[n] = next[n];
                    }
                    if (n0 == 0) load_v(t);                 // (behind the wait for this tile's keys)
                    if (n0 + PAIR == TILES) load_k(t + 1);
                    float x[PAIR][8];
#pragma unroll
                    for (int n = 0; n < PAIR; ++n) {
                        const int d = draft_of(n0 + n), own = d - key0;         // a chain: keys up to the draft itself
                        uint32_t sees = own >= 31 ? ~0u : own < 0 ? 0u : (2u << own) - 1u;
                        if (a.mask) sees = mask[(uint32_t)(d * words + t)];
                        sees &= there;
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[n][i] = acc[n][i >> 2][i & 3] * a.scale;
                        if (!__all(sees == ~0u)) {
                            const uint32_t mine = sees >> (4 * g4);
#pragma unroll
                            for (int i = 0; i < 8; ++i) x[n][i] = mine >> (i < 4 ? i : 12 + i) & 1u ? x[n][i] : SQ_NEG_INF;
                        }
                    }
                    fold_scores<PAIR>(st.m + n0, st.l + n0, st.o + n0, x, one, pr + n0);
                    if (Q_IN_LDS) __builtin_amdgcn_sched_barrier(0);
                }
                // (for the values, which the compiler does not count; the next keys have been waited for already, with the words of the mask)
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                h8 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const h8 *>(s_v + (4 * g4 + (i < 4 ? i : 12 + i)) * (D * 2) + 16 * c16);
                uint32_t odd = 0;                           // bit 15 or 31: an infinity or NaN among the lane's values
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) odd |= (__builtin_bit_cast(u4v, v[i])[c] & 0x7fff7fffu) + 0x04000400u;
                if (__builtin_expect(__any((odd & 0x80008000u) != 0u), 0)) {
                    strange = true;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            uint32_t &w = reinterpret_cast<uint32_t *>(&v[i])[c];
                            if ((w & 0x7c00u) == 0x7c00u) w &= 0xffff0000u;
                            if ((w & 0x7c000000u) == 0x7c000000u) w &= 0xffffu;
                        }
                }
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                    const h8 vf = h8{v[0][dt], v[1][dt], v[2][dt], v[3][dt], v[4][dt], v[5][dt], v[6][dt], v[7][dt]};
#pragma unroll
                    for (int n = 0; n < TILES; ++n) st.o[n][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pr[n], st.o[n][dt], 0, 0, 0);
                }
            }
            if (__builtin_expect(strange, 0)) {
                // Infinities and NaN among the values, which the products left out, reach the columns that see their draft, and no others.
#pragma clang loop unroll(disable)
                for (int key = d0 * QT; key < min(d1 * QT, n_drafts); ++key) {
                    h8 z[4];
                    bool any = false;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        z[c] = *reinterpret_cast<global<h8>>(Vd + (row_at(key) + 64 * g4) + 16 * c);
#pragma unroll
                        for (int dt = 0; dt < 8; ++dt) {
                            const bool finite = (float)z[c][dt] - (float)z[c][dt] == 0.0f;
                            any = any || !finite;
                            if (finite) z[c][dt] = (_Float16)0.0f;
                        }
                    }
                    if (!__any(any)) continue;
#pragma unroll
                    for (int n = 0; n < TILES; ++n) {
                        const int d = draft_of(n);
                        bool seen = key <= d;
                        if (a.mask) seen = mask[(uint32_t)(d * words + (key >> 5))] >> (key & 31) & 1u;
                        if (seen)
#pragma unroll
                            for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                                for (int c = 0; c < 4; ++c) st.o[n][dt][c] += (float)z[c][dt];
                    }
                }
            }
        }

        // Results: the waves' are joined in two buffers, waves 0 and 1 writing and 2 and 3 adding; a lane has dimensions 32 g4 + 8 i .. + 7 of
        // its columns, i = 0 .. 3.
        const TreeAttnArgs &r = arguments();
        const bool whole = lo == 0 && hi == total;
        wave_lds_sync();                                    // (s_draft has been read)
        auto out = [&](int buffer, int row, int place) {    // four dimensions of a row
            return reinterpret_cast<f4 *>(s_mem) + (buffer * 16 * TILES + row) * (D / 4) + (place ^ (row & 15));
        };
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            const float l = cross16_sum(st.l[n]);
            if (g4 == 0) {
                s_ml[0][wave][n * 16 + c16] = st.m[n];
                s_ml[1][wave][n * 16 + c16] = l;
            }
        }
        __syncthreads();                                    // (and the queries have been read)
        auto largest = [&](int c) { return fmaxf(fmaxf(s_ml[0][0][c], s_ml[0][1][c]), fmaxf(s_ml[0][2][c], s_ml[0][3][c])); };
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            const float m = largest(n * 16 + c16), f = __builtin_amdgcn_exp2f(st.m[n] - (m == SQ_NEG_INF ? 0.0f : m));
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) st.o[n][dt] *= f;
        }
        if (wave < 2) {
#pragma unroll
            for (int n = 0; n < TILES; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    *out(wave, n * 16 + c16, 8 * g4 + 2 * i) = f4{st.o[n][0][i], st.o[n][1][i], st.o[n][2][i], st.o[n][3][i]};
                    *out(wave, n * 16 + c16, 8 * g4 + 2 * i + 1) = f4{st.o[n][4][i], st.o[n][5][i], st.o[n][6][i], st.o[n][7][i]};
                }
        }
        __syncthreads();
        if (wave >= 2) {
#pragma unroll
            for (int n = 0; n < TILES; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    *out(wave - 2, n * 16 + c16, 8 * g4 + 2 * i) += f4{st.o[n][0][i], st.o[n][1][i], st.o[n][2][i], st.o[n][3][i]};
                    *out(wave - 2, n * 16 + c16, 8 * g4 + 2 * i + 1) += f4{st.o[n][4][i], st.o[n][5][i], st.o[n][6][i], st.o[n][7][i]};
                }
        }
        __syncthreads();
#pragma clang loop unroll(disable)
        for (int n = 0; n < TILES; ++n) {
            const int here = thread_here(), row = n * 16 + (here >> 4), d = 8 * (here & 15);
            if (row0 + row >= end_row) break;
            const float m = largest(row), mu = m == SQ_NEG_INF ? 0.0f : m;
            float ls = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) ls += __builtin_amdgcn_exp2f(s_ml[0][w][row] - mu) * s_ml[1][w][row];
            const f4 x = *out(0, row, d / 4) + *out(1, row, d / 4), y = *out(0, row, d / 4 + 1) + *out(1, row, d / 4 + 1);
            if (whole) store_dims(r, u, row0 + row, d, m, ls, x, y);
            else {
                float *p = r.part + ((size_t)slot * 16 * TILES + row) * PART_STRIDE;
                *reinterpret_cast<f4 *>(p + 4 + d) = x;
                *reinterpret_cast<f4 *>(p + 8 + d) = y;
                if (d == 0) *reinterpret_cast<float2 *>(p) = make_float2(m, ls);
            }
        }
        __syncthreads();
        if (plan.splits == 1) return;
        if (tid == 0 && lo == 0) {
            const int last = share0 + (unit_start + ahead + total - 1) / per;
            r.info[ui] = int2{slot, whole ? 0 : last - share + 1};      // (its other partial results are the first of their shares)
        }
        unit_start += ahead + total;
        if (unit_start >= t1) break;
        slot = 2 * share + 1;
        do u = unit_of(r, ++ui, TILES);
        while (u.total == 0);
    }
}

// Rows of blocks that several workgroups took: GROUPS times 16 lanes a row, eight dimensions a lane, each group of lanes every GROUPS-th
// partial result, four of them read side by side.  Bound by the chain of reads: 4 to 7 us for what is a few MB (10 for the rows of a long chain).
template <int GROUPS>
__global__ __launch_bounds__(256) void tree_merge_kernel(TreeAttnArgs a, TreePlan plan)
{
    const int rows = 16 * plan.tiles, at = (blockIdx.x * 16 + (threadIdx.x >> 4)) / GROUPS, grp = (threadIdx.x >> 4) % GROUPS, d = 8 * (threadIdx.x & 15);
    const int ui = at / rows, in_block = at - ui * rows;
    Unit u = place_of(a, ui);                               // (as many threads as rows of units)
    const Counts c = counts_of(a, u);
    const int2 info = a.info[ui];
    count(a, c, plan.tiles, u);
    const int row = u.block * rows + in_block;
    if (row >= u.n * a.G || info.y == 0) return;            // (nobody wrote the numbers of a unit without rows)
    float M = SQ_NEG_INF, ls = 0.0f;
    f4 x = {0.f, 0.f, 0.f, 0.f}, y = x;
    auto fold = [&](float pm, float pl, f4 px, f4 py) {
        const float mn = fmaxf(M, pm), mu = mn == SQ_NEG_INF ? 0.0f : mn;
        const float fa = exp2f(M - mu), fb = exp2f(pm - mu);
        ls = ls * fa + pl * fb;
        x = x * fa + px * fb;
        y = y * fa + py * fb;
        M = mn;
    };
    for (int i = grp; i < info.y; i += 4 * GROUPS) {
        float2 ml[4];
        f4 px[4], py[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int j = min(i + k * GROUPS, info.y - 1);
            const float *p = a.part + ((size_t)(j == 0 ? info.x : 2 * ((info.x >> 1) + j)) * rows + in_block) * PART_STRIDE;
            ml[k] = *reinterpret_cast<const float2 *>(p);
            px[k] = *reinterpret_cast<const f4 *>(p + 4 + d);
            py[k] = *reinterpret_cast<const f4 *>(p + 8 + d);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k * GROUPS < info.y) fold(ml[k].x, ml[k].y, px[k], py[k]);
    }
#pragma unroll
    for (int k = 16; k < 16 * GROUPS; k <<= 1) {
        const float pm = __shfl_xor(M, k), pl = __shfl_xor(ls, k);
        f4 px, py;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            px[e] = __shfl_xor(x[e], k);
            py[e] = __shfl_xor(y[e], k);
        }
        fold(pm, pl, px, py);
    }
    if (grp == 0) store_dims(a, u, row, d, M, ls, x, y);
}

TreePlan tree_plan(int B, int H, int rows, long long keys)
{
    TreePlan p{};
    // Rows of a block.  More of them share what a key costs (its codes to f16, its values turned); fewer make more blocks, which are begun and
    // ended side by side, but read the keys again.  us at 64 / 32 rows, 36K keys a head of which 1/8 and 2K user keys: 8 blocks of 64 29.3 / 23.1,
    // 32 32.4 / 30.0, 64 45.6 / 43.3, 128 63.5 / 68.2, 256 99 / 113; with 1/16, 1/8 and 0.3 kept: 64 blocks, 32K keys 33 / 28, 39 / 33, 53 / 51;
    // 32, 128K 39 / 34, 53 / 53, 89 / 106; 64, 128K 53 / 51, 78 / 80, 141 / 169.  Up to 64 blocks, then, and 3M keys of all of them (what is
    // kept is not known here).  Of a cache the room that its table has counts, since what it holds is not known here either: with room for 2M tokens and
    // 512 held, blocks of 64 rows are made where 32 were better (8 blocks 27 / 22 us, 16 29.6 / 24.1, 32 32 / 28, 64 over the cache alone 28 / 20; four blocks over 4K keys in shares
    // and not in parts of their own 12.7 / 11.5); counted as 16K at most, caches that are full would have 32 where 64 are better, which costs more
    // (128K held: 8 blocks 94 / 68, 16 174 / 117, 32 304 / 221).  48 where that makes no more blocks: a quarter less of the softmax (36 rows 44.6 / 37.3).
    const int at64 = (rows + 63) / 64;
    const long long blocks64 = (long long)B * H * at64;
    const bool few = blocks64 <= 64 && blocks64 * keys <= TREE_FEW_KEYS;
    p.tiles = rows <= 16 ? 1 : rows <= 32 || few ? 2 : (rows + 47) / 48 == at64 ? 3 : 4;
    p.blocks = (rows + 16 * p.tiles - 1) / (16 * p.tiles);
    const long long units = (long long)B * H * p.blocks, most = (keys + QT - 1) / QT + 3;      // tiles: of three sources
    p.units = (int)std::min(units, 0x7fffffffll);
    p.splits = units > TREE_SHARED_UNITS ? 1 : units * ((most + 3) / 4) <= TREE_SHARES ? (int)((most + 3) / 4) : 0;
    p.grid = p.splits ? (long long)p.units * p.splits : TREE_SHARES;
    return p;
}

hipError_t launch_tree_attn(TreeAttnArgs a, hipStream_t s)
{
    const long long keys = (a.ranges ? a.L : 0) + (a.seq_len ? (long long)a.max_pages << a.p_log : 0) + (a.Kd ? a.T : 0);
    const TreePlan p = tree_plan(a.B, a.H, a.G * a.T, keys);
    const bool wide = ((size_t)a.n_pages * a.H << a.p_log) * D > (1ull << 32);
    a.blocks = p.blocks;
    auto *kernel = p.tiles == 1 ? (wide ? tree_attn_kernel<1, true> : tree_attn_kernel<1, false>)
                   : p.tiles == 2 ? (wide ? tree_attn_kernel<2, true> : tree_attn_kernel<2, false>)
                   : p.tiles == 3 ? (wide ? tree_attn_kernel<3, true> : tree_attn_kernel<3, false>)
                                  : (wide ? tree_attn_kernel<4, true> : tree_attn_kernel<4, false>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)p.grid), dim3(256), 0, s, a, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    // (few units are in many parts each.  us, 16 / 64 lanes a row: 32 units of 32 rows 8.7 / 5.5, 64 6.9 / 5.2, 128 5.6 / 6.2, 128 of 64 rows
    // 6.8 / 9.1, 1024 in two or three parts 10 / 26)
    if (p.units <= TREE_SHARES / 8) hipLaunchKernelGGL(tree_merge_kernel<4>, dim3((unsigned)(p.units * p.tiles * 4)), dim3(256), 0, s, a, p);
    else hipLaunchKernelGGL(tree_merge_kernel<1>, dim3((unsigned)(p.units * p.tiles)), dim3(256), 0, s, a, p);
    return hipGetLastError();
}

}  // namespace sq
